"""4-bit weights with group scales on the GPU against plain implementations: the quantizer's codes bit for bit (binary32
operations in the order the header states) and its values in 64 bits, the dequantizer, and the product with activations.

Tolerance of the product, derived from how it is summed: within 128 columns the codes times activations are exact products added in
binary32, at most 32 additions deep (16-term tensor-core sums, eight of them, a tree across lanes), then one addition per 64
columns or fewer of a longer row; each addition may truncate (2^-23). So |error| <= (32 + cols / 32) 2^-23 sum |x w|, plus the
rounding of the result to its type. One missing or misplaced column is 1 / cols of that sum, far more.
"""
import pytest
import torch

from paper_2309_01507_b200 import lpmm

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -24}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _unpack(m):
    """Codes of a W4Matrix as int64, rows x cols."""
    k = torch.arange(m.cols, device="cuda")
    return (m.codes[:, k // 2].long() >> (4 * (k % 2))) & 15


def _zeros_of(m):
    k = torch.arange(m.cols, device="cuda") // m.group
    return m.zeros[:, k].long() if m.zeros is not None else torch.full((1, 1), 8, device="cuda")


def _values64(m):
    k = torch.arange(m.cols, device="cuda") // m.group
    return (_unpack(m) - _zeros_of(m)).double() * m.scales.double()[:, k]


def _random_matrix(rows, cols, group=128, zeros=False, scale_dtype=F32, seed=0, extra_pitch=0):
    """Every code, and garbage (not zeros) in the bytes behind a row's end."""
    g = _gen(seed)
    pitch = -(-cols // 32) * 16 + extra_pitch
    codes = torch.randint(0, 256, (rows, pitch), generator=g, device="cuda", dtype=torch.uint8)
    groups = -(-cols // group)
    scales = (0.01 * torch.exp(torch.randn(rows, groups, generator=g, device="cuda"))).to(scale_dtype)
    z = torch.randint(0, 16, (rows, groups), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    return lpmm.W4Matrix(codes, scales, cols, group=group, zeros=z)


def _check_product(m, x, y, bias=None):
    w = _values64(m)
    x64 = x.double().reshape(-1, m.cols)
    want = x64 @ w.T
    size = x64.abs() @ w.abs().T
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    err = (y.double().reshape(want.shape) - want).abs()
    bound = (32 + m.cols / 32) * 2.0 ** -23 * size
    bound = bound + ROUND[y.dtype] * (want.abs() + bound) + TINY[y.dtype]
    assert torch.isfinite(y).all()
    assert (err <= bound).all(), f"{((err - bound).max())} over, worst ratio {(err / bound.clamp(min=1e-300)).max()}"


# ------------------------------------------------------------------------------------------------------- product

@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 129), (7, 31), (16, 32), (17, 33), (64, 128), (127, 96), (129, 1000), (300, 257), (2000, 2048)])
def test_product_shapes(dtype, rows, cols):
    for tokens in (1, 2, 3, 8, 9):
        m = _random_matrix(rows, cols, seed=rows + cols)
        x = torch.randn(tokens, cols, generator=_gen(tokens), device="cuda").to(dtype)
        _check_product(m, x, lpmm.w4_matvec(m, x))


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens", [4, 5, 10, 11, 16, 17, 21, 22, 32, 33, 63, 64, 65, 100, 200])
def test_product_numbers_of_tokens(dtype, tokens):
    m = _random_matrix(200, 1160, group=64, zeros=True, scale_dtype=dtype, seed=tokens)
    x = torch.randn(tokens, 1160, generator=_gen(tokens), device="cuda").to(dtype)
    _check_product(m, x, lpmm.w4_matvec(m, x))


@pytest.mark.parametrize("zeros", [False, True], ids=["symmetric", "zeros"])
@pytest.mark.parametrize("scale_dtype", [F32, BF16, F16], ids=["sf32", "sbf16", "sf16"])
@pytest.mark.parametrize("group", [32, 64, 128, 256, 384, 4096])
def test_product_groups_and_scales(group, scale_dtype, zeros):
    for cols in (group, group + 1, 3 * group - 17, 1000):
        m = _random_matrix(50, cols, group, zeros, scale_dtype, seed=group + cols)
        for dtype in (F32, BF16, F16):
            x = torch.randn(3, cols, generator=_gen(cols), device="cuda").to(dtype)
            _check_product(m, x, lpmm.w4_matvec(m, x))


@pytest.mark.parametrize("rows,cols,tokens", [(4096, 4096, 1), (32000, 4096, 1), (11008, 4096, 8), (4096, 11008, 32), (50265, 1024, 3), (5, 100003, 2), (70001, 33, 2), (11008, 4096, 16), (4096, 11008, 33),
                                              (1000, 20000, 5), (2500, 131072, 1), (40, 131072, 16)])
def test_product_of_layers(rows, cols, tokens):
    for dtype in (BF16, F32):
        m = _random_matrix(rows, cols, seed=1)
        x = torch.randn(tokens, cols, generator=_gen(2), device="cuda").to(dtype)
        _check_product(m, x, lpmm.w4_matvec(m, x))


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_product_strides_bias_and_fp32_result(dtype):
    g = _gen(5)
    for cols, extra, off in ((384, 5, 1), (384, 8, 0), (130, 3, 3)):
        m = _random_matrix(77, cols, 32, True, BF16, seed=cols, extra_pitch=48)
        buf = torch.full((9, cols + extra + off), float("nan"), device="cuda", dtype=dtype)   # what lies between the rows is not read
        x = buf[:, off:off + cols]
        x.copy_(torch.randn(9, cols, generator=g, device="cuda"))
        bias = torch.randn(77, generator=g, device="cuda")
        out = torch.full((9, 80), 7.0, device="cuda", dtype=dtype)
        y = lpmm.w4_matvec(m, x, bias=bias, out=out[:, 2:79])
        _check_product(m, x, y, bias)
        assert (out[:, :2] == 7).all() and (out[:, 79:] == 7).all()
        y32 = lpmm.w4_matvec(m, x, bias=bias, out_dtype=F32)
        assert y32.dtype == F32
        _check_product(m, x, y32, bias)
        y1 = lpmm.w4_matvec(m, x[4], bias=bias)
        assert y1.shape == (77,) and y1.dtype == dtype
        _check_product(m, x[4:5], y1, bias)
    # a slice of rows of a larger matrix is a matrix
    m = _random_matrix(300, 512, seed=9)
    part = lpmm.W4Matrix(m.codes[100:133], m.scales[100:133], 512)
    x = torch.randn(2, 512, generator=g, device="cuda").to(dtype)
    _check_product(part, x, lpmm.w4_matvec(part, x))


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_product_keeps_tokens_apart_and_ends_of_the_range(dtype):
    m = _random_matrix(100, 700, seed=3)
    x = torch.randn(6, 700, generator=_gen(4), device="cuda").to(dtype)
    clean = lpmm.w4_matvec(m, x)
    for bad in (float("nan"), float("inf"), -float("inf")):
        spoiled = x.clone()
        spoiled[2, 699] = bad
        y = lpmm.w4_matvec(m, spoiled)
        keep = [0, 1, 3, 4, 5]
        assert torch.equal(y[keep], clean[keep])
        q = _unpack(m)[:, 699]
        if bad == bad:      # infinity times the sign of the weight; 0 * infinity is NaN
            assert torch.isinf(y[2][q != 8]).all() and torch.isnan(y[2][q == 8]).all()
            assert ((y[2][q != 8] > 0) == ((q[q != 8] > 8) == (bad > 0))).all()
        else:
            assert torch.isnan(y[2]).all()
    assert torch.equal(lpmm.w4_matvec(m, x), clean)                        # the same bits every time
    small = (x.double() * 2.0 ** (-14 if dtype == F16 else -100)).to(dtype)   # subnormal halves, small floats
    y = lpmm.w4_matvec(m, small, out_dtype=F32)
    _check_product(m, small, y)
    zero = torch.zeros(6, 700, device="cuda", dtype=dtype)
    assert (lpmm.w4_matvec(m, zero) == 0).all()
    assert lpmm.w4_matvec(m, x[:0]).shape == (0, 100)                      # no tokens: nothing to do


def test_product_on_another_stream():
    m = _random_matrix(3000, 2048, seed=6)
    x = torch.randn(4, 2048, generator=_gen(7), device="cuda").to(BF16)
    want = lpmm.w4_matvec(m, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lpmm.w4_matvec(m, x, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_a_chain_in_a_graph():
    """Weights requantized, used and taken back within one captured chain: each call waits for the one before it."""
    w = torch.randn(700, 1000, generator=_gen(8), device="cuda")
    x = torch.randn(3, 1000, generator=_gen(9), device="cuda")
    src = w.clone()

    def chain(a):
        m = lpmm.w4_quantize(a, group=64, zero_points=True)
        y = lpmm.w4_matvec(m, x)
        z = lpmm.w4_matvec(m, x * y[:, :1])
        return y, z, lpmm.w4_dequantize(m, BF16)

    chain(src)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain(src)
    for k in range(6):
        src.copy_(w * (k - 2.5))
        graph.replay()
        for a, b in zip(got, chain(w * (k - 2.5))):
            assert torch.equal(a, b)


# ----------------------------------------------------------------------------------------- quantizer, dequantizer

def _plain_quantize(w, group, zero_points, scale_dtype):
    """The header's operations, one binary32 rounding each, on the CPU. Returns codes, scales, zeros."""
    w = w.float().cpu()
    codes, scales, zeros = [], [], []
    for a in range(0, w.shape[1], group):
        v = w[:, a:a + group]
        lo, hi = v.amin(1, keepdim=True).clamp(max=0), v.amax(1, keepdim=True).clamp(min=0)
        if zero_points:
            s = (hi - lo) * torch.tensor(1 / 15, dtype=F32)
        else:
            s = torch.maximum(hi, -lo) * torch.tensor(1 / 7, dtype=F32)
        if scale_dtype == F16:
            s = s.clamp(max=65504.0)
        s = s.to(scale_dtype)
        r = torch.where(s.float() >= torch.finfo(F32).tiny, torch.ones(()) / s.float(), torch.zeros(()))
        z = (-lo * r).round().clamp(0, 15) if zero_points else torch.full_like(lo, 8)
        codes.append(((v * r).round() + z).clamp(0, 15))
        scales.append(s)
        zeros.append(z)
    return torch.cat(codes, 1), torch.cat(scales, 1), torch.cat(zeros, 1)


@pytest.mark.parametrize("zeros", [False, True], ids=["symmetric", "zeros"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 32), (33, 129), (17, 1001), (64, 1024), (2, 5000)])
def test_quantizer(rows, cols, dtype, zeros):
    g = _gen(rows * cols)
    w = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    w[rows // 2] = w[rows // 2].abs()      # one-sided rows
    w[rows // 3] = 0                       # a row of zeros
    w = w.to(dtype)
    for group in (32, 64, 128, 256, 1024):
        for scale_dtype in (F32, dtype):
            m = lpmm.w4_quantize(w, group=group, zero_points=zeros, scale_dtype=scale_dtype)
            codes, scales, z = _plain_quantize(w, group, zeros, scale_dtype)
            assert torch.equal(m.scales.cpu(), scales)
            if zeros:
                assert torch.equal(m.zeros.cpu().float(), z)
            assert torch.equal(_unpack(m).cpu().float(), codes)
            # in 64 bits: a value is half a step away at most, a step where the code had to be clamped; types round the scale
            k = torch.arange(cols, device="cuda") // group
            step = m.scales.double()[:, k]
            off = (w.double() - _values64(m)).abs()
            clamped = (_unpack(m) == 0) | (_unpack(m) == 15)
            slack = 2.0 ** -10 + 15 * ROUND[scale_dtype]
            tiny = 15 * (TINY[scale_dtype] + 2.0 ** -126)     # steps below the types' range
            assert (off <= step * torch.where(clamped, 1.0 + slack, 0.5 + 2.0 ** -10) + tiny).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_quantizer_strides_and_extremes(dtype):
    g = _gen(11)
    buf = torch.full((20, 523), float("nan"), device="cuda", dtype=dtype)
    w = buf[:, 3:516]
    w.copy_(torch.randn(20, 513, generator=g, device="cuda"))
    m = lpmm.w4_quantize(w, group=32)
    assert torch.equal(_unpack(m).cpu().float(), _plain_quantize(w, 32, False, F32)[0])
    top = torch.finfo(dtype).max
    ends = torch.tensor([[top, -top, 0, top / 2], [-top, 0, 0, 0], [top, top, top, top]], device="cuda").to(dtype)
    m = lpmm.w4_quantize(ends, group=32)
    assert torch.equal(_unpack(m).cpu().float(), _plain_quantize(ends, 32, False, F32)[0])
    assert torch.isfinite(lpmm.w4_dequantize(m, F32)).all()
    low = (torch.randn(4, 64, generator=g, device="cuda") * (2.0 ** -24 if dtype == F16 else 1e-41)).to(dtype)   # subnormal
    m = lpmm.w4_quantize(low, group=64)
    assert torch.equal(_unpack(m).cpu().float(), _plain_quantize(low, 64, False, F32)[0])
    bad = torch.full((2, 64), float("nan"), device="cuda", dtype=dtype)       # unspecified, but codes stay codes
    bad[1] = float("inf")
    assert (_unpack(lpmm.w4_quantize(bad)) <= 15).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128, 512])
def test_dequantizer(dtype, group):
    for rows, cols in ((1, 1), (9, 31), (40, 1001), (64, 2048)):
        for zeros, sd in ((False, F32), (True, BF16), (True, F16)):
            m = _random_matrix(rows, cols, group, zeros, sd, seed=rows + cols, extra_pitch=16)
            want = _values64(m)
            got = lpmm.w4_dequantize(m, dtype)
            # one rounding of the binary32 product, one to the type
            assert ((got.double() - want).abs() <= want.abs() * (2.0 ** -24 + ROUND[dtype] * (1 + 2.0 ** -20)) + TINY[dtype]).all()
            out = torch.full((rows, cols + 3), 5.0, device="cuda", dtype=dtype)
            assert torch.equal(lpmm.w4_dequantize(m, out=out[:, 1:1 + cols]), got)
            assert (out[:, 0] == 5).all() and (out[:, cols + 1:] == 5).all()


def test_a_matrix_of_more_than_2_31_codes():
    rows, cols = 70_000, 32_768       # 2.3 G weights: row offsets pass 32 bits
    m = _random_matrix(rows, cols, seed=1)
    x = torch.randn(2, cols, generator=_gen(2), device="cuda").to(BF16)
    y = lpmm.w4_matvec(m, x)
    tail = lpmm.W4Matrix(m.codes[-100:], m.scales[-100:], cols)
    _check_product(tail, x, y[:, -100:])
    head = lpmm.W4Matrix(m.codes[:100], m.scales[:100], cols)
    _check_product(head, x, y[:, :100])
