"""Cases and plain forms of the operators around the optimizer step: products with 4-bit weights, their quantizer, and the
loss that distils a teacher's top logits into a student, with its gradient.

    listed()             the cases that are measured by name
    draw(rng)            one more case of the same ranges
    prepare(case, seed)  a case's inputs on the GPU, made from the seed alone
    run(state)           one pass: the plain form in elementary torch operations (fp32, rounded once at the end), or, with
                         own = True, the calls a user makes of the library
    exact(case, seed)    the same outputs from the definition, in 64 bits
    work(case)           the bytes and operations a pass cannot do without

Definitions (i a row of the weight, k a column, G = ceil(cols / group) groups per row, j a vocabulary entry):
    w4_quantize   symmetric: s = round(max |w| / 7), q = clamp(rint(w / s), -8, 7) + 8, value (q - 8) s;
                  with zero points: s = round((hi - lo) / 15), hi = max(w, 0), lo = min(w, 0), z = clamp(rint(-lo / s), 0, 15),
                  q = clamp(rint(w / s) + z, 0, 15), value (q - z) s. round() is to the type the scales are kept in.
    w4_matvec     y[m, i] = sum_k x[m, k] (q[i, k] - z[i, k / group]) s[i, k / group] + bias[i]
    distill       p = softmax(z / tau) over the vocabulary; q over a row's K listed entries, softmax(t / tau) over those
                  entries, or exp(t / tau - lse) when the teacher's log-sum-exp is given (then the entries left out form one
                  more class: q_rest = 1 - sum q, p_rest = 1 - sum p).  loss = weight * sum q (log q - log p)  (+ that class),
                  gradient = weight / tau * (p_j Q - q_j), and for entries left out p_j (Q - q_rest / p_rest); Q = sum q.
"""
import math

import torch

own = False

_DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _es(name):
    return 4 if name == "float32" else 2


def _matvec(name, tokens, rows, cols, group=128, dtype="bfloat16", scale="float32", zeros=False, bias=False):
    case = {"op": "w4_matvec", "tokens": tokens, "rows": rows, "cols": cols, "group": group, "dtype": dtype, "scale": scale,
            "zeros": zeros, "bias": bias}
    return dict(case, name=name) if name else case


def _quantize(name, rows, cols, group=128, dtype="bfloat16", scale="float32", zeros=False):
    case = {"op": "w4_quantize", "rows": rows, "cols": cols, "group": group, "dtype": dtype, "scale": scale, "zeros": zeros}
    return dict(case, name=name) if name else case


def _distill(name, op, tokens, vocab, top, dtype="bfloat16", tail=False, tau=1.0, masked=0.0, padded=0, pitch=0):
    case = {"op": op, "tokens": tokens, "vocab": vocab, "top": top, "dtype": dtype, "tail": tail, "tau": tau, "masked": masked,
            "padded": padded, "pitch": pitch}
    return dict(case, name=name) if name else case


def listed():
    return [
        # One token through an attention projection of a 4096-wide decoder: the smallest product, where latency counts.
        _matvec("token_4096x4096", 1, 4096, 4096),
        # One token through that decoder's output head, the largest matrix a token has to pass.
        _matvec("token_head_32000x4096", 1, 32000, 4096),
        # Eight sequences decoded together through the wide half of the feed-forward block; asymmetric codes, 16-bit scales.
        _matvec("batch8_11008x4096_zeros", 8, 11008, 4096, group=64, scale="bfloat16", zeros=True),
        # Thirty-two sequences through the narrow half, whose rows are long; the finest groups, half precision.
        _matvec("batch32_4096x11008_f16", 32, 4096, 11008, group=32, dtype="float16", scale="float16"),
        # Three positions through a masked-language-model head with its bias: an odd number of rows, fp32 activations.
        _matvec("mlm_head_50265x1024_f32", 3, 50265, 1024, dtype="float32", bias=True),
        # A bf16 head matrix to 4 bits and back, as done once when a trained model is put into service.
        _quantize("quantize_32000x4096", 32000, 4096),
        # An fp32 matrix with odd extents, asymmetric, fine groups: rows that end inside a group and inside a byte.
        _quantize("quantize_odd_50265x1001_f32", 50265, 1001, group=32, dtype="float32", scale="float16", zeros=True),
        # The loss alone over an evaluation batch.
        _distill("eval_2048x32000", "distill_loss", 2048, 32000, 32, tau=2.0),
        # The loss alone over a large vocabulary, few rows, fp16 logits in a padded buffer: a row is split over several SMs.
        _distill("eval_64x131073_f16", "distill_loss", 64, 131073, 256, dtype="float16", tail=True, padded=17, pitch=7),
        # Four positions of one short sample: the smallest training call.
        _distill("step_4x32000", "distill_grad", 4, 32000, 16),
        # An ordinary training micro-batch with the class of the entries left out, a tenth of it padding.
        _distill("step_4096x32000_tail", "distill_grad", 4096, 32000, 64, tail=True, tau=2.0, masked=0.1),
        # fp32 logits over an odd vocabulary where only the masked positions of a sample carry a loss.
        _distill("step_1001x50265_f32", "distill_grad", 1001, 50265, 100, dtype="float32", masked=0.15),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["w4_matvec", "w4_matvec", "w4_quantize", "distill_loss", "distill_grad", "distill_grad"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    if op in ("w4_matvec", "w4_quantize"):
        rows, cols = _log(rng, 64, 50265), _log(rng, 64, 16384)
        if rng.random() < 0.5:  # half of them whole multiples, as most layers are
            rows, cols = max(64, rows // 64 * 64), max(64, cols // 64 * 64)
        rows = min(rows, 50265 * 1001 // cols if dtype == "float32" else 32000 * 4096 // cols)
        group, zeros = rng.choice([32, 64, 128, 128]), rng.random() < 0.4
        scale = rng.choice(["float32", dtype])
        if op == "w4_quantize":
            return _quantize(None, rows, cols, group, dtype, scale, zeros)
        return _matvec(None, _log(rng, 1, 64), rows, cols, group, dtype, scale, zeros, rng.random() < 0.3)
    vocab = _log(rng, 1000, 200000)
    tokens = min(_log(rng, 1, 8192), 262_000_000 // _es(dtype) // vocab)
    return _distill(None, op, max(1, tokens), vocab, min(_log(rng, 4, 512), vocab // 2), dtype, rng.random() < 0.5,
                    rng.choice([1.0, 2.0, 4.0]), rng.choice([0.0, 0.0, 0.1, 0.5]), rng.choice([0, 0, 5, 64]), rng.choice([0, 0, 0, 8, 3]))


# ---------------------------------------------------------------------------------------------------------------- inputs

def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kw = dict(generator=gen, device="cuda")
    dtype = _DTYPES[case["dtype"]]
    if case["op"] in ("w4_matvec", "w4_quantize"):
        rows, cols, group = case["rows"], case["cols"], case["group"]
        ngroups = -(-cols // group)
        if case["op"] == "w4_quantize":   # a trained matrix: rows of unequal size, a few large entries
            w = torch.randn(rows, cols, **kw) * (0.02 * torch.exp(0.3 * torch.randn(rows, 1, **kw)))
            w += (torch.rand(rows, cols, **kw) < 1e-3) * torch.randn(rows, cols, **kw) * 0.2
            return {"w": w.to(dtype)}
        pitch = -(-cols // 32) * 16   # bytes per row of codes: two codes per byte, rows at 16-byte boundaries
        mean = torch.randint(5, 11, (rows, 1), **kw).float() if case["zeros"] else 8.0
        q = (torch.randn(rows, 2 * pitch, **kw) * 2.5 + mean).round_().clamp_(0, 15).to(torch.uint8)
        s = {"codes": q[:, 0::2] | (q[:, 1::2] << 4)}
        s["scales"] = (0.005 * torch.exp(0.4 * torch.randn(rows, ngroups, **kw))).to(_DTYPES[case["scale"]])
        s["zeros"] = (mean + torch.randint(-1, 2, (rows, ngroups), **kw)).to(torch.uint8) if case["zeros"] else None
        s["bias"] = 0.1 * torch.randn(rows, **kw) if case["bias"] else None
        x = torch.randn(case["tokens"], cols, **kw)   # activations after a norm: unit size, a few outlier channels
        s["x"] = (x * (1 + 20 * (torch.rand(1, cols, **kw) < 0.002))).to(dtype)
        return s
    tokens, vocab, top = case["tokens"], case["vocab"], case["top"]
    z = torch.randn(tokens, vocab + case["pitch"], **kw).mul_(2.5)
    t = torch.randn(tokens, vocab, **kw).mul_(1.5).add_(z[:, :vocab])
    if case["padded"]:    # entries behind the tokenizer's last one, masked by the model with the type's lowest value
        z[:, vocab - case["padded"]:vocab] = torch.finfo(dtype).min
        t[:, vocab - case["padded"]:] = -math.inf
    values, ids = torch.topk(t, top, dim=1)
    s = {"logits": z.to(dtype)[:, :vocab], "ids": ids, "top": values, "lse": None, "weights": None}
    if case["tail"]:
        s["lse"] = torch.logsumexp(t.mul_(1 / case["tau"]), dim=1)
    keep = torch.rand(tokens, **kw) >= case["masked"]
    if case["masked"]:    # padding or unmasked positions: no loss, no gradient
        s["weights"] = keep.float() / keep.sum().clamp(min=1)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own and case["op"] == "w4_matvec":   # the handle a program keeps beside its weights: pointers and sizes, nothing computed
        from paper_2309_01507_b200 import lpmm
        s["weight"] = lpmm.W4Matrix(s["codes"], s["scales"], case["cols"], group=case["group"], zeros=s["zeros"])
    return s


# ----------------------------------------------------------------------------------------------------------- plain forms

def _values(codes, scales, zeros, cols, group):
    """The fp32 matrix that 4-bit codes stand for."""
    q = torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1)[:, :cols].float()
    z = zeros.float().repeat_interleave(group, dim=1)[:, :cols] if zeros is not None else 8.0
    return (q - z) * scales.float().repeat_interleave(group, dim=1)[:, :cols]


def _plain_matvec(s, c):
    y = s["x"].float() @ _values(s["codes"], s["scales"], s["zeros"], c["cols"], c["group"]).T
    return (y + s["bias"] if s["bias"] is not None else y).to(s["x"].dtype)


def _plain_quantize(s, c):
    rows, cols, group = c["rows"], c["cols"], c["group"]
    w = torch.nn.functional.pad(s["w"].float(), (0, -cols % group)).reshape(rows, -1, group)
    if c["zeros"]:
        lo, hi = w.amin(2, keepdim=True).clamp(max=0), w.amax(2, keepdim=True).clamp(min=0)
        scale = ((hi - lo) * (1 / 15)).to(_DTYPES[c["scale"]])
        r = 1 / scale.float()
        zero = (-lo * r).round().clamp(0, 15)
        q = ((w * r).round() + zero).clamp(0, 15)
    else:
        scale = (w.abs().amax(2, keepdim=True) * (1 / 7)).to(_DTYPES[c["scale"]])
        zero = torch.full_like(scale, 8, dtype=torch.float32)
        q = ((w * (1 / scale.float())).round() + 8).clamp(0, 15)
    values = ((q - zero) * scale.float()).reshape(rows, -1)[:, :cols].to(s["w"].dtype)
    return {"values": values, "scales": scale[:, :, 0], "zeros": zero[:, :, 0].to(torch.uint8) if c["zeros"] else None}


def _plain_distill(s, c):
    it = 1 / c["tau"]
    x = s["logits"].float() * it
    x = x - x.amax(1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    t = s["top"] * it
    if c["tail"]:
        log_q = t - s["lse"][:, None]
    else:
        t = t - t.amax(1, keepdim=True)
        log_q = t - torch.log(torch.exp(t).sum(1, keepdim=True))
    q = torch.exp(log_q)
    loss = (q * (log_q - (x.gather(1, s["ids"]) - torch.log(total)))).sum(1)
    p = e / total
    if c["tail"]:
        rest = (1 - q.sum(1, keepdim=True)).clamp(min=0)
        p_rest = p.scatter(1, s["ids"], 0.0).sum(1, keepdim=True)
        loss = loss + (rest * (torch.log(rest) - torch.log(p_rest)))[:, 0]
        grad = (p * (1 - rest / p_rest)).scatter(1, s["ids"], p.gather(1, s["ids"]) - q)
    else:
        grad = p.scatter(1, s["ids"], p.gather(1, s["ids"]) - q)
    w = s["weights"] if s["weights"] is not None else torch.ones_like(loss)
    loss = torch.where(w != 0, loss * w, 0.0)
    if c["op"] == "distill_loss":
        return loss
    return {"loss": loss, "grad": (grad * (w * it)[:, None]).to(s["logits"].dtype)}


def run(state):
    c = state["case"]
    if not own:
        return {"w4_matvec": _plain_matvec, "w4_quantize": _plain_quantize, "distill_loss": _plain_distill,
                "distill_grad": _plain_distill}[c["op"]](state, c)
    from paper_2309_01507_b200 import lpmm
    if c["op"] == "w4_matvec":
        return lpmm.w4_matvec(state["weight"], state["x"], bias=state["bias"])
    if c["op"] == "w4_quantize":
        m = lpmm.w4_quantize(state["w"], group=c["group"], zero_points=c["zeros"], scale_dtype=_DTYPES[c["scale"]])
        return {"values": lpmm.w4_dequantize(m, state["w"].dtype), "scales": m.scales, "zeros": m.zeros}
    args = (state["logits"], state["ids"], state["top"])
    kw = dict(temperature=c["tau"], teacher_lse=state["lse"], weights=state["weights"])
    if c["op"] == "distill_loss":
        return lpmm.distill_loss(*args, **kw)
    loss, grad = lpmm.distill_grad(*args, **kw)
    return {"loss": loss, "grad": grad}


# --------------------------------------------------------------------------------------------------- definition in 64 bits

def _exact_matvec(s, c):
    k = torch.arange(c["cols"], device="cuda")
    out = []
    for a in range(0, c["rows"], 8192):
        part = slice(a, min(a + 8192, c["rows"]))
        q = (s["codes"][part][:, k // 2].long() >> (4 * (k % 2))) & 15
        z = s["zeros"][part][:, k // c["group"]].long() if c["zeros"] else 8
        out.append(s["x"].double() @ ((q - z).double() * s["scales"][part].double()[:, k // c["group"]]).T)
    y = torch.cat(out, 1)
    return y + s["bias"].double() if c["bias"] else y


def _exact_quantize(s, c):
    values, scales, zeros = [], [], []
    for a in range(0, c["cols"], c["group"]):
        w = s["w"][:, a:a + c["group"]].double()
        if c["zeros"]:
            lo = w.min(1, keepdim=True).values.clamp(max=0)
            scale = ((w.max(1, keepdim=True).values.clamp(min=0) - lo) / 15).to(_DTYPES[c["scale"]]).double()
            zero = torch.round(-lo / scale).clamp(0, 15)
            q = (torch.round(w / scale) + zero).clamp(0, 15) - zero
            zeros.append(zero)
        else:
            scale = (w.abs().max(1, keepdim=True).values / 7).to(_DTYPES[c["scale"]]).double()
            q = torch.round(w / scale).clamp(-8, 7)
        values.append(q * scale)
        scales.append(scale)
    return {"values": torch.cat(values, 1), "scales": torch.cat(scales, 1),
            "zeros": torch.cat(zeros, 1).to(torch.uint8) if zeros else None}


def _exact_distill(s, c):
    losses, grads = [], []
    rows_at_once = max(1, 40_000_000 // c["vocab"])
    for a in range(0, c["tokens"], rows_at_once):
        part = slice(a, a + rows_at_once)
        ids, tau = s["ids"][part], c["tau"]
        logp = torch.log_softmax(s["logits"][part].double() / tau, 1)
        t = s["top"][part].double() / tau
        logq = t - s["lse"][part].double()[:, None] if c["tail"] else torch.log_softmax(t, 1)
        q = logq.exp()
        w = s["weights"][part].double() if s["weights"] is not None else torch.ones(len(t), dtype=torch.float64, device="cuda")
        loss = (q * (logq - logp.gather(1, ids))).sum(1)
        p = logp.exp_()
        grad = p
        if c["tail"]:
            rest = (1 - q.sum(1)).clamp(min=0)
            left_out = torch.ones_like(p, dtype=torch.bool).scatter_(1, ids, False)
            p_rest = (p * left_out).sum(1)
            loss = loss + rest * (rest / p_rest).log()
            grad = torch.where(left_out, p * (1 - rest / p_rest)[:, None], p)
        losses.append(loss * w)
        if c["op"] == "distill_grad":
            grads.append((grad.scatter_add(1, ids, -q) * (w / tau)[:, None]))
    loss = torch.cat(losses)
    return {"loss": loss, "grad": torch.cat(grads)} if grads else loss


def exact(case, seed):
    s = _inputs(case, seed)
    return {"w4_matvec": _exact_matvec, "w4_quantize": _exact_quantize, "distill_loss": _exact_distill,
            "distill_grad": _exact_distill}[case["op"]](s, case)


def work(case):
    if case["op"] in ("w4_matvec", "w4_quantize"):
        rows, cols = case["rows"], case["cols"]
        weight = rows * (-(-cols // 2)) + rows * -(-cols // case["group"]) * (_es(case["scale"]) + int(case["zeros"]))
        if case["op"] == "w4_quantize":   # the matrix read, the codes written; the codes read, the values written
            return {"bytes": 2 * rows * cols * _es(case["dtype"]) + 2 * weight, "flops": 4 * rows * cols}
        m = case["tokens"]
        return {"bytes": weight + m * (rows + cols) * _es(case["dtype"]) + 4 * rows * int(case["bias"]), "flops": 2 * m * rows * cols}
    t, v, es = case["tokens"], case["vocab"], _es(case["dtype"])
    live = t * (1 - case["masked"])       # the logits of positions without a loss need not be read
    b = live * (v * es + 12 * case["top"] + 4 * int(case["tail"])) + 4 * t * (1 + int(case["masked"] > 0))
    if case["op"] == "distill_grad":
        b += t * v * es
    return {"bytes": int(b), "flops": int((4 if case["op"] == "distill_loss" else 7) * live * v)}
