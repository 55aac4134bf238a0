"""Operators of a language model's training step and of its scoring, as they are measured.

A case is a dict of plain values.  Its "kind" names the operator:

  norm         h = x + residual; y = RMS norm of h, coded in 8 bits with a power-of-two scale per group of columns
  norm_grad    the norm's backward pass, from the residual stream in its own type or from its 8-bit codes
  checkpoint   rows coded in 8 bits, and decoded again when the backward pass needs them
  weight_grad  weight gradient of a linear layer, dW = dY^T X, with X in 8-bit codes
  logprob      log probability of a given token per row of logits, entropy, and the most likely alternatives
  logprob_grad gradient of the logits from those of the log probability and of the entropy

`own` False: elementary torch operations in 32 bits; True: the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token on its way through a layer of 8192 features: latency is all there is
        dict(name="norm_one_token", kind="norm", T=1, K=8192, type="bf16", group=128, residual=True, pad=0),
        # a training batch of 8192 tokens, 4096 features, fine scales
        dict(name="norm_train", kind="norm", T=8192, K=4096, type="bf16", group=32, residual=True, pad=0),
        # small model in 32 bits with an odd width, the residual stream kept in 8 bits, rows inside a wider buffer
        dict(name="norm_grad_odd", kind="norm_grad", T=1023, K=1001, type="f32", group=64, coded=True, residual=False, pad=7),
        # backward of a training batch, with the gradient that comes down the residual stream
        dict(name="norm_grad_train", kind="norm_grad", T=16384, K=4096, type="bf16", group=32, coded=False, residual=True, pad=0),
        # activations of a small model, odd sizes
        dict(name="checkpoint_odd", kind="checkpoint", T=333, K=2051, type="f16", group=64, pad=5),
        # the widest activation of a large layer
        dict(name="checkpoint_large", kind="checkpoint", T=16384, K=8192, type="bf16", group=32, pad=0),
        # a layer of a small model in 32 bits: gradient of odd sizes
        dict(name="weight_grad_odd", kind="weight_grad", T=1000, N=515, K=2051, type="f32", group=64, pad=1),
        # a layer of a large model over a training batch: the largest case
        dict(name="weight_grad_train", kind="weight_grad", T=16384, N=8192, K=4096, type="bf16", group=32, pad=0),
        # one token of an answer: its log probability and twenty alternatives
        dict(name="logprob_one_token", kind="logprob", T=1, V=128_000, type="bf16", top=20, masked=False, pad=0),
        # scoring a batch over an odd vocabulary that ends in entries that are masked out
        dict(name="logprob_batch", kind="logprob", T=4096, V=100_003, type="bf16", top=8, masked=True, pad=0),
        # loss gradient of a few hundred rows in 32 bits, over as many classes as a sparse text set has features
        dict(name="logprob_grad_odd", kind="logprob_grad", T=509, V=47_236, type="f32", masked=True, pad=3),
        # loss gradient of a training batch
        dict(name="logprob_grad_train", kind="logprob_grad", T=8192, V=32_768, type="bf16", masked=False, pad=0),
    ]


def draw(rng):
    def size(lo, hi):
        """Log-uniform, odd more often than not."""
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, v | 1 if rng.random() < 0.6 else v))

    kind = rng.choice(["norm", "norm_grad", "checkpoint", "weight_grad", "weight_grad", "logprob", "logprob_grad"])
    c = dict(kind=kind, type=rng.choice(["bf16", "bf16", "f32", "f16"]), pad=rng.choice([0, 0, 0, 1, 8, 13]))
    if kind in ("norm", "norm_grad", "checkpoint"):
        K = size(64, 16384)
        c.update(T=size(1, min(16384, (1 << 25) // K)), K=K, group=rng.choice([32, 64, 128]))
        if kind != "checkpoint":
            c.update(residual=rng.random() < 0.7)
        if kind == "norm_grad":
            c.update(coded=rng.random() < 0.5)
    elif kind == "weight_grad":
        N, K = size(16, 8192), size(16, 8192)
        c.update(T=size(1, min(16384, (1 << 37) // (N * K))), N=N, K=K, group=rng.choice([32, 64, 128]))
    else:
        V = size(2, 200_000)
        c.update(T=size(1, min(8192, (1 << 27) // V)), V=V, masked=rng.random() < 0.4)
        if kind == "logprob":
            c.update(top=rng.choice([0, 1, min(V, 5), min(V, 20), min(V, 64)]))
    return c


def work(case):
    c, t = case, BYTES[case["type"]]
    if c["kind"] in ("norm", "norm_grad", "checkpoint"):
        E, coded = c["T"] * c["K"], c["T"] * (c["K"] + -(-c["K"] // c["group"]))
        if c["kind"] == "norm":            # x, residual, h; codes and the values they stand for; weight; rstd
            return dict(bytes=E * (t * (3 if c["residual"] else 2) + 2) + coded + 4 * c["K"] + 4 * c["T"], flops=8 * E)
        if c["kind"] == "checkpoint":      # two calls: x -> codes, codes -> values
            return dict(bytes=E * (t + 2) + 2 * coded, flops=4 * E)
        h = coded if c["coded"] else E * t
        return dict(bytes=E * t * (3 if c["residual"] else 2) + h + 8 * c["K"] + 4 * c["T"], flops=10 * E)
    if c["kind"] == "weight_grad":
        T, N, K = c["T"], c["N"], c["K"]
        return dict(bytes=T * N * t + T * (K + -(-K // c["group"])) + 4 * N * K, flops=2 * T * N * K)
    E = c["T"] * c["V"]
    if c["kind"] == "logprob":
        return dict(bytes=E * t + c["T"] * (20 + 8 * c["top"]), flops=6 * E)
    return dict(bytes=2 * E * t + c["T"] * 24, flops=6 * E)


# ---- inputs ------------------------------------------------------------------------------------------------


def values_of(v, group):
    """What v's 8-bit codes stand for, in 32 bits: per row and `group` columns the smallest power of two, 2^-126 at
    least, by which the largest magnitude is at most 127, and the nearest whole multiples of it, ties to even; NaN
    for a group that is not finite."""
    return _decode(*codes_of(v, group), group, v.shape[1])


def codes_of(v, group):
    T, K = v.shape
    p = torch.nn.functional.pad(v, (0, -K % group)).view(T, -1, group)
    most = p.abs().amax(dim=2)
    e = (((most.view(torch.int32) + 0x1FFFF) >> 23) - 6).clamp(min=1)
    e = torch.where(torch.isfinite(most), e, torch.full_like(e, 255))
    inv = torch.where(e == 255, torch.zeros_like(e), 254 - e)
    q = p * (inv << 23).view(torch.float32).unsqueeze(2)
    q = torch.where((e == 255).unsqueeze(2), torch.zeros_like(q), torch.round(q))
    return q.view(T, -1)[:, :K].to(torch.int8), e.to(torch.uint8)


def _decode(codes, scales, group, K):
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    s = torch.where(scales == 255, torch.full_like(s, math.nan), s)
    return codes.float() * s.repeat_interleave(group, dim=1)[:, :K]


def _rows(gen, T, K, type_, pad, scale=1.0):
    """T rows of K values inside rows of K + pad."""
    v = torch.randn(T, K + pad, generator=gen, device="cuda") * scale
    return v.to(TYPES[type_])[:, :K]


def _stream(gen, c):
    """A residual stream: rows of different sizes and a few features that stand out."""
    T, K = c["T"], c["K"]
    v = torch.randn(T, K + c["pad"], generator=gen, device="cuda")
    v *= torch.exp(0.5 * torch.randn(T, 1, generator=gen, device="cuda"))
    v *= 1.0 + 7.0 * (torch.rand(K + c["pad"], generator=gen, device="cuda") < 0.01)
    return v.to(TYPES[c["type"]])[:, :K]


def _coded_buffers(c):
    K, g = c["K"], c["group"]
    stride = -(-K // 16) * 16
    return (torch.zeros(c["T"], stride, dtype=torch.int8, device="cuda"),
            torch.zeros(c["T"], -(-K // g), dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    c, dev = dict(case), "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t = TYPES[c["type"]]
    s = dict(c=c, layout=None, ws=None)

    def f32(*shape):
        return torch.empty(*shape, dtype=torch.float32, device=dev)

    if c["kind"] in ("norm", "norm_grad", "checkpoint"):
        T, K = c["T"], c["K"]
        s["x"] = _stream(gen, c)
        s["codes"], s["scales"] = _coded_buffers(c)
        if c["kind"] != "checkpoint":
            s["weight"] = 1.0 + 0.2 * torch.randn(K, generator=gen, device=dev)
            s["rstd"] = f32(T)
        if c["kind"] == "norm":
            s["residual"] = _rows(gen, T, K, c["type"], c["pad"]) if c["residual"] else None
            s["h"] = torch.empty(T, K, dtype=t, device=dev)
        if c["kind"] == "norm_grad":
            s["dy"] = _rows(gen, T, K, c["type"], c["pad"], 0.05)
            s["dh"] = _rows(gen, T, K, c["type"], c["pad"], 0.05) if c["residual"] else None
            h = s["x"].float()
            if c["coded"]:
                codes, s["scales"] = codes_of(h, c["group"])
                s["codes"][:, :K] = codes
                h = _decode(codes, s["scales"], c["group"], K)
            s["rstd"] = torch.rsqrt((h * h).mean(dim=1) + EPS)
            s["dx"] = torch.empty(T, K, dtype=t, device=dev)
            s["dweight"] = f32(K)
        else:
            s["y"] = torch.empty(T, K, dtype=torch.bfloat16, device=dev)
    elif c["kind"] == "weight_grad":
        s["dy"] = _rows(gen, c["T"], c["N"], c["type"], c["pad"], 0.02)
        s["codes"], s["scales"] = _coded_buffers(c)
        codes, s["scales"] = codes_of(_stream(gen, dict(c, pad=0)).float(), c["group"])
        s["codes"][:, :c["K"]] = codes
        s["dw"] = f32(c["N"], c["K"])
    else:
        T, V = c["T"], c["V"]
        x = 2.5 * torch.randn(T, V + c["pad"], generator=gen, device=dev)
        x += 9.0 * (torch.rand(T, V + c["pad"], generator=gen, device=dev) < 2e-5)
        y = torch.randint(0, V, (T,), generator=gen, device=dev)
        y = torch.where(torch.rand(T, generator=gen, device=dev) < 0.5, y, x[:, :V].argmax(dim=1))
        if c["masked"]:  # the vocabulary's end is masked out, a row has no target, and one has nothing at all
            x[:, V - V // 50:] = -math.inf
            y[T // 3] = -1
            x[T // 2] = -math.inf
        s["x"], s["target"] = x.to(t)[:, :V], y.to(torch.int32)
        s["stats"], s["entropy"], s["logprob"] = f32(T, 2), f32(T), f32(T)
        if c["kind"] == "logprob":
            s["top_logprob"] = f32(T, c["top"])
            s["top_index"] = torch.empty(T, c["top"], dtype=torch.int32, device=dev)
        else:
            s["stats"], s["entropy"] = _softmax_numbers(s["x"].float())
            s["g_logprob"] = -torch.rand(T, generator=gen, device=dev) / T
            s["g_entropy"] = -0.01 * torch.rand(T, generator=gen, device=dev) / T
            s["dx"] = torch.empty(T, V, dtype=t, device=dev)
    if own:
        import paper_2208_05631_amd as qa

        s["type"] = dict(f32=qa.QA_F32, bf16=qa.QA_BF16, f16=qa.QA_F16)[c["type"]]
        need = 0
        if "K" in c:
            s["layout"] = qa.CodedRows.make(c["T"], c["K"], c["group"])
            if c["kind"] == "norm_grad":
                need = qa.qa_rows_workspace_bytes(s["layout"], qa.QA_OP_NORM_GRAD, s["type"], 0)
            if c["kind"] == "weight_grad":
                need = qa.qa_rows_workspace_bytes(s["layout"], qa.QA_OP_WEIGHT_GRAD, s["type"], c["N"])
        elif c["kind"] == "logprob":
            need = qa.qa_token_workspace_bytes(c["T"], c["V"], c["top"])
        s["ws"] = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    return s


# ---- one pass ----------------------------------------------------------------------------------------------


def run(state):
    s, c = state, state["c"]
    if own:
        return _call(s, c)
    t = TYPES[c["type"]]
    if c["kind"] == "norm":
        h = s["x"].float()
        if c["residual"]:
            h = h + s["residual"].float()
        rstd = torch.rsqrt((h * h).mean(dim=1) + EPS)
        y = h * rstd.unsqueeze(1) * s["weight"]
        return dict(h=h.to(t), y=values_of(y, c["group"]).to(torch.bfloat16), rstd=rstd)
    if c["kind"] == "checkpoint":
        return dict(y=values_of(s["x"].float(), c["group"]).to(torch.bfloat16))
    if c["kind"] == "norm_grad":
        h = _decode(s["codes"][:, :c["K"]], s["scales"], c["group"], c["K"]) if c["coded"] else s["x"].float()
        dy = s["dy"].float()
        r = s["rstd"].unsqueeze(1)
        n, g = h * r, dy * s["weight"]
        dx = r * (g - n * (g * n).mean(dim=1, keepdim=True))
        if c["residual"]:
            dx = dx + s["dh"].float()
        return dict(dx=dx.to(t), dweight=(dy * n).sum(dim=0))
    if c["kind"] == "weight_grad":
        x = _decode(s["codes"][:, :c["K"]], s["scales"], c["group"], c["K"])
        return dict(dw=s["dy"].float().t().contiguous() @ x)
    x, y = s["x"].float(), s["target"].long()
    has = y >= 0
    at = y.clamp(min=0).unsqueeze(1)
    if c["kind"] == "logprob":
        stats, entropy = _softmax_numbers(x)
        lp = _logp(x.gather(1, at), stats).squeeze(1)
        top, index = _top(x, c["top"])
        return dict(logprob=torch.where(has, lp, torch.zeros_like(lp)), entropy=entropy, stats=stats,
                    top_logprob=_logp(top, stats), top_index=index)
    lp = _logp(x, s["stats"])
    p = torch.exp(lp)
    a = torch.where(has, s["g_logprob"], torch.zeros_like(s["g_logprob"])).unsqueeze(1)
    lp = torch.where(p > 0, lp, torch.zeros_like(lp)) + s["entropy"].unsqueeze(1)
    dx = -p * (a + s["g_entropy"].unsqueeze(1) * lp)
    return dict(dx=dx.scatter_add_(1, at, a).to(t))


def _softmax_numbers(x):
    """Largest logit and logarithm of the sum of exponentials relative to it, and entropy, per row; -inf, 0 and 0 for a
    row of -inf."""
    m = x.amax(dim=1, keepdim=True)
    d = x - torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(d)
    z = e.sum(dim=1)
    w = (e * torch.where(e > 0, d, torch.zeros_like(d))).sum(dim=1)
    empty = m.squeeze(1) == -math.inf
    zero = torch.zeros_like(z)
    log_sum = torch.where(empty, zero, torch.log(z))
    return torch.stack((m.squeeze(1), log_sum), dim=1), torch.where(empty, zero, log_sum - w / z)


def _logp(x, stats):
    """Logarithms of probabilities; -inf in a row of -inf."""
    m, log_sum = stats[:, :1], stats[:, 1:]
    return torch.where(m == -math.inf, torch.full_like(x, -math.inf), (x - m) - log_sum)


def _top(x, k):
    """The k largest values per row and where they are; of equal ones the lowest index first."""
    bits = x.contiguous().view(torch.int32)
    bits = torch.where(bits == -0x80000000, torch.zeros_like(bits), bits)     # -0 equals 0
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32
    order += (1 << 31) - 1 - torch.arange(x.shape[1], device=x.device)
    index = (1 << 31) - 1 - (torch.topk(order, k, dim=1).values & 0xFFFFFFFF)
    return x.gather(1, index), index.to(torch.int32)


def _call(s, c):
    import paper_2208_05631_amd as qa

    L, t, ws = s["layout"], s["type"], s["ws"]
    if c["kind"] == "norm":
        x, r, h, y = s["x"], s["residual"], s["h"], s["y"]
        qa.qa_rms_norm(L, t, x, x.stride(0), r, 0 if r is None else r.stride(0), s["weight"], EPS, h, h.stride(0),
                       s["codes"], s["scales"], y, y.stride(0), s["rstd"])
        return dict(h=h, y=y, rstd=s["rstd"])
    if c["kind"] == "checkpoint":
        qa.qa_rows_pack(L, t, s["x"], s["x"].stride(0), s["codes"], s["scales"])
        qa.qa_rows_unpack(L, s["codes"], s["scales"], qa.QA_BF16, s["y"], s["y"].stride(0))
        return dict(y=s["y"])
    if c["kind"] == "norm_grad":
        h, dh, coded = s["x"], s["dh"], c["coded"]
        qa.qa_rms_norm_grad(L, t, s["dy"], s["dy"].stride(0), None if coded else h, h.stride(0),
                            s["codes"] if coded else None, s["scales"] if coded else None, s["weight"], s["rstd"],
                            dh, 0 if dh is None else dh.stride(0), s["dx"], s["dx"].stride(0), s["dweight"], 0, ws)
        return dict(dx=s["dx"], dweight=s["dweight"])
    if c["kind"] == "weight_grad":
        qa.qa_rows_weight_grad(L, s["codes"], s["scales"], t, s["dy"], s["dy"].stride(0), c["N"], s["dw"],
                               s["dw"].stride(0), 0, ws)
        return dict(dw=s["dw"])
    x = s["x"]
    if c["kind"] == "logprob":
        qa.qa_token_logprob(t, c["T"], c["V"], x, x.stride(0), s["target"], c["top"], s["logprob"], s["entropy"],
                            s["stats"], s["top_logprob"] if c["top"] else None, s["top_index"] if c["top"] else None, ws)
        return {k: s[k] for k in ("logprob", "entropy", "stats", "top_logprob", "top_index")}
    qa.qa_token_logprob_grad(t, c["T"], c["V"], x, x.stride(0), s["target"], s["stats"], s["entropy"], s["g_logprob"],
                             s["g_entropy"], s["dx"], s["dx"].stride(0))
    return dict(dx=s["dx"])


# ---- the definitions in 64 bits ------------------------------------------------------------------------------


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    c = s["c"]

    def expand(scales, K):
        b = scales.double()
        s = torch.where(b == 255, torch.full_like(b, math.nan), torch.exp2(b - 127))
        return s.unsqueeze(2).expand(-1, -1, c["group"]).reshape(s.shape[0], -1)[:, :K]

    def coded(v):
        """The values of v's codes, group by group."""
        out = torch.empty_like(v)
        for k in range(0, v.shape[1], c["group"]):
            part = v[:, k:k + c["group"]]
            mantissa, exponent = torch.frexp(part.abs().amax(dim=1, keepdim=True))      # in [0.5, 1) times 2^exponent
            step = torch.exp2((exponent - 7 + (mantissa > 127 / 128).int()).double().clamp(min=-126))
            out[:, k:k + c["group"]] = torch.round(part / step) * step
        return out

    if c["kind"] == "norm":
        h = s["x"].double() + (s["residual"].double() if c["residual"] else 0.0)
        rstd = (h.pow(2).sum(dim=1) / c["K"] + EPS).pow(-0.5)
        return dict(h=h, y=coded(h * rstd[:, None] * s["weight"].double()), rstd=rstd)
    if c["kind"] == "checkpoint":
        return dict(y=coded(s["x"].double()))
    if c["kind"] == "norm_grad":
        h = s["codes"][:, :c["K"]].double() * expand(s["scales"], c["K"]) if c["coded"] else s["x"].double()
        n, dy = h * s["rstd"].double()[:, None], s["dy"].double()
        g = dy * s["weight"].double()
        dx = s["rstd"].double()[:, None] * (g - n * ((g * n).sum(dim=1, keepdim=True) / c["K"]))
        return dict(dx=dx + s["dh"].double() if c["residual"] else dx, dweight=torch.sum(dy * n, dim=0))
    if c["kind"] == "weight_grad":
        x = s["codes"][:, :c["K"]].double() * expand(s["scales"], c["K"])
        return dict(dw=torch.mm(s["dy"].double().t().contiguous(), x))
    T, V = c["T"], c["V"]
    got = []
    step = max(1, (1 << 26) // V)
    for i in range(0, T, step):                 # some rows at a time: 64 bits of everything take much memory
        x, y = s["x"][i:i + step].double(), s["target"][i:i + step].long()
        lse = torch.logsumexp(x, dim=1)
        logp = torch.where(torch.isinf(lse)[:, None], torch.full_like(x, -math.inf), x - lse[:, None])
        p = logp.exp()
        if c["kind"] == "logprob":
            given = logp.gather(1, y.clamp(min=0)[:, None])[:, 0]
            entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(dim=1)
            most = x.max(dim=1).values
            got.append((torch.where(y < 0, torch.zeros_like(given), given), entropy,
                        torch.stack((most, torch.where(torch.isinf(lse), torch.zeros_like(lse), lse - most)), dim=1),
                        logp.topk(c["top"], dim=1).values))
        else:
            a = torch.where(y < 0, torch.zeros_like(lse), s["g_logprob"][i:i + step].double())[:, None]
            e = s["g_entropy"][i:i + step].double()[:, None]
            entropy = s["entropy"][i:i + step].double()[:, None]
            dx = -a * p - e * torch.where(p > 0, p * (logp + entropy), torch.zeros_like(p))
            dx[torch.arange(dx.shape[0], device=dx.device), y.clamp(min=0)] += a[:, 0]
            got.append((dx,))
    got = [torch.cat(v) for v in zip(*got)]
    if c["kind"] == "logprob_grad":
        return dict(dx=got[0])
    return dict(logprob=got[0], entropy=got[1], stats=got[2], top_logprob=got[3], top_index=None)
