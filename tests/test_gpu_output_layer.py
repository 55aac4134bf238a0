"""Log probabilities under an output layer and their gradient against the formulas in 64 bits.

Tolerances.  u = 2^-24.  A logit of 16-bit operands is a sum of exact products in binary32, k taken sixteen at a time: at most (K / 16 + 16)
roundings of partial sums, each at most u sum|x w|.  Binary32 operands are two parts of 22 bits and a sign: 2^-23 of each factor,
2^-22 for the product of the two small parts that is left out, and three times the sums.  So a logit is off by at most
    dz = ((P K / 16 + 16) u + (P == 3) 2^-21) max_v sum|x w|          (P: products, 1 or 3),
log p by 2 dz and the statistics' own errors (SUM as in the other operators' tests), the entropy by dz sum p |log p + H| <= dz (2 H + 2)."""
import math
import zlib

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")

F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
U = 2.0 ** -24
SUM = 64 * U


def code_of(t):
    return {"f32": qa.QA_F32, "bf16": qa.QA_BF16, "f16": qa.QA_F16}[t]


def gen_of(*what):
    return torch.Generator().manual_seed(zlib.crc32(repr(what).encode()))


def inside(v, t, pad=0, lead=0):
    """v rounded to the type, and on the device as rows of a wider buffer of NaN that begins `lead` elements after an aligned place."""
    v = v.to(TYPES[t])
    T, K = v.shape
    flat = torch.full((lead + T * (K + pad) + 8,), math.nan, dtype=TYPES[t])
    flat[lead:lead + T * (K + pad)].view(T, K + pad)[:, :K] = v
    return v.to(F64), flat.to(DEV)[lead:lead + T * (K + pad)].view(T, K + pad)[:, :K]


def layer_of(gen, T, V, H, t, pad=0, lead=0, scale=2.0):
    w = torch.randn(V, H, generator=gen) * (scale / math.sqrt(H))
    y = torch.randint(0, V, (T,), generator=gen)
    x = torch.randn(T, H, generator=gen) + 1.5 * (torch.rand(T, 1, generator=gen) < 0.5) * w[y] / scale
    x64, xd = inside(x, t, pad, lead)
    w64, wd = inside(w, t, pad, lead)
    return qa.OutputLayer.make(T, V, H, H + pad, H + pad), x64, xd, w64, wd, y


def room(layer, op, t):
    """Filled with NaN: nothing that a call reads there may be older than the call."""
    return torch.full((qa.qa_output_workspace_bytes(layer, op, code_of(t)) // 4,), math.nan, device=DEV)


def dz_of(x, w, t):
    P = 3 if t == "f32" else 1
    most = (x.abs() @ w.abs().t()).amax(dim=1)
    return ((P * x.shape[1] / 16 + 16) * U + (2.0 ** -21 if P == 3 else 0.0)) * most


def score(layer, xd, wd, y, t):
    T = layer.rows
    lp, h, st = (torch.full(s, 5.0, device=DEV) for s in ((T + 1,), (T + 1,), (T + 1, 2)))
    qa.qa_output_logprob(layer, code_of(t), xd, wd, y.to(torch.int32).to(DEV), lp, h, st, room(layer, qa.QA_OP_LOGPROB, t))
    assert (lp[T:] == 5.0).all() and (h[T:] == 5.0).all() and (st[T:] == 5.0).all()
    return lp[:T].cpu().to(F64), h[:T].cpu().to(F64), st[:T].cpu().to(F64)


def check_score(t, x, w, y, got):
    z, lp, h, st = ref.score(x, w, y)
    dz = dz_of(x, w, t)
    assert ((got[2][:, 0] - st[:, 0]).abs() <= dz + U * st[:, 0].abs()).all()
    assert ((got[2][:, 1] - st[:, 1]).abs() <= 2 * dz + SUM * (1 + st[:, 1])).all()
    assert ((got[0] - lp).abs() <= 2 * dz + SUM * (1 + lp.abs())).all()
    assert ((got[1] - h).abs() <= dz * (2 * h + 2) + SUM * (1 + 4 * st[:, 1])).all()


SHAPES = [(1, 1, 1, 0), (1, 1000, 64, 0), (1, 333, 100, 0), (3, 129, 32, 0), (16, 64, 96, 8), (17, 257, 33, 0), (64, 500, 128, 0), (65, 511, 160, 0),
          (100, 65, 257, 1), (130, 1030, 64, 8), (300, 700, 72, 0), (1, 70000, 32, 0), (513, 130, 515, 3), (48, 4097, 320, 0)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,H,pad", SHAPES)
def test_logprob(t, T, V, H, pad):
    gen = gen_of(t, T, V, H)
    layer, x, xd, w, wd, y = layer_of(gen, T, V, H, t, pad)
    y[T // 2] = -1 if T > 2 else y[T // 2]
    check_score(t, x, w, y, score(layer, xd, wd, y, t))


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_logprob_in_large_tiles(t):
    """Enough tiles for those of 256 x 256, ends inside a tile on both sides."""
    gen = gen_of("large", t)
    layer, x, xd, w, wd, y = layer_of(gen, 2101, 6101, 64, t)
    check_score(t, x, w, y, score(layer, xd, wd, y, t))


def check_grad(t, T, V, H, pad=0, lead=0, entropy=False, ignored=0.0, wants="xw", accumulate=False, seed=0, kept=None):
    gen = gen_of(t, T, V, H, entropy, ignored, seed)
    layer, x, xd, w, wd, y = layer_of(gen, T, V, H, t, pad, lead)
    if ignored:
        y = torch.where(torch.rand(T, generator=gen) < ignored, torch.full_like(y, -1), y)
    z, _, h, st = ref.score(x, w, y)
    st32, h32 = st.float(), h.float()
    a = -torch.rand(T, generator=gen) - 0.5
    e = 0.3 * torch.randn(T, generator=gen) if entropy else None
    if kept is not None:
        skip = torch.ones(T, dtype=torch.bool)
        skip[kept] = False
        a[skip] = 0.0
        xd[skip.to(DEV)] = math.nan
    dx = torch.full((T, H + 1), 5.0, dtype=TYPES[t], device=DEV) if "x" in wants else None
    dw = torch.full((V, H + 2), 3.0, device=DEV) if "w" in wants else None
    qa.qa_output_logprob_grad(layer, code_of(t), xd, wd, y.to(torch.int32).to(DEV), st32.to(DEV), h32.to(DEV) if entropy else None, a.to(DEV),
                              e.to(DEV) if entropy else None, dx, H + 1, dw, H + 2, int(accumulate), room(layer, qa.QA_OP_LOGPROB_GRAD, t))
    c, none = ref.logits_grad(z, y, st32.to(F64), h32.to(F64), a.to(F64), e.to(F64) if entropy else None)
    # c: log p is off by dz and the roundings of z, m and log_sum; p relatively by as much and the exponential's 2^-21
    lp = z - st32.to(F64)[:, :1] - st32.to(F64)[:, 1:]
    off = dz_of(x, w, t)[:, None] + 8 * U * (z.abs() + st[:, :1].abs() + st[:, 1:]) + 2.0 ** -21
    size = a.abs().to(F64)[:, None] * torch.exp(lp) * off
    if entropy:
        size = size + e.abs().to(F64)[:, None] * torch.exp(lp) * (lp.abs() + h[:, None] + 1) * off
    size = torch.where(none[:, None], torch.zeros_like(c), size + 4 * U * c.abs())
    most = float((a.abs() + (18 * e.abs() if entropy else 0)).max())
    part = 2.0 ** -11 if t != "f32" else 2.0 ** -21               # of c, and of w where it has two parts
    small = 2.0 ** -38 * most                                     # what binary16 has no bits for, of the scaled c
    sums = (3 * max(T, V) / 16 + 64) * U
    if dx is not None:
        assert (dx[:, H:] == 5.0).all()
        want = c @ w
        tol = (size + (part + sums) * c.abs() + small) @ w.abs() + HALF_ULP[t] * 1.01 * want.abs() + (2.0 ** -24 if t == "f16" else 0.0)
        got = dx[:, :H].cpu().to(F64)
        assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())
        assert (got[none] == 0).all()
    if dw is not None:
        assert (dw[:, H:] == 3.0).all()
        want = c.t() @ x + (3.0 if accumulate else 0.0)
        tol = (size + (2.0 ** -21 + sums) * c.abs() + small).t() @ x.abs() + 2 * U * want.abs()
        got = dw[:, :H].cpu().to(F64)
        assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,H,pad", SHAPES)
@pytest.mark.parametrize("entropy", [False, True])
def test_grad(t, T, V, H, pad, entropy):
    check_grad(t, T, V, H, pad, entropy=entropy, ignored=0.3 if T > 2 else 0.0)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("wants", ["x", "w"])
def test_grad_of_one_side(t, wants):
    check_grad(t, 77, 301, 96, wants=wants, accumulate=wants == "w", entropy=True)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_grad_accumulates_and_begins_anywhere(t):
    check_grad(t, 70, 200, 96, lead=1, accumulate=True)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_grad_in_large_tiles(t):
    check_grad(t, 2101, 6101, 64, ignored=0.1)


def test_rows_of_padding_hold_anything():
    """Rows without target and without weight: NaN and infinities in x, statistics of NaN; every other number is as without them."""
    gen = gen_of("padding")
    T, V, H = 200, 600, 96
    layer, x, xd, w, wd, y = layer_of(gen, T, V, H, "bf16")
    st, h = (v.float().to(DEV) for v in ref.score(x, w, y)[3:1:-1])
    a, e = torch.rand(T, device=DEV), torch.rand(T, device=DEV)
    none = torch.arange(T) % 3 == 0
    y[none], e[none.to(DEV)] = -1, 0.0
    got = []
    for junk in (0.0, math.nan, math.inf, 3e38):
        xj, stj = xd.clone(), st.clone()
        xj[none.to(DEV)] = junk
        stj[none.to(DEV)] = math.nan if junk else 0.0
        dx, dw = torch.full((T, H), 5.0, dtype=torch.bfloat16, device=DEV), torch.full((V, H), 5.0, device=DEV)
        qa.qa_output_logprob_grad(layer, qa.QA_BF16, xj, wd, y.to(torch.int32).to(DEV), stj, h, a, e, dx, H, dw, H, 0, room(layer, qa.QA_OP_LOGPROB_GRAD, "bf16"))
        assert (dx[none.to(DEV)] == 0).all()
        got.append((dx, dw))
    assert bool(torch.isfinite(got[0][1]).all())
    for dx, dw in got[1:]:
        assert torch.equal(dx, got[0][0]) and torch.equal(dw, got[0][1])


def test_a_row_that_is_not_finite_spoils_its_own_numbers_alone():
    gen = gen_of("nan")
    layer, x, xd, w, wd, y = layer_of(gen, 70, 300, 64, "bf16")
    clean = score(layer, xd, wd, y, "bf16")
    for bad in (math.nan, math.inf):
        xb = xd.clone()
        xb[33, 5] = bad
        lp, h, st = score(layer, xb, wd, y, "bf16")
        others = torch.arange(70) != 33
        assert math.isnan(float(lp[33])) and math.isnan(float(h[33])) and math.isnan(float(st[33, 1]))
        for a, b in zip((lp, h, st), clean):
            assert torch.equal(a[others], b[others])


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 60])
def test_binary32_of_any_size(scale):
    """x small by as much as w is large: the logits are the same to the bit, as scales are powers of two."""
    gen = gen_of("sizes")
    layer, x, xd, w, wd, y = layer_of(gen, 40, 200, 50, "f32")
    a, b = score(layer, xd, wd, y, "f32"), score(layer, xd * scale, wd / scale, y, "f32")
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_targets_outside_the_vocabulary_and_outputs_left_out():
    gen = gen_of("outside")
    layer, x, xd, w, wd, y = layer_of(gen, 20, 100, 32, "f16")
    full = score(layer, xd, wd, y, "f16")
    y2 = y.clone()
    y2[3], y2[4], y2[5] = 100, -7, 2 ** 31 - 1
    lp, h, st = score(layer, xd, wd, y2, "f16")
    assert (lp[3:6] == 0).all() and torch.equal(h, full[1]) and torch.equal(st, full[2])
    only = torch.empty(20, device=DEV)
    ws = room(layer, qa.QA_OP_LOGPROB, "f16")
    qa.qa_output_logprob(layer, qa.QA_F16, xd, wd, None, None, only, None, ws)
    assert torch.equal(only.cpu().to(F64), h)
    qa.qa_output_logprob(layer, qa.QA_F16, xd, wd, y.to(torch.int32).to(DEV), only, None, None, ws)
    assert torch.equal(only.cpu().to(F64), full[0])


def test_no_rows():
    layer = qa.OutputLayer.make(0, 50, 32)
    w = torch.zeros(50, 32, device=DEV)
    dw = torch.full((50, 40), 3.0, device=DEV)
    qa.qa_output_logprob(layer, qa.QA_F32, None, w, None, None, None, None, None)
    qa.qa_output_logprob_grad(layer, qa.QA_F32, None, w, None, None, None, None, None, None, 32, dw, 40, 1, None)
    assert (dw == 3.0).all()
    qa.qa_output_logprob_grad(layer, qa.QA_F32, None, w, None, None, None, None, None, None, 32, dw, 40, 0, None)
    assert (dw[:, :32] == 0).all() and (dw[:, 32:] == 3.0).all()


def test_the_gradient_is_the_slope_of_the_loss():
    """Central differences in 64 bits of sum(a log p + e H) over single elements, step d: off by d^2 / 6 of a third derivative of the
    gradient's own order, plus the gradient's rounding (dz and parts of 2^-21, of numbers below 3)."""
    gen = gen_of("slope")
    T, V, H, d = 4, 9, 6, 1e-4
    layer, x, xd, w, wd, y = layer_of(gen, T, V, H, "f32")
    y[2] = -1
    a, e = torch.randn(T, generator=gen), 0.5 * torch.randn(T, generator=gen)
    _, _, h, st = ref.score(x, w, y)
    dx, dw = torch.empty(T, H, device=DEV), torch.empty(V, H, device=DEV)
    qa.qa_output_logprob_grad(layer, qa.QA_F32, xd, wd, y.to(torch.int32).to(DEV), st.float().to(DEV), h.float().to(DEV), a.to(DEV), e.to(DEV), dx, H, dw, H, 0,
                              room(layer, qa.QA_OP_LOGPROB_GRAD, "f32"))

    def loss(x, w):
        _, lp, h, _ = ref.score(x, w, y)
        return float((a.to(F64) * lp + e.to(F64) * h).sum())
    for v, got in ((x, dx), (w, dw)):
        for i in range(v.numel()):
            keep = float(v.view(-1)[i])
            v.view(-1)[i] = keep + d
            up = loss(x, w)
            v.view(-1)[i] = keep - d
            down = loss(x, w)
            v.view(-1)[i] = keep
            assert abs((up - down) / (2 * d) - float(got.view(-1)[i])) < 3e-5


# ---- calls as programs make them ------------------------------------------------------------------------------------------------


def buffers(T, V, H, t):
    return dict(lp=torch.empty(T, device=DEV), h=torch.empty(T, device=DEV), st=torch.empty(T, 2, device=DEV), dx=torch.empty(T, H, dtype=TYPES[t], device=DEV),
                dw=torch.empty(V, H, device=DEV))


def forward_and_back(layer, t, x, w, y, a, b, ws, ws2, stream=None):
    c, H = code_of(t), layer.features
    qa.qa_output_logprob(layer, c, x, w, y, b["lp"], b["h"], b["st"], ws, stream)
    qa.qa_output_logprob_grad(layer, c, x, w, y, b["st"], b["h"], a, a, b["dx"], H, b["dw"], H, 0, ws2, stream)


@pytest.mark.parametrize("t,T,V,H", [("bf16", 40, 3000, 96), ("f16", 300, 2500, 128), ("f32", 70, 900, 50)])
def test_captured_and_replayed_among_eager_calls(t, T, V, H):
    """Replays give what eager calls give, bit for bit, with eager calls of the same buffers and other inputs between them; two graphs
    share a workspace, one after the other."""
    gen = gen_of("graph", t)
    layer, _, xd, _, wd, y = layer_of(gen, T, V, H, t)
    y, a = y.to(torch.int32).to(DEV), torch.randn(T, generator=gen).to(DEV)
    ws, ws2 = room(layer, qa.QA_OP_LOGPROB, t), room(layer, qa.QA_OP_LOGPROB_GRAD, t)
    x, b = xd.clone(), buffers(T, V, H, t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward_and_back(layer, t, x, wd, y, a, b, ws, ws2)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            forward_and_back(layer, t, x, wd, y, a, b, ws, ws2)
        graphs.append(g)
    for i in range(6):
        fresh = (xd * (1 + 0.1 * i)).clone()
        want = buffers(T, V, H, t)
        forward_and_back(layer, t, fresh, wd, y, a, want, ws, ws2)
        torch.cuda.synchronize()
        x.copy_(fresh)
        for v in b.values():
            v.fill_(7.0)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        for k in b:
            assert torch.equal(b[k], want[k]), (i, k)


@pytest.mark.parametrize("t,T,V,H", [("bf16", 600, 30000, 64), ("f16", 300, 2500, 128), ("f32", 270, 9000, 50)])
def test_replayed_with_other_rows_that_count(t, T, V, H):
    """A graph that was captured where all rows count, replayed where some do, one or none, and where all do again; and each twice, bit for bit."""
    gen = gen_of("replayed rows", t)
    layer, _, xd, _, wd, y = layer_of(gen, T, V, H, t)
    y, a, b = y.to(torch.int32).to(DEV), torch.ones(T, device=DEV), buffers(T, V, H, t)
    ws = room(layer, qa.QA_OP_LOGPROB_GRAD, t)
    qa.qa_output_logprob(layer, code_of(t), xd, wd, y, b["lp"], b["h"], b["st"], room(layer, qa.QA_OP_LOGPROB, t))
    call = lambda to: qa.qa_output_logprob_grad(layer, code_of(t), xd, wd, y, b["st"], None, a, None, to["dx"], H, to["dw"], H, 0, ws)  # noqa: E731
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        call(b)
    for kept in (range(0), range(7, 8), range(0, T, 3), range(T // 2, T), range(T), range(100, 130)):
        weights = torch.zeros(T)
        weights[list(kept)] = torch.randn(len(kept), generator=gen)
        for _ in range(2):
            a.copy_(weights)
            want = buffers(T, V, H, t)
            call(want)
            torch.cuda.synchronize()
            b["dx"].fill_(7.0), b["dw"].fill_(7.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(b["dx"], want["dx"]) and torch.equal(b["dw"], want["dw"])
            skip = weights == 0
            assert bool((b["dx"].cpu()[skip] == 0).all())
            if not len(kept):
                assert bool((b["dw"] == 0).all())


def test_on_another_stream():
    gen = gen_of("stream")
    T, V, H, t = 130, 4000, 64, "bf16"
    layer, _, xd, _, wd, y = layer_of(gen, T, V, H, t)
    y, a = y.to(torch.int32).to(DEV), torch.randn(T, generator=gen).to(DEV)
    want, got = buffers(T, V, H, t), buffers(T, V, H, t)
    forward_and_back(layer, t, xd, wd, y, a, want, room(layer, qa.QA_OP_LOGPROB, t), room(layer, qa.QA_OP_LOGPROB_GRAD, t))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = [(buffers(T, V, H, t), room(layer, qa.QA_OP_LOGPROB, t), room(layer, qa.QA_OP_LOGPROB_GRAD, t)) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):                                            # two calls at once, each with its own workspace
        for s, (b, ws, ws2) in zip(streams, both):
            forward_and_back(layer, t, xd, wd, y, a, b, ws, ws2, s)
    torch.cuda.synchronize()
    for b, _, _ in both:
        assert all(torch.equal(b[k], want[k]) for k in want)
    del got


@pytest.mark.parametrize("t,T", [("bf16", 20), ("bf16", 100), ("f32", 3)])
def test_offsets_beyond_32_bits(t, T):
    """Rows of w 150000 and more elements apart, 20000 of them: offsets of 6 GB and more, strides that are read in place and ones that are not."""
    gen = gen_of("far", t)
    V, H = 20000, 64
    for stride in (150000, 150001):
        wide = torch.zeros(V, stride, dtype=TYPES[t], device=DEV)
        wide[:, :H] = (torch.randn(V, H, generator=gen) / 4).to(TYPES[t]).to(DEV)
        w = wide[:, :H]
        x = torch.randn(T, H, generator=gen).to(TYPES[t]).to(DEV)
        y = torch.randint(0, V, (T,), generator=gen)
        y[0] = V - 1
        layer = qa.OutputLayer.make(T, V, H, H, stride)
        check_score(t, x.cpu().to(F64), w.cpu().to(F64), y, score(layer, x, w, y, t))
        del wide, w
        torch.cuda.empty_cache()


def test_dw_of_far_rows():
    """dw rows a few hundred thousand elements apart, past 2^31 elements."""
    gen = gen_of("far dw")
    T, V, H, stride = 33, 9000, 48, 250000
    layer, x, xd, w, wd, y = layer_of(gen, T, V, H, "bf16")
    _, _, h, st = ref.score(x, w, y)
    a = torch.rand(T, generator=gen) + 0.5
    dw, near = torch.zeros(V, stride, device=DEV), torch.empty(V, H, device=DEV)
    ws = room(layer, qa.QA_OP_LOGPROB_GRAD, "bf16")
    for to, s in ((dw, stride), (near, H)):
        qa.qa_output_logprob_grad(layer, qa.QA_BF16, xd, wd, y.to(torch.int32).to(DEV), st.float().to(DEV), None, a.to(DEV), None, None, H, to, s, 0, ws)
    assert torch.equal(dw[:, :H], near) and bool((dw[:, H:H + 100] == 0).all())


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,V,H", [(700, 300, 64), (700, 300, 50), (5000, 200, 32), (700, 20011, 40)])
@pytest.mark.parametrize("kept", [(), (699,), (0, 1, 255, 256, 257, 511, 512), range(100, 116), range(37, 163), range(300, 700)])
def test_few_of_many_rows_count(t, T, V, H, kept):
    """The others' dx is 0, whatever x holds there.  None, one, up to a whole step of 16 and more, within one share of the rows and in several."""
    check_grad(t, T, V, H, accumulate=True, kept=list(kept))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_pieces_of_the_rows(t):
    """So many rows that they are scored in pieces."""
    T, V, H = 260000, 50001, 32
    gen = torch.Generator(device=DEV).manual_seed(4)
    w = (torch.randn(V, H, generator=gen, device=DEV) * (2 / math.sqrt(H))).to(TYPES[t])
    x = torch.randn(T, H, generator=gen, device=DEV).to(TYPES[t])
    y = torch.randint(0, V, (T,), generator=gen, device=DEV)
    layer = qa.OutputLayer.make(T, V, H)
    assert 4 * 3 * (V // 128) * T > qa.qa_output_workspace_bytes(layer, qa.QA_OP_LOGPROB, code_of(t))       # less than all chunks' numbers
    b = buffers(T, V, H, t)
    qa.qa_output_logprob(layer, code_of(t), x, w, y.to(torch.int32), b["lp"], b["h"], b["st"], room(layer, qa.QA_OP_LOGPROB, t))
    for rows in (slice(0, 500), slice(100000, 240000, 173), slice(T - 300, T)):
        check_score(t, x[rows].to(F64), w.to(F64), y[rows], [b[n][rows].to(F64) for n in ("lp", "h", "st")])


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_pieces_of_the_vocabulary(t):
    """So many rows that the vocabulary is taken in pieces: the sums of dx go on from piece to piece."""
    T, V, H = (20000, 20011, 32) if t == "bf16" else (9000, 20011, 20)
    gen = torch.Generator(device=DEV).manual_seed(3)
    w = (torch.randn(V, H, generator=gen, device=DEV) * (2 / math.sqrt(H))).to(TYPES[t])
    x = torch.randn(T, H, generator=gen, device=DEV).to(TYPES[t])
    y = torch.randint(0, V, (T,), generator=gen, device=DEV)
    layer = qa.OutputLayer.make(T, V, H)
    b = buffers(T, V, H, t)
    qa.qa_output_logprob(layer, code_of(t), x, w, y.to(torch.int32), b["lp"], b["h"], b["st"], room(layer, qa.QA_OP_LOGPROB, t))
    a = -torch.rand(T, generator=gen, device=DEV) - 0.5
    qa.qa_output_logprob_grad(layer, code_of(t), x, w, y.to(torch.int32), b["st"], None, a, None, b["dx"], H, b["dw"], H, 0, room(layer, qa.QA_OP_LOGPROB_GRAD, t))
    x64, w64, dx, dw, sizes = x.to(F64), w.to(F64), [], torch.zeros(V, H, dtype=F64, device=DEV), torch.zeros(V, H, dtype=F64, device=DEV)
    off_x = []
    for i in range(0, T, 2000):
        z, lp, h, st = ref.score(x64[i:i + 2000], w64, y[i:i + 2000])
        dz = dz_of(x64[i:i + 2000], w64, t)
        assert ((b["lp"][i:i + 2000] - lp).abs() <= 2 * dz + SUM * (1 + lp.abs())).all()
        c, _ = ref.logits_grad(z, y[i:i + 2000], b["st"][i:i + 2000].to(F64), None, a[i:i + 2000].to(F64), None)
        off = c.abs() * (dz[:, None] + 8 * U * (z.abs() + 30) + 2.0 ** -21 + (3 * T / 16 + 64) * U)
        dx.append(c @ w64)
        off_x.append((off + c.abs() * (2.0 ** -11 if t != "f32" else 2.0 ** -21) + 2.0 ** -38 * 1.5) @ w64.abs())
        dw += c.t() @ x64[i:i + 2000]
        sizes += (off + c.abs() * 2.0 ** -21 + 2.0 ** -38 * 1.5).t() @ x64[i:i + 2000].abs()
    dx, off_x = torch.cat(dx), torch.cat(off_x)
    assert ((b["dx"].to(F64) - dx).abs() <= off_x + 1.01 * HALF_ULP[t] * dx.abs()).all()
    assert ((b["dw"].to(F64) - dw).abs() <= sizes + 2 * U * dw.abs()).all()
