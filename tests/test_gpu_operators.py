"""The operators on activations and logits against the formulas in 64 bits.

Tolerances.  u = 2^-24 is binary32's rounding, v half an ulp of the output type (2^-24, 2^-8, 2^-11 relative at most).  A sum of n
terms in binary32, whatever its order, is off by at most n u sum|terms|; the kernels add in trees and in runs of at most
some hundred terms, so SUM = 64 u = 4e-6 of sum|terms| is a generous bound at every size here.  exp2 and log2 of the
hardware are good to about 2^-22 relative; a logit difference d enters with |d| 2u more."""
import math
import zlib

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    DEV = torch.device("cuda:0")

F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SUM = 64 * 2.0 ** -24


def code_of(t):
    return {"f32": qa.QA_F32, "bf16": qa.QA_BF16, "f16": qa.QA_F16}[t]


def rows_of(gen, T, K, t, pad=0, scale=1.0, lead=0):
    """Rows inside a wider buffer that begins `lead` elements after an aligned place; what is around them is NaN."""
    flat = torch.full((lead + T * (K + pad) + 8,), math.nan, dtype=TYPES[t])
    v = flat[lead:lead + T * (K + pad)].view(T, K + pad)[:, :K] if T else flat[:0].view(0, K)
    if T:
        v.copy_((torch.randn(T, K, generator=gen) * scale).to(TYPES[t]))
    d = flat.to(DEV)
    return v, d[lead:lead + T * (K + pad)].view(T, K + pad)[:, :K] if T else d[:0].view(0, K)


def coded_rows(T, K, group, fill=77):
    L = qa.CodedRows.make(T, K, group)
    codes = torch.full((max(T, 1), L.code_stride), fill, dtype=torch.int8, device=DEV)
    scales = torch.full((max(T, 1), L.scale_stride + 3), fill, dtype=torch.uint8, device=DEV)
    L.scale_stride += 3
    return L, codes, scales


def unpack(L, codes, scales, t):
    out = torch.full((L.rows, L.cols + 1), 5.0, dtype=TYPES[t], device=DEV)
    qa.qa_rows_unpack(L, codes, scales, code_of(t), out, L.cols + 1)
    assert (out[:, L.cols] == 5.0).all()
    return out[:, :L.cols].cpu()


def gen_of(*what):
    g = torch.Generator()
    g.manual_seed(zlib.crc32(repr(what).encode()))
    return g


# ---- rows in 8 bits ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,K,group,pad,lead", [(1, 1, 32, 0, 0), (3, 31, 32, 0, 1), (5, 96, 32, 1, 0), (7, 257, 64, 0, 3),
                                                (33, 2048, 128, 0, 0), (2, 16385, 64, 7, 0), (300, 100, 128, 4, 2)])
def test_pack_is_the_definition_and_unpack_its_inverse(t, T, K, group, pad, lead):
    gen = gen_of(t, T, K, group)
    x, xd = rows_of(gen, T, K, t, pad, 3.0, lead)
    L, codes, scales = coded_rows(T, K, group)
    qa.qa_rows_pack(L, code_of(t), xd, K + pad, codes, scales)
    want_s = ref.scale_bytes(x.to(F64), group)
    want = ref.code(x.to(F64), want_s, group)
    G = want_s.shape[1]
    assert torch.equal(scales[:, :G].cpu().long(), want_s) and (scales[:, G:] == 77).all()
    assert torch.equal(codes[:, :K].cpu().long(), want) and (codes[:, K:] == 77).all()
    values = ref.decode(want, want_s, group)
    for to in ("bf16", "f32"):
        assert torch.equal(unpack(L, codes, scales, to).to(F64), values)         # exact in either
    assert torch.equal(unpack(L, codes, scales, "f16"), values.to(torch.float16))


def test_groups_at_the_edges_of_the_code():
    """Groups of zeros, of the smallest and the largest numbers, on either side of a scale, with an infinity, with a NaN."""
    big = torch.finfo(torch.float32).max
    just = 127 * 2.0 ** -10
    firsts = [0.0, -0.0, 1e-45, 2.0 ** -126, 2.0 ** -120 * 127, just, torch.nextafter(torch.tensor(just), torch.tensor(1.0)).item(),
              -just, 1.0, 127.0, 127.5, 128.0, big, -big, math.inf, -math.inf, math.nan, 0.5, 2.5 / 64]
    x = torch.zeros(len(firsts), 64)
    x[:, 5] = torch.tensor(firsts)
    x[:, 6] = 0.4999 * x[:, 5]
    x[:, 40] = 1.0                                   # the second group is untouched by the first
    L, codes, scales = coded_rows(len(firsts), 64, 32)
    qa.qa_rows_pack(L, qa.QA_F32, x.to(DEV), 64, codes, scales)
    want_s = ref.scale_bytes(x.to(F64), 32)
    assert torch.equal(scales[:, :2].cpu().long(), want_s)
    assert torch.equal(codes[:, :64].cpu().long(), ref.code(torch.nan_to_num(x.to(F64), 0, 0, 0), want_s, 32))
    got = unpack(L, codes, scales, "bf16").to(F64)
    bad = want_s[:, 0] == 255
    assert int(bad.sum()) == 3 and torch.isnan(got[bad, :32]).all() and torch.isfinite(got[~bad]).all()
    assert (got[:, 40] == 1.0).all()


# ---- norm ------------------------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 1, 32, 0), (1, 8192, 128, 0), (3, 33, 32, 1), (9, 511, 64, 0), (13, 1024, 32, 8), (5, 1025, 32, 0), (7, 2048, 64, 0),
               (4, 4095, 128, 3), (3, 5003, 32, 0), (2, 16384, 64, 0), (2, 20011, 32, 5), (2100, 72, 32, 0), (1100, 1280, 64, 0)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,K,group,pad", NORM_SHAPES)
@pytest.mark.parametrize("residual", [True, False])
def test_norm(t, T, K, group, pad, residual):
    gen = gen_of(t, T, K, group, residual)
    x, xd = rows_of(gen, T, K, t, pad, 2.0, 1)
    r, rd = rows_of(gen, T, K, t, pad + 1) if residual else (None, None)
    w = 1 + 0.3 * torch.randn(K, generator=gen)
    L, codes, scales = coded_rows(T, K, group)
    h = torch.full((T, K + 2), 5.0, dtype=TYPES[t], device=DEV)
    y = torch.full((T, K + 3), 5.0, dtype=torch.bfloat16, device=DEV)
    rstd = torch.empty(T, device=DEV)
    qa.qa_rms_norm(L, code_of(t), xd, K + pad, rd, K + pad + 1 if residual else 0, w.to(DEV), 1e-5, h, K + 2, codes, scales, y, K + 3, rstd)
    assert (h[:, K:] == 5.0).all() and (y[:, K:] == 5.0).all() and (codes[:, K:] == 77).all()
    h32 = x.float() + r.float() if residual else x.float()
    assert torch.equal(h[:, :K].cpu(), h32.to(TYPES[t]))                         # one rounding of the binary32 sum
    want_rstd, want = ref.norm(x.to(F64) + (r.to(F64) if residual else 0), w.to(F64), 1e-5)
    assert (rstd.cpu().to(F64) / want_rstd - 1).abs().max() < SUM
    G = -(-K // group)
    s, q = scales[:, :G].cpu().long(), codes[:, :K].cpu()
    value = ref.decode(q, s, group)
    assert torch.equal(y[:, :K].cpu().to(F64), value)
    # the scale is the one of y, or of a y that binary32's error moves over the next power of two
    near = [ref.scale_bytes(want * f, group) for f in (1 - 2 * SUM, 1 + 2 * SUM)]
    assert ((s >= near[0]) & (s <= near[1])).all()
    step = torch.exp2((s - 127).to(F64)).repeat_interleave(group, dim=1)[:, :K]
    assert ((value - want).abs() <= step / 2 + 2 * SUM * want.abs()).all()


def test_norm_in_place_and_with_outputs_left_out():
    gen = gen_of("in place")
    T, K = 37, 1000
    L, codes, scales = coded_rows(T, K, 64)
    w = torch.ones(K, device=DEV)
    for K_long in (K, 20000):
        L, codes, scales = coded_rows(T, K_long, 64)
        w = torch.ones(K_long, device=DEV)
        x, xd = rows_of(gen, T, K_long, "bf16")
        r, rd = rows_of(gen, T, K_long, "bf16")
        h = (x.float() + r.float()).to(torch.bfloat16)
        first = xd.clone()
        qa.qa_rms_norm(L, qa.QA_BF16, first, K_long, rd, K_long, w, 1e-6, first, K_long, codes, scales, None, 0, None)
        assert torch.equal(first.cpu(), h)
        second = rd.clone()
        y = torch.empty(T, K_long, dtype=torch.bfloat16, device=DEV)
        qa.qa_rms_norm(L, qa.QA_BF16, xd, K_long, second, K_long, w, 1e-6, second, K_long, None, None, y, K_long, None)
        assert torch.equal(second.cpu(), h)
        assert torch.equal(y.cpu(), unpack(L, codes, scales, "bf16"))


def test_norm_of_rows_without_size():
    """A row of zeros has y = 0 with an eps and NaN without one; an infinity makes its row NaN and no other."""
    x = torch.ones(4, 64)
    x[1], x[2, 3] = 0.0, math.inf
    for eps, zero in ((1e-6, 0.0), (0.0, math.nan)):
        L, codes, scales = coded_rows(4, 64, 32)
        y = torch.empty(4, 64, dtype=torch.bfloat16, device=DEV)
        qa.qa_rms_norm(L, qa.QA_F32, x.to(DEV), 64, None, 0, torch.ones(64, device=DEV), eps, None, 0, codes, scales, y, 64, None)
        y = y.cpu().float()
        assert (y[0] == 1.0).all() and (y[3] == 1.0).all()
        assert torch.isnan(y[1]).all() if math.isnan(zero) else (y[1] == 0).all()
        assert torch.isnan(y[2, :32]).all() and (y[2, 32:] == 0).all()        # 1 / infinity is 0, infinity times 0 is NaN


# ---- the norm's backward pass ------------------------------------------------------------------------------------


def run_norm_grad(t, T, K, group, pad, dh, coded, accumulate=False, same=None):
    gen = gen_of(t, T, K, group, dh, coded)
    dy, dyd = rows_of(gen, T, K, t, pad, 0.5, 1)
    x, xd = rows_of(gen, T, K, t, pad + 2, 2.0)
    g, gd = rows_of(gen, T, K, t, 0, 0.5) if dh else (None, None)
    w = 1 + 0.3 * torch.randn(K, generator=gen)
    L, codes, scales = coded_rows(T, K, group)
    h = x.to(F64)
    if coded:
        qa.qa_rows_pack(L, code_of(t), xd, K + pad + 2, codes, scales)
        h = ref.decode(codes[:, :K].cpu(), scales[:, :-(-K // group)].cpu(), group)
    rstd = (1 / torch.sqrt((h * h).mean(dim=1) + 1e-6)).float()
    dx = torch.full((T, K + 1), 5.0, dtype=TYPES[t], device=DEV)
    dw = torch.full((K + 1,), 2.0, device=DEV)
    ws = torch.empty(max(256, qa.qa_rows_workspace_bytes(L, qa.QA_OP_NORM_GRAD, code_of(t), 0)), dtype=torch.uint8, device=DEV)
    to, stride = (dx, K + 1) if same is None else {"dy": (dyd, K + pad), "dh": (gd, K)}[same]
    qa.qa_rms_norm_grad(L, code_of(t), dyd, K + pad, None if coded else xd, K + pad + 2, codes if coded else None,
                        scales if coded else None, w.to(DEV), rstd.to(DEV), gd, K if dh else 0, to, stride, dw, int(accumulate), ws)
    if same is None:
        assert (dx[:, K:] == 5.0).all()
    assert (dw[K:] == 2.0).all()
    dy64, w64, r64 = dy.to(F64), w.to(F64), rstd.to(F64)
    want, want_w = ref.norm_grad(dy64, h, w64, r64, g.to(F64) if dh else None)
    got = to[:, :K].cpu().to(F64)
    n = (h * r64[:, None]).abs()
    terms = r64[:, None] * ((dy64 * w64).abs() + n * (dy64 * w64 * n).abs().mean(dim=1, keepdim=True))
    if dh:
        terms = terms + g.to(F64).abs()
    tiny = 2.0 ** -24 if t == "f16" else 0.0
    assert ((got - want).abs() <= HALF_ULP[t] * want.abs() * 1.01 + SUM * terms + tiny).all()
    each = (dy64.abs() * n).sum(dim=0)
    assert ((dw[:K].cpu().to(F64) - (2.0 if accumulate else 0.0) - want_w).abs() <= SUM * each + 2.0 ** -22).all()


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,K,group,pad", NORM_SHAPES)
@pytest.mark.parametrize("dh,coded", [(True, False), (False, True)])
def test_norm_grad(t, T, K, group, pad, dh, coded):
    run_norm_grad(t, T, K, group, pad, dh, coded)


@pytest.mark.parametrize("K", [700, 4096, 20011])
def test_norm_grad_accumulates_and_writes_over_its_inputs(K):
    run_norm_grad("bf16", 50, K, 32, 0, True, True, accumulate=True)
    run_norm_grad("f32", 50, K, 32, 0, True, False, same="dy")
    run_norm_grad("f32", 50, K, 32, 0, True, False, same="dh")


def test_norm_grad_is_the_slope_of_the_norm():
    """Central differences in 64 bits of sum(dy y) over single components of h and of the weight, step d: their error is d^2 / 6 of a third
    derivative that is of the order of the gradient itself."""
    gen = gen_of("slope")
    T, K, d, eps = 2, 40, 1e-4, 1e-3
    h, w = torch.randn(T, K, generator=gen).float(), (1 + 0.3 * torch.randn(K, generator=gen)).float()
    dy = torch.randn(T, K, generator=gen).float()
    rstd, _ = ref.norm(h.to(F64), w.to(F64), eps)
    L = qa.CodedRows.make(T, K, 32)
    dx, dw = torch.empty(T, K, device=DEV), torch.empty(K, device=DEV)
    ws = torch.empty(qa.qa_rows_workspace_bytes(L, qa.QA_OP_NORM_GRAD, qa.QA_F32, 0), dtype=torch.uint8, device=DEV)
    qa.qa_rms_norm_grad(L, qa.QA_F32, dy.to(DEV), K, h.to(DEV), K, None, None, w.to(DEV), rstd.float().to(DEV), None, 0, dx, K, dw, 0, ws)

    def total(h, w):
        return float((dy.to(F64) * ref.norm(h, w, eps)[1]).sum())
    for t in range(T):
        for k in range(K):
            e = torch.zeros(T, K, dtype=F64)
            e[t, k] = d
            slope = (total(h.to(F64) + e, w.to(F64)) - total(h.to(F64) - e, w.to(F64))) / (2 * d)
            assert abs(slope - float(dx[t, k])) < 1e-5
    for k in range(K):
        e = torch.zeros(K, dtype=F64)
        e[k] = d
        slope = (total(h.to(F64), w.to(F64) + e) - total(h.to(F64), w.to(F64) - e)) / (2 * d)
        assert abs(slope - float(dw[k])) < 1e-5


# ---- weight gradient -----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,N,K,group,pad", [(1, 1, 1, 32, 0), (1, 128, 128, 32, 0), (31, 5, 40, 64, 1), (32, 256, 96, 128, 0), (33, 130, 257, 32, 6),
                                             (515, 100, 130, 64, 0), (1000, 515, 333, 32, 1), (4097, 64, 72, 32, 0), (700, 2050, 1025, 128, 2),
                                             (520, 4096, 1024, 32, 0), (96, 777, 1300, 32, 8), (1100, 256, 512, 64, 8), (2048, 512, 768, 128, 0)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_weight_grad(t, T, N, K, group, pad, accumulate):
    """Products are exact and sums are of at most some hundred terms in a row, or of their sums."""
    gen = gen_of(t, T, N, K, accumulate)
    x, xd = rows_of(gen, T, K, "f32", 0, 2.0)
    dy, dyd = rows_of(gen, T, N, t, pad, 0.1, 1 if pad % 2 else 0)
    L, codes, scales = coded_rows(T, K, group)
    qa.qa_rows_pack(L, qa.QA_F32, xd, K, codes, scales)
    values = ref.decode(codes[:, :K].cpu(), scales[:, :-(-K // group)].cpu(), group)
    dw = torch.full((N, K + 3), 0.5, device=DEV)
    need = qa.qa_rows_workspace_bytes(L, qa.QA_OP_WEIGHT_GRAD, code_of(t), N)
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV) if need else None
    qa.qa_rows_weight_grad(L, codes, scales, code_of(t), dyd, N + pad, N, dw, K + 3, accumulate, ws)
    assert (dw[:, K:] == 0.5).all()
    want = dy.to(F64).t() @ values + 0.5 * accumulate
    each = dy.to(F64).abs().t() @ values.abs() + 0.5 * accumulate
    assert ((dw[:, :K].cpu().to(F64) - want).abs() <= SUM * each).all()
    again = torch.full((N, K + 3), 0.5, device=DEV)
    qa.qa_rows_weight_grad(L, codes, scales, code_of(t), dyd, N + pad, N, again, K + 3, accumulate, ws)
    assert torch.equal(dw, again)                         # bit for bit


def test_weight_grad_keeps_every_bit_of_dy():
    """One row: each product is one binary32 number times a code, exact but for the last rounding."""
    gen = gen_of("bits")
    N, K = 300, 64
    dy = torch.randn(1, N, generator=gen) * torch.exp2(torch.randint(-60, 60, (1, N), generator=gen).float())
    dy[0, 0], dy[0, 1] = torch.finfo(torch.float32).max / 256, 0.0
    x = torch.ones(1, K)
    L, codes, scales = coded_rows(1, K, 32)
    qa.qa_rows_pack(L, qa.QA_F32, x.to(DEV), K, codes, scales)
    dw = torch.empty(N, K, device=DEV)
    qa.qa_rows_weight_grad(L, codes, scales, qa.QA_F32, dy.to(DEV), N, N, dw, K, 0, None)
    assert torch.equal(dw.cpu(), dy.t().expand(N, K).contiguous())


@pytest.mark.parametrize("N,K", [(200, 130), (512, 512)])
def test_weight_grad_of_what_is_not_a_number(N, K):
    """A group without values and an infinity reach the sums that they enter, and no other."""
    gen = gen_of("nan", N)
    T = 300
    x, dy = torch.randn(T, K, generator=gen), torch.randn(T, N, generator=gen).to(torch.bfloat16)
    x[17, 40] = math.nan
    dy[250, 9] = math.inf
    L, codes, scales = coded_rows(T, K, 32)
    qa.qa_rows_pack(L, qa.QA_F32, x.to(DEV), K, codes, scales)
    ws = torch.empty(max(1, qa.qa_rows_workspace_bytes(L, qa.QA_OP_WEIGHT_GRAD, qa.QA_BF16, N)), dtype=torch.uint8, device=DEV)
    dw = torch.zeros(N, K, device=DEV)
    qa.qa_rows_weight_grad(L, codes, scales, qa.QA_BF16, dy.to(DEV), N, N, dw, K, 0, ws)
    bad = torch.zeros(N, K, dtype=torch.bool)
    bad[:, 32:64] = True
    bad[9] = True
    assert torch.equal(~torch.isfinite(dw.cpu()), bad)


# ---- log probabilities ---------------------------------------------------------------------------------------------


def run_token(t, x, target, top, pad=0, lead=0, ws_fill=0xA5):
    T, V = x.shape
    flat = torch.full((lead + T * (V + pad) + 8,), 50.0, dtype=TYPES[t])            # what must not be read would be the largest
    flat[lead:lead + T * (V + pad)].view(T, V + pad)[:, :V] = x
    xd = flat.to(DEV)[lead:]
    out = {k: torch.full((T + 1,), 7.0, device=DEV) for k in ("logprob", "entropy")}
    stats = torch.full((T + 1, 2), 7.0, device=DEV)
    tl = torch.full((T * top + 1,), 7.0, device=DEV)
    ti = torch.full((T * top + 1,), -9, dtype=torch.int32, device=DEV)
    need = qa.qa_token_workspace_bytes(T, V, top)
    ws = torch.full((need,), ws_fill, dtype=torch.uint8, device=DEV) if need else None
    qa.qa_token_logprob(code_of(t), T, V, xd, V + pad, target.to(DEV), top, out["logprob"], out["entropy"], stats,
                        tl if top else None, ti if top else None, ws)
    for v in out.values():
        assert v[T] == 7.0
    assert tl[-1] == 7.0 and ti[-1] == -9 and (stats[T] == 7.0).all()
    return (*(out[k][:T].cpu() for k in ("logprob", "entropy")), stats[:T].cpu(), tl[:-1].view(T, top).cpu(), ti[:-1].view(T, top).cpu())


def check_token(t, x, target, top, **how):
    got = run_token(t, x, target, top, **how)
    x64 = x.to(F64)
    lp, entropy, stats, logp = ref.token_logprob(x64, target)

    def near(a, b, slack):
        a = a.to(F64)
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.isinf(a), torch.isinf(b))
        fine = torch.isfinite(b)
        assert torch.equal(a[~fine & ~torch.isnan(b)], b[~fine & ~torch.isnan(b)])
        assert ((a - b).abs()[fine] <= slack.expand_as(b)[fine]).all(), ((a - b).abs()[fine] - slack.expand_as(b)[fine]).max()
    # the largest logit as it is, the sum of exponentials to SUM and its logarithm rounded; log p is two differences
    bad = torch.isnan(stats[:, 1])
    assert torch.equal(got[2][~bad, 0].to(F64), stats[~bad, 0])
    near(got[2][:, 1], stats[:, 1], 2 * SUM + 2.0 ** -22 * torch.nan_to_num(stats[:, 1]))
    near(got[0], lp, 2 * SUM + 2.0 ** -22 * (torch.nan_to_num(lp, 0, 0, 0).abs() + 20))
    near(got[1], entropy, SUM * (8 + 2 * torch.nan_to_num(entropy)))
    want = ref.top(x64, top)
    assert torch.equal(got[4].long(), want)
    at = logp.gather(1, want)
    at = torch.where(bad[:, None], torch.full_like(at, math.nan), at)
    near(got[3], at, 2 * SUM + 2.0 ** -22 * (torch.nan_to_num(at, 0, 0, 0).abs() + 20))


TOKEN_SHAPES = [(1, 1, 1), (3, 2, 2), (5, 63, 20), (4, 64, 64), (9, 511, 5), (2, 513, 64), (7, 4096, 8), (1030, 700, 3), (600, 4500, 2),
                (1, 4097, 20), (3, 50021, 64), (1, 131072, 20), (520, 9000, 7), (2, 100003, 0), (2, 300, 0), (530, 5000, 0)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V,top", TOKEN_SHAPES)
def test_token_logprob(t, T, V, top):
    gen = gen_of(t, T, V, top)
    x = (3 * torch.randn(T, V, generator=gen)).to(TYPES[t])
    target = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    target[0] = V - 1
    if T > 2:
        target[1], target[2] = -1, V
    check_token(t, x, target, top, pad=V % 3, lead=V % 5)


@pytest.mark.parametrize("V", [40, 600, 4096, 9001, 70001])
@pytest.mark.parametrize("T", [6, 513])
def test_token_logprob_of_ties_and_masks(V, T):
    """Constant rows, rows of few values, descending and ascending ones, masked ones (by -infinity and by the type's lowest value), and rows that
    the mask leaves empty."""
    gen = gen_of(V, T)
    x = torch.randint(-2, 3, (T, V), generator=gen).float()
    x[0] = 1.5
    x[1] = torch.arange(V).float().flip(0) / 64
    x[2] = torch.arange(V).float() / 64
    x[3] = -math.inf
    x[4] = -math.inf
    x[4, V // 2], x[4, V - 1] = 2.0, 3.0
    x[5] = torch.finfo(torch.float32).min
    x[5, V // 3] = 4.0
    target = torch.zeros(T, dtype=torch.int32)
    target[4] = 1                                      # a target that is masked out
    check_token("f32", x, target, min(V, 20))
    low = x.to(torch.bfloat16)
    low[5] = torch.finfo(torch.bfloat16).min           # all of them: a uniform row
    check_token("bf16", low, target, min(V, 64))
    signs = torch.zeros(T, V)
    signs[:, ::2] = -0.0
    check_token("f32", signs, target, 5)


@pytest.mark.parametrize("V", [40, 4096, 9001, 70001])
def test_token_logprob_of_rows_that_are_not_numbers(V):
    x = torch.zeros(4, V)
    x[:, 1] = 1.0
    x[1, V - 2] = math.nan
    x[2, V // 2] = math.inf
    x[3, :-3] = math.nan
    target = torch.ones(4, dtype=torch.int32)
    got = run_token("f32", x, target, 6)
    for row in (1, 2, 3):
        for v in (got[0], got[1], got[2][:, 1], got[3]):
            assert torch.isnan(v[row]).all()
    check_token("f32", x[:1], target[:1], 6)
    assert torch.equal(got[4].long(), ref.top(x, 6))


def test_token_logprob_with_a_large_offset():
    """Logits far from 0 lose only what their own rounding loses."""
    gen = gen_of("offset")
    x = (1000 + torch.randn(3, 30000, generator=gen)).float()
    check_token("f32", x, torch.zeros(3, dtype=torch.int32), 4)
    check_token("f32", -x, torch.zeros(3, dtype=torch.int32), 4)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 7), (9, 1000), (2, 8193), (1, 50021), (300, 257)])
@pytest.mark.parametrize("in_place", [False, True])
def test_token_logprob_grad(t, T, V, in_place):
    gen = gen_of(t, T, V)
    x = (3 * torch.randn(T, V, generator=gen)).to(TYPES[t])
    target = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    if T > 2:
        target[0], target[1] = -1, V
        x[2] = -math.inf
        x[1, : V // 2] = -math.inf
        x[T - 1] = torch.finfo(TYPES[t]).min if T > 3 else x[T - 1]        # a mask that leaves nothing: uniform
    a, e = torch.randn(T, generator=gen), torch.randn(T, generator=gen)
    x64 = x.to(F64)
    _, entropy, stats, logp = ref.token_logprob(x64, target)
    want = ref.token_logprob_grad(x64, target, a.to(F64), e.to(F64))
    pad = 1
    flat = torch.full((T, V + pad), 5.0, dtype=TYPES[t], device=DEV)
    flat[:, :V] = x.to(DEV)
    out = flat if in_place else torch.full((T, V + pad), 5.0, dtype=TYPES[t], device=DEV)
    f = lambda v: v.float().to(DEV)  # noqa: E731
    qa.qa_token_logprob_grad(code_of(t), T, V, flat, V + pad, target.to(DEV), f(stats), f(entropy), a.to(DEV), e.to(DEV), out, V + pad)
    assert (out[:, V:] == 5.0).all()
    p = torch.exp(logp)
    reach = torch.where(p == 0, torch.zeros_like(p), (logp - entropy[:, None]).abs()) + 1
    # log p is two differences of numbers of its size and of log_sum's, each rounded: so many units in the exponent
    units = torch.nan_to_num(logp, 0, 0, 0).abs() + stats[:, 1:] + 4
    off = p * (a.abs()[:, None] + e.abs()[:, None] * reach) * 2.0 ** -21 * units + 2.0 ** -23 * a.abs()[:, None]
    tiny = 2.0 ** -24 if t == "f16" else 0.0
    got = out[:, :V].cpu().to(F64)
    assert ((got - want).abs() <= HALF_ULP[t] * 1.01 * want.abs() + off + tiny).all()


def test_token_logprob_grad_is_the_slope():
    gen = gen_of("token slope")
    T, V, d = 3, 20, 1e-4
    x = torch.randn(T, V, generator=gen).float()
    x[1, 4] = -math.inf
    target = torch.tensor([3, 7, -1], dtype=torch.int32)
    a, e = torch.randn(T, generator=gen), torch.randn(T, generator=gen)
    _, entropy, stats, _ = ref.token_logprob(x.to(F64), target)
    dx = torch.empty(T, V, device=DEV)
    f = lambda v: v.float().to(DEV)  # noqa: E731
    qa.qa_token_logprob_grad(qa.QA_F32, T, V, x.to(DEV), V, target.to(DEV), f(stats), f(entropy), f(a), f(e), dx, V)

    def total(x):
        lp, entropy, _, _ = ref.token_logprob(x, target)
        return float((a.to(F64) * lp + e.to(F64) * entropy).sum())
    for t in range(T):
        for j in range(V):
            step = torch.zeros(T, V, dtype=F64)
            step[t, j] = d
            slope = (total(x.to(F64) + step) - total(x.to(F64) - step)) / (2 * d)
            assert abs(slope - float(dx[t, j])) < 1e-5


def test_token_logprob_grad_without_entropy_or_target():
    x = torch.randn(4, 300, generator=gen_of("parts"))
    target = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    _, entropy, stats, _ = ref.token_logprob(x.to(F64), target)
    f = lambda v: v.float().to(DEV)  # noqa: E731
    a, zero = torch.ones(4), torch.zeros(4)
    out = torch.empty(4, 300, device=DEV)
    qa.qa_token_logprob_grad(qa.QA_F32, 4, 300, x.to(DEV), 300, target.to(DEV), f(stats), None, f(a), None, out, 300)
    assert (out.cpu() - ref.token_logprob_grad(x.to(F64), target, a.to(F64), zero.to(F64))).abs().max() < 1e-6
    qa.qa_token_logprob_grad(qa.QA_F32, 4, 300, x.to(DEV), 300, None, f(stats), f(entropy), None, f(a), out, 300)
    assert (out.cpu() - ref.token_logprob_grad(x.to(F64), target, zero.to(F64), a.to(F64))).abs().max() < 1e-6


# ---- calls ---------------------------------------------------------------------------------------------------------


def test_calls_without_rows():
    L = qa.CodedRows.make(0, 100, 32)
    none = torch.empty(0, device=DEV)
    dw = torch.full((100,), 3.0, device=DEV)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    qa.qa_rows_pack(L, qa.QA_F32, none, 100, none, none)
    qa.qa_rows_unpack(L, none, none, qa.QA_F32, none, 100)
    qa.qa_rms_norm(L, qa.QA_F32, none, 100, None, 0, none, 1e-6, None, 0, none, none, None, 0, None)
    qa.qa_token_logprob(qa.QA_F32, 0, 10, none, 10, None, 0, None, None, None, None, None, None)
    qa.qa_token_logprob_grad(qa.QA_F32, 0, 10, none, 10, None, none, None, None, None, none, 10)
    qa.qa_rms_norm_grad(L, qa.QA_F32, none, 100, none, 100, None, None, none, none, None, 0, none, 100, dw, 1, ws)
    assert (dw == 3.0).all()
    qa.qa_rms_norm_grad(L, qa.QA_F32, none, 100, none, 100, None, None, none, none, None, 0, none, 100, dw, 0, ws)
    assert (dw == 0.0).all()
    more = torch.full((3, 101), 3.0, device=DEV)
    qa.qa_rows_weight_grad(L, none, none, qa.QA_BF16, none, 3, 3, more, 101, 1, None)
    assert (more == 3.0).all()
    qa.qa_rows_weight_grad(L, none, none, qa.QA_BF16, none, 3, 3, more, 101, 0, None)
    assert (more[:, :100] == 0.0).all() and (more[:, 100] == 3.0).all()


def test_calls_on_another_stream_and_in_a_graph():
    """Every call enqueues on the stream it is given and can be recorded; a replay repeats the call bit for bit."""
    gen = gen_of("graph")
    T, K, N, V, top = 600, 200, 136, 6000, 5
    L, codes, scales = coded_rows(T, K, 32)
    x, r, dy = (torch.randn(T, K, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(3))
    dz = torch.randn(T, N, generator=gen).to(torch.bfloat16).to(DEV)
    logits = torch.randn(T, V, generator=gen).to(DEV)
    target = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32).to(DEV)
    w, one = torch.ones(K, device=DEV), torch.ones(T, device=DEV)
    h, y, dx = (torch.zeros(T, K, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    rstd, lp, entropy, stats = (torch.zeros(s, device=DEV) for s in (T, T, T, (T, 2)))
    tl, ti = torch.zeros(T, top, device=DEV), torch.zeros(T, top, dtype=torch.int32, device=DEV)
    dw, dn, dl = torch.zeros(N, K, device=DEV), torch.zeros(K, device=DEV), torch.zeros(T, V, device=DEV)
    room = lambda n: torch.zeros(max(n, 1), dtype=torch.uint8, device=DEV)  # noqa: E731
    ws = [room(qa.qa_rows_workspace_bytes(L, qa.QA_OP_WEIGHT_GRAD, qa.QA_BF16, N)), room(qa.qa_rows_workspace_bytes(L, qa.QA_OP_NORM_GRAD, qa.QA_BF16, 0)),
          room(qa.qa_token_workspace_bytes(T, V, top))]

    def calls(stream=None):
        qa.qa_rms_norm(L, qa.QA_BF16, x, K, r, K, w, 1e-6, h, K, codes, scales, y, K, rstd, stream=stream)
        qa.qa_rows_weight_grad(L, codes, scales, qa.QA_BF16, dz, N, N, dw, K, 0, ws[0], stream=stream)
        qa.qa_rms_norm_grad(L, qa.QA_BF16, dy, K, h, K, None, None, w, rstd, None, 0, dx, K, dn, 0, ws[1], stream=stream)
        qa.qa_token_logprob(qa.QA_F32, T, V, logits, V, target, top, lp, entropy, stats, tl, ti, ws[2], stream=stream)
        qa.qa_token_logprob_grad(qa.QA_F32, T, V, logits, V, target, stats, entropy, one, one, dl, V, stream=stream)

    outs = (h, y, dx, rstd, lp, entropy, stats, tl, ti, dw, dn, dl)
    calls()
    torch.cuda.synchronize()
    want = [v.clone() for v in outs]
    side = torch.cuda.Stream()
    for v in outs:
        v.zero_()
    side.wait_stream(torch.cuda.current_stream())
    calls(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        for v in outs:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_offsets_beyond_32_bits(t):
    """Three rows, 2^31 + 24 elements apart: the last begins at 8 or 17 GB."""
    gen, K, far = gen_of("far", t), 100, (1 << 31) + 24
    flat = torch.empty(2 * far + K, dtype=TYPES[t], device=DEV)
    rows = flat.as_strided((3, K), (far, 1))
    x = torch.randn(3, K, generator=gen).to(TYPES[t])
    rows.copy_(x)
    L, codes, scales = coded_rows(3, K, 32)
    qa.qa_rows_pack(L, code_of(t), flat, far, codes, scales)
    want_s = ref.scale_bytes(x.to(F64), 32)
    assert torch.equal(codes[:, :K].cpu().long(), ref.code(x.to(F64), want_s, 32))
    y = torch.empty(3, K, dtype=torch.bfloat16, device=DEV)
    rstd = torch.empty(3, device=DEV)
    ones = torch.ones(K, device=DEV)
    qa.qa_rms_norm(L, code_of(t), flat, far, flat, far, ones, 0.0, None, 0, codes, scales, y, K, rstd)
    want, _ = ref.norm(2 * x.to(F64), torch.ones(K, dtype=F64), 0.0)
    assert (rstd.cpu().to(F64) / want - 1).abs().max() < SUM
    ws = torch.empty(qa.qa_rows_workspace_bytes(L, qa.QA_OP_NORM_GRAD, code_of(t)), dtype=torch.uint8, device=DEV)
    dx = torch.empty(3, K, dtype=TYPES[t], device=DEV)
    dw = torch.empty(K, device=DEV)
    qa.qa_rms_norm_grad(L, code_of(t), flat, far, flat, far, None, None, ones, ones, flat, far, dx, K, dw, 0, ws)
    want_dx, want_dw = ref.norm_grad(x.to(F64), x.to(F64), torch.ones(K, dtype=F64), torch.ones(3, dtype=F64), x.to(F64))
    assert (dw.cpu().to(F64) - want_dw).abs().max() < 1e-5
    assert ((dx.cpu().to(F64) - want_dx).abs() <= HALF_ULP[t] * 1.01 * want_dx.abs() + SUM * 40).all()
    target = torch.tensor([1, 2, 3], dtype=torch.int32)
    lp, entropy, stats = torch.empty(3, device=DEV), torch.empty(3, device=DEV), torch.empty(3, 2, device=DEV)
    qa.qa_token_logprob(code_of(t), 3, K, flat, far, target.to(DEV), 0, lp, entropy, stats, None, None, None)
    want_lp = ref.token_logprob(x.to(F64), target)[0]
    assert (lp.cpu().to(F64) - want_lp).abs().max() < 1e-5
    qa.qa_token_logprob_grad(code_of(t), 3, K, flat, far, target.to(DEV), stats, None, ones, None, flat, far)
    want_dx = ref.token_logprob_grad(x.to(F64), target, torch.ones(3, dtype=F64), torch.zeros(3, dtype=F64))
    assert ((rows.cpu().to(F64) - want_dx).abs() <= HALF_ULP[t] * 1.01 * want_dx.abs() + 1e-6).all()


def test_more_rows_than_a_launch_has_work_groups_for():
    """Numbers of up to seven bits come back as they are."""
    T = (1 << 24) + 77
    x = (torch.arange(T, device=DEV) % 255 - 127).float()[:, None]
    L = qa.CodedRows.make(T, 1, 32)
    codes = torch.empty(T, 16, dtype=torch.int8, device=DEV)
    scales, back = torch.empty(T, 1, dtype=torch.uint8, device=DEV), torch.empty(T, 1, device=DEV)
    qa.qa_rows_pack(L, qa.QA_F32, x, 1, codes, scales)
    qa.qa_rows_unpack(L, codes, scales, qa.QA_F32, back, 1)
    assert torch.equal(back, x)
    T = 300_001
    logits = torch.zeros(T, 3, device=DEV)
    logits[:, 1] = 1.0
    index, top = torch.full((T, 2), -1, dtype=torch.int32, device=DEV), torch.empty(T, 2, device=DEV)
    entropy = torch.empty(T, device=DEV)
    qa.qa_token_logprob(qa.QA_F32, T, 3, logits, 3, None, 2, None, entropy, None, top, index, None)
    assert torch.equal(index, torch.tensor([[1, 0]], dtype=torch.int32, device=DEV).expand(T, 2))
    assert (entropy == entropy[0]).all() and (top == top[0]).all()


def test_tiles_that_the_whole_width_does_not_fill():
    """A large enough gradient for the large tiles, with ends inside one in all three directions, against a product in 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(7)
    T, N, K = 335, 3851, 4099
    x = torch.randn(T, K, generator=gen, device=DEV)
    for t in ("bf16", "f16", "f32"):
        dy = torch.randn(T, N + 5, generator=gen, device=DEV).to(TYPES[t])[:, :N]
        L, codes, scales = coded_rows(T, K, 64)
        qa.qa_rows_pack(L, qa.QA_F32, x, K, codes, scales)
        values = torch.empty(T, K, device=DEV)
        qa.qa_rows_unpack(L, codes, scales, qa.QA_F32, values, K)
        ws = torch.empty(max(1, qa.qa_rows_workspace_bytes(L, qa.QA_OP_WEIGHT_GRAD, code_of(t), N)), dtype=torch.uint8, device=DEV)
        for accumulate in (0, 1):
            dw = torch.full((N, K + 1), 0.25, device=DEV)
            qa.qa_rows_weight_grad(L, codes, scales, code_of(t), dy, N + 5, N, dw, K + 1, accumulate, ws)
            assert (dw[:, K] == 0.25).all()
            want = dy.double().t().contiguous() @ values.double() + 0.25 * accumulate
            each = dy.double().abs().t().contiguous() @ values.double().abs() + 0.25
            assert ((dw[:, :K].double() - want).abs() <= SUM * each).all()


# ---- many rows ---------------------------------------------------------------------------------------------------

# Rows that a work-group goes over, one read ahead, in every form; the last are more than the caches hold.
MANY = [(40000, 5, 32, 0), (20000, 8, 64, 1), (18000, 43, 32, 0), (17001, 64, 128, 3), (9000, 120, 64, 1), (5000, 200, 32, 0), (2300, 511, 32, 0),
        (2100, 1003, 64, 1), (1100, 2047, 32, 0), (700, 3001, 32, 2), (600, 4097, 128, 0), (300, 9001, 32, 0)]
MANY_TYPES = [(*shape, t) for shape in MANY for t in ("f32", "bf16")] + [(9400, 4099, 32, 0, "bf16")]


@pytest.mark.parametrize("T,K,group,pad,t", MANY_TYPES)
def test_norm_of_many_rows(T, K, group, pad, t):
    test_norm(t, T, K, group, pad, True)


@pytest.mark.parametrize("T,K,group,pad,t", MANY_TYPES)
@pytest.mark.parametrize("coded", [False, True])
def test_norm_grad_of_many_rows(T, K, group, pad, t, coded):
    run_norm_grad(t, T, K, group, pad, True, coded)


@pytest.mark.parametrize("T,V,t", [(4200, 16500, "bf16"), (2100, 16500, "f32"), (4200, 8200, "f32")])
@pytest.mark.parametrize("in_place", [False, True])
def test_token_logprob_grad_of_many_rows(T, V, t, in_place):
    """More than the caches hold, rows at every offset inside 16 bytes; all rows against each other's bits, some against 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(11)
    x = torch.full((T, V + 1), 5.0, dtype=TYPES[t], device=DEV)
    x[:, :V] = 3 * torch.randn(T, V, generator=gen, device=DEV)
    x[T // 2:, :V] = x[:T - T // 2, :V]                                          # at other offsets
    target = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    target[0], target[1] = 0, V - 1
    target[T // 2:] = target[:T - T // 2].clone()
    a, e = (torch.randn(T, generator=gen, device=DEV) for _ in range(2))
    a[T // 2:], e[T // 2:] = a[:T - T // 2].clone(), e[:T - T // 2].clone()
    rows = torch.tensor([0, 1, 2, 3, 5, T // 3, T // 2 - 1, T // 2, T - 1])
    x64, some = x[rows.to(DEV), :V].cpu().to(F64), target[rows.to(DEV)].cpu()
    entropy, stats = torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV)
    logprob = torch.empty(T, device=DEV)
    qa.qa_token_logprob(code_of(t), T, V, x, V + 1, target, 0, logprob, entropy, stats, None, None, None)
    entropy[T // 2:], stats[T // 2:] = entropy[:T - T // 2].clone(), stats[:T - T // 2].clone()
    out = x if in_place else torch.full((T, V + 1), 5.0, dtype=TYPES[t], device=DEV)
    qa.qa_token_logprob_grad(code_of(t), T, V, x, V + 1, target, stats, entropy, a, e, out, V + 1)
    assert (out[:, V] == 5.0).all()
    assert torch.equal(out[T // 2:, :V], out[:T - T // 2, :V])
    _, entropy64, stats64, logp = ref.token_logprob(x64, some)
    a64, e64 = a[rows.to(DEV)].cpu().to(F64), e[rows.to(DEV)].cpu().to(F64)
    want = ref.token_logprob_grad(x64, some, a64, e64)
    p = torch.exp(logp)
    reach = (logp - entropy64[:, None]).abs() + 1
    units = logp.abs() + stats64[:, 1:] + 4
    # stats and entropy are the call's own, good to SUM of the largest |log p| that enters them
    off = p * (a64.abs()[:, None] + e64.abs()[:, None] * reach) * (2.0 ** -21 * units + 4 * SUM * units) + 2.0 ** -23 * a64.abs()[:, None]
    assert ((out[rows.to(DEV), :V].cpu().to(F64) - want).abs() <= HALF_ULP[t] * 1.01 * want.abs() + off).all()
