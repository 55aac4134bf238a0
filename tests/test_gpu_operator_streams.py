"""Calls that read and write more than 256 MiB go past the caches, most of them in kernels of their own.  Each is compared bit for bit
(the logits' gradient number for number) with calls on thirds of its rows, which the caches hold and which the other tests compare
with the formulas, and some rows with the formulas in 64 bits.  Tolerances are those of tests/test_gpu_operators.py."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    from test_gpu_operators import F64, HALF_ULP, SUM, TYPES, code_of
    DEV = torch.device("cuda:0")

HELD = 256 << 20
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def rows_for(bytes_of_a_row):
    """Rows that are a few percent more than the caches hold; a third of them is less."""
    return int(1.05 * HELD / bytes_of_a_row) + 1


def thirds(T):
    return [(T * i // 3, T * (i + 1) // 3) for i in range(3)]


def some_of(T):
    return torch.tensor(sorted({0, 1, 2, 3, 5, T // 3 - 1, T // 2, T - 2, T - 1} & set(range(T))))


def random(gen, T, K, t, pad=0, scale=1.0):
    """Rows inside wider ones, with NaN between them."""
    v = torch.full((T, K + pad), math.nan, dtype=TYPES[t], device=DEV)
    v[:, :K] = (scale * torch.randn(T, K, generator=gen, device=DEV)).to(TYPES[t])
    return v[:, :K]


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---- rows in 8 bits ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("t,K,group,pad", [("bf16", 8209, 32, 3), ("f32", 8192, 64, 0), ("f16", 100, 128, 1), ("f32", 1031, 32, 0), ("bf16", 5, 32, 0)])
def test_rows_pack_and_unpack(t, K, group, pad):
    T = rows_for(K * (BYTES[t] + 1))
    gen = torch.Generator(device=DEV).manual_seed(K)
    x = random(gen, T, K, t, pad, 3.0)
    x[T // 2, K // 2] = math.inf
    L = qa.CodedRows.make(T, K, group)
    new = lambda: (torch.full((T, L.code_stride), 77, dtype=torch.int8, device=DEV),  # noqa: E731
                   torch.full((T, L.scale_stride), 77, dtype=torch.uint8, device=DEV), torch.full((T, K + 1), 5.0, dtype=TYPES[t], device=DEV))
    codes, scales, back = new()
    qa.qa_rows_pack(L, code_of(t), x, K + pad, codes, scales)
    qa.qa_rows_unpack(L, codes, scales, code_of(t), back, K + 1)
    assert (codes[:, K:] == 77).all() and (back[:, K] == 5.0).all()
    codes3, scales3, back3 = new()
    for a, b in thirds(T):
        part = qa.CodedRows.make(b - a, K, group)
        qa.qa_rows_pack(part, code_of(t), x[a:], K + pad, codes3[a:], scales3[a:])
        qa.qa_rows_unpack(part, codes3[a:], scales3[a:], code_of(t), back3[a:], K + 1)
    assert same(codes, codes3) and same(scales, scales3) and same(back, back3)
    some = some_of(T)
    v = x[some.to(DEV)].cpu().to(F64)
    want_s = ref.scale_bytes(v, group)
    assert torch.equal(scales[some.to(DEV)].cpu().long(), want_s)
    assert torch.equal(codes[some.to(DEV), :K].cpu().long(), ref.code(torch.nan_to_num(v, 0, 0, 0), want_s, group))


# ---- norm ------------------------------------------------------------------------------------------------------------

# every number of lanes that a row can have, aligned and not
FORMS = [("bf16", 6, 32, 0), ("f32", 43, 32, 1), ("bf16", 64, 64, 0), ("f16", 120, 32, 0), ("f32", 200, 128, 0), ("bf16", 511, 64, 2), ("f32", 1003, 32, 0),
         ("bf16", 2047, 32, 0), ("f32", 3001, 128, 1), ("f16", 4096, 32, 0), ("bf16", 4097, 32, 0), ("f32", 8192, 64, 0), ("bf16", 9001, 32, 0),
         ("bf16", 20011, 64, 0)]


@pytest.mark.parametrize("t,K,group,pad", FORMS)
@pytest.mark.parametrize("in_place", [False, True])
def test_norm(t, K, group, pad, in_place):
    T = rows_for(K * (3 * BYTES[t] + 3))
    gen = torch.Generator(device=DEV).manual_seed(K)
    x, r = random(gen, T, K, t, pad, 2.0), random(gen, T, K, t, pad)
    w = 1 + 0.3 * torch.randn(K, generator=gen, device=DEV)
    L = qa.CodedRows.make(T, K, group)
    stride = K + pad if in_place else K + 1

    def new():
        h = random(gen, 0, K, t) if in_place else torch.full((T, stride), 5.0, dtype=TYPES[t], device=DEV)
        return (h, torch.full((T, L.code_stride), 77, dtype=torch.int8, device=DEV), torch.full((T, L.scale_stride), 77, dtype=torch.uint8, device=DEV),
                torch.full((T, K + 1), 5.0, dtype=torch.bfloat16, device=DEV), torch.empty(T, device=DEV))

    three = new()
    three_x = x.as_strided((T, K + pad), (K + pad, 1)).clone() if in_place else x
    for a, b in thirds(T):
        h, codes, scales, y, rstd = (v[a:] for v in three)
        xa = three_x[a:]
        qa.qa_rms_norm(qa.CodedRows.make(b - a, K, group), code_of(t), xa, K + pad, r[a:], K + pad, w, 1e-5, xa if in_place else h, stride,
                       codes, scales, y, K + 1, rstd[:])
    some = some_of(T).to(DEV)
    want_rstd, want = ref.norm((x[some].cpu().to(F64) + r[some].cpu().to(F64)), w.cpu().to(F64), 1e-5)
    h, codes, scales, y, rstd = new()
    qa.qa_rms_norm(L, code_of(t), x, K + pad, r, K + pad, w, 1e-5, x if in_place else h, stride, codes, scales, y, K + 1, rstd)
    assert same(codes, three[1]) and same(scales, three[2]) and same(y, three[3]) and same(rstd, three[4])
    assert same(x, three_x[:, :K]) if in_place else same(h, three[0])
    assert (codes[:, K:] == 77).all() and (y[:, K] == 5.0).all()
    assert (rstd[some].cpu().to(F64) / want_rstd - 1).abs().max() < SUM
    s = scales[some].cpu().long()
    step = torch.exp2((s - 127).to(F64)).repeat_interleave(group, dim=1)[:, :K]
    assert ((ref.decode(codes[some, :K].cpu(), s, group) - want).abs() <= step / 2 + 2 * SUM * want.abs()).all()


@pytest.mark.parametrize("t,K,group,pad", FORMS)
@pytest.mark.parametrize("coded,same_as", [(False, None), (True, None), (False, "dy"), (True, "dh")])
def test_norm_grad(t, K, group, pad, coded, same_as):
    T = rows_for(K * (3 * BYTES[t] + (1 if coded else BYTES[t])))
    gen = torch.Generator(device=DEV).manual_seed(K)
    dy, dh, h = random(gen, T, K, t, pad, 0.5), random(gen, T, K, t, pad, 0.5), random(gen, T, K, t, pad, 2.0)
    w = 1 + 0.3 * torch.randn(K, generator=gen, device=DEV)
    L = qa.CodedRows.make(T, K, group)
    codes = torch.empty(T, L.code_stride, dtype=torch.int8, device=DEV)
    scales = torch.empty(T, L.scale_stride, dtype=torch.uint8, device=DEV)
    if coded:
        qa.qa_rows_pack(L, code_of(t), h, K + pad, codes, scales)
        h = torch.empty(T, K, device=DEV)
        qa.qa_rows_unpack(L, codes, scales, qa.QA_F32, h, K)
    rstd = torch.rsqrt((h.double() ** 2).mean(dim=1) + 1e-6).float()
    ws = torch.empty(qa.qa_rows_workspace_bytes(L, qa.QA_OP_NORM_GRAD, code_of(t)), dtype=torch.uint8, device=DEV)
    stride = K + pad if same_as else K + 1

    def call(a, b, dy, dh, dx, dw):
        part = qa.CodedRows.make(b - a, K, group)
        qa.qa_rms_norm_grad(part, code_of(t), dy[a:], K + pad, None if coded else h[a:], K + pad, codes[a:] if coded else None,
                            scales[a:] if coded else None, w, rstd[a:], dh[a:], K + pad, {None: dx, "dy": dy, "dh": dh}[same_as][a:], stride,
                            dw, int(a > 0), ws)

    def run(pieces):
        whole = lambda v: v.as_strided((T, K + pad), (K + pad, 1)).clone()  # noqa: E731
        a_dy, a_dh = whole(dy) if same_as == "dy" else dy, whole(dh) if same_as == "dh" else dh
        dx = torch.full((T if same_as is None else 1, K + 1), 5.0, dtype=TYPES[t], device=DEV)
        dw = torch.empty(K, device=DEV)
        for a, b in pieces:
            call(a, b, a_dy, a_dh, dx, dw)
        return {None: dx, "dy": a_dy, "dh": a_dh}[same_as], dw

    dx, dw = run([(0, T)])
    dx3, _ = run(thirds(T))
    assert same(dx[:, :K], dx3[:, :K]) and (same_as or (dx[:, K] == 5.0).all())
    some = some_of(T).to(DEV)
    c = lambda v: v[some].cpu().to(F64)  # noqa: E731
    want, _ = ref.norm_grad(c(dy), c(h), w.cpu().to(F64), c(rstd), c(dh))
    n = (c(h) * c(rstd)[:, None]).abs()
    g = c(dy) * w.cpu().to(F64)
    terms = c(rstd)[:, None] * (g.abs() + n * (g * n).abs().mean(dim=1, keepdim=True)) + c(dh).abs()
    tiny = 2.0 ** -24 if t == "f16" else 0.0
    assert ((c(dx[:, :K]) - want).abs() <= HALF_ULP[t] * want.abs() * 1.01 + SUM * terms + tiny).all()
    want_w, each = torch.zeros(K, dtype=F64, device=DEV), torch.zeros(K, dtype=F64, device=DEV)
    for a, b in [(T * i // 16, T * (i + 1) // 16) for i in range(16)]:                  # some rows at a time: 64 bits take memory
        p = dy[a:b].double() * (h[a:b].double() * rstd[a:b].double()[:, None])
        want_w += p.sum(dim=0)
        each += p.abs().sum(dim=0)
    assert ((dw.double() - want_w).abs() <= SUM * each).all()


# ---- log probabilities -------------------------------------------------------------------------------------------------


def logits(gen, T, V, t, pad):
    x = torch.full((T, V + pad), 50.0, dtype=TYPES[t], device=DEV)                     # what must not be read would be the largest
    x[:, :V] = (3 * torch.randn(T, V, generator=gen, device=DEV)).to(TYPES[t])
    x[2, :V] = -math.inf
    x[3, V // 2:V] = -math.inf
    x[T - 2, V // 3] = math.nan
    target = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    target[0], target[1] = -1, V - 1
    return x, target


@pytest.mark.parametrize("t,V,pad", [("bf16", 50021, 0), ("f32", 70001, 1), ("f16", 4097, 2), ("bf16", 32768, 0), ("bf16", 70001, 0),
                                     ("f32", 32768, 0), ("f16", 131072, 0)])
@pytest.mark.parametrize("top", [0, 8, 64])
def test_token_logprob(t, V, pad, top):
    T = rows_for(V * BYTES[t])
    gen = torch.Generator(device=DEV).manual_seed(V)
    x, target = logits(gen, T, V, t, pad)

    def run(pieces):
        logprob, entropy, stats = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV)
        best, index = torch.empty(T, top, device=DEV), torch.empty(T, top, dtype=torch.int32, device=DEV)
        for a, b in pieces:
            need = qa.qa_token_workspace_bytes(b - a, V, top)
            assert need == 0                        # neither the whole nor a third is split: the same order of additions
            qa.qa_token_logprob(code_of(t), b - a, V, x[a:], V + pad, target[a:], top, logprob[a:], entropy[a:], stats[a:],
                                best[a:] if top else None, index[a:] if top else None, None)
        return logprob, entropy, stats, best, index

    got, want = run([(0, T)]), run(thirds(T))
    assert all(same(a, b) for a, b in zip(got, want))
    some = torch.tensor([0, 1, 2, 3, 5, T // 2, T - 1])
    x64, y = x[some.to(DEV), :V].cpu().to(F64), target[some.to(DEV)].cpu()
    lp, entropy, stats, logp = ref.token_logprob(x64, y)
    logprob, h, st, best, index = (v[some.to(DEV)].cpu() for v in got)
    full = torch.isfinite(stats[:, 0])
    assert torch.equal(st[:, 0].to(F64), stats[:, 0])
    near = lambda a, b: ((a.to(F64) - b).abs() <= 2 * SUM + 2.0 ** -22 * (b.abs() + 20)) | (a.to(F64) == b)  # noqa: E731
    assert near(st[:, 1], stats[:, 1]).all() and near(logprob, lp).all()
    assert ((h.to(F64) - entropy).abs() <= SUM * (8 + 2 * entropy))[full].all() and (h[~full] == 0).all()
    assert torch.equal(index.long(), ref.top(x64, top))
    assert near(best, logp.gather(1, index.long())).all()
    assert torch.isnan(got[1][T - 2]) and torch.isnan(got[2][T - 2, 1])


@pytest.mark.parametrize("t,V,pad", [("bf16", 2048, 0), ("f32", 1001, 0), ("f16", 7, 0), ("bf16", 2049, 1), ("f16", 8193, 0), ("f32", 47236, 3), ("f32", 217, 1), ("f32", 512, 0),
                                     ("bf16", 16387, 0), ("f16", 7001, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_token_logprob_grad(t, V, pad, in_place):
    T = rows_for(2 * V * BYTES[t])
    gen = torch.Generator(device=DEV).manual_seed(V)
    x, target = logits(gen, T, V, t, pad)
    x[T - 2, V // 3] = 1.0
    entropy, stats, logprob = torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV), torch.empty(T, device=DEV)
    ws = torch.empty(max(1, qa.qa_token_workspace_bytes(T, V, 0)), dtype=torch.uint8, device=DEV)
    qa.qa_token_logprob(code_of(t), T, V, x, V + pad, target, 0, logprob, entropy, stats, None, None, ws)
    a, e = (torch.randn(T, generator=gen, device=DEV) for _ in range(2))
    some = some_of(T)
    x64, y = x[some.to(DEV), :V].cpu().to(F64), target[some.to(DEV)].cpu()

    def run(pieces):
        from_ = x.clone() if in_place else x
        out = from_ if in_place else torch.full((T, V + pad), 5.0, dtype=TYPES[t], device=DEV)
        for i, j in pieces:
            qa.qa_token_logprob_grad(code_of(t), j - i, V, from_[i:], V + pad, target[i:], stats[i:], entropy[i:], a[i:], e[i:], out[i:], V + pad)
        assert (out[:, V:] == (50.0 if in_place else 5.0)).all()
        return out

    out = run([(0, T)])
    # equal numbers: a zero's sign depends on whether its vector of eight has the target, and pieces begin elsewhere in a third
    assert torch.equal(out, run(thirds(T)))
    _, entropy64, stats64, logp = ref.token_logprob(x64, y)
    a64, e64 = a[some.to(DEV)].cpu().to(F64), e[some.to(DEV)].cpu().to(F64)
    want = ref.token_logprob_grad(x64, y, a64, e64)
    p = torch.exp(logp)
    reach = torch.where(p == 0, torch.zeros_like(p), (logp - entropy64[:, None]).abs()) + 1
    units = torch.nan_to_num(logp, 0, 0, 0).abs() + stats64[:, 1:] + 4
    # stats and entropy are the call's own, good to SUM of the largest |log p| that enters them
    off = p * (a64.abs()[:, None] + e64.abs()[:, None] * reach) * (2.0 ** -21 * units + 4 * SUM * units) + 2.0 ** -23 * a64.abs()[:, None]
    tiny = 2.0 ** -24 if t == "f16" else 0.0
    assert ((out[some.to(DEV), :V].cpu().to(F64) - want).abs() <= HALF_ULP[t] * 1.01 * want.abs() + off + tiny).all()
