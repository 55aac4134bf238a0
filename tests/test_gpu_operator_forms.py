"""Forms of the operators on activations and logits that only some sizes and values reach, against the formulas in 64 bits.

Tolerances are those of tests/test_gpu_operators.py: u = 2^-24 is binary32's rounding, and a sum in binary32 that is added in trees
and in runs of at most some hundred terms is off by at most SUM = 64 u of the sum of its terms' magnitudes."""
import math

import pytest
import torch

import operator_reference as ref
from weight_grad_shapes import FEW, LARGE, LARGE_SPLIT, SMALL

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    from test_gpu_operators import F64, SUM, TYPES, check_token, code_of, coded_rows, gen_of
    DEV = torch.device("cuda:0")


# ---- rows in 8 bits ------------------------------------------------------------------------------------------------


def test_error_of_a_code():
    """Half a scale, and 1/127 of the group's largest magnitude; at the largest scale less than a whole one, and 1/64."""
    gen = gen_of("error")
    most = torch.exp2(torch.randint(-115, 128, (3000, 1), generator=gen).double()) * (1 + torch.rand(3000, 1, generator=gen).double())
    most[-600:] = 2.0 ** 127 * (1.9 + 0.1 * torch.rand(600, 1, generator=gen).double())
    x = (most.clamp(max=torch.finfo(torch.float32).max) * (2 * torch.rand(3000, 32, generator=gen) - 1).double()).float()
    x[:, 7] = most.clamp(max=torch.finfo(torch.float32).max)[:, 0].float()
    L, codes, scales = coded_rows(3000, 32, 32)
    qa.qa_rows_pack(L, qa.QA_F32, x.to(DEV), 32, codes, scales)
    s = scales[:, :1].cpu().long()
    off = (ref.decode(codes[:, :32].cpu(), s, 32) - x.to(F64)).abs() / torch.exp2((s - 127).to(F64))
    share = (ref.decode(codes[:, :32].cpu(), s, 32) - x.to(F64)).abs() / x.to(F64).abs().amax(dim=1, keepdim=True)
    last = (s == 249)[:, 0]
    assert last.sum() > 50 and (off[last] < 1).all() and (share[last] < 1 / 64).all()
    assert (off[~last] <= 0.5).all() and (share[~last] <= 1 / 127).all()


# ---- weight gradient ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,N,K", [SMALL, FEW, LARGE[1]])
def test_weight_grad_of_groups_with_the_largest_scales(t, T, N, K):
    """Groups whose largest magnitude is up to binary32's largest number, with zeros beside it: their codes stand for finite
    values, and dY is small enough that every sum is finite.  An infinity makes its group's columns NaN and no others."""
    gen = gen_of("scales", t, T, N, K)
    G = -(-K // 32)
    tops = torch.tensor([0.0, 1.0, 127 * 2.0 ** 119, 127 * 2.0 ** 120, 127 * 2.0 ** 121, 1.2 * 2.0 ** 127, torch.finfo(torch.float32).max])
    most = tops[torch.randint(0, len(tops), (T, G), generator=gen)].repeat_interleave(32, dim=1)[:, :K]
    x = most * (2 * torch.rand(T, K, generator=gen) - 1) * (torch.rand(T, K, generator=gen) < 0.8)
    x[:, ::32] = most[:, ::32]
    x[3, 70] = math.inf
    dy = (1e-3 * torch.randn(T, N, generator=gen)).to(TYPES[t])
    L, codes, scales = coded_rows(T, K, 32)
    qa.qa_rows_pack(L, qa.QA_F32, x.to(DEV), K, codes, scales)
    s = scales[:, :G].cpu().long()
    assert all((s == b).any() for b in (0 + 1, 246, 247, 248, 249, 255))
    values = ref.decode(codes[:, :K].cpu(), s, 32)
    bad = torch.zeros(K, dtype=torch.bool)
    bad[64:96] = True
    assert torch.equal(torch.isnan(values).any(dim=0), bad)
    ws = torch.empty(max(1, qa.qa_rows_workspace_bytes(L, qa.QA_OP_WEIGHT_GRAD, code_of(t), N)), dtype=torch.uint8, device=DEV)
    dw = torch.empty(N, K, device=DEV)
    qa.qa_rows_weight_grad(L, codes, scales, code_of(t), dy.to(DEV), N, N, dw, K, 0, ws)
    assert (~torch.isfinite(dw[:, bad.to(DEV)])).all()
    values, dy = torch.nan_to_num(values).to(DEV), dy.to(F64).to(DEV)
    want, each = dy.t().contiguous() @ values, dy.abs().t().contiguous() @ values.abs()
    ok = (dw.to(F64) - want).abs() <= SUM * each
    assert ok[:, ~bad.to(DEV)].all()


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,N,K", LARGE + LARGE_SPLIT)
@pytest.mark.parametrize("accumulate", [0, 1])
def test_weight_grad_of_large_tiles(t, T, N, K, accumulate):
    """Rows, columns of dY and of X that end inside a tile, in one piece and split, against a product in 64 bits; one row to
    the last bit, where a product of dY's 8 or 11 bits and a code's 7 is a binary32 number."""
    gen = torch.Generator(device=DEV).manual_seed(T + N)
    x = 2 * torch.randn(T, K, generator=gen, device=DEV)
    pad = N % 3
    dy = (0.1 * torch.randn(T, N + pad, generator=gen, device=DEV)).to(TYPES[t])[:, :N]
    L, codes, scales = coded_rows(T, K, 64)
    qa.qa_rows_pack(L, qa.QA_F32, x, K, codes, scales)
    values = torch.empty(T, K, device=DEV)
    qa.qa_rows_unpack(L, codes, scales, qa.QA_F32, values, K)
    need = qa.qa_rows_workspace_bytes(L, qa.QA_OP_WEIGHT_GRAD, code_of(t), N)
    assert (need > 0) == ((T, N, K) in LARGE_SPLIT)
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV) if need else None
    got = []
    for _ in range(2):
        dw = torch.full((N, K + 1), 0.25, device=DEV)
        qa.qa_rows_weight_grad(L, codes, scales, code_of(t), dy, N + pad, N, dw, K + 1, accumulate, ws)
        got.append(dw)
    assert torch.equal(*got) and (dw[:, K] == 0.25).all()
    want = dy.double().t().contiguous() @ values.double() + 0.25 * accumulate
    each = dy.double().abs().t().contiguous() @ values.double().abs() + 0.25 * accumulate
    assert ((dw[:, :K].double() - want).abs() <= SUM * each).all()
    if T == 1 and not accumulate and t != "f32":
        assert torch.equal(dw[:, :K], want.float())


def test_weight_grad_of_large_tiles_keeps_every_bit_of_dy():
    """One row of codes that are powers of two: each product has the 24 bits of a binary32 number."""
    _, N, K = LARGE[0]
    gen = gen_of("bits of large tiles")
    dy = torch.randn(1, N, generator=gen) * torch.exp2(torch.randint(-60, 60, (1, N), generator=gen).float())
    x = torch.exp2(torch.randint(-6, 1, (1, K), generator=gen).float())
    x[:, ::32] = 1.0
    L, codes, scales = coded_rows(1, K, 32)
    qa.qa_rows_pack(L, qa.QA_F32, x.to(DEV), K, codes, scales)
    dw = torch.empty(N, K, device=DEV)
    qa.qa_rows_weight_grad(L, codes, scales, qa.QA_F32, dy.to(DEV), N, N, dw, K, 0, None)
    assert torch.equal(dw.cpu(), dy.t() @ x)


@pytest.mark.parametrize("T,N,K", [SMALL, LARGE[1]])
def test_weight_grad_of_the_smallest_numbers(T, N, K):
    """binary32 elements of dY lose what lies below 2^-133, and bfloat16 ones nothing."""
    gen = gen_of("smallest", T, N, K)
    dy = torch.zeros(T, N)
    dy[0] = torch.randn(N, generator=gen) * torch.exp2(torch.randint(-140, -100, (N,), generator=gen).double()).float()
    L, codes, scales = coded_rows(T, K, 32)
    qa.qa_rows_pack(L, qa.QA_F32, torch.full((T, K), 2.0 ** 100, device=DEV), K, codes, scales)
    for t, lost in (("f32", 2.0 ** -133), ("bf16", 0.0)):
        d = dy.to(TYPES[t])
        dw = torch.empty(N, K, device=DEV)
        ws = torch.empty(max(1, qa.qa_rows_workspace_bytes(L, qa.QA_OP_WEIGHT_GRAD, code_of(t), N)), dtype=torch.uint8, device=DEV)
        qa.qa_rows_weight_grad(L, codes, scales, code_of(t), d.to(DEV), N, N, dw, K, 0, ws)
        assert ((dw[:, 0].cpu().to(F64) * 2.0 ** -100 - d[0].to(F64)).abs() <= lost).all()
        assert (dw == dw[:, :1]).all()


# ---- log probabilities of long rows ----------------------------------------------------------------------------------


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(1, 131073), (1, 199999), (3, 200001), (2, 1_100_003)])
@pytest.mark.parametrize("top", [0, 1, 64])
def test_token_logprob_of_more_splits_than_lanes(t, T, V, top):
    """65 to 512 splits of a row: the join's bound comes from several of them per lane."""
    gen = gen_of("splits", t, T, V, top)
    x = (3 * torch.randn(T, V, generator=gen)).to(TYPES[t])
    target = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    need = qa.qa_token_workspace_bytes(T, V, top)
    assert 64 < need // (T * (16 + 8 * top)) <= 512
    check_token(t, x, target, top, pad=V % 2, lead=V % 3)
    if T > 1:                                          # all of one row's best in one split, ties, a mask that leaves nothing
        x[0] = -math.inf
        x[1, : V // 2] = 1.0
        x[1, V // 2:] = -2.0
        x[T - 1, 5000:5100] = 30.0 + torch.arange(100) % 7
        check_token(t, x, target, top)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("V", [196_609, 200_000])
@pytest.mark.parametrize("top", [0, 20])
def test_token_logprob_of_many_rows_that_are_too_long_for_one_piece(t, V, top):
    """More chunks than a work-group notes: split although there are rows enough.  Rows against their copies' bits, at the same place
    inside 16 bytes, and some in 64 bits."""
    T, stride = 260, -(-V // 8) * 8
    gen = torch.Generator(device=DEV).manual_seed(V)
    x = torch.full((T, stride), 50.0, dtype=TYPES[t], device=DEV)[:, :V]
    x.copy_(3 * torch.randn(T, V, generator=gen, device=DEV))
    x[T // 2:] = x[:T // 2].clone()
    x[7] = -math.inf
    x[9, : V - 40] = -math.inf
    x[11] = 2.0
    target = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    target[T // 2:] = target[:T // 2].clone()
    need = qa.qa_token_workspace_bytes(T, V, top)
    assert need == T * 2 * (16 + 8 * top)
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV)
    logprob, entropy, stats = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV)
    best, index = torch.empty(T, top, device=DEV), torch.empty(T, top, dtype=torch.int32, device=DEV)
    qa.qa_token_logprob(code_of(t), T, V, x, stride, target, top, logprob, entropy, stats, best if top else None, index if top else None, ws)
    keep = [i for i in range(T // 2) if i not in (7, 9, 11)]
    for v in (logprob, entropy, stats, best, index):
        assert torch.equal(v[:T // 2][keep], v[T // 2:][keep])
    some = torch.tensor([0, 1, 7, 9, 11, T - 1])
    x64, y = x[some.to(DEV)].cpu().to(F64), target[some.to(DEV)].cpu()
    lp, want_h, want_s, logp = ref.token_logprob(x64, y)
    logprob, entropy, stats, best, index = (v[some.to(DEV)].cpu().to(F64) for v in (logprob, entropy, stats, best, index))
    near = lambda a, b: ((a - b).abs() <= 2 * SUM + 2.0 ** -22 * (b.abs() + 20)) | (a == b)  # noqa: E731
    assert torch.equal(stats[:, 0], want_s[:, 0]) and near(stats[:, 1], want_s[:, 1]).all() and near(logprob, lp).all()
    assert ((entropy - want_h).abs() <= SUM * (8 + 2 * want_h)).all()
    assert torch.equal(index.long(), ref.top(x64, top)) and near(best, logp.gather(1, index.long())).all()


def test_token_logprob_of_more_splits_than_the_bound_looks_at():
    """A row of more than 512 pieces: the bound comes from the first 512, and the best may lie in the others."""
    V, top = 512 * 196_608 + 12_345, 20
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(1, V, generator=gen, device=DEV)
    places = torch.tensor([5, 196_608, 100_000_000, V - 12_000, V - 1, V // 2])
    x[0, places.to(DEV)] = torch.tensor([9.0, 9.0, 11.0, 10.0, 12.0, 8.5], device=DEV)
    need = qa.qa_token_workspace_bytes(1, V, top)
    assert need == 513 * (16 + 8 * top)
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV)
    target = torch.tensor([V - 1], dtype=torch.int32, device=DEV)
    logprob, entropy, stats = torch.empty(1, device=DEV), torch.empty(1, device=DEV), torch.empty(1, 2, device=DEV)
    best, index = torch.empty(1, top, device=DEV), torch.empty(1, top, dtype=torch.int32, device=DEV)
    qa.qa_token_logprob(qa.QA_F32, 1, V, x, V, target, top, logprob, entropy, stats, best, index, ws)
    x64 = x.double()
    log_sum = torch.log(torch.exp(x64 - 12.0).sum())
    logp = x64 - 12.0 - log_sum
    want_h = -(torch.exp(logp) * logp).sum()
    order = torch.sort(x64[0], descending=True, stable=True).indices[:top]
    assert torch.equal(index[0].long(), order) and float(stats[0, 0]) == 12.0
    slack = 2 * SUM + 2.0 ** -22 * 40
    assert abs(float(stats[0, 1] - log_sum)) <= slack and abs(float(logprob[0] - logp[0, V - 1])) <= slack
    assert (best[0] - logp[0, order]).abs().max() <= slack and abs(float(entropy[0] - want_h)) <= SUM * (8 + 2 * float(want_h))
