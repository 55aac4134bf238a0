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
    from test_gpu_operators import F64, SUM, TYPES, code_of, coded_rows, gen_of
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
