"""Forms of the operators on activations and logits that only some sizes and values reach, against the formulas in 64 bits.

Tolerances are those of tests/test_gpu_operators.py: u = 2^-24 is binary32's rounding, and a sum in binary32 that is added in trees
and in runs of at most some hundred terms is off by at most SUM = 64 u of the sum of its terms' magnitudes."""
import math

import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2208_05631_amd as qa
    from test_gpu_operators import F64, SUM, TYPES, code_of, coded_rows, gen_of
    DEV = torch.device("cuda:0")


# ---- weight gradient ---------------------------------------------------------------------------------------------

# Small tiles, and large ones.
SMALL, LARGE = (70, 40, 200), (70, 4099, 4100)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,N,K", [SMALL, (70, 5, 200), LARGE])
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
