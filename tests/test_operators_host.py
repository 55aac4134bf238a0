"""Host-side checks of the operators on activations and logits that need no GPU: sizes of workspaces, and refusals
before anything is launched."""
import ctypes as C

import pytest

qa = pytest.importorskip("paper_2208_05631_amd", reason="libqadagrad.so not built")
from paper_2208_05631_amd import binding as B  # noqa: E402

FAKE = 0x10000        # non-null and aligned, never dereferenced: checks fail first
F32, BF16, F16 = qa.QA_F32, qa.QA_BF16, qa.QA_F16
INVALID, ALIGNMENT, WORKSPACE = -1, -2, -3

BAD_ROWS = [qa.CodedRows(-1, 64, 32, 64, 2), qa.CodedRows(1 << 31, 64, 32, 64, 2), qa.CodedRows(4, 0, 32, 64, 2),
            qa.CodedRows(4, 1 << 24, 32, 1 << 24, 1 << 20), qa.CodedRows(4, 64, 48, 64, 2), qa.CodedRows(4, 64, 16, 64, 4),
            qa.CodedRows(4, 64, 32, 48, 2), qa.CodedRows(4, 60, 32, 60, 2), qa.CodedRows(4, 65, 32, 80, 2)]


def rows(**change):
    r = qa.CodedRows.make(4, 100, 32)
    for k, v in change.items():
        setattr(r, k, v)
    return r


def call(name, L, **change):
    """The entry point with arguments that pass every check, but for `change`."""
    p = C.byref(L) if isinstance(L, qa.CodedRows) else L
    args = {
        "qa_rows_pack": dict(rows=p, type=BF16, x=FAKE, x_stride=100, codes=FAKE, scales=FAKE, stream=None),
        "qa_rows_unpack": dict(rows=p, codes=FAKE, scales=FAKE, type=BF16, x=FAKE, x_stride=100, stream=None),
        "qa_rows_weight_grad": dict(rows=p, codes=FAKE, scales=FAKE, type=BF16, dy=FAKE, dy_stride=7, n=7, dw=FAKE, dw_stride=100,
                                    accumulate=0, ws=None, ws_bytes=0, stream=None),
        "qa_rms_norm": dict(rows=p, type=BF16, x=FAKE, x_stride=100, residual=FAKE, residual_stride=100, weight=FAKE, eps=1e-6,
                            h=FAKE, h_stride=100, codes=FAKE, scales=FAKE, y=FAKE, y_stride=100, rstd=FAKE, stream=None),
        "qa_rms_norm_grad": dict(rows=p, type=BF16, dy=FAKE, dy_stride=100, h=FAKE, h_stride=100, codes=None, scales=None, weight=FAKE,
                                 rstd=FAKE, dh=FAKE, dh_stride=100, dx=FAKE, dx_stride=100, dweight=FAKE, accumulate=0, ws=FAKE,
                                 ws_bytes=1 << 20, stream=None),
        "qa_token_logprob": dict(type=BF16, rows=4, vocab=100, logits=FAKE, stride=100, target=FAKE, top=5, logprob=FAKE, entropy=FAKE,
                                 stats=FAKE, top_logprob=FAKE, top_index=FAKE, ws=None, ws_bytes=0, stream=None),
        "qa_token_logprob_grad": dict(type=BF16, rows=4, vocab=100, logits=FAKE, stride=100, target=FAKE, stats=FAKE, entropy=FAKE,
                                      g_logprob=FAKE, g_entropy=FAKE, dlogits=FAKE, dlogits_stride=100, stream=None),
    }[name]
    assert set(change) <= set(args), change
    args.update(change)
    return getattr(B._lib, name)(*args.values())


@pytest.mark.parametrize("name", ["qa_rows_pack", "qa_rows_unpack", "qa_rows_weight_grad", "qa_rms_norm", "qa_rms_norm_grad"])
def test_rows_that_no_call_takes(name):
    for bad in BAD_ROWS:
        assert call(name, bad) == INVALID
        assert qa.qa_rows_workspace_bytes(bad, qa.QA_OP_NORM_GRAD, BF16) == 0
    assert call(name, None) == INVALID
    assert call(name, rows(), type=3) == INVALID and call(name, rows(), type=-1) == INVALID


def test_pack_and_unpack():
    for name in ("qa_rows_pack", "qa_rows_unpack"):
        assert call(name, rows(), x_stride=99) == INVALID
        for k in ("x", "codes", "scales"):
            assert call(name, rows(), **{k: None}) == INVALID
        assert call(name, rows(), x=FAKE + 1) == ALIGNMENT
        assert call(name, rows(), type=F32, x=FAKE + 2) == ALIGNMENT
        assert call(name, rows(), codes=FAKE + 8) == ALIGNMENT


def test_weight_grad():
    name = "qa_rows_weight_grad"
    for bad in (dict(n=0), dict(n=8), dict(n=1 << 24, dy_stride=1 << 24), dict(dw_stride=99), dict(accumulate=2), dict(dw=None), dict(dy=None),
                dict(codes=None), dict(scales=None)):
        assert call(name, rows(), **bad) == INVALID, bad
    for bad in (dict(dy=FAKE + 1), dict(dw=FAKE + 2), dict(codes=FAKE + 4)):
        assert call(name, rows(), **bad) == ALIGNMENT, bad
    long = qa.CodedRows.make(10000, 100, 32)
    need = qa.qa_rows_workspace_bytes(long, qa.QA_OP_WEIGHT_GRAD, BF16, 7)
    assert need >= 2 * 7 * 100 * 4
    assert call(name, long) == WORKSPACE and call(name, long, ws=FAKE, ws_bytes=need - 1) == WORKSPACE
    assert call(name, long, ws=FAKE + 16, ws_bytes=need) == ALIGNMENT
    assert qa.qa_rows_workspace_bytes(rows(), qa.QA_OP_WEIGHT_GRAD, BF16, 7) == 0            # few rows: one pass
    assert qa.qa_rows_workspace_bytes(long, qa.QA_OP_WEIGHT_GRAD, 9, 7) == 0
    assert qa.qa_rows_workspace_bytes(long, qa.QA_OP_WEIGHT_GRAD, BF16, 0) == 0
    assert qa.qa_rows_workspace_bytes(long, qa.QA_OP_STEP, BF16, 7) == 0


def test_norm():
    name = "qa_rms_norm"
    for bad in (dict(x_stride=99), dict(residual_stride=99), dict(h_stride=99), dict(y_stride=99), dict(eps=-1e-6), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(x=None), dict(weight=None), dict(codes=None), dict(scales=None), dict(codes=None, scales=None, y=None)):
        assert call(name, rows(), **bad) == INVALID, bad
    for bad in (dict(x=FAKE + 1), dict(residual=FAKE + 1), dict(h=FAKE + 1), dict(y=FAKE + 1), dict(weight=FAKE + 2), dict(rstd=FAKE + 2),
                dict(codes=FAKE + 8)):
        assert call(name, rows(), **bad) == ALIGNMENT, bad


def test_norm_grad():
    name = "qa_rms_norm_grad"
    for bad in (dict(dy_stride=99), dict(h_stride=99), dict(dh_stride=99), dict(dx_stride=99), dict(accumulate=-1), dict(dy=None), dict(weight=None),
                dict(rstd=None), dict(dx=None), dict(h=None), dict(codes=FAKE, scales=FAKE), dict(h=None, codes=FAKE),
                dict(h=None, scales=FAKE), dict(scales=FAKE)):
        assert call(name, rows(), **bad) == INVALID, bad
    for bad in (dict(dy=FAKE + 1), dict(h=FAKE + 1), dict(dh=FAKE + 1), dict(dx=FAKE + 1), dict(weight=FAKE + 2), dict(rstd=FAKE + 2),
                dict(dweight=FAKE + 2), dict(h=None, codes=FAKE + 8, scales=FAKE), dict(ws=FAKE + 16)):
        assert call(name, rows(), **bad) == ALIGNMENT, bad
    need = qa.qa_rows_workspace_bytes(rows(), qa.QA_OP_NORM_GRAD, BF16)
    assert need >= 100 * 4
    assert call(name, rows(), ws=None) == WORKSPACE and call(name, rows(), ws_bytes=need - 1) == WORKSPACE


def test_token_logprob():
    name = "qa_token_logprob"
    for bad in (dict(type=3), dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=1 << 31, stride=1 << 31), dict(stride=99), dict(top=-1),
                dict(top=65), dict(vocab=4), dict(logits=None), dict(target=None), dict(logprob=None), dict(top_logprob=None), dict(top_index=None)):
        assert call(name, None, **bad) == INVALID, bad
    for bad in (dict(logits=FAKE + 1), dict(target=FAKE + 2), dict(logprob=FAKE + 2), dict(entropy=FAKE + 2), dict(stats=FAKE + 2),
                dict(top_logprob=FAKE + 2), dict(top_index=FAKE + 2)):
        assert call(name, None, **bad) == ALIGNMENT, bad
    need = qa.qa_token_workspace_bytes(1, 100000, 5)
    assert need > 0 and qa.qa_token_workspace_bytes(1, 100, 5) == 0 and qa.qa_token_workspace_bytes(4096, 100000, 5) == 0
    long = dict(rows=1, vocab=100000, stride=100000)
    assert call(name, None, **long) == WORKSPACE and call(name, None, **long, ws=FAKE, ws_bytes=need - 1) == WORKSPACE
    assert call(name, None, **long, ws=FAKE + 8, ws_bytes=need) == ALIGNMENT
    assert qa.qa_token_workspace_bytes(1, 100000, 65) == 0 and qa.qa_token_workspace_bytes(1, 3, 4) == 0


def test_token_logprob_grad():
    name = "qa_token_logprob_grad"
    for bad in (dict(type=7), dict(rows=-1), dict(vocab=0), dict(stride=99), dict(dlogits_stride=99), dict(logits=None), dict(stats=None),
                dict(dlogits=None), dict(entropy=None), dict(g_entropy=None)):
        assert call(name, None, **bad) == INVALID, bad
    for bad in (dict(logits=FAKE + 1), dict(dlogits=FAKE + 1), dict(target=FAKE + 2), dict(stats=FAKE + 2), dict(entropy=FAKE + 2),
                dict(g_logprob=FAKE + 2), dict(g_entropy=FAKE + 2)):
        assert call(name, None, **bad) == ALIGNMENT, bad
