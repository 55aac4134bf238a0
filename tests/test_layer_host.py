"""Host-side checks of the output layer's operators and of the orthogonal step that need no GPU: sizes of workspaces, and refusals
before anything is launched."""
import ctypes as C
import math

import pytest

qa = pytest.importorskip("paper_2208_05631_amd", reason="libqadagrad.so not built")
from paper_2208_05631_amd import binding as B  # noqa: E402

FAKE = 0x10000        # non-null and aligned, never dereferenced: checks fail first
F32, BF16, F16 = qa.QA_F32, qa.QA_BF16, qa.QA_F16
INVALID, ALIGNMENT, WORKSPACE = -1, -2, -3

BAD_LAYERS = [qa.OutputLayer(-1, 10, 8, 8, 8), qa.OutputLayer(1 << 24, 10, 8, 8, 8), qa.OutputLayer(4, 0, 8, 8, 8), qa.OutputLayer(4, 1 << 24, 8, 8, 8),
              qa.OutputLayer(4, 10, 0, 8, 8), qa.OutputLayer(4, 10, 1 << 20, 1 << 20, 1 << 20), qa.OutputLayer(4, 10, 8, 7, 8),
              qa.OutputLayer(4, 10, 8, 8, 7), qa.OutputLayer(4, 10, 8, 1 << 40, 8), qa.OutputLayer(4, 10, 8, 8, 1 << 40)]
BAD_MATRICES = [qa.Matrices(-1, 4, 4, 4, 16), qa.Matrices(1 << 16, 4, 4, 4, 16), qa.Matrices(1, 0, 4, 4, 16), qa.Matrices(1, 1 << 20, 4, 4, 1 << 22),
                qa.Matrices(1, 4, 0, 4, 16), qa.Matrices(1, 4, 1 << 20, 1 << 20, 1 << 22), qa.Matrices(1, 4, 4, 3, 16), qa.Matrices(2, 4, 4, 4, 15),
                qa.Matrices(1, 4, 4, 1 << 40, 16), qa.Matrices(2, 4, 4, 4, 1 << 56)]


def call(name, what, **change):
    """The entry point with arguments that pass every check, but for `change`."""
    p = C.byref(what) if what is not None else None
    args = {
        "qa_output_logprob": dict(layer=p, type=BF16, x=FAKE, w=FAKE, target=FAKE, logprob=FAKE, entropy=FAKE, stats=FAKE, ws=FAKE, ws_bytes=1 << 40, stream=None),
        "qa_output_logprob_grad": dict(layer=p, type=BF16, x=FAKE, w=FAKE, target=FAKE, stats=FAKE, entropy=FAKE, g_logprob=FAKE, g_entropy=FAKE, dx=FAKE,
                                       dx_stride=100, dw=FAKE, dw_stride=100, accumulate=0, ws=FAKE, ws_bytes=1 << 40, stream=None),
        "qa_orthogonalize": dict(matrices=p, type=BF16, g=FAKE, steps=5, coefficients=None, out=FAKE, ws=FAKE, ws_bytes=1 << 40, stream=None),
        "qa_step_orthogonal": dict(matrices=p, g=FAKE, momentum=FAKE, x=FAKE, mu=0.9, nesterov=1, steps=5, coefficients=None, eta=0.1, shrink=1.0, ws=FAKE,
                                   ws_bytes=1 << 40, stream=None),
    }[name]
    assert set(change) <= set(args), change
    args.update(change)
    return getattr(B._lib, name)(*args.values())


def layer(**change):
    v = qa.OutputLayer.make(4, 50, 100)
    for k, x in change.items():
        setattr(v, k, x)
    return v


def matrices(**change):
    v = qa.Matrices.make(2, 200, 300)
    for k, x in change.items():
        setattr(v, k, x)
    return v


@pytest.mark.parametrize("name,op", [("qa_output_logprob", qa.QA_OP_LOGPROB), ("qa_output_logprob_grad", qa.QA_OP_LOGPROB_GRAD)])
def test_layers_that_no_call_takes(name, op):
    for bad in BAD_LAYERS:
        assert call(name, bad) == INVALID
        assert qa.qa_output_workspace_bytes(bad, op, BF16) == 0
    assert call(name, None) == INVALID and call(name, layer(), type=3) == INVALID and call(name, layer(), type=-1) == INVALID
    assert qa.qa_output_workspace_bytes(layer(), op, 3) == 0 and qa.qa_output_workspace_bytes(layer(), qa.QA_OP_STEP, BF16) == 0
    assert qa.qa_output_workspace_bytes(layer(rows=0), op, BF16) == 0
    for t in (F32, BF16, F16):
        need = qa.qa_output_workspace_bytes(layer(), op, t)
        assert need > 0 and need % 256 == 0
        assert call(name, layer(), type=t, ws=None) == WORKSPACE and call(name, layer(), type=t, ws_bytes=need - 1) == WORKSPACE
    assert call(name, layer(), ws=FAKE + 16) == ALIGNMENT


def test_output_logprob():
    name = "qa_output_logprob"
    for bad in (dict(x=None), dict(w=None), dict(target=None), dict(logprob=None)):
        assert call(name, layer(), **bad) == INVALID, bad
    for bad in (dict(x=FAKE + 1), dict(w=FAKE + 1), dict(type=F32, x=FAKE + 2), dict(type=F32, w=FAKE + 2), dict(target=FAKE + 2), dict(logprob=FAKE + 2),
                dict(entropy=FAKE + 2), dict(stats=FAKE + 2)):
        assert call(name, layer(), **bad) == ALIGNMENT, bad
    assert call(name, layer(rows=0), x=None, w=None, ws=None, ws_bytes=0) == 0


def test_output_logprob_grad():
    name = "qa_output_logprob_grad"
    for bad in (dict(x=None), dict(w=None), dict(stats=None), dict(entropy=None), dict(g_entropy=None), dict(target=None), dict(dx=None, dw=None),
                dict(dx_stride=99), dict(dw_stride=99), dict(accumulate=2), dict(accumulate=-1)):
        assert call(name, layer(), **bad) == INVALID, bad
    for bad in (dict(x=FAKE + 1), dict(w=FAKE + 1), dict(dx=FAKE + 1), dict(type=F32, dx=FAKE + 2), dict(dw=FAKE + 2), dict(target=FAKE + 2), dict(stats=FAKE + 2),
                dict(entropy=FAKE + 2), dict(g_logprob=FAKE + 2), dict(g_entropy=FAKE + 2)):
        assert call(name, layer(), **bad) == ALIGNMENT, bad


def test_workspaces_hold_no_logits_of_a_large_vocabulary():
    """8192 rows of a vocabulary of 2^20 would be 32 GiB of binary32 logits."""
    big = qa.OutputLayer.make(8192, 1 << 20, 1024)
    assert qa.qa_output_workspace_bytes(big, qa.QA_OP_LOGPROB, BF16) < 2 << 30
    assert qa.qa_output_workspace_bytes(big, qa.QA_OP_LOGPROB_GRAD, BF16) < 2 << 30
    many = layer(rows=(1 << 24) - 1, vocab=1 << 17)
    assert qa.qa_output_workspace_bytes(many, qa.QA_OP_LOGPROB, BF16) < 2 << 30


@pytest.mark.parametrize("name", ["qa_orthogonalize", "qa_step_orthogonal"])
def test_matrices_that_no_call_takes(name):
    for bad in BAD_MATRICES:
        assert call(name, bad) == INVALID
        assert qa.qa_orthogonal_workspace_bytes(bad, F32) == 0
    assert call(name, None) == INVALID
    for steps in (0, -1, qa.QA_ORTHOGONAL_STEPS_MAX + 1):
        assert call(name, matrices(), steps=steps) == INVALID
    for v in (64.0, -64.0, math.inf, math.nan):
        assert call(name, matrices(), coefficients=(C.c_float * 15)(*([1.0] * 14), v)) == INVALID
    need = qa.qa_orthogonal_workspace_bytes(matrices(), F32)
    assert need >= 2 * 200 * 300 * 4 and need % 256 == 0
    assert call(name, matrices(), ws=None) == WORKSPACE and call(name, matrices(), ws_bytes=need - 1) == WORKSPACE
    assert call(name, matrices(), ws=FAKE + 16) == ALIGNMENT
    assert qa.qa_orthogonal_workspace_bytes(matrices(), 7) == 0 and qa.qa_orthogonal_workspace_bytes(matrices(count=0), F32) == 0
    assert call(name, matrices(count=0), g=None, ws=None, ws_bytes=0) == 0


def test_small_matrices_need_no_workspace():
    for R, Cc in ((1, 1), (96, 96), (128, 128), (64, 512), (512, 64), (288, 96)):
        assert qa.qa_orthogonal_workspace_bytes(qa.Matrices.make(3, R, Cc), F32) == 0
    for R, Cc in ((129, 129), (64, 513), (128, 256)):
        assert qa.qa_orthogonal_workspace_bytes(qa.Matrices.make(3, R, Cc), F32) > 0


def test_orthogonalize():
    name = "qa_orthogonalize"
    assert call(name, matrices(), type=3) == INVALID
    for bad in (dict(g=None), dict(out=None)):
        assert call(name, matrices(), **bad) == INVALID, bad
    for bad in (dict(g=FAKE + 1), dict(out=FAKE + 1), dict(type=F32, g=FAKE + 2), dict(type=F32, out=FAKE + 2)):
        assert call(name, matrices(), **bad) == ALIGNMENT, bad
    with pytest.raises(ValueError):
        qa.qa_orthogonalize(matrices(), F32, None, 5, [(1.0, 0.0, 0.0)] * 4, None, None, stream=0)


def test_step_orthogonal():
    name = "qa_step_orthogonal"
    for bad in (dict(g=None), dict(x=None), dict(mu=-0.1), dict(mu=1.1), dict(mu=math.nan), dict(nesterov=2), dict(eta=-1.0), dict(eta=math.inf), dict(eta=math.nan),
                dict(shrink=-0.1), dict(shrink=1.5), dict(shrink=math.nan)):
        assert call(name, matrices(), **bad) == INVALID, bad
    for bad in (dict(g=FAKE + 2), dict(momentum=FAKE + 2), dict(x=FAKE + 2)):
        assert call(name, matrices(), **bad) == ALIGNMENT, bad


def test_a_gradients_workspace_does_not_grow_with_c():
    """c of 2^20 rows would be 4 GiB for 1024 words, in pieces of the vocabulary alone; copies and sums of a piece of the rows are what is left."""
    need = lambda rows, vocab, features, t: qa.qa_output_workspace_bytes(qa.OutputLayer.make(rows, vocab, features), qa.QA_OP_LOGPROB_GRAD, t)  # noqa: E731
    for rows in (1 << 16, (1 << 16) + 1, 100003, 1 << 20, (1 << 24) - 1):
        for t in (F32, BF16, F16):
            assert need(rows, 32768, 64, t) < 1 << 30
            assert need(rows, 50, 64, t) < 2 << 30
    assert need(1 << 20, 32768, 1024, BF16) < 2 << 30
    # two pieces of 35072 rows need no more than one of 65536
    for t in (F32, BF16, F16):
        assert need(70000, 32768, 64, t) <= need(1 << 16, 32768, 64, t)


def test_workspaces_of_matrices_are_what_the_header_says():
    up = lambda k: -(-k // 16) * 16  # noqa: E731
    for count, R, Cc in ((1, 1, 4096), (1, 4096, 1), (3, 2, 1024), (7, 17, 5000), (1, 300, 300), (2, 129, 129), (5000, 40, 600), (1, 4096, 8192)):
        n, m = min(R, Cc), max(R, Cc)
        least = count * 8 * up(n) * (up(m) + n)
        for t in (F32, BF16, F16):
            assert least <= qa.qa_orthogonal_workspace_bytes(qa.Matrices.make(count, R, Cc), t) <= least + count * 8192 + 1280
