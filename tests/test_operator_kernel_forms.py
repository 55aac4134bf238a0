"""Which kernels of the operators the library holds: every form is one that calls reach, and binary32 has none past the caches but
where it gains by it (a form that is compiled and not launched, or launched where it loses, shows here first)."""
import os
import re
import subprocess

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2208_05631_amd", "libqadagrad.so")
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def forms():
    if not os.path.exists(LIB):
        pytest.skip("libqadagrad.so not built")
    out = subprocess.run(["nm", "-C", LIB], check=True, capture_output=True, text=True).stdout
    found = {}
    for name, args in re.findall(r"__device_stub__(\w+)<([^<>]*)>", out):
        found.setdefault(name, set()).add(tuple({"true": True, "false": False}.get(a.strip(), a.strip()) for a in args.split(",")))
    return {k: {tuple(int(a) if isinstance(a, str) else a for a in f) for f in v} for k, v in found.items()
            if k.startswith(("rms_norm", "token_"))}


def test_norm(forms):
    assert {f[0] for f in forms["rms_norm_kernel"] if f[3]} == {BF16, F16}
    assert {f[0] for f in forms["rms_norm_grad_kernel"] if f[4]} == {BF16, F16}
    assert {f[0] for f in forms["rms_norm_kernel"] if not f[3]} == {F32, BF16, F16}


def test_token(forms):
    past = {(f[0], f[2]) for f in forms["token_wide_kernel"] if f[3]}                # type, alternatives
    assert past == {(F32, False), (BF16, False), (F16, False), (BF16, True), (F16, True)}
    assert {f[0] for f in forms["token_grad_kernel"] if f[2]} == {BF16, F16}
    assert {f[0] for f in forms["token_grad_narrow_kernel"] if f[1]} == {F32, BF16, F16}
