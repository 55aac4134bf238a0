"""Compile-time guard for the weight gradient's buffers in LDS: its kernels promise the compiler that the buffers of one step lie
apart, so that it may move reads of one across writes of another.  Kernels for binary32 and binary16 have two buffers, and may
speak of two only: a third name would be a second one for the buffer that the step writes."""
import collections
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2208_05631_amd", "csrc")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Per kernel: the names of memory known to lie apart that its accesses of LDS bear, by the step they belong to."""
    import __graft_entry__ as entry
    out = str(tmp_path_factory.mktemp("ir") / "weight_grad.ll")
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run(["hipcc", *flags, "--cuda-device-only", "-emit-llvm", "-S", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                    os.path.join(CSRC, "qa_weight_grad.hip"), "-o", out], check=True, capture_output=True)
    text = open(out).read()
    node = dict(re.findall(r"^!(\d+) = (.*)$", text, re.M))
    found = {}
    for m in re.finditer(r"^define [^\n]*@(\S*weight_grad_kernel\w*).*?\n}", text, re.M | re.S):
        names = collections.defaultdict(set)
        for line in m.group(0).split("\n"):
            scopes = re.search(r"!alias\.scope !(\d+)", line)
            if not scopes or not ("ds.read.tr" in line or re.search(r"(load|store) .*addrspace\(3\)", line)):
                continue
            for scope in re.findall(r"!(\d+)", node[scopes.group(1)]):
                itself, domain, name = re.match(r'distinct !\{!(\d+), !(\d+), !"(.*)"\}', node[scope]).groups()
                assert itself == scope
                names[domain, (re.search(r":It\d+$", name) or [""])[0]].add(scope)
        found[m.group(1)] = names
    return found


def test_steps_of_two_buffers_speak_of_two(kernels):
    two = {k: v for k, v in kernels.items() if re.search(r"weight_grad_kernelILi[02]E", k)}
    assert len(two) == 6 and all(two.values())
    assert max(len(s) for v in two.values() for s in v.values()) == 2


def test_steps_of_three_buffers_speak_of_three(kernels):
    three = {k: v for k, v in kernels.items() if "weight_grad_kernelILi1E" in k}
    assert len(three) == 3 and all(three.values())
    assert {max(len(s) for s in v.values()) for v in three.values()} == {3}
