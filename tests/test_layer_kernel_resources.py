"""Compile-time guard for the kernels of products: waves and LDS that their forms count on, scratch only outside the loop (tiles of
256 x 256 use all 512 registers of a lane, and their results' addresses a few words more), and a loop that waits for what it counts."""
import os
import re
import subprocess

import pytest

from test_kernel_resources import CSRC, ROOT


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """Per source: resources of its kernels, and the assembly."""
    import __graft_entry__ as entry
    tmp = tmp_path_factory.mktemp("asm")
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    running = {}
    for source in ("qa_output.hip", "qa_orthogonal.hip"):
        running[source] = subprocess.Popen(["hipcc", *flags, "--cuda-device-only", "-S", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(CSRC, source),
                                            "-o", str(tmp / source) + ".s", "-Rpass-analysis=kernel-resource-usage"], stderr=subprocess.PIPE, text=True)
    out = {}
    pattern = (r"Function Name: (\S+).*?VGPRs: (\d+).*?ScratchSize \[bytes/lane\]: (\d+)"
               r".*?Occupancy \[waves/SIMD\]: (\d+).*?LDS Size \[bytes/block\]: (\d+)")
    for source, p in running.items():
        said = p.communicate()[1]
        assert p.returncode == 0, said[-2000:]
        kernels = {m.group(1): dict(scratch=int(m.group(3)), waves=int(m.group(4)), lds=int(m.group(5))) for m in re.finditer(pattern, said, re.S)}
        out[source] = kernels, open(str(tmp / source) + ".s").read()
    return out


def form(name):
    """(WM, WN, FM, FN, SHARE) of a product kernel's tiles."""
    return tuple(int(v) for v in re.search(r"4LiesE\dELS2_\dELi(\d)ELi(\d)ELi(\d)ELi(\d)ELi(\d)E", name).groups())


def test_products(compiled):
    seen = set()
    for kernels, _ in compiled.values():
        for name, v in kernels.items():
            if "product_kernel" not in name:
                continue
            f = form(name)
            seen.add(f)
            assert v["lds"] <= 160 * 1024, name
            assert v["scratch"] <= (256 if f[2] * f[3] == 16 else 0), (name, v)
            # what LDS leaves room for, two of which registers have to
            room = (160 * 1024 // v["lds"]) * f[0] * f[1] * f[4] // 4
            assert v["waves"] >= min(room, 1 if f[2] * f[3] == 16 else 2), (name, v)
    assert {(2, 2, 4, 4, 1), (2, 2, 3, 3, 1), (2, 2, 2, 2, 1), (2, 2, 2, 2, 2), (2, 2, 1, 1, 2), (1, 1, 2, 2, 4), (4, 1, 2, 2, 1)} == seen


def test_the_others(compiled):
    output, orthogonal = (compiled[s][0] for s in ("qa_output.hip", "qa_orthogonal.hip"))
    small = {k: v for k, v in orthogonal.items() if "small_kernel" in k}
    assert len(small) == 16
    assert all(v["scratch"] == 0 and v["waves"] >= 4 for v in small.values()), small
    stream = {k: v for k, v in output.items() if "stream_kernel" in k}
    assert len(stream) == 9 and all(v["waves"] >= 4 and v["lds"] <= 80 * 1024 and v["scratch"] <= 80 for v in stream.values()), stream
    rest = {k: v for k, v in {**output, **orthogonal}.items() if "product_kernel" not in k and "stream_kernel" not in k}
    assert rest and not {k: v for k, v in rest.items() if v["scratch"]}


@pytest.mark.parametrize("source,least", [("qa_output.hip", 60), ("qa_orthogonal.hip", 30)])
def test_loops_of_products_wait_for_what_they_count(compiled, source, least):
    """The loop's barrier waits until a known number of loads is on its way: there is no other access of memory in the loop (a spill would be
    one), and no other wait for loads, which the compiler would set in front of reads of LDS if it took the buffers for one."""
    bodies = re.findall(r"^(\S*product_kernel\S*):[^\n]*\n(.*?)\n\.Lfunc_end", compiled[source][1], re.M | re.S)
    assert len(bodies) >= least
    for name, body in bodies:
        lines = body.split("\n")
        labels = {m.group(1): i for i, m in enumerate(re.match(r"(\.LBB\d+_\d+):", line) for line in lines) if m}
        loops = []
        for i, line in enumerate(lines):
            to = re.search(r"\bs_c?branch\w* (\.LBB\d+_\d+)", line)
            # (a block may also stand behind the function's end and branch back)
            if to and labels.get(to.group(1), i + 1) <= i and "Loop Header" in lines[labels[to.group(1)]]:
                loop = "\n".join(lines[labels[to.group(1)]:i + 1])
                if "v_mfma" in loop:
                    loops.append(loop)
        assert len(loops) == 1, (name, len(loops))
        assert not re.search(r"scratch_|global_load_(?!lds)|global_store|buffer_|flat_", loops[0]), name
        waits = re.findall(r"vmcnt\((\d+)\)", loops[0])
        assert loops[0].count("s_barrier") == 1 and len(waits) == 1 and int(waits[0]) > 0, (name, waits)
