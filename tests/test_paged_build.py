"""What the compiler made of the paged operators' kernels, and what their sources say of tensor memory: the CTAs that the launches count on
an SM fit its registers, nothing spills, and a kernel that allocates tensor memory, by the instruction or through the helper that issues
it, lets its successor start behind the allocation only."""
import glob
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21759_b200", "csrc")


def _kernels(source):
    """{kernel, template arguments: (registers per thread, spilled bytes)} of a source."""
    r = subprocess.run(["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xptxas", "-v", "-c", os.path.join(CSRC, source),
                        "-o", os.devnull], capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr[-2000:]
    out = {}
    for b in re.split(r"ptxas info\s*: Compiling entry function '", r.stderr)[1:]:
        m = re.search(r".*\d(paged_[a-z_]+_kernel)(I(?:L[ib]\d+E)+E)?", b.split("'", 1)[0])
        key = (m.group(1), *map(int, re.findall(r"L[ib](\d+)E", m.group(2) or "")))
        assert key not in out
        out[key] = (int(re.search(r"Used (\d+) registers", b).group(1)), sum(int(x) for x in re.findall(r"(\d+) bytes spill", b)))
    return out


LAUNCHES = {  # source: {kernel: (threads, CTAs on an SM)}
    "paged_layout.cu": {("paged_layout_kernel",): (256, 2)},
    "paged_store.cu": {("paged_store_kernel", d, i, w): (64, 14) for d in (64, 128) for i in (0, 1) for w in (0, 1)},
    "paged_attention.cu": {("paged_attention_kernel", d): (160, 2) for d in (64, 128)},
    "paged_attention_tc.cu": {("paged_attention_tc_kernel", d, q): (192 * q, 3 - q) for d in (64, 128) for q in (1, 2)}
    | {("paged_merge_kernel", d): (128, 8) for d in (64, 128)},
}


@pytest.mark.parametrize("source", LAUNCHES)
def test_kernels_fit_and_spill_nothing(source):
    seen = _kernels(source)
    assert set(seen) == set(LAUNCHES[source])
    for kernel, (threads, ctas) in LAUNCHES[source].items():
        registers, spills = seen[kernel]
        assert ctas * threads * (-(-registers // 8) * 8) <= 65536 and spills == 0, (kernel, registers, spills)


def test_successors_start_behind_an_allocation_through_the_helper_too():
    seen = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for body in text.split("__global__")[1:]:
            name = re.search(r"(\w+_kernel)\s*\(", body).group(1)
            at = [m.start() for m in re.finditer(r"tcgen05\.alloc|\btmem_alloc\s*\(", body)]
            starts = [m.start() for m in re.finditer(r"pdl_launch_dependents\(\)", body)]
            if at and starts:
                seen[name] = min(starts) > max(at)
    assert set(seen) == {"gemm_kernel", "gemm_rows_kernel", "attention_tc_kernel", "paged_attention_tc_kernel"}
    assert all(seen.values()), seen
    # whoever else issues the instruction is a helper that this scan has to know
    helpers = {os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*.cuh")) if "tcgen05.alloc" in open(p).read()}
    assert helpers == {"attention_tc.cuh"}, helpers
