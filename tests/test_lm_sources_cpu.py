"""Properties of the local step's kernels that only their sources show."""

import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def sources():
    files = sorted(glob.glob(os.path.join(ROOT, "paper_2504_17672_b200", "csrc", "lm_*")))
    assert len(files) >= 6
    for f in files:
        with open(f) as h:
            yield os.path.basename(f), re.sub(r"//[^\n]*", "", h.read())


def test_kernels_that_start_early_read_by_ordinary_loads():
    """They exist while the kernel before them still writes; the read-only path is for data that is constant for a kernel's lifetime."""
    for name, text in sources():
        found = re.findall(r"__ldg\b|ld\.global(?:\.\w+)*\.nc\b|__restrict__", text)
        assert not found, (name, found)


def test_every_kernel_waits_for_the_one_before_it_first():
    for name, text in sources():
        for body in re.findall(r"__global__ void[^;{]*\{(.*?)\n\}", text, re.S):
            before = body[:body.index("wait_for_previous();")]
            # until then only shared memory and parameters
            assert not re.search(r"tma_load|record\(|atomic|token_at|tmem_alloc", before), name


def test_lanes_come_together_before_aligned_instructions():
    """tcgen05 and cluster-barrier instructions marked .aligned stand in wrappers that first bring the warp's lanes together; a wait for
    loads follows the loads themselves, and mma.sync stands where no branch is taken by some lanes only, or after __syncwarp()."""
    wrappers = 0
    for name, text in sources():
        for m in re.finditer(r"(?:tcgen05\.(?:alloc|dealloc|ld)|barrier\.cluster\.arrive)[^\"]*\.aligned", text):
            body = text[text.rindex("__forceinline__", 0, m.start()):m.start()]
            assert "__syncwarp();" in body, (name, m.group(0))
            wrappers += 1
    assert wrappers >= 4
    for name, text in sources():
        for m in re.finditer(r"load_end\(tokens", text):
            assert re.match(r"[^}]*__syncwarp\(\);\s*multiply\(", text[m.start():]), name
