"""How a CTA of the tensor-core kernels ends, checked on the CPU from the kernels' sources: whatever gives up, the products and copies that were
issued are through before its tensor memory and shared memory go."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2112_13935_b200", "csrc")
KERNELS = ["layer_mma_kernel.cu", "layer_f32_kernel.cu"]


def source(name):
    return open(os.path.join(CSRC, name)).read()


def kernel(name):
    s = source(name)
    return s[s.index("__global__"):s.index("tmem_free")]


@pytest.mark.parametrize("name", KERNELS)
def test_products_are_through_before_a_cta_ends(name):
    k = kernel(name)
    issue, last = k.index("} else if (warp == 1) {"), k.index("commit<CG>(drained)" if "CG>" in k else "commit<1>(drained)")
    assert issue < k.index("mma", issue) < k.rindex("commit<", 0, last) < last          # committed to behind every product
    end = k[k.rindex("__syncthreads();"):]
    assert re.search(r"if \(warp == 1\) drain\(drained, \*gave_up != 0, ns\);", end)
    if "CG" in k:      # neither CTA of a pair leaves before that
        assert end.index("drain(drained") < end.index("barrier.cluster.arrive")
    assert "bar_init(drained, 1);" in k and "*gave_up = 0;" in k


@pytest.mark.parametrize("name", KERNELS)
def test_every_role_that_gives_up_says_so(name):
    k = kernel(name)
    roles = re.split(r"\n  (?:if \(warp == 0\) \{|\} else if \(warp [^\n]*\{|\} else \{)", k)[1:]
    assert len(roles) == {"layer_mma_kernel.cu": 3, "layer_f32_kernel.cu": 4}[name]
    for role in roles:
        assert "bar_wait(" in role and "*gave_up = 1" in role


def test_every_wait_is_bounded():
    shared = source("layer_mma.cuh")
    assert re.search(r"if \(now - from > most_ns\) return false;", shared)
    for name in KERNELS:
        for call in re.findall(r"bar_wait\((.*)$", kernel(name), re.M):
            assert re.search(r", ns\)", call), call


@pytest.mark.parametrize("name", KERNELS)
def test_a_warp_that_gave_up_hands_no_tensor_memory_back(name):
    """A barrier counts arrivals, not who arrives: one warp running ahead would stand for another that still reads."""
    k = kernel(name)
    assert re.search(r"ok = __all_sync\(~0u, bar_wait\(acc_full", k)          # a warp gives up as a whole
    given = re.findall(r"if \(lane == 0( && ok)?\)[^;]*acc_empty", k)
    assert given and all(given), given
