"""What the MXFP4 product may wait for without a limit, and what may be parked beside it.  Neither shows at run time until a call
stops making progress, so the sources are read."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1910_06188_b200", "csrc")


@pytest.fixture(scope="module")
def kernel():
    with open(os.path.join(CSRC, "q8_mx4_gemm_sm100.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    return re.search(r"\nmx4_gemm_kernel\(.*?\n}\n", text, re.S).group(0)


def test_no_kernel_is_parked_beside_a_pair_or_a_long_product(kernel):
    """The next kernel's CTAs are let in early by single CTAs with few rounds of tiles only, a condition that is the same for the whole grid."""
    released = re.findall(r"grid_dependency_release_next\((.*)\);", kernel)
    assert released == ["CTAS == 1 && (a.offsets != nullptr ? table.tile[a.E] : plan.tiles) <= kRoundsBeside * tile_step"]
    assert "constexpr int kRoundsBeside = FUSED ? 3 : 1;" in kernel
    assert "griddepcontrol" not in kernel


def test_the_next_kernel_is_let_in_behind_the_allocation(kernel):
    """A CTA that has started but does not have its tensor memory yet would wait for a parked one that has it, which waits for the first."""
    allocated, met, released = (kernel.index(t) for t in ("tmem_alloc(", "barrier.cta.sync 1", "grid_dependency_release_next("))
    assert allocated < met < released
    assert re.search(r"if \(goes_ahead\) asm volatile\(\"barrier\.cta\.arrive", kernel) and "if (!goes_ahead) grid_dependency_release_next(" in kernel


def test_every_stage_is_given_back_before_a_cta_ends(kernel):
    """The issuer's last arrivals, in a pair at the barriers of both CTAs, are waited for while the CTA still owns them (with a limit)."""
    producers = kernel[kernel.index("if (warp == 0 || (warp == 2 && !FUSED))"):kernel.index("} else if (warp == 1)")]
    behind = producers[producers.rindex("++issued;"):]
    assert re.search(r"for \(int i = 0; ok && i < C::kStages; \+\+i\) \{\s*ok = wait_for\(smem_u32\(empty_bar \+ s\), phase \^ 1u, abort_flag, a\.status\);", behind)
