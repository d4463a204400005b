"""Hand-overs of the attention over pages, read from its source: what a wait that is missing or gives up would leave behind."""
import os

from conftest import ROOT

SRC = open(os.path.join(ROOT, "paper_2607_21927_gb300", "csrc", "attn_paged.cu")).read()
KERNEL = SRC[SRC.index("k_paged_tiles(const __grid_constant__"):SRC.index("// ---------------------------------------------------------------- host side")]
LOADERS = KERNEL[KERNEL.index("if (warp == kLoadQK) {\n                const uint32_t q_bytes"):KERNEL.index("// The issuing warps, all lanes")]
ISSUERS = KERNEL[KERNEL.index("// The issuing warps, all lanes"):KERNEL.index("setmaxnreg.inc")]
SOFTMAX = KERNEL[KERNEL.index("setmaxnreg.inc"):]


def test_copies_and_products_are_waited_for_before_a_pass_ends():
    """Also after a wait that gave up: with the waits' own limit, whatever a test asked for."""
    for bar in ("B_Q_FULL", "B_K_FULL"):
        assert f"mbar_wait_own<1>(bar(L::{bar}" in LOADERS[:LOADERS.index("} else if (warp == kLoadV) {")]
    assert "mbar_wait_own<1>(bar(L::B_V_FULL" in LOADERS[LOADERS.index("} else if (warp == kLoadV) {"):]
    assert LOADERS.count("tma_load_4d(") == 2 and LOADERS.count("tma_load_3d<1>(") == 1 and "tma_load" not in ISSUERS + SOFTMAX
    # a commit for each barrier that the end waits on, and no other
    commits = {line.split("tc_commit<1>(bar(L::")[1].split(" ")[0].rstrip(")") for line in ISSUERS.split(";") if "tc_commit<1>(" in line}
    assert commits == {"B_S_FULL", "B_K_FREE", "B_Q_FREE", "B_PV_DONE", "B_V_FREE"}
    end = ISSUERS[ISSUERS.index("every commit of this warp has arrived"):]
    assert "warp == kScores ? L::B_S_FULL : L::B_PV_DONE" in end and "warp == kScores ? L::B_K_FREE : L::B_V_FREE" in end
    assert end.count("mbar_wait_own<1>(") == 3 and "mbar_wait_own<1>(bar(L::B_Q_FREE)" in end
    assert end.index("mbar_wait_own") < end.index("while (another_pass());")


def test_everyone_meets_between_passes_and_before_tensor_memory_is_given_back():
    """Every role ends a pass at the same barrier, and barriers are set up anew by one warp between two of them."""
    meet = KERNEL[KERNEL.index("auto another_pass"):KERNEL.index("setmaxnreg.dec")]
    assert meet.count("barrier.cta.sync 0") == 2
    assert meet.index("barrier.cta.sync 0") < meet.index("wrong != 1u") < meet.index("mbarrier.inval") < meet.index("set_up();") < meet.rindex("barrier.cta.sync 0")
    assert ISSUERS.count("another_pass()") == 1 and SOFTMAX.count("another_pass()") == 2
    assert SOFTMAX.rindex("another_pass()") < SOFTMAX.index("tmem_dealloc<1")


def test_a_places_last_values_have_been_used_before_a_warp_writes_to_it():
    """A softmax warp that changes a tile's values has waited for the product over the values before them in that place (the scores came
    without it), and for the values' copy; its writes are handed to the product before the weights' arrival."""
    edge = SOFTMAX[SOFTMAX.index("(a thread takes a key)"):SOFTMAX.index("mbar_arrive_if(lane == 0, bar(L::B_P_GO + buf));")]
    order = ["B_PV_DONE + (unsigned)(t - 2) % NS", "B_V_FULL + t % NSV", "make_uint4(0u, 0u, 0u, 0u)", "clean_values<D>", "fence.proxy.async"]
    assert [edge.index(x) for x in order] == sorted(edge.index(x) for x in order)
