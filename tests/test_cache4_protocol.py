"""Copies of the 4-bit attention into its rings, read from the source: a wait that gives up must leave none under way."""
import os

from conftest import ROOT

SRC = open(os.path.join(ROOT, "paper_2607_21927_gb300", "csrc", "cache4.cu")).read()
KERNEL = SRC[SRC.index("k_cache4_attend(const Cache4AttendArgs"):SRC.index("// Joins the parts of a list.")]
LOOP = KERNEL[KERNEL.index("for (int s0 = warp * per; ok && s0 < n; s0 += s_step)"):]


def test_a_wait_that_gives_up_takes_what_was_asked_for():
    """Before the loop over a part's stages is left, so before the rings take the warps' parts and before the CTA ends: of the
    stages from this one on those that the ring holds, each in its place and phase, as they were asked for."""
    gave_up = LOOP[LOOP.index("if (!ok) {"):LOOP.index("break;")]
    assert "for (int i = 0; i < kStages && s0 < n && !a.debug_no_loads; ++i, s0 += s_step)" in gave_up
    assert gave_up.index("mbar_wait(bars + 8 * used, phase);") < gave_up.index("if (++used == kStages) used = 0, phase ^= 1;")
    assert LOOP.index("break;") < LOOP.index("__syncthreads()")
    assert "int64_t limit = kWaitLimit" in SRC  # (with the waits' own limit, whatever a test asked for)


def test_copies_are_asked_for_while_all_is_well_alone():
    """A part's first stages where no wait gave up before, the later ones after the wait for the stage whose place they take."""
    assert KERNEL.count("fetch(") == 2 and KERNEL.count("bulk_load(") == 4  # (all four of a stage on its barrier)
    assert "if (lane == 0 && ok && !a.debug_no_loads)\n                for (int i = 0, s0 = warp * per, slot = used; i < kStages && s0 < n;" in KERNEL
    assert LOOP.index("break;") < LOOP.index("fetch(s0 + kStages * s_step, used);")
