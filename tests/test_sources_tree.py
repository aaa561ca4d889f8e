"""How the trees' tensor-core kernel leaves when a wait is out of time: what no run can show, since
the runs that would go wrong are the ones that must not be made."""
import re

from tests.test_sources import _code


def _loaders(code):
    """The fetching warps' part."""
    return code[code.index("if (warp >= 5) {"):code.index("} else if (warp == 4) {")]


def test_every_load_of_16_bit_pages_has_landed_when_a_cta_leaves():
    # a warp that has fetched its last blocks waits for them whether or not its own waits ended
    # well: the role that gave up may be another
    part = re.sub(r"\s+", " ", _loaders(_code("paged_tree_tc.cu")))
    assert part.rstrip(" }").endswith("nullptr);")
    end = part[part.rindex("copies_landed();"):]
    assert end.startswith("copies_landed(); if (!kCodes) { for (int i = max(0, n - ST); i < n; ++i) "
                          "mbar_wait(&full[i % ST], i / ST & 1, nullptr); } else if (!ok) {")


def test_softmax_warps_agree_before_the_copies_join():
    # each decides for itself whether a wait ended well: they do so together before barriers that
    # all four have to reach, and no wait stands between those
    code = _code("paged_tree_tc.cu")
    part = code[code.index("} else if (warp == 4) {"):]
    agree = part.index("if constexpr (C > 1) ok = all_say(ok);")
    assert part[agree:].split("\n", 2)[1].strip() == "if (!ok) break;"
    join = part[agree:part.index("cta_warp == 8) tmem_dealloc")]
    assert "named_bar_sync(1 + team, 128)" in join and "wait_for(" not in join
    # (what looks for values that are not finite is called from the join)
    helper = part.index("auto find_not_finite")
    before = part[:helper] + part[part.index("auto put_not_finite"):agree]
    assert "named_bar_sync(1 + team" not in before and "find_not_finite(" not in before
    assert "find_not_finite(c, CP);" in join
