"""What a warp does whose bounded wait has run out, read from the sources of the 8-bit kernels: it still comes to every barrier at which
others would wait for it.  (The waits end after a second; a barrier has no limit.)"""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_1611_08035_b200" / "csrc"


def source(name):
    return re.sub(r"//[^\n]*", "", (CSRC / name).read_text())


def body(text, start):
    """The text from the brace after `start` to the one that closes it."""
    at = text.index("{", text.index(start))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at : i + 1]


def test_barriers_of_some_warps_carry_the_verdict():
    for f in sorted(CSRC.glob("f8*")):
        assert not re.search(r'"bar(rier)?\.(cta\.)?(sync|arrive)', source(f.name)), f"{f.name}: a barrier of some warps that none of them can call off"


def test_scale_warps_leave_together():
    """Between two meetings of the four warps that bring the scales, nothing but their common verdict ends a loop."""
    text = source("f8_mx.cu")
    role = text[text.index("setmaxnreg.dec.sync.aligned.u32 80") : text.index("setmaxnreg.inc.sync.aligned.u32 184")]
    tiles = re.search(r"for \(int tile = [^;]*;([^;]*);", role)[1]
    assert "go" in tiles and not re.search(r"\bok\b", tiles)
    blocks = body(role, "for (int kb = 0")
    assert re.findall(r"(\S[^\n]*?)\s*break;", blocks) == ["if (!go)"] and "return" not in blocks
    assert re.search(r"go = named_barrier_all<1, 128>\(ok\);", blocks)


def test_joining_warps_all_reach_their_barrier():
    join, add = body(source("f8_out.cuh"), "void f8_split_join("), body(source("f8_out.cuh"), "void f8_add_shares(")
    assert "named_barrier_all<2, WORKERS>(true)" in add and add.count("named_barrier_all") == 1
    assert re.search(r"if \(worker >= 0 && !ok\) \{\s*if \(!p\.vec\) \(void\)named_barrier_all<2, 32 \* EW>\(false\);", join)
    before = add[: add.index("named_barrier_all")]
    assert re.search(r"if \(!p\.vec\) \{\s*if \(!$", before) and "return" not in before  # the same condition, and no way around it
    for name in ("f8_gemm.cu", "f8_wgrad.cu"):
        assert not re.search(r"ok \? tid", source(name)), f"{name}: a warp whose wait ran out is not numbered among the joining ones"
