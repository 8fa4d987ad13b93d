"""The build's checks of scalar bases and of copies of a ring of loads on small hand-written listings: along paths, not lines."""
import pytest

from paper_2412_14590_amd import asm_scan, build

LOAD = "\t;;#ASMSTART\n\tglobal_load_dwordx4 v[0:3], v4, s[6:7] offset:0\n\t;;#ASMEND\n"
LANE = "\tv_readlane_b32 s6, v40, s3\n"
FIVE = "\tv_add_u32_e32 v9, v8, v7\n" * 5


def bases(text, function=True):
    build.check_scalar_bases(("\t.type\tk,@function\nk:\n" if function else "") + text + "\ts_endpgm\n", "listing")


# reported: the lane read reaches the load in fewer than five wait states on some path
SOON = {
    "a scalar instruction that only reads": LANE + "\ts_cmp_lg_u32 s6, 0\n" + LOAD,
    "... a pair": LANE + "\ts_cmp_lg_u64 s[6:7], 0\n" + LOAD,
    "... a bit test": LANE + "\ts_bitcmp1_b32 s6, 3\n" + LOAD,
    "a scalar instruction that may write": LANE + "\ts_cmov_b32 s6, s9\n" + LOAD,
    "a wait": LANE + "\ts_waitcnt lgkmcnt(0)\n" + LOAD,
    "around a loop": ".LBB0_1:\n" + LOAD + FIVE + LANE + "\ts_cbranch_scc1 .LBB0_1\n",
    "over a skipped rewrite": LANE + "\ts_cbranch_scc1 .LBB0_2\n\ts_mov_b32 s6, s9\n.LBB0_2:\n" + LOAD,
    "over skipped waits": LANE + "\ts_cbranch_execz .LBB0_2\n" + FIVE + ".LBB0_2:\n" + LOAD,
    "a forward branch over other code": LANE + "\ts_branch .LBB0_2\n.LBB0_1:\n" + FIVE + "\ts_endpgm\n.LBB0_2:\n" + LOAD,
    "a comparison": "\tv_cmp_gt_u32_e64 s[6:7], v1, v2\n" + LOAD,
    "a carry": "\tv_add_co_u32 v1, s[6:7], v1, v2\n" + LOAD,
    "the upper half": "\tv_readfirstlane_b32 s7, v40\n" + LOAD,
    "the condition as a base": "\tv_cmp_gt_u32_e32 vcc, v1, v2\n" + LOAD.replace("s[6:7]", "vcc"),
    "a comment is no wait": LANE + "\t;;#ASMSTART\n\t; ring drained\n\t;;#ASMEND\n" + "\tv_add_u32_e32 v9, v8, v7\n" * 4 + LOAD,
}
FAR = {
    "five wait states": LANE + FIVE + LOAD,
    "five on either path": LANE + "\ts_cbranch_scc1 .LBB0_2\n" + "\ts_nop 0\n" + ".LBB0_2:\n\ts_nop 3\n" + LOAD,
    "waits behind the load of a loop": ".LBB0_1:\n\ts_nop 4\n" + LOAD + LANE + "\ts_cbranch_scc1 .LBB0_1\n",
    "written by the scalar unit": LANE + "\ts_mov_b64 s[6:7], s[8:9]\n" + LOAD,
    "code that no path comes from": "\ts_branch .LBB0_2\n.LBB0_1:\n" + LANE + "\ts_endpgm\n.LBB0_2:\n" + LOAD,
    "another register": "\tv_readlane_b32 s8, v40, s3\n" + LOAD,
    "a vector register of the same number": "\tv_mov_b32_e32 v6, v7\n" + LOAD,
    "the compiler's own load": LANE + "\tglobal_load_dwordx4 v[0:3], v4, s[6:7]\n",
}


@pytest.mark.parametrize("name", list(SOON))
@pytest.mark.parametrize("function", [True, False])
def test_a_base_read_too_soon_on_any_path_is_reported(name, function):
    with pytest.raises(RuntimeError, match="too early"):
        bases(SOON[name], function)


@pytest.mark.parametrize("name", list(FAR))
@pytest.mark.parametrize("function", [True, False])
def test_a_base_that_is_there_passes(name, function):
    bases(FAR[name], function)


RING = "\t;;#ASMSTART\n\tglobal_load_dwordx4 v[{0}:{1}], v60, s[6:7] offset:0 nt\n\t;;#ASMEND\n"
DRAINED = "\t;;#ASMSTART\n\t; ring drained\n\t;;#ASMEND\n"
COPY = "\tv_mov_b32_e32 v{0}, v{1}\n"


def copies(body):
    (name, n), = asm_scan.ring_copies("\t.type\tthe_kernel,@function\nthe_kernel:\n" + body + "\ts_endpgm\n\t.type\tother,@function\nother:\n" +
                                      RING.format(4, 7) + COPY.format(9, 4) + "\ts_endpgm\n", "the_kernel")
    assert name == "the_kernel"
    return n


def test_copies_of_a_ring_are_counted_along_paths():
    request = RING.format(4, 7)
    assert copies(request + COPY.format(20, 4)) == 1
    assert copies(request + COPY.format(4, 20)) == 1
    assert copies(request + COPY.format(20, 21)) == 0
    assert copies(COPY.format(20, 4) + request) == 0                       # before the first request
    assert copies(request + DRAINED + COPY.format(20, 4)) == 0
    assert copies(request + DRAINED + RING.format(8, 11) + COPY.format(20, 4) + COPY.format(20, 8)) == 1
    # a latch that stands behind the marker, while the loop that it closes goes on
    latch = ".LBB0_1:\n" + request + "\ts_cbranch_scc1 .LBB0_3\n" + DRAINED + "\ts_endpgm\n.LBB0_3:\n" + COPY.format(20, 4) * 3 + "\ts_branch .LBB0_1\n"
    assert copies(latch) == 3
    # drained on one way to the copy only
    assert copies(request + "\ts_cbranch_scc1 .LBB0_2\n" + DRAINED + ".LBB0_2:\n" + COPY.format(20, 4)) == 1


def test_the_limit_of_copies_is_checked(monkeypatch):
    listing = "\t.type\tthe_kernel,@function\nthe_kernel:\n" + RING.format(4, 7) + COPY.format(20, 4) * 3 + "\ts_endpgm\n"
    for limit in (2, 3):
        monkeypatch.setattr(build, "RING_COPY_LIMIT", {"x.hip": ("the_kernel", limit)})
        if limit == 2:
            with pytest.raises(RuntimeError, match="3 register copies"):
                build.check_ring_copies(listing, "x.hip")
        else:
            build.check_ring_copies(listing, "x.hip")
