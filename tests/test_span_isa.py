"""The tiles of attention over parts of the keys read their fragments from LDS by inline
assembly with hand-placed waits, and set m0 for their copies; these tests check the gfx950
assembly as for the other attention kernels."""
import os
import re
import shutil

import pytest

from lds_hazards import check
from paper_2606_16264_amd import build

pytestmark = pytest.mark.skipif(shutil.which(build.HIPCC) is None and not os.path.exists(build.HIPCC),
                                reason="hipcc not available")
KERNEL = "(span_attn|small_span)_kernel"


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    return open(build.device_asm("attention_span.hip", str(tmp_path_factory.mktemp("s") / "span.s"))).read()


def test_no_lds_read_hazard(asm):
    res = {k: v for k, v in check(asm).items() if re.search(KERNEL, k)}
    # two head dims: with tiles, streams alone; each also for small calls
    assert len(res) == 8, sorted(res)
    bad = {k: v[:3] for k, v in res.items() if v}
    assert not bad, bad


def test_copies_alone_use_m0(asm):
    ops = [l.split(";")[0].strip() for l in asm.splitlines()]
    ops = [l for l in ops if l and not l.startswith(".") and not l.endswith(":")]
    uses = [i for i, l in enumerate(ops) if re.search(r"\bm0\b", l)]
    copies = [i for i, l in enumerate(ops) if l.startswith("global_load_lds")]
    assert copies and [i + 2 for i in uses] == copies
    for i in uses:
        assert re.fullmatch(r"s_mov_b32 m0, s\d+", ops[i]) and ops[i + 1] == "s_nop 0", ops[i:i + 3]
        assert re.fullmatch(r"global_load_lds_dwordx4 v\d+, s\[\d+:\d+\]", ops[i + 2]), ops[i + 2]


def test_no_spills(asm):
    """A spilled register's reload is a vector-memory load: it would count among the copies, whose
    waits are placed by hand, and come back behind them."""
    meta = re.findall(r"\.name:\s+(\S*(?:span_attn|small_span)_kernel\S*)\n(.*?)\.wavefront_size", asm, re.S)
    assert len(meta) == 8
    for name, body in meta:
        assert re.search(r"\.private_segment_fixed_size:\s+0\b", body), name


def test_the_loops_wait_for_copies_by_hand_alone(asm):
    """A loop of a tile that holds its 32 matrix products waits for vector memory once, at its top,
    with the count of one chunk's copies: any other such wait would hold for the copies in flight."""
    found = 0
    for hd, copies in ((128, 4), (64, 2)):
        fn = re.search(rf"^\S*span_attn_kernelILi{hd}ELb1E\S*:[^\n]*\n(.*?)^\.Lfunc_end", asm, re.S | re.M).group(1)
        for block in re.split(r"\n(?=\.LBB)", fn):
            if block.count("v_mfma") != hd // 4 or "global_load_lds" not in block:
                continue
            found += 1
            waits = re.findall(r"s_waitcnt[^\n;]*vmcnt\((\d+)\)", block)
            assert waits == [str(copies)], (hd, waits)
    assert found >= 8
