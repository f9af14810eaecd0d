"""The 8-bit attention's prefill tiles read their fragments and scales from LDS by inline
assembly with hand-placed waits, and set m0 for their copies; these tests check the
gfx950 assembly as for the bf16 kernels."""
import os
import re
import shutil

import pytest

from lds_hazards import check
from paper_2606_16264_amd import build

pytestmark = pytest.mark.skipif(shutil.which(build.HIPCC) is None and not os.path.exists(build.HIPCC),
                                reason="hipcc not available")


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    return open(build.device_asm("attention_f8.hip", str(tmp_path_factory.mktemp("s") / "f8.s"))).read()


def test_no_lds_read_hazard(asm):
    res = {k: v for k, v in check(asm).items() if re.search("(paged|small)_attn_f8_kernel", k)}
    assert len(res) == 6, sorted(res)  # two head dims: with weights, without, small calls
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


def test_no_spills_in_the_prefill_tiles(asm):
    """A spilled register's reload is a vector-memory load: it would count among the copies, whose
    waits are placed by hand."""
    meta = re.findall(r"\.name:\s+(\S*(?:paged|small)_attn_f8_kernel\S*)\n(.*?)\.wavefront_size", asm, re.S)
    assert len(meta) == 6
    for name, body in meta:
        assert re.search(r"\.private_segment_fixed_size:\s+0\b", body), name
