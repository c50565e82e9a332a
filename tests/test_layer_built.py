"""The layer norm's kernels that are built are those that some row takes."""
import json
import os
import re

import pytest

from paper_2401_04658_amd import build

# lanes and 16-byte pieces a lane of a row, by the number of pieces of the row up to which they are taken
LOW = [(8, 8, 1), (16, 16, 1), (32, 32, 1), (64, 64, 1), (128, 64, 2)]
SPLITS = {
    ("fwd", 16): LOW + [(256, 64, 4), (512, 256, 2), (1024, 512, 2), (2048, 512, 4)],
    ("fwd", 32): LOW + [(256, 64, 4), (512, 256, 2), (1024, 512, 2), (2048, 512, 4), (4096, 1024, 4)],
    ("bwd", 16): LOW + [(256, 256, 1), (512, 256, 2), (1024, 1024, 1), (2048, 512, 4)],
    ("bwd", 32): LOW + [(256, 64, 4), (512, 256, 2), (1024, 512, 2), (2048, 512, 4), (4096, 1024, 4)],
}


@pytest.mark.parametrize("way,bits", sorted(SPLITS))
def test_no_kernel_without_a_row(way, bits):
    if not os.path.exists(build.RESOURCES):
        build.build()
    with open(build.RESOURCES) as f:
        names = list(json.load(f))
    for code in ("f",) if bits == 32 else ("DF16b", "DF16_"):
        built = {tuple(int(x) for x in m.groups()) for m in (re.search(r"\dlayer_norm_%s_kernelI%sLi(\d+)ELi(\d+)E" % (way, code), k) for k in names) if m}
        assert built == {s[1:] for s in SPLITS[way, bits]}, code
