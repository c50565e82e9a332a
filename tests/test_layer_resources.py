"""Registers, scratch and LDS of the kernels around the recurrence, as the compiler reported them at build time.  The tiled products sit
at the LDS and register limits of their occupancy; a spill in their loop costs a third of their speed and fails no other test."""
import json
import os
import re

import pytest

from paper_2401_04658_amd import build

FAMILIES = {   # scratch bytes per lane, waves per SIMD at least
    "layer_norm_fwd_kernel": (0, 2), "layer_norm_bwd_kernel": (0, 2), "layer_norm_wide_fwd_kernel": (0, 4), "layer_norm_wide_bwd_kernel": (0, 4),
    "layer_norm_wide_columns_kernel": (0, 4), "column_sum_kernel": (0, 4), "linear_few_kernel": (0, 2), "linear_join_kernel": (0, 4),
    "linear_prepare_kernel": (0, 2), "product_kernel": (0, 2), "product_pair_kernel": (0, 2), "beam_chunk_kernel": (0, 4),
    "beam_merge_kernel": (0, 2), "beam_reorder_kernel": (0, 3),
}


@pytest.fixture(scope="module")
def resources():
    if not os.path.exists(build.RESOURCES):
        build.build()
    with open(build.RESOURCES) as f:
        return json.load(f)


def family(name):
    for f in sorted(FAMILIES, key=len, reverse=True):
        if re.search(r"\d" + f, name):
            return f
    return None


def test_every_family_is_built_and_within_its_limits(resources):
    seen = set()
    for k, v in resources.items():
        f = family(k)
        if f is None:
            continue
        seen.add(f)
        scratch, waves = FAMILIES[f]
        assert v["ScratchSize"] <= scratch and v["SGPRs_Spill"] == 0, (k, v["ScratchSize"], v["SGPRs_Spill"])
        assert v["Occupancy"] >= waves, (k, v["Occupancy"])
    assert seen == set(FAMILIES)


def test_two_workgroups_of_the_middle_tile_share_a_unit(resources):
    for k, v in resources.items():
        if family(k) in ("product_kernel", "product_pair_kernel"):
            lds = v["LDS"]
            if "ILi256ELi256" in k:
                assert lds == 131072, (k, lds)
            else:
                assert 2 * lds <= build_lds(), (k, lds)


def build_lds():
    return 160 * 1024
