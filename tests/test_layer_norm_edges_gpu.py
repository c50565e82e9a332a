"""Layer normalisation where its launches are at their limits."""
import pytest
import torch

import layer_reference as ref
import paper_2401_04658_amd as la2

pytestmark = pytest.mark.gpu


def test_more_columns_than_one_launch_sums():
    """2^25 features and some: d_weight and d_bias are 2^26 columns of sums, which one grid does not hold."""
    rows, width = 3, (1 << 25) + 1000
    x = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda").normal_()
    dy = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda").normal_()
    _, mean, rstd = la2.la2_layer_norm_fwd(x)
    dx, dw, db = la2.la2_layer_norm_bwd(dy, x, mean, rstd)
    # the first columns, those on both sides of 2^24 and 2^25 (where a launch ends, counted over both sums or one), the last
    for at in (slice(0, 4096), slice((1 << 24) - 2048, (1 << 24) + 2048), slice((1 << 25) - 2048, width)):
        h = (ref.d(x[:, at]) - ref.d(mean)[:, None]) * ref.d(rstd)[:, None]
        g = ref.d(dy[:, at])
        # a term's h is off by 4 roundings of it and of the mean's share, sums of three terms by three
        off = 8 * ref.U32 * (g.abs() * (h.abs() + (ref.d(mean) * ref.d(rstd)).abs()[:, None])).sum(0)
        ref.within("d_weight", dw[at], (g * h).sum(0), off)
        ref.within("d_bias", db[at], g.sum(0), 4 * ref.U32 * g.abs().sum(0))
    assert not bool(torch.isnan(dx).any())
