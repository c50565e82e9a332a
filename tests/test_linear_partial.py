"""Backward passes of the linear layer that want only some of the gradients: the workspace that the query names is enough for each of them (host
code only), and each is right where one product alone is cut otherwise than beside the other."""
import ctypes
import itertools

import pytest
import torch

import layer_reference as ref
import paper_2401_04658_amd as la2
from paper_2401_04658_amd import binding

WORKSPACE, LAUNCH = 5, 6
P = 0x10000   # an aligned "device pointer"
SIZES = [1, 17, 64, 300, 511, 512, 768, 1001, 1024, 2048, 2192, 4096, 8192]
SUBSETS = [s for s in itertools.product((False, True), repeat=3) if any(s)]


@pytest.mark.parametrize("dtype", [binding.LA2_BF16, binding.LA2_F16, binding.LA2_F32])
@pytest.mark.parametrize("act", [0, 2])
def test_the_workspace_of_the_query_is_enough_for_any_of_the_gradients(dtype, act):
    if torch.cuda.is_available():
        pytest.skip("a call with enough workspace would launch")
    lib = binding.load()
    for rows, k, n in itertools.product([1, 33, 512, 1024, 3295, 4096, 16384, 65536], SIZES, SIZES):
        desc = binding.la2_linear_desc(rows, k, n, dtype, act, k, k, n)
        size = lib.la2_linear_workspace_bytes(ctypes.byref(desc), binding.LA2_OP_BWD)
        for dx, dw, db in SUBSETS:
            st = lib.la2_linear_bwd(ctypes.byref(desc), P, P, P, P, P if dx else None, P if dw else None, P if db else None, P, size, None)
            assert st == LAUNCH, (rows, k, n, dx, dw, db, st)


@pytest.mark.gpu
@pytest.mark.parametrize("m,k,n,dtype,act", [(512, 1024, 4096, torch.bfloat16, "none"), (4096, 1024, 1024, torch.bfloat16, "none"),
                                             (1024, 512, 2048, torch.float16, "gelu"), (3295, 352, 2192, torch.float32, "silu"),
                                             (512, 512, 512, torch.float32, "none"), (600, 1001, 333, torch.bfloat16, "relu")])
def test_gradients_one_at_a_time(m, k, n, dtype, act):
    g = torch.Generator().manual_seed(m + k + n)
    x, w, dy, z = (torch.randn(*s, generator=g).mul(f).to(dtype).cuda() for s, f in (((m, k), 1.0), ((n, k), k ** -0.5), ((m, n), 1.0), ((m, n), 1.0)))
    r = ref.linear_bwd(dy, x, w, z, act)
    for want in SUBSETS:
        got = la2.la2_linear_bwd(dy, x, w, pre=None if act == "none" else z, act=act, want_dx=want[0], want_dw=want[1], want_d_bias=want[2])
        for i, name in enumerate(("dx", "dw", "d_bias")):
            assert (got[i] is not None) == want[i]
            if want[i]:
                ref.within("%s of %s" % (name, want), got[i], r[2 * i], r[2 * i + 1])
