"""How linear layers are planned (CPU: launchers that only write down what they are asked for)."""
import ctypes
import os
import subprocess

import pytest
import torch

import layer_reference as ref
import paper_2401_04658_amd as la2
from paper_2401_04658_amd import binding, build

HERE = os.path.dirname(os.path.abspath(__file__))
P = 1 << 30   # an aligned address; nothing reads it
SHAPE = 2
DTYPES = [binding.LA2_BF16, binding.LA2_F16, binding.LA2_F32]
THREADS = (256, 256, 512)   # of the tiles of 64, 128 and 256


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    bdir = os.path.join(os.path.dirname(binding.lib_path()), "_build")
    if not os.path.exists(build.RESOURCES):
        build.build()
    folder = str(tmp_path_factory.mktemp("routes"))
    obj, so = os.path.join(folder, "recorder.o"), os.path.join(folder, "libroutes.so")
    subprocess.check_call([build.HIPCC, "-O1", "-std=c++17", "--offload-host-only", "-fPIC", "-Wall", "-Wno-unused-command-line-argument", "-c",
                           os.path.join(HERE, "layer_route_recorder.hip"), "-o", obj])
    subprocess.check_call([build.HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", so, obj,
                           os.path.join(bdir, "la2_layer_api.o"), os.path.join(bdir, "la2_linear.o")])
    lib = ctypes.CDLL(so)
    lib.la2_linear_workspace_bytes.restype = ctypes.c_size_t
    return lib


def plan(lib, op, rows, k, n, dtype, dx=True, dw=True):
    """(status, products) of a call without activation and bias."""
    p = ctypes.c_void_p
    d = binding.la2_linear_desc(rows, k, n, dtype, 0, k, k, n)
    size = ctypes.c_size_t(lib.la2_linear_workspace_bytes(ctypes.byref(d), op))
    if op == binding.LA2_OP_FWD:
        st = lib.la2_linear_fwd(ctypes.byref(d), p(P), p(P), p(0), p(0), p(P), p(0), p(P), size, p(0))
    else:
        st = lib.la2_linear_bwd(ctypes.byref(d), p(P), p(P), p(0), p(P), p(P if dx else 0), p(P if dw else 0), p(0), p(P), size, p(0))
    out = ctypes.create_string_buffer(4096)
    assert lib.routes_take(out, 4096) >= 0
    words = [line.split() for line in out.value.decode().splitlines()]
    return st, [dict(((k, int(v)) for k, v in (w.split("=") for w in ws[1:])), kind=ws[0]) for ws in words]


@pytest.mark.parametrize("dtype", DTYPES)
def test_grids_stay_below_the_largest(lib, dtype):
    """A grid has at most 2^32 - 1 work-items: larger tiles where the small ones would be more, extents that no tile holds are refused."""
    refused = taken = 0
    most = (1 << 31) - (1 << 26)
    tiles = lambda a, b: -(-a // 256) * -(-b // 256)
    for rows in (1 << 20, 1 << 26, 1 << 28, (1 << 29) + 1, 1 << 30, (1 << 30) + 64, 1500000000, most - 1, most, (1 << 31) - 1):
        for k, n in ((8, 8), (64, 8), (8, 64), (72, 8), (256, 256), (512, 8), (8, 1024), (2048, 2048)):
            if (dtype == binding.LA2_F32 and max(k, n) > 1 << 19) or rows * max(k, n) > 1 << 40:
                continue
            for op in (binding.LA2_OP_FWD, binding.LA2_OP_BWD):
                for dx, dw in ((True, True), (True, False), (False, True)):
                    st, products = plan(lib, op, rows, k, n, dtype, dx, dw)
                    if st == SHAPE:
                        refused += 1
                        assert max(tiles(rows, n), tiles(rows, k) + tiles(n, k)) >= (1 << 23) - (1 << 18), (rows, k, n)
                        continue
                    assert products
                    taken += 1
                    items = sum(-(-x["I"] // (64 << x["tile"])) * -(-x["J"] // (64 << x["tile"])) * x["splits"] * THREADS[x["tile"]] for x in products)
                    assert items + (n + 15) // 16 * 512 < 1 << 32, (rows, k, n, products)
    assert refused and taken


@pytest.mark.gpu
def test_more_rows_than_small_tiles_take():
    """2^30 rows and some of 8 features, 16 GiB a tensor."""
    rows, f = (1 << 30) + 77, 8
    x = torch.empty(rows, f, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn(f, f, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    places = (slice(0, 500), slice(rows // 2, rows // 2 + 500), slice(rows - 500, rows))
    y, _ = la2.la2_linear_fwd(x, w)
    for at in places:
        ry, ey, _, _ = ref.linear_fwd(x[at], w, None, None, "none")
        ref.within("y", y[at], ry, ey)
    dx, _, _ = la2.la2_linear_bwd(x, y, w, want_dw=False, want_d_bias=False)
    for at in places:
        rdx, edx = ref.linear_bwd(x[at], y[at], w, None, "none")[:2]
        ref.within("dx", dx[at], rdx, edx)
