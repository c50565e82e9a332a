"""Which tensors the binding of the operators around the recurrence takes and which it refuses (host code only; nothing is launched)."""
import ctypes

import pytest
import torch

from paper_2401_04658_amd import binding

ALIGN, LAUNCH = 4, 6


@pytest.fixture
def entries(monkeypatch):
    """The binding's functions on CPU tensors; a call that passes every check ends with LA2_ERR_LAUNCH, there being no device."""
    if torch.cuda.is_available():
        pytest.skip("a call that passes the checks would launch")
    monkeypatch.setattr(binding, "_on_gpu", lambda t, what: None)
    monkeypatch.setattr(binding, "_call", lambda entry, t, *args: entry(*args, 0))
    return binding


def zeros(*size, dtype=torch.bfloat16):
    return torch.zeros(size, dtype=dtype)


def scratch(size=1 << 20):
    """A workspace at a multiple of 256, as device memory is and host memory is not always."""
    t = torch.empty(size + 256, dtype=torch.uint8)
    skip = -t.data_ptr() % 256
    return t[skip:skip + size]


def calls(la2, t):
    """Every entry point that takes t [a, b, 128] as rows of features, t in each of the places where it does."""
    lead, dense, w, ws = t.shape[:-1], zeros(*t.shape), zeros(128, 128), scratch()
    stats = zeros(*lead, dtype=torch.float32)
    return {
        "layer_norm_fwd x": lambda: la2.la2_layer_norm_fwd(t),
        "layer_norm_bwd x, dy": lambda: la2.la2_layer_norm_bwd(t, t, stats, stats, workspace=ws),
        "linear_fwd x": lambda: la2.la2_linear_fwd(t, w),
        "linear_fwd residual": lambda: la2.la2_linear_fwd(dense, w, residual=t),
        "linear_fwd out": lambda: la2.la2_linear_fwd(dense, w, out=t),
        "linear_bwd x": lambda: la2.la2_linear_bwd(dense, t, w, workspace=ws),
        "linear_bwd dy": lambda: la2.la2_linear_bwd(t, dense, w, workspace=ws),
        "beam_select logits": lambda: la2.la2_beam_select(t, stats, workspace=ws),
    }


EXPANDED = [  # size before expand(3, 4, 128)
    (3, 1, 128),    # the middle: a gradient per sequence for all its positions, logits of a prompt for all its beams
    (1, 4, 128),    # the leading dimension
    (1, 1, 128),    # both
]


@pytest.mark.parametrize("size", EXPANDED)
def test_rows_that_share_memory_are_refused(entries, size):
    t = zeros(*size).expand(3, 4, 128)
    for name, call in calls(entries, t).items():
        try:
            got = call()
        except ValueError:
            continue
        assert got == ALIGN, name


def test_more_leading_dimensions(entries):
    for size, full in (((2, 3, 1, 64), (2, 3, 4, 64)), ((2, 1, 4, 64), (2, 3, 4, 64)), ((1, 3, 4, 64), (2, 3, 4, 64)), ((2, 1, 1, 64), (2, 3, 4, 64)),
                       ((1, 64), (4, 64)), ((1, 1, 64), (4, 1, 64))):
        t = zeros(*size).expand(*full)
        try:
            got = entries.la2_layer_norm_fwd(t)
        except ValueError:
            continue
        assert got == ALIGN, size
    # overlapping rather than expanded
    for stride in ((64, 64, 1), (128, 64, 1), (96, 96, 1)):
        with pytest.raises(ValueError):
            entries.la2_layer_norm_fwd(zeros(2000).as_strided((3, 4, 64), stride))
    assert entries.la2_layer_norm_fwd(zeros(2000).as_strided((3, 4, 64), (128, 32, 1))) == ALIGN


def test_rows_at_one_distance_are_taken(entries):
    wide = zeros(6, 4, 192)
    for t in (zeros(3, 4, 128), zeros(12, 160)[:, :128].view(3, 4, 128), wide[::2, :, :128][:, :1], wide[:3, :1, :128], wide[:1, ::2, :128],
              zeros(3, 1, 128), zeros(1, 1, 128), zeros(1, 1, 128).expand(1, 1, 128), zeros(3, 128).unsqueeze(1)):
        for name, call in calls(entries, t).items():
            assert call() == LAUNCH, (name, t.shape, t.stride())


def test_no_rows_at_any_distance(entries):
    """Tensors without elements: whatever their strides say, as torch leaves them behind slicing."""
    for t in (zeros(3, 0, 128), zeros(0, 4, 128), zeros(3, 4, 128)[:, :0], zeros(3, 4, 192)[:0, :, :128], zeros(3, 8, 192)[:, 4:4, :128]):
        stats = zeros(*t.shape[:-1], dtype=torch.float32)
        assert entries.la2_layer_norm_fwd(t)[0].shape == t.shape
        assert entries.la2_linear_fwd(t, zeros(64, 128))[0].shape == t.shape[:-1] + (64,)
        assert entries.la2_layer_norm_bwd(t, t, stats, stats, want_d_weight=False, want_d_bias=False)[0].shape == t.shape
        assert entries.la2_linear_bwd(t, t, zeros(128, 128), want_dw=False, want_d_bias=False)[0].shape == t.shape


def test_an_extent_that_does_not_fit_raises():
    x = torch.empty(0, 2 ** 31, dtype=torch.bfloat16)
    v = torch.empty(0)
    lib = binding._module()
    for call in (lambda: lib.layer_norm_fwd(x, None, None, 1e-5, None, None, None, 0),
                 lambda: lib.layer_norm_bwd(x, x, v, v, None, False, False, None, None, 0),
                 lambda: lib.linear_fwd(x, x, None, None, 0, False, None, None, None, 0)):
        with pytest.raises(OverflowError):
            call()


def test_tensors_without_storage_raise():
    """What torch.func hands to a function it transforms has sizes and strides but no memory: an error, with the interpreter lock held."""
    lib, x, w, square = binding._module(), zeros(2, 4, 64), zeros(2, 32, 64), zeros(2, 64, 64)
    v, scores, parent = torch.zeros(4), torch.zeros(2, 2), torch.zeros(2, 2, dtype=torch.int32)
    for call in (lambda: torch.func.vmap(lambda t: lib.layer_norm_fwd(t, None, None, 1e-5, None, None, None, 0))(x),
                 lambda: torch.func.vmap(lambda t: lib.layer_norm_bwd(x[0], t, v, v, None, False, False, None, None, 0), randomness="same")(x),
                 lambda: torch.func.vmap(lambda t, u: lib.linear_fwd(t, u, None, None, 0, False, None, None, None, 0))(x, w),
                 lambda: torch.func.vmap(lambda t, u: lib.linear_bwd(t, t, u, None, 0, True, True, True, None, 0))(x, square),
                 lambda: torch.func.vmap(lambda t: lib.beam_select(t, scores, None, -1, None, 0))(torch.zeros(2, 2, 2, 9)),
                 lambda: torch.func.vmap(lambda t: lib.beam_reorder([t], parent, 0))(torch.zeros(2, 4, 8))):
        with pytest.raises(RuntimeError, match="data pointer"):
            call()


def test_a_workspace_without_its_bytes_is_refused(entries):
    """One byte expanded to many counts as many and has one."""
    x, w, v = zeros(300, 128), zeros(64, 128), torch.zeros(300)
    dy, logits, scores = zeros(300, 64), zeros(2, 2, 9), torch.zeros(2, 2)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 30), torch.zeros(1, 1 << 10).expand(1 << 10, 1 << 10), scratch()[::2]):
        for call in (lambda: entries.la2_layer_norm_bwd(x, x, v, v, workspace=ws), lambda: entries.la2_linear_fwd(x, w, workspace=ws),
                     lambda: entries.la2_linear_bwd(dy, x, w, workspace=ws), lambda: entries.la2_beam_select(logits, scores, workspace=ws)):
            with pytest.raises(ValueError):
                call()


def test_strides_of_dimensions_of_one_entry_do_not_count(entries):
    """A step's [batch, 1, features] sliced out of a longer tensor lies as a dense one does."""
    ws, v, w = scratch(), torch.zeros(1, 1), zeros(64, 64)
    long = zeros(1, 7, 64)
    one, dense = long[:, 3:4], zeros(1, 1, 64)
    dense_b, part_b = zeros(5, 1, 64), zeros(5, 1, 64).as_strided((5, 1, 64), (64, 9, 1))
    vb = torch.zeros(5, 1)
    assert one.stride() != dense.stride() and part_b.stride() != dense_b.stride()
    for a, b, s in ((one, dense, v), (dense, one, v), (part_b, dense_b, vb), (dense_b, part_b, vb)):
        for call in (lambda: entries.la2_layer_norm_fwd(a, out=b), lambda: entries.la2_layer_norm_bwd(a, b, s, s, workspace=ws),
                     lambda: entries.la2_linear_fwd(a, w, residual=a, out=b, pre=a.clone()),
                     lambda: entries.la2_linear_bwd(a, b, w, pre=b, act="gelu", workspace=ws)):
            assert call() == LAUNCH, (a.stride(), b.stride())
    columns = zeros(4, 6).t()[:, :1]   # features of one entry: [6, 1], rows one element apart
    assert entries.la2_layer_norm_fwd(columns, out=zeros(6, 1)) == LAUNCH
    with pytest.raises(ValueError):
        entries.la2_layer_norm_fwd(zeros(5, 1, 96)[:, :, :64], out=dense_b)


def test_states_larger_than_a_grid_are_refused():
    """A grid has at most 2^32 - 1 work-items of 16 bytes each, in whole workgroups of 256."""
    if torch.cuda.is_available():
        pytest.skip("a call that passes the checks would launch")
    lib, P, SHAPE = binding.load(), 0x10000, 2
    call = lambda row: lib.la2_beam_reorder(1, (ctypes.c_void_p * 1)(P), 1, 2, row, P, None)
    for row in ((1 << 36) - 4096 + 16, 1 << 36, 1 << 40):
        assert call(row) == SHAPE, row
    assert call((1 << 36) - 4096) == LAUNCH and call(64) == LAUNCH
