"""What the layer norm, window attention and paged cache calls refuse, on the host: through the C ABI with pointers
that are never followed, and through the binding and autograd with CPU tensors (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2310_01655_amd import autograd
from paper_2310_01655_amd import binding as psf

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGNMENT = 0, 1, 2, 3, 4, 6
P = 4096                                        # an aligned address that nothing reads before the refusal


def changed(desc, **fields):
    out = type(desc).from_buffer_copy(desc)
    for name, value in fields.items():
        setattr(out, name, value)
    return out


WINDOW = psf.make_window_desc(2, 8, 1000, 64, 100, 4, kv_heads=2)


@pytest.mark.parametrize("fields,code", [
    ({}, OK), (dict(batch=0), SHAPE), (dict(heads=-1), SHAPE), (dict(kv_heads=3), SHAPE), (dict(kv_heads=0), SHAPE), (dict(n=0), SHAPE),
    (dict(d=0), SHAPE), (dict(window=0), SHAPE), (dict(sinks=-1), SHAPE), (dict(dtype=2), UNSUPPORTED), (dict(layout=2), UNSUPPORTED),
    (dict(d=60), UNSUPPORTED), (dict(d=136), UNSUPPORTED), (dict(n=(1 << 24) + 1), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED),
    (dict(scale=float("inf")), UNSUPPORTED), (dict(scale=float("nan")), UNSUPPORTED), (dict(scale=-0.5), OK),
    (dict(batch=8, heads=8192, kv_heads=1, n=1 << 16, d=8), UNSUPPORTED), (dict(heads=16384, kv_heads=1, d=128), UNSUPPORTED),
    (dict(window=2 ** 31 - 1), OK), (dict(sinks=2 ** 31 - 1), OK), (dict(d=128, n=1), OK),
])
def test_window_descriptor(fields, code):
    desc = changed(WINDOW, **fields)
    assert psf.check_window_desc(desc) == code
    assert (psf.window_bwd_workspace_bytes(desc) > 0) == (code == OK)
    assert psf.lib().psf_window_attn_fwd(ctypes.byref(desc), None, P, P, None, P, None, None) == (code or NULL)


def test_window_pointers():
    L, ref = psf.lib(), ctypes.byref(WINDOW)
    assert psf.lib().psf_check_window_desc(None) == NULL
    for k in (0, 1, 2, 4):
        args = [P, P, P, None, P, None, None]
        args[k] = None
        assert L.psf_window_attn_fwd(ref, *args) == NULL
        args[k] = P + 8
        assert L.psf_window_attn_fwd(ref, *args) == ALIGNMENT
    need = psf.window_bwd_workspace_bytes(WINDOW)
    good = [P, P, P, None, P, P, P, P, P, P, P, need, None]
    for k in (0, 1, 2, 4, 5, 6, 7, 8, 9, 10):
        assert L.psf_window_attn_bwd(ref, *[None if i == k else a for i, a in enumerate(good)]) == NULL
    for k in (0, 1, 2, 4, 6, 7, 8, 9):
        assert L.psf_window_attn_bwd(ref, *[P + 2 if i == k else a for i, a in enumerate(good)]) == ALIGNMENT
    assert L.psf_window_attn_bwd(ref, *good[:11], need - 1, None) == WORKSPACE
    assert L.psf_window_attn_bwd(ref, *good[:10], P + 128, need, None) == WORKSPACE


@pytest.mark.parametrize("rows,width,dtype,eps,code", [
    (0, 64, 1, 1e-6, SHAPE), (-1, 64, 1, 1e-6, SHAPE), (5, 0, 0, 1e-6, SHAPE), (5, 64, 2, 1e-6, UNSUPPORTED), (5, 8193, 0, 1e-6, UNSUPPORTED),
    (1 << 31, 8, 1, 1e-6, UNSUPPORTED), (5, 64, 1, 0.0, UNSUPPORTED), (5, 64, 1, -1.0, UNSUPPORTED), (5, 64, 1, float("nan"), UNSUPPORTED),
])
def test_layer_norm_sizes(rows, width, dtype, eps, code):
    L = psf.lib()
    assert L.psf_layer_norm_fwd(rows, width, dtype, eps, P, P, P, P, None, None) == code
    if eps == 1e-6:
        assert L.psf_layer_norm_bwd_workspace_bytes(rows, width, dtype) == 0
        assert L.psf_layer_norm_bwd(rows, width, dtype, P, P, P, P, P, P, P, P, 1 << 40, None) == code


def test_layer_norm_pointers():
    L = psf.lib()
    for k in (0, 1, 3):
        assert L.psf_layer_norm_fwd(5, 64, 1, 1e-6, *[None if i == k else P for i in range(5)], None) == NULL
    for k in (0, 1, 2, 3):
        assert L.psf_layer_norm_fwd(5, 64, 1, 1e-6, *[P + 1 if i == k else P for i in range(5)], None) == ALIGNMENT
        assert L.psf_layer_norm_fwd(5, 64, 0, 1e-6, *[P + 2 if i == k else P for i in range(5)], None) == ALIGNMENT
    assert L.psf_layer_norm_fwd(5, 64, 1, 1e-6, P, P, P, P, P + 4, None) == ALIGNMENT
    need = L.psf_layer_norm_bwd_workspace_bytes(5, 64, 1)
    assert need >= 2 * 64 * 4
    for k in (0, 1, 2, 3, 4, 5, 7):
        assert L.psf_layer_norm_bwd(5, 64, 1, *[None if i == k else P for i in range(8)], need, None) == NULL
    assert L.psf_layer_norm_bwd(5, 64, 1, *[P] * 8, need - 1, None) == WORKSPACE
    assert L.psf_layer_norm_bwd(5, 64, 1, *[P] * 7, P + 64, need, None) == WORKSPACE
    assert L.psf_layer_norm_bwd(5, 64, 1, *[P] * 6, P + 1, P, need, None) == ALIGNMENT


CACHE = psf.make_cache_desc(100, 16, 4, 64, 8, 200)


@pytest.mark.parametrize("fields,code", [
    ({}, OK), (dict(pages=0), SHAPE), (dict(page=0), SHAPE), (dict(kv_heads=-1), SHAPE), (dict(d=0), SHAPE), (dict(seqs=0), SHAPE),
    (dict(cols=0), SHAPE), (dict(dtype=3), UNSUPPORTED), (dict(d=12), UNSUPPORTED), (dict(d=136), UNSUPPORTED),
    (dict(pages=(1 << 20) + 1), UNSUPPORTED), (dict(pages=1 << 20, page=512, kv_heads=4), UNSUPPORTED), (dict(page=1 << 27), UNSUPPORTED),
    (dict(seqs=1 << 16, cols=1 << 15), UNSUPPORTED), (dict(cols=1 << 27), UNSUPPORTED), (dict(pages=1 << 20, kv_heads=1), OK),
])
def test_cache_descriptor(fields, code):
    desc, L = changed(CACHE, **fields), psf.lib()
    ref = ctypes.byref(desc)
    assert psf.check_cache_desc(desc) == code
    assert L.psf_cache_append(ref, 1, None, P, P, P, P, P, None, None) == (code or NULL)
    assert L.psf_cache_fork(ref, 1, None, P, P, P, P, P, P, None) == (code or NULL)
    assert L.psf_cache_compact(ref, None, P, P, P, P, P, P, 1 << 40, None) == (code or NULL)
    assert L.psf_paged_attn(ref, desc.kv_heads, 1, 0, 1.0, None, P, P, P, P, P, P, 1 << 40, None) == (code or NULL)
    assert (L.psf_cache_compact_workspace_bytes(ref) > 0) == (code == OK)


def test_cache_pointers_and_sizes():
    L, ref = psf.lib(), ctypes.byref(CACHE)
    assert L.psf_check_cache_desc(None) == NULL
    assert L.psf_cache_append(ref, 0, *[P] * 7, None) == SHAPE and L.psf_cache_append(ref, 1 << 30, *[P] * 7, None) == UNSUPPORTED
    for k in range(6):
        assert L.psf_cache_append(ref, 3, *[None if i == k else P for i in range(7)], None) == NULL
    for k in range(4):
        assert L.psf_cache_append(ref, 3, *[P + 8 if i == k else P for i in range(7)], None) == ALIGNMENT
    assert L.psf_cache_fork(ref, 0, *[P] * 7, None) == SHAPE and L.psf_cache_fork(ref, 65536, *[P] * 7, None) == UNSUPPORTED
    for k in range(7):
        assert L.psf_cache_fork(ref, 2, *[None if i == k else P for i in range(7)], None) == NULL
    assert L.psf_cache_fork(ref, 2, P + 4, *[P] * 6, None) == ALIGNMENT
    need = L.psf_cache_compact_workspace_bytes(ref)
    for k in range(7):
        assert L.psf_cache_compact(ref, *[None if i == k else P for i in range(7)], need, None) == NULL
    assert L.psf_cache_compact(ref, *[P] * 7, need - 1, None) == WORKSPACE
    assert L.psf_cache_compact(ref, *[P] * 6, P + 16, need, None) == WORKSPACE
    assert L.psf_cache_compact(ref, P, P + 8, *[P] * 5, need, None) == ALIGNMENT


def test_paged_attention_sizes():
    L, ref = psf.lib(), ctypes.byref(CACHE)
    need = psf.paged_workspace_bytes(CACHE, 8)
    assert need > 0 and psf.paged_workspace_bytes(CACHE, 7) == 0 and psf.paged_workspace_bytes(CACHE, 0) == 0
    call = lambda heads=8, window=1, sinks=0, args=(P,) * 7, room=need: L.psf_paged_attn(ref, heads, window, sinks, 1.0, *args, room, None)
    assert call(heads=6) == SHAPE and call(heads=0) == SHAPE and call(window=0) == SHAPE and call(sinks=-1) == SHAPE
    assert call(heads=4 << 20) == UNSUPPORTED
    for scale in (float("inf"), float("nan")):
        assert L.psf_paged_attn(ref, 8, 1, 0, scale, *[P] * 7, need, None) == UNSUPPORTED
    for k in range(7):
        assert call(args=[None if i == k else P for i in range(7)]) == NULL
    for k in (0, 1, 2, 5):
        assert call(args=[P + 8 if i == k else P for i in range(7)]) == ALIGNMENT
    assert call(room=need - 1) == WORKSPACE and call(args=[P] * 6 + [P + 128]) == WORKSPACE


def test_cpu_tensors_are_refused():
    x, w = torch.zeros(4, 64), torch.ones(64)
    heads = torch.zeros(1, 2, 8, 64)
    for call in (lambda: autograd.layer_norm(x, w), lambda: psf.psf_layer_norm_fwd(x, w),
                 lambda: psf.psf_layer_norm_bwd(x, w, torch.zeros(4, 2), x),
                 lambda: autograd.causal_window_attention(heads, heads, heads, 4),
                 lambda: psf.psf_cache_append(psf.make_cache_desc(4, 16, 2, 64, 1, 2, "f32"), heads, heads, heads, heads, heads, heads),
                 lambda: psf.psf_paged_attn(psf.make_cache_desc(4, 16, 2, 64, 1, 2, "f32"), heads, heads, heads, heads, heads)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError):
        autograd.layer_norm(x.double(), w.double())
    with pytest.raises(ValueError):
        autograd.causal_window_attention(x, x, x, 4)
    with pytest.raises(psf.PsfError):
        autograd.causal_window_attention(heads, heads, heads, 0)
    with pytest.raises(psf.PsfError):
        autograd.causal_window_attention(heads[..., :60], heads[..., :60], heads[..., :60], 3)
