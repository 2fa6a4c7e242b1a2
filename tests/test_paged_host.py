"""Refusals of the paged cache's entry points, through the C ABI and the binding (no GPU needed): every bad
argument returns its status before any device work, and a well-formed call fails only for want of a device."""
import ctypes

import pytest
import torch

import paper_2609_03235_amd as sg

A = 1 << 20  # an aligned address; nothing here is dereferenced


def _gpu():
    try:
        return torch.cuda.is_available()
    except Exception:
        return False


def _pool(**kw):
    f = dict(k_pages=A, v_pages=A, num_pages=10, page_size=16, head_dim=128, dtype=sg.DTYPE_BF16, reserved=0)
    f.update(kw)
    return sg.PagePool(*f.values())


def _status(fn, *args):
    lib = sg.load_library()
    st = getattr(lib, fn)(*[ctypes.byref(x) if isinstance(x, ctypes.Structure) else x for x in args])
    assert st == sg.OK or lib.sgdkv_last_error()
    return st


def _update(ptrs=None, **kw):
    f = dict(batch=2, num_kv_heads=2, page_size=16, max_pages=8, by_segment=0, reserved=0, num_free=50, num_slots=4)
    f.update(kw)
    p = [A] * 10
    for i, x in (ptrs or {}).items():
        p[i] = x
    return _status("sgdkv_page_update", sg.PageDesc(*f.values()), *p, None)


@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(num_kv_heads=0), dict(page_size=8), dict(page_size=24), dict(page_size=2048), dict(max_pages=0),
    dict(max_pages=2**27), dict(by_segment=2), dict(reserved=1), dict(num_free=0), dict(num_free=2**31),
    dict(num_slots=-1), dict(num_slots=2**30), dict(num_slots=2**31, by_segment=1)])
def test_page_update_sizes(kw):
    assert _update(**kw) == sg.ERR_INVALID_ARG


def test_page_update_pointers_and_limits():
    for i in range(10):
        assert _update({i: None}) == sg.ERR_INVALID_ARG
        assert _update({i: A + 4}) == sg.ERR_INVALID_ARG
    assert _update(batch=2049) == sg.ERR_UNSUPPORTED
    assert _status("sgdkv_page_update", None, *[A] * 10, None) == sg.ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(num_pages=0), 1), (dict(num_pages=2**27), 1), (dict(page_size=15), 1), (dict(page_size=1 << 11), 1),
    (dict(head_dim=96), 2), (dict(dtype=2), 1), (dict(reserved=3), 1), (dict(k_pages=None), 1),
    (dict(v_pages=A + 8), 1)])
def test_bad_pools(kw, status):
    pool = _pool(**kw)
    assert _status("sgdkv_paged_store", pool, A, A, A, 4, None) == status
    assert _status("sgdkv_norm_rope_store", pool, _rope_desc(), *[A] * 9, None) == status
    assert _status("sgdkv_paged_attention", pool, _attn_desc(), A, A, A, A, A, A, A, 1 << 40, None) == status


def test_paged_store_refusals():
    for p in ((None, A, A), (A, None, A), (A, A, None), (A + 2, A, A), (A, A, A + 4)):
        assert _status("sgdkv_paged_store", _pool(), *p, 4, None) == sg.ERR_INVALID_ARG
    for n in (-1, 1 << 40):
        assert _status("sgdkv_paged_store", _pool(), A, A, A, n, None) == sg.ERR_INVALID_ARG
    assert _status("sgdkv_paged_store", None, A, A, A, 4, None) == sg.ERR_INVALID_ARG


def _rope_desc(**kw):
    f = dict(num_tokens=3, num_q_heads=4, num_kv_heads=2, q_stride=512, k_stride=256, v_stride=256, rot_dim=128,
             interleaved=0, eps=1e-6, reserved=0)
    f.update(kw)
    return sg.NormRopeDesc(*f.values())


@pytest.mark.parametrize("kw", [
    dict(num_tokens=-1), dict(num_tokens=2**31), dict(num_q_heads=-1), dict(num_kv_heads=0), dict(q_stride=511),
    dict(q_stride=516), dict(k_stride=255), dict(v_stride=0), dict(v_stride=2**31), dict(rot_dim=144),
    dict(rot_dim=-16),
    dict(rot_dim=24), dict(interleaved=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(reserved=1)])
def test_norm_rope_sizes(kw):
    assert _status("sgdkv_norm_rope_store", _pool(), _rope_desc(**kw), *[A] * 9, None) == sg.ERR_INVALID_ARG


def test_norm_rope_pointers():
    for i in range(9):
        args = [A] * 8 + [2 * A]
        args[i] = A + 4
        assert _status("sgdkv_norm_rope_store", _pool(), _rope_desc(), *args, None) == sg.ERR_INVALID_ARG
        if i not in (6, 7):  # the weights are optional
            args[i] = None
            assert _status("sgdkv_norm_rope_store", _pool(), _rope_desc(), *args, None) == sg.ERR_INVALID_ARG
    assert _status("sgdkv_norm_rope_store", _pool(), None, *[A] * 9, None) == sg.ERR_INVALID_ARG
    assert _status("sgdkv_norm_rope_store", _pool(), _rope_desc(num_q_heads=9000, q_stride=9000 * 128), *[A] * 9,
                   None) == sg.ERR_UNSUPPORTED
    # q_out may be q only where q is dense
    assert _status("sgdkv_norm_rope_store", _pool(), _rope_desc(q_stride=1024), *[A] * 9, None) == sg.ERR_INVALID_ARG


def _attn_desc(**kw):
    f = dict(batch=2, num_q_heads=8, num_kv_heads=2, out_dtype=0, num_tokens=6, max_new=4, max_pages=8, causal=1,
             scale=0.0)
    f.update(kw)
    return sg.PagedDesc(*f.values())


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), 1), (dict(num_q_heads=0), 1), (dict(num_kv_heads=0), 1), (dict(num_kv_heads=3), 1),
    (dict(num_q_heads=34), 2), (dict(num_q_heads=8448, num_kv_heads=528), 2), (dict(batch=40000), 2),
    (dict(out_dtype=3), 1), (dict(num_tokens=-1), 1), (dict(num_tokens=2**31), 1), (dict(max_new=0), 1),
    (dict(causal=2), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(max_pages=0), 1),
    (dict(max_pages=2**27), 1)])
def test_paged_attention_sizes(kw, status):
    n = ctypes.c_size_t(0)
    if "max_pages" not in kw:
        assert _status("sgdkv_paged_attention_workspace_size", _pool(), _attn_desc(**kw), ctypes.byref(n)) == status
    assert _status("sgdkv_paged_attention", _pool(), _attn_desc(**kw), A, A, A, A, A, A, A, 1 << 40, None) == status


@pytest.mark.parametrize("scale", [3e38, -3e38, 2.4e38, float("-inf")])
def test_paged_attention_scales_that_the_kernels_cannot_hold(scale):
    """The kernels take scale * log2(e) in fp32: past 2.358e38 that is infinite, and every logit of 0 would be NaN."""
    n = ctypes.c_size_t(0)
    desc = _attn_desc(scale=scale)
    assert _status("sgdkv_paged_attention_workspace_size", _pool(), desc, ctypes.byref(n)) == sg.ERR_INVALID_ARG
    assert _status("sgdkv_paged_attention", _pool(), desc, *[A] * 7, 1 << 40, None) == sg.ERR_INVALID_ARG
    assert _status("sgdkv_paged_attention_workspace_size", _pool(), _attn_desc(scale=2.3e38), ctypes.byref(n)) == sg.OK


def test_paged_attention_pointers_and_workspace():
    for i in range(6):
        args = [A] * 6
        args[i] = A + 4
        assert _status("sgdkv_paged_attention", _pool(), _attn_desc(), *args, A, 1 << 40, None) == sg.ERR_INVALID_ARG
        if i != 5:  # lse_out is optional
            args[i] = None
            assert _status("sgdkv_paged_attention", _pool(), _attn_desc(), *args, A, 1 << 40,
                           None) == sg.ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    assert _status("sgdkv_paged_attention_workspace_size", _pool(), _attn_desc(), ctypes.byref(n)) == sg.OK
    assert 0 < n.value <= 70_000_000
    for ws, size in ((None, n.value), (A + 128, n.value), (A, n.value - 1)):
        assert _status("sgdkv_paged_attention", _pool(), _attn_desc(), *[A] * 6, ws, size, None) == sg.ERR_WORKSPACE
    assert _status("sgdkv_paged_attention_workspace_size", _pool(), _attn_desc(), None) == sg.ERR_INVALID_ARG
    assert _status("sgdkv_paged_attention_workspace_size", _pool(), None, ctypes.byref(n)) == sg.ERR_INVALID_ARG


def test_workspace_grows_with_the_bound():
    size = lambda max_new: sg.paged_attention_workspace_size(torch.zeros(1, 8, 128), 2, 1, max_new=max_new)
    sizes = [size(n) for n in (1, 4, 5, 8, 9, 1000, 1 << 30)]
    assert sizes == sorted(sizes) and sizes[-1] <= 70_000_000


@pytest.mark.skipif(_gpu(), reason="checks the no-device path")
def test_no_device_fails_after_validation():
    assert _update() == sg.ERR_HIP
    assert _status("sgdkv_paged_store", _pool(), A, A, A, 4, None) == sg.ERR_HIP
    assert _status("sgdkv_norm_rope_store", _pool(), _rope_desc(), *[A] * 8, 2 * A, None) == sg.ERR_HIP
    assert _status("sgdkv_paged_attention", _pool(), _attn_desc(), *[A] * 6, A, 1 << 40, None) == sg.ERR_HIP


# ------------------------------------------------------------------ the binding
def _refused(fn, *args, **kw):
    with pytest.raises(sg.SgdkvError) as e:
        fn(*args, **kw)
    assert e.value.status == sg.ERR_INVALID_ARG


def test_binding_refuses_shapes_types_and_host_tensors():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    pages = torch.zeros(4, 16, 64)
    _refused(sg.page_update, i32(2), i32(2), i32(2, 4), i32(9), i32(1), page_size=16, n_slots=2)  # not on a GPU
    _refused(sg.paged_store, torch.zeros(3, 64), torch.zeros(3, 64), i32(3), pages, pages)
    _refused(sg.norm_rope_store, None, torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), i32(3), i32(3, 2), pages, pages)
    _refused(sg.paged_attention, torch.zeros(3, 4, 64), pages, pages, i32(2, 4), i32(2), i32(2), 2, max_new=3)
    for bad in ((pages[:, :, :32], pages[:, :, :32]), (pages, pages[:2]), (pages, pages.bfloat16()),
                (pages[0], pages[0]), (pages.half(), pages.half())):
        _refused(sg.page_pool, *bad)
