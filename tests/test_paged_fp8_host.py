"""Refusals of the 8-bit paged cache's entry points, through the C ABI and the binding (no GPU needed), and their host
layer under the sanitizers: every bad argument returns its status before any device work, and a well-formed call fails
only for want of a device."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_03235_amd as sg
from test_paged_host import A, _attn_desc, _gpu, _refused, _rope_desc, _status

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _pool(**kw):
    f = dict(k_pages=A, v_pages=A, k_scales=A, v_scales=A, num_pages=10, page_size=16, head_dim=128,
             row_dtype=sg.DTYPE_BF16, reserved=0)
    f.update(kw)
    return sg.PagePoolFp8(*f.values())


def _rope(pool, desc, ptrs, factor=1.0):
    return _status("sgdkv_norm_rope_store_fp8", pool, desc, factor, *ptrs, None)


@pytest.mark.parametrize("kw,status", [
    (dict(num_pages=0), 1), (dict(num_pages=2**27), 1), (dict(page_size=15), 1), (dict(page_size=8), 1),
    (dict(page_size=1 << 11), 1), (dict(head_dim=96), 2), (dict(row_dtype=2), 1), (dict(row_dtype=-1), 1),
    (dict(reserved=3), 1), (dict(k_pages=None), 1), (dict(v_pages=A + 8), 1), (dict(k_scales=None), 1),
    (dict(v_scales=None), 1), (dict(k_scales=A + 1), 1), (dict(v_scales=A + 4), 1)])
def test_bad_pools(kw, status):
    pool = _pool(**kw)
    assert _status("sgdkv_paged_store_fp8", pool, A, A, A, 4, None) == status
    assert _rope(pool, _rope_desc(), [A] * 9) == status
    assert _status("sgdkv_paged_attention_fp8", pool, _attn_desc(), *[A] * 7, 1 << 40, None) == status


def test_paged_store_fp8_refusals():
    for p in ((None, A, A), (A, None, A), (A, A, None), (A + 2, A, A), (A, A + 8, A), (A, A, A + 4)):
        assert _status("sgdkv_paged_store_fp8", _pool(), *p, 4, None) == sg.ERR_INVALID_ARG
    for n in (-1, 1 << 40):
        assert _status("sgdkv_paged_store_fp8", _pool(), A, A, A, n, None) == sg.ERR_INVALID_ARG
    assert _status("sgdkv_paged_store_fp8", None, A, A, A, 4, None) == sg.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(num_tokens=-1), dict(num_tokens=2**31), dict(num_q_heads=-1), dict(num_kv_heads=0), dict(q_stride=511),
    dict(q_stride=516), dict(k_stride=255), dict(v_stride=0), dict(v_stride=2**31), dict(rot_dim=144),
    dict(rot_dim=-16), dict(rot_dim=24), dict(interleaved=2), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(reserved=1)])
def test_norm_rope_store_fp8_sizes(kw):
    assert _rope(_pool(), _rope_desc(**kw), [A] * 9) == sg.ERR_INVALID_ARG


def test_norm_rope_store_fp8_pointers_and_factor():
    for i in range(9):
        args = [A] * 8 + [2 * A]
        args[i] = A + 4
        assert _rope(_pool(), _rope_desc(), args) == sg.ERR_INVALID_ARG
        if i not in (6, 7):  # the weights are optional
            args[i] = None
            assert _rope(_pool(), _rope_desc(), args) == sg.ERR_INVALID_ARG
    for factor in (float("nan"), float("inf"), -float("inf")):
        assert _rope(_pool(), _rope_desc(), [A] * 8 + [2 * A], factor) == sg.ERR_INVALID_ARG
    assert _rope(_pool(), None, [A] * 9) == sg.ERR_INVALID_ARG
    assert _rope(None, _rope_desc(), [A] * 9) == sg.ERR_INVALID_ARG
    assert _rope(_pool(), _rope_desc(num_q_heads=9000, q_stride=9000 * 128), [A] * 9) == sg.ERR_UNSUPPORTED
    # q_out may be q only where q is dense
    assert _rope(_pool(), _rope_desc(q_stride=1024), [A] * 9) == sg.ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), 1), (dict(num_q_heads=0), 1), (dict(num_kv_heads=0), 1), (dict(num_kv_heads=3), 1),
    (dict(num_q_heads=34), 2), (dict(num_q_heads=8448, num_kv_heads=528), 2), (dict(batch=40000), 2),
    (dict(out_dtype=3), 1), (dict(num_tokens=-1), 1), (dict(num_tokens=2**31), 1), (dict(max_new=0), 1),
    (dict(causal=2), 1), (dict(scale=float("nan")), 1), (dict(scale=3e38), 1), (dict(max_pages=0), 1),
    (dict(max_pages=2**27), 1)])
def test_paged_attention_fp8_sizes(kw, status):
    n = ctypes.c_size_t(0)
    if "max_pages" not in kw:
        assert _status("sgdkv_paged_attention_fp8_workspace_size", _pool(), _attn_desc(**kw),
                       ctypes.byref(n)) == status
    assert _status("sgdkv_paged_attention_fp8", _pool(), _attn_desc(**kw), *[A] * 7, 1 << 40, None) == status


def test_paged_attention_fp8_pointers_and_workspace():
    for i in range(6):
        args = [A] * 6
        args[i] = A + 4
        assert _status("sgdkv_paged_attention_fp8", _pool(), _attn_desc(), *args, A, 1 << 40,
                       None) == sg.ERR_INVALID_ARG
        if i != 5:  # lse_out is optional
            args[i] = None
            assert _status("sgdkv_paged_attention_fp8", _pool(), _attn_desc(), *args, A, 1 << 40,
                           None) == sg.ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    size = "sgdkv_paged_attention_fp8_workspace_size"
    assert _status(size, _pool(k_pages=None, v_scales=None), _attn_desc(), ctypes.byref(n)) == sg.OK
    assert 0 < n.value <= 70_000_000
    for ws, have in ((None, n.value), (A + 128, n.value), (A, n.value - 1)):
        assert _status("sgdkv_paged_attention_fp8", _pool(), _attn_desc(), *[A] * 6, ws, have,
                       None) == sg.ERR_WORKSPACE
    assert _status(size, _pool(), _attn_desc(), None) == sg.ERR_INVALID_ARG
    assert _status(size, _pool(), None, ctypes.byref(n)) == sg.ERR_INVALID_ARG
    assert _status(size, None, _attn_desc(), ctypes.byref(n)) == sg.ERR_INVALID_ARG
    for kw, status in ((dict(reserved=1), 1), (dict(row_dtype=7), 1), (dict(head_dim=32), 2)):
        assert _status(size, _pool(**kw), _attn_desc(), ctypes.byref(n)) == status


def test_workspace_grows_with_the_bound():
    for dtype in (torch.float32, torch.bfloat16):
        q = torch.zeros(1, 8, 128, dtype=dtype)
        sizes = [sg.paged_attention_fp8_workspace_size(q, 2, 1, max_new=n) for n in (1, 4, 5, 8, 9, 1000, 1 << 30)]
        assert sizes == sorted(sizes) and sizes[-1] <= 70_000_000


@pytest.mark.skipif(_gpu(), reason="checks the no-device path")
def test_no_device_fails_after_validation():
    assert _status("sgdkv_paged_store_fp8", _pool(), A, A, A, 4, None) == sg.ERR_HIP
    assert _rope(_pool(), _rope_desc(), [A] * 8 + [2 * A]) == sg.ERR_HIP
    assert _status("sgdkv_paged_attention_fp8", _pool(), _attn_desc(), *[A] * 7, 1 << 40, None) == sg.ERR_HIP


# ------------------------------------------------------------------ the binding
def test_binding_refuses_shapes_types_and_host_tensors():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    pages = torch.zeros(4, 16, 64, dtype=torch.float8_e4m3fn)
    scales = torch.zeros(4, 16, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    pool = (pages, pages, scales, scales)
    rows = torch.zeros(3, 64)
    _refused(sg.paged_store_fp8, rows, rows, i32(3), *pool)  # not on a GPU
    _refused(sg.norm_rope_store_fp8, None, rows[:, None], rows[:, None], i32(3), i32(3, 1), *pool)
    _refused(sg.paged_attention_fp8, torch.zeros(3, 4, 64), *pool, i32(2, 4), i32(2), i32(2), 2, max_new=3)
    sg.page_pool_fp8(*pool, torch.float32)
    sg.page_pool_fp8(*pool, torch.bfloat16)
    half = scales.view(torch.uint8)
    for bad in ((pages[:, :, :32], pages[:, :, :32], scales, scales), (pages, pages[:2], scales, scales),
                (pages, pages, scales[:2], scales), (pages, pages, scales, scales[:, :8]),
                (pages[0], pages[0], scales, scales),
                (pages.float(), pages, scales, scales), (pages, pages.view(torch.uint8), scales, scales),
                (pages, pages, half, scales), (pages, pages, scales, scales.float()),
                (pages, pages, scales, scales.t().contiguous().t())):
        _refused(sg.page_pool_fp8, *bad, torch.float32)
    for dtype in (torch.float16, torch.float64, torch.float8_e4m3fn, torch.int32):
        _refused(sg.page_pool_fp8, *pool, dtype)


@pytest.mark.parametrize("out_dtype", [None, torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_results_are_dense_whatever_the_strides_of_one_token(dtype, out_dtype):
    """One token cut from a wider projection is contiguous for torch with any stride between tokens; the results that
    the attention calls allocate are not laid out after it."""
    q = torch.zeros(1, 12, 64, dtype=dtype)[:, :4]
    assert q.is_contiguous() and q.stride() == (768, 64, 1)
    i32 = torch.zeros(4, dtype=torch.int32)
    desc = sg._paged_desc(q, 2, 1, 1, 4, out_dtype, True, 0.0)
    done = lambda *args: 0  # stands in for the library's call
    out, lse = sg._attend(done, None, sg.PagePool(), desc, q, i32, i32, i32, True, None, None, i32, None)
    assert out.shape == (1, 4, 64) and out.stride() == (256, 64, 1) and out.dtype is (out_dtype or dtype)
    assert lse.shape == (1, 4) and lse.stride() == (4, 1) and lse.dtype is torch.float32


# ------------------------------------------------------------------ the launchers
@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/lib/libamdhip64.so"),
                    reason="needs g++ and the HIP host runtime")
@pytest.mark.skipif(_gpu(), reason="host-only run")
def test_the_launcher_of_many_rows_refuses_queries_it_has_no_instance_for(tmp_path):
    sg.load_library()
    package = os.path.dirname(sg.__file__)
    exe = str(tmp_path / "paged_fp8_launch")
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-isystem", "/opt/rocm/include", "-I",
                    os.path.join(package, "csrc"), os.path.join(ROOT, "tests", "sanitize", "paged_fp8_launch.cpp"), "-o",
                    exe, "-L" + package, "-l:libsgdkv.so", "-Wl,-rpath," + package, "-L/opt/rocm/lib",
                    "-Wl,-rpath,/opt/rocm/lib", "-lamdhip64"], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "REFUSED\n", r.stdout + r.stderr


# ------------------------------------------------------------------ sanitizers
@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/lib/libamdhip64.so"),
                    reason="needs g++ and the HIP host runtime")
@pytest.mark.skipif(_gpu(), reason="host-only run: the device entry points are driven through validation only")
def test_paged_fp8_host_under_sanitizers(tmp_path):
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1"]
    csrc, here = os.path.join(ROOT, "paper_2609_03235_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize")
    exe = str(tmp_path / "paged_fp8_driver")
    sources = [os.path.join(csrc, f) for f in ("sgdkv_host.cpp", "paged_fp8_host.cpp", "profile.cpp")]
    sources += [os.path.join(here, f) for f in ("launch_stubs.cpp", "paged_fp8_driver.cpp")]
    subprocess.run(["g++", "-std=c++17", *san, "-ffp-contract=off", "-fno-fast-math", "-D__HIP_PLATFORM_AMD__",
                    "-isystem", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc, *sources, "-o",
                    exe, "-L/opt/rocm/lib", "-Wl,-rpath,/opt/rocm/lib", "-lamdhip64", "-lm"], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, f"sanitizer run failed (rc {r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-6000:]}"
    assert "SANITIZE PASS" in r.stdout
