"""The 8-bit floating point layers without a GPU: what the library refuses before it touches the device, and the reference that the
GPU tests go by against torch's own E4M3 conversion."""
import ctypes as C
import os

import numpy as np
import pytest

import fp8_reference as ref
import paper_2510_26771_amd as st
from paper_2510_26771_amd import fp8


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(st.lib_path()):
        from paper_2510_26771_amd.build import build
        build(verbose=False)
    return st.load_library()


def _create(lib, W=256, scales=256, bias=None, **kw):
    d = st.Fp8Desc(**{**dict(d_in=256, d_out=128), **kw})
    h = C.c_void_p()
    rc = lib.stamp_fp8_plan_create(C.byref(d.to_c()), W, scales, bias, None, C.byref(h))
    assert not h.value
    return rc


@pytest.mark.parametrize("kw,expect", [
    (dict(d_in=0), 2), (dict(d_out=0), 2), (dict(d_in=-4), 2), (dict(experts=-1), 2), (dict(gated=2), 2), (dict(gated=1), 2), (dict(x_dtype=2), 2),
    (dict(y_dtype=5), 2), (dict(w_dtype=3), 2), (dict(scale_format=2), 2), (dict(w_is_out_by_in=3), 2), (dict(d_in=65537), 3), (dict(d_out=(1 << 20) + 1), 3),
    (dict(experts=1025), 3), (dict(w_is_out_by_in=0), 3), (dict(W=None), 1), (dict(scales=None), 1), (dict(w_dtype=0), 1),  # scales beside fp32 weights
    (dict(experts=2, gated=1, bias=256), 3)])
def test_plan_create_refuses_before_any_device_call(lib, kw, expect):
    assert _create(lib, **kw) == expect


def test_null_and_empty(lib):
    r = fp8._Routing(0, 4, 2, None, None, None, None, None)
    assert lib.stamp_fp8_plan_create(None, None, None, None, None, None) == 1
    assert lib.stamp_fp8_plan_destroy(None) == 1
    assert lib.stamp_fp8_workspace_bytes(None, 5) == 0
    assert lib.stamp_fp8_quantize_act(None, 1, None, 0, None, None, 0, None) == 1
    assert lib.stamp_fp8_linear_forward(None, 1, None, 0, None, 0, None, 0, None) == 1
    assert lib.stamp_fp8_linear_forward_q(None, 1, None, None, 0, None, 0, None, 0, None) == 1
    assert lib.stamp_fp8_grouped_forward(None, 1, None, None, 0, None, 0, None, 0, None) == 1
    assert lib.stamp_fp8_debug_weight_codes(None, None, None) == 1
    assert lib.stamp_fp8_debug_route(None, 4) == 0
    assert lib.stamp_route_topk(None, None, 0, 0, 1, None, 0, None) == 1
    assert lib.stamp_route_topk(C.byref(r), None, 0, 4, 1, None, 0, None) == 1
    assert lib.stamp_experts_workspace_bytes(None, None, 4, 2) == 0
    assert lib.stamp_experts_forward(None, None, None, None, 0, None, 0, None, 0, None) == 1


@pytest.mark.parametrize("tokens,experts,top_k,ld,dtype,renorm,expect", [
    (-1, 4, 1, 4, 0, 1, 2), (4, 0, 1, 4, 0, 1, 2), (4, 4, 0, 4, 0, 1, 2), (4, 1025, 1, 1025, 0, 1, 3), (4, 64, 33, 64, 0, 1, 3), ((1 << 22) + 1, 4, 1, 4, 0, 1, 3),
    (4, 4, 1, 3, 0, 1, 2), (4, 4, 1, 4, 2, 1, 2), (4, 4, 1, 4, 0, 2, 2), (4, 4, 1, (1 << 21) + 1, 0, 1, 3), (4, 4, 1, 4, 0, 1, 4)])
def test_router_refuses_before_any_device_call(lib, tokens, experts, top_k, ld, dtype, renorm, expect):
    r = fp8._Routing(tokens, experts, top_k, 256, 256, 256, 256, 256)
    assert lib.stamp_route_topk(C.byref(r), 256, dtype, ld, renorm, None, 0, None) == expect


def test_router_workspace_grows_with_the_tokens(lib):
    sizes = [lib.stamp_route_workspace_bytes(t, 64, 4) for t in (0, 1, 128, 129, 4096, 1 << 22)]
    assert all(s > 0 and s % 256 == 0 for s in sizes) and sizes == sorted(sizes)
    assert lib.stamp_route_workspace_bytes(1, 0, 1) == 0 and lib.stamp_route_workspace_bytes(1, 4, 33) == 0


def test_reference_codes_are_e4m3():
    import torch
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(every, ref.E4M3.astype(np.float32), equal_nan=True)
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-460, 460, 20000), rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 6, 20000), ref.E4M3[:127][:-1] + np.diff(ref.E4M3[:127]) / 2])
    v = v.astype(np.float32)
    assert np.array_equal(ref.encode(v), torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("pow2", [0, 1])
def test_reference_scales(pow2):
    """No code beyond 448, the error of a value at most half a step of its binade, a power of two where one is asked for."""
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((50, 300)) * 2.0 ** rng.integers(-20, 20, (50, 1))).astype(np.float32)
    codes, scales = ref.quantize(x, pow2)
    v = ref.values(codes, scales, 300)
    sc = np.repeat(scales.astype(np.float64), 128, 1)[:, :300]
    assert np.all(np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, sc * 2.0 ** -10) * (1 + 1e-6))
    if pow2:
        assert np.all(np.frexp(scales)[0] == 0.5)
