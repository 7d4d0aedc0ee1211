"""Epilogue, dense MLP and layer of experts without a GPU: what is refused before the device is touched, and that the GPU tests' bounds see
mistakes."""
import ctypes as C

import numpy as np
import pytest
import torch

import fp8_block_reference as block
import fp8_reference as ref
import paper_2510_26771_amd as st
from paper_2510_26771_amd import fp8
from test_fp8_calls_host import D, EXPERTS, N, ROWS, OnGpu, lib, on_cpu  # noqa: F401  (fixtures)


def test_null(lib):  # noqa: F811
    ep, router = C.byref(fp8._Epilogue(0, None, 0)), C.byref(fp8._Router(None, 0, 1, None))
    r = fp8._Routing(4, 4, 2, None, None, None, None, None)
    for e in (None, ep):
        assert lib.stamp_fp8_linear_forward_act(None, 1, None, 0, e, None, 0, None, 0, None) == 1
        assert lib.stamp_fp8_linear_forward_q_act(None, 1, None, None, 0, e, None, 0, None, 0, None) == 1
        assert lib.stamp_fp8_grouped_forward_act(None, 1, None, None, 0, e, None, 0, None, 0, None) == 1
        assert lib.stamp_mlp_forward(None, None, 1, None, 0, e, None, 0, None, 0, None) == 1
        assert lib.stamp_moe_forward(router, None, None, C.byref(r), None, 0, e, None, 0, None, 0, None) == 1
    assert lib.stamp_mlp_workspace_bytes(None, None, 4) == 0
    assert lib.stamp_moe_workspace_bytes(None, None, 4, 2) == 0
    assert lib.stamp_moe_debug_route(None, None, 4, 2) == 0


def _calls(plan, r):
    """(call of keyword tensors, those tensors) of every entry point."""
    bf16 = torch.bfloat16
    x, y, codes, scales = torch.zeros(ROWS, D, dtype=bf16), torch.zeros(ROWS, N, dtype=bf16), torch.zeros(ROWS, D, dtype=torch.uint8), torch.zeros(2, 8)
    ws, offsets, z = torch.zeros(4096, dtype=torch.uint8), torch.zeros(EXPERTS + 1, dtype=torch.int32), torch.zeros(ROWS, D, dtype=bf16)
    dense, back, grouped = plan(), plan(d_in=N, d_out=D), plan(experts=EXPERTS)
    up, down = plan(experts=EXPERTS, gated=1), plan(d_in=N, d_out=D, experts=EXPERTS)
    return {
        "linear": (lambda X, Y, workspace, residual: dense.linear_forward(X, Y, workspace, activation="gelu", residual=residual), dict(X=x, Y=y, workspace=ws, residual=y)),
        "linear_q": (lambda codes, scales, Y, workspace, residual: dense.linear_forward_q(codes, scales, Y, workspace, residual=residual),
                     dict(codes=codes, scales=scales, Y=y, workspace=ws, residual=y)),
        "grouped": (lambda X, offsets, Y, workspace, residual: grouped.grouped_forward(X, offsets, Y, workspace, activation="relu", residual=residual),
                    dict(X=x, offsets=offsets, Y=y, workspace=ws, residual=y)),
        "mlp": (lambda X, Y, workspace, residual: st.mlp_forward(dense, back, X, Y, workspace, "silu", residual=residual), dict(X=x, Y=z, workspace=ws, residual=z)),
        "moe": (lambda router, router_bias, X, Y, workspace, residual: st.moe_forward(router, up, down, X, r, Y, workspace, router_bias=router_bias, residual=residual),
                dict(router=torch.zeros(EXPERTS, D, dtype=bf16), router_bias=torch.zeros(EXPERTS), X=x, Y=z, workspace=ws, residual=z)),
    }


NAMES = ("linear", "linear_q", "grouped", "mlp", "moe")


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_the_host_or_another_gpu_are_refused(on_cpu, name):  # noqa: F811
    lib, plan, r = on_cpu  # noqa: F811
    call, tensors = _calls(plan, r)[name]
    for which in tensors:
        for bad in (tensors[which], OnGpu(tensors[which], 1)):
            with pytest.raises(ValueError):
                call(**{n: bad if n == which else OnGpu(t) for n, t in tensors.items()})
            assert not lib.names, f"{which} got through"
    call(**{n: OnGpu(t) for n, t in tensors.items()})
    assert len(lib.names) == 1


@pytest.mark.parametrize("name", NAMES)
def test_workspaces_with_gaps_and_tensors_of_other_shapes_or_types_are_refused(on_cpu, name):  # noqa: F811
    lib, plan, r = on_cpu  # noqa: F811
    call, tensors = _calls(plan, r)[name]
    good = {n: OnGpu(t) for n, t in tensors.items()}
    for which, t in tensors.items():
        wrong = [None, OnGpu(torch.zeros(64, 128, dtype=torch.uint8)[:, :64])] if which == "workspace" else [OnGpu(t.double())]
        if which not in ("workspace", "offsets", "router_bias"):
            wrong.append(OnGpu(t[:, :-1]))
        for bad in wrong:
            with pytest.raises(ValueError):
                call(**{**good, which: bad})
    assert not lib.names


def test_an_unknown_activation_is_refused(on_cpu):  # noqa: F811
    lib, plan, r = on_cpu  # noqa: F811
    x, y, ws = OnGpu(torch.zeros(ROWS, D, dtype=torch.bfloat16)), OnGpu(torch.zeros(ROWS, N, dtype=torch.bfloat16)), OnGpu(torch.zeros(64, dtype=torch.uint8))
    for name in ("tanh", "", None, 1):
        with pytest.raises(ValueError):
            plan().linear_forward(x, y, ws, activation=name)
    assert not lib.names


def test_calls_without_an_epilogue_are_what_they_were(on_cpu):  # noqa: F811
    lib, plan, r = on_cpu  # noqa: F811
    x, y, ws = OnGpu(torch.zeros(ROWS, D, dtype=torch.bfloat16)), OnGpu(torch.zeros(ROWS, N, dtype=torch.bfloat16)), OnGpu(torch.zeros(64, dtype=torch.uint8))
    plan().linear_forward(x, y, ws, activation="none", residual=None)
    plan().linear_forward(x, y, ws, activation="relu")
    assert lib.names == ["stamp_fp8_linear_forward", "stamp_fp8_linear_forward_act"]


# ---- the reference ----

def test_activations_are_torchs():
    z = torch.linspace(-12, 12, 4001, dtype=torch.float64)
    for name, f in (("relu", torch.relu), ("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu),
                    ("gelu_tanh", lambda v: torch.nn.functional.gelu(v, approximate="tanh"))):
        assert np.allclose(block.activation(z.numpy(), name), f(z).numpy(), rtol=1e-9, atol=1e-12), name


def test_the_bounds_tell_one_activation_from_another_and_see_lost_terms():
    rng = np.random.default_rng(0)
    rows, d, ff, n = 20, 300, 257, 140
    x = rng.standard_normal((rows, d)).astype(np.float32)
    w, ws = ref.quantize_weights((rng.standard_normal((ff, d)) / 17).astype(np.float32), 0)
    w2, ws2 = ref.quantize_weights((rng.standard_normal((n, ff)) / 10).astype(np.float32), 0)
    bias, res = rng.standard_normal(ff).astype(np.float32), rng.standard_normal((rows, ff))
    for y in ("f32", "bf16"):
        want, tol = block.layer(x, w, ws, bias, "gelu", res, y, 0, y == "f32")
        for other in (block.layer(x, w, ws, bias, "silu", res, y, 0, True), block.layer(x, w, ws, bias, "gelu", None, y, 0, True), block.layer(x, w, ws, None, "gelu", res, y, 0, True)):
            assert np.mean(np.abs(other[0] - want) > tol) > 0.5
    want, tol = block.layer(x, w, ws, bias, "gelu", res, "f32", 0, True)
    assert np.mean(np.abs(block.layer(x, w, ws, bias, "gelu_tanh", res, "f32", 0, True)[0] - want) > tol) > 0.5
    want, tol = block.mlp(x, w, ws, bias, w2, ws2, None, "silu", None, "f32", 0)
    assert np.median(tol / np.abs(want)) < 0.01
    codes, scales = ref.quantize(x, 0)
    h, _ = block.hidden(codes, scales, w, ws, bias, "silu")
    rounded = torch.from_numpy(h.astype(np.float32)).to(torch.bfloat16).float().numpy()  # h held in bf16 ahead of its codes
    lost = ref.values(*ref.quantize(rounded, 0), ff) @ ref.weight_values(w2, ws2).T
    assert np.mean(np.abs(lost - want) > tol) > 0.3


def test_looks_of_no_plan(lib):  # noqa: F811
    assert lib.stamp_moe_debug_set_looks(None, 0) == 1


def test_the_route_of_no_mlp(lib):  # noqa: F811
    out = (C.c_int32 * 3)(7, 7, 7)
    assert lib.stamp_mlp_debug_route(None, None, 4, out) == 1 and lib.stamp_mlp_debug_route(None, None, 4, None) == 1
    assert list(out) == [7, 7, 7]
