"""Calls of the 8-bit floating point layers and the router at their limits, without a GPU."""
import os

import pytest
import torch

import paper_2510_26771_amd as st
from paper_2510_26771_amd import fp8


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(st.lib_path()):
        from paper_2510_26771_amd.build import build
        build(verbose=False)
    return st.load_library()


@pytest.mark.parametrize("experts", [1, 20, 64, 255, 256, 257, 1000, 1024])
def test_a_router_workspace_serves_every_smaller_call(lib, experts):
    """Around every step of the tokens of a workgroup (64 or 16 at once, 256 workgroups at most), up to the largest call."""
    tokens = sorted({t for m in range(1, 40) for t in (4096 * m - 1, 4096 * m, 4096 * m + 1)} | {0, 1, 15, 16, 17, 63, 64, 65, (1 << 22) - 1, 1 << 22})
    sizes = [lib.stamp_route_workspace_bytes(t, experts, 4) for t in tokens]
    falls = [(tokens[i], sizes[i], tokens[i + 1], sizes[i + 1]) for i in range(len(tokens) - 1) if sizes[i + 1] < sizes[i]]
    assert not falls, f"{len(falls)} steps down, the first (tokens, bytes): {falls[0]}"


def test_the_cut_of_no_plan(lib):
    assert lib.stamp_fp8_debug_cut(None, 4, None) == 1


# ---- what the Python calls refuse: the library gets addresses, and a host's or another GPU's would fault the kernels ----

class OnGpu:
    """A host tensor that says it lies on a GPU."""

    def __init__(self, tensor, index=0):
        self.tensor, self.is_cuda, self.get_device = tensor, True, lambda: index

    def __getattr__(self, name):
        return getattr(self.tensor, name)


class Calls:
    """The library's place: notes the names of the calls that get through."""

    def __init__(self):
        self.names, self.arguments = [], []

    def __getattr__(self, name):
        def call(*arguments):
            self.names.append(name)
            self.arguments.append(arguments)
            return 0
        return call


ROWS, D, N, EXPERTS = 6, 256, 128, 2


@pytest.fixture
def on_cpu(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: 0)
    lib = Calls()

    def plan(**kw):
        p = object.__new__(fp8.Fp8Plan)
        p.lib, p.desc, p._h = lib, st.Fp8Desc(**{**dict(d_in=D, d_out=N), **kw}), None
        p._x_dtype = p._y_dtype = torch.bfloat16
        p.gpu = 0
        return p
    r = object.__new__(st.Routing)
    r.lib, r.tokens, r.experts, r.top_k, r.gpu, r._c = lib, ROWS, EXPERTS, 1, 0, fp8._Routing(ROWS, EXPERTS, 1)
    r.workspace = OnGpu(torch.empty(512, dtype=torch.uint8))
    return lib, plan, r


def _calls(plan, r):
    """(call of keyword tensors, those tensors) of every entry point."""
    bf16 = torch.bfloat16
    x, y, codes, scales = torch.zeros(ROWS, D, dtype=bf16), torch.zeros(ROWS, N, dtype=bf16), torch.zeros(ROWS, D, dtype=torch.uint8), torch.zeros(2, 8)
    ws, offsets = torch.zeros(4096, dtype=torch.uint8), torch.zeros(EXPERTS + 1, dtype=torch.int32)
    dense, grouped, up, down = plan(), plan(experts=EXPERTS), plan(experts=EXPERTS, gated=1), plan(d_in=N, d_out=D, experts=EXPERTS)
    return {
        "quantize_act": (lambda X, codes, scales: dense.quantize_act(X, codes, scales), dict(X=x, codes=codes, scales=scales)),
        "linear_forward": (lambda X, Y, workspace: dense.linear_forward(X, Y, workspace), dict(X=x, Y=y, workspace=ws)),
        "linear_forward_q": (lambda codes, scales, Y, workspace: dense.linear_forward_q(codes, scales, Y, workspace),
                             dict(codes=codes, scales=scales, Y=y, workspace=ws)),
        "grouped_forward": (lambda X, offsets, Y, workspace: grouped.grouped_forward(X, offsets, Y, workspace), dict(X=x, offsets=offsets, Y=y, workspace=ws)),
        "route_topk": (lambda logits: st.route_topk(logits, r), dict(logits=torch.zeros(ROWS, EXPERTS))),
        "experts_forward": (lambda X, Y, workspace: st.experts_forward(up, down, X, r, Y, workspace), dict(X=x, Y=torch.zeros_like(x), workspace=ws)),
    }


NAMES = ("quantize_act", "linear_forward", "linear_forward_q", "grouped_forward", "route_topk", "experts_forward")


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_the_host_or_another_gpu_are_refused(on_cpu, name):
    lib, plan, r = on_cpu
    call, tensors = _calls(plan, r)[name]
    for which in tensors:
        for bad in (tensors[which], OnGpu(tensors[which], 1)):
            with pytest.raises(ValueError):
                call(**{n: bad if n == which else OnGpu(t) for n, t in tensors.items()})
            assert not lib.names, f"{which} got through"
    call(**{n: OnGpu(t) for n, t in tensors.items()})
    assert len(lib.names) == 1


@pytest.mark.parametrize("name", ["linear_forward", "linear_forward_q", "grouped_forward", "experts_forward"])
def test_a_workspace_with_gaps_is_refused_and_any_type_counts_its_bytes(on_cpu, name):
    lib, plan, r = on_cpu
    call, tensors = _calls(plan, r)[name]
    on_gpu = {n: OnGpu(t) for n, t in tensors.items()}
    for bad in (None, OnGpu(torch.zeros(64, 128, dtype=torch.uint8)[:, :64])):
        with pytest.raises(ValueError):
            call(**{**on_gpu, "workspace": bad})
    assert not lib.names
    call(**{**on_gpu, "workspace": OnGpu(torch.zeros(1024))})
    assert lib.arguments[0][-2] == 4096


def test_a_plan_of_another_gpu_than_the_current_is_refused(on_cpu, monkeypatch):
    lib, plan, r = on_cpu
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call, tensors in _calls(plan, r).values():
        with pytest.raises(ValueError):
            call(**{n: OnGpu(t) for n, t in tensors.items()})
    with pytest.raises(ValueError):
        st.Fp8Plan(st.Fp8Desc(d_in=D, d_out=N, w_dtype=st.STAMP_BF16), OnGpu(torch.zeros(N, D, dtype=torch.bfloat16)))
    assert not lib.names


def test_a_stream_of_another_gpu_is_refused(on_cpu):
    lib, plan, r = on_cpu

    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 0
    x, y = OnGpu(torch.zeros(ROWS, D, dtype=torch.bfloat16)), OnGpu(torch.zeros(ROWS, N, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        plan().linear_forward(x, y, OnGpu(torch.zeros(4096, dtype=torch.uint8)), stream=Stream())
    with pytest.raises(ValueError):
        st.route_topk(OnGpu(torch.zeros(ROWS, EXPERTS)), r, stream=Stream())
    assert not lib.names


def test_a_plans_scales_and_bias_lie_on_its_gpu(on_cpu, monkeypatch):
    lib, _, _ = on_cpu
    monkeypatch.setattr(fp8, "load_library", lambda: lib)
    w, ws, bias = torch.zeros(N, D, dtype=torch.uint8), torch.zeros(1, 2), torch.zeros(N)
    for scales_on, bias_on in ((1, 0), (0, 1)):
        with pytest.raises(ValueError):
            st.Fp8Plan(st.Fp8Desc(d_in=D, d_out=N), OnGpu(w), OnGpu(ws, scales_on), OnGpu(bias, bias_on))
    assert "stamp_fp8_plan_create" not in lib.names
    st.Fp8Plan(st.Fp8Desc(d_in=D, d_out=N), OnGpu(w), OnGpu(ws), OnGpu(bias))
    assert "stamp_fp8_plan_create" in lib.names


def test_a_routing_of_the_host_is_refused():
    with pytest.raises(ValueError):
        st.Routing(4, 8, 2, device="cpu")
