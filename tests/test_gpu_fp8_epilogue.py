"""Activations at minus infinity and in every kernel, how near they are to their definitions (fp8_block_reference.py), and that calls repeat."""
import numpy as np
import pytest

import fp8_block_reference as block
from test_gpu_fp8 import _activations, _code, _dt, _gpu, _weights
from test_gpu_fp8_block import _smaller, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _of_bias(st, z, y, rows, d=128):  # noqa: F811
    """A layer whose weights are zero: Y is the activation of the bias."""
    import torch
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=z.size, y_dtype=_code(st, y)), torch.zeros((z.size, d), dtype=torch.uint8, device="cuda"),
                      torch.ones((-(-z.size // 128), -(-d // 128)), device="cuda"), _gpu(z))
    X = torch.randn((rows, d), device="cuda").to(torch.bfloat16)
    return plan, X, torch.empty((rows, z.size), dtype=_dt(y), device="cuda"), plan.alloc_workspace(rows)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,parts", [(3, 128, 0), (40, 128, 0), (300, 128, 0), (130, 4096, 1)])
def test_activations_at_the_ends_of_their_range(st, rows, d, parts, y):  # noqa: F811
    import torch
    z = np.resize(np.float32([-np.inf, np.inf, np.nan, 0.0, -0.0, 2.0, -3e38, 3e38, -1e-38]), 290)
    plan, X, Y, ws = _of_bias(st, z, y, rows, d)
    assert not parts or plan.cut(rows)[1] > 1  # by rule: the activation where the parts of the depth are joined
    low = {"none": -np.inf, "relu": 0.0, "silu": np.nan, "gelu": np.nan, "gelu_tanh": np.nan}  # of minus infinity: x times 0
    big = float(torch.tensor(3e38).to(_dt(y)))
    for route in ("", "rows", "tiles_64", "tiles_128") + (("tiles_256",) if y == "bf16" else ()):
        plan.set_route(route)
        for act in block.ACTIVATIONS:
            Y.fill_(-7.0)
            plan.linear_forward(X, Y, ws, activation=act)
            got = Y.float().cpu().numpy()
            two = block.activation(np.float64(2.0), act)
            want = [low[act], np.inf, np.nan, 0.0, 0.0, None, -big if act == "none" else 0.0, big, None]
            for i, w in enumerate(want):
                if w is not None:
                    assert np.array_equal(got[:, i::9], np.full_like(got[:, i::9], w), equal_nan=True), (route, act, z[i])
            assert (np.abs(got[:, 5::9] - two) <= (2.0 ** -8 if y == "bf16" else 2.0 ** -20) * two).all()
            assert (np.abs(got[:, 8::9]) <= 1.01e-38).all()
    plan.destroy()


def _arguments():
    rng = np.random.default_rng(0)
    return np.concatenate([rng.uniform(-12, 12, 1 << 19), rng.uniform(-100, 100, 1 << 18), rng.uniform(-1, 1, 1 << 18)]).astype(np.float32)


def test_activations_beside_their_argument(st):  # noqa: F811
    """The bounds that stamp.h states, over a million arguments."""
    z = _arguments()
    plan, X, Y, ws = _of_bias(st, z, "f32", 1)
    for act, bound, own in (("silu", 1.5e-7, 1e-6), ("gelu", 2.7e-7, 1e-5), ("gelu_tanh", 1.5e-7, 1e-5)):
        plan.linear_forward(X, Y, ws, activation=act)
        want = block.activation(z.astype(np.float64), act)
        off = np.abs(Y[0].cpu().numpy() - want)
        assert (off <= bound * np.abs(z) + 1e-37).all(), (act, np.max(off / np.abs(z)))
        assert (off <= own * np.abs(want) + 1e-37)[z >= -6].all(), (act, np.max((off / np.abs(want))[z >= -6]))
    plan.destroy()


@pytest.mark.parametrize("rows,d", [(1, 128), (80, 128), (200, 128), (130, 4096)])
def test_gelu_keeps_its_digits_in_fp32(st, rows, d):  # noqa: F811
    """exp(-t^2 / 2): two products and a constant's half rounding, each 2^-24 of an exponent that counts t^2 / 2 times; 14 such roundings for the fit (2.7), the
    polynomial (3), the reciprocal (2), the power of two (2), the products and the sum."""
    n = 1 << 10 if rows > 1 else 1 << 20
    z = _arguments()[:: (1 << 20) // n]
    z = z[z >= -8]
    want = block.activation(z.astype(np.float64), "gelu")
    plan, X, Y, ws = _of_bias(st, z, "f32", rows, d)
    for route in ("", "rows", "tiles_64", "tiles_128"):
        plan.set_route(route)
        plan.linear_forward(X, Y, ws, activation="gelu")
        off = np.abs(Y.cpu().numpy() - want)
        assert (off <= (1.25 * z.astype(np.float64) ** 2 + 14) * 2.0 ** -24 * np.abs(want) + 1e-37).all(), (route, np.max(off / np.abs(want)))
    plan.destroy()


@pytest.mark.parametrize("rows,d,n", [(2048, 1152, 1500), (700, 4096, 300), (8192, 256, 1152)])
def test_the_same_call_gives_the_same_bits(st, rows, d, n):  # noqa: F811
    """A layer's epilogue in tiles, dense and by expert, an MLP and a layer of experts, with other calls between and anything in the workspace; a bf16 Y is as far from the
    definition as the nearest bf16 numbers are, in norm, but for 1e-4: the FP8 instructions lose 6e-5 of a sum at most for exponents all over the range."""
    import torch
    rng = np.random.default_rng(rows)
    x, X = _activations(rng, rows, d, "bf16")
    X2 = torch.randn_like(X)

    def plan(d_in, d_out, experts=0, gated=0):
        lead = ((experts,) if experts else ()) + ((2,) if gated else ())
        w, ws = _weights(rng, lead, d_out, d_in, 0)
        return st.Fp8Plan(st.Fp8Desc(d_in=d_in, d_out=d_out, experts=experts, gated=gated), _gpu(w), _gpu(_smaller(ws))), w, _smaller(ws)
    (lin, w, ws), (grp, *_), (up, *_), (down, *_), (gup, *_), (gdown, *_) = plan(d, n), plan(d, n, 4), plan(d, 520), plan(520, d), plan(d, 520, 4, 1), plan(520, d, 4)
    offsets = _gpu(np.int32([0, rows // 3, rows // 3, rows - 5, rows - 5]))
    rt, r = torch.randn((4, d), device="cuda"), st.Routing(rows, 4, 2)
    R, Rd = (torch.randn((rows, c), device="cuda").to(torch.bfloat16) for c in (n, d))
    calls = [(n, lin.alloc_workspace(rows), lambda x, y, room: lin.linear_forward(x, y, room, activation="gelu", residual=R)),
             (n, grp.alloc_workspace(rows), lambda x, y, room: grp.grouped_forward(x, offsets, y, room, activation="silu", residual=R)),
             (d, st.mlp_workspace(up, down, rows), lambda x, y, room: st.mlp_forward(up, down, x, y, room, "gelu_tanh", residual=Rd)),
             (d, st.moe_workspace(gup, gdown, rows, 2), lambda x, y, room: st.moe_forward(rt, gup, gdown, x, r, y, room, residual=Rd))]
    for i, (cols, room, call) in enumerate(calls):
        first, Y = (torch.full((rows, cols), -7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        call(X, first, room)
        for value in (255, 0, 60):
            call(X2, Y, room)
            assert not torch.equal(Y, first)
            room.fill_(value)
            Y.fill_(-7.0)
            call(X, Y, room)
            assert torch.equal(Y, first), i
        if i == 0:
            some = rng.permutation(rows)[:200]
            want, _ = block.layer(x[some], w, ws, None, "gelu", R[_gpu(some)].double().cpu().numpy(), "bf16", 0, False)
            got = first[_gpu(some)].double().cpu().numpy()
            nearest = torch.from_numpy(want).to(torch.bfloat16).double().numpy()
            off, own = (np.linalg.norm(a - want) / np.linalg.norm(want) for a in (got, nearest))
            assert off <= own + 1e-4, (off, own)
    for p in (lin, grp, up, down, gup, gdown):
        p.destroy()
