"""Activations at minus infinity and in every kernel, and how near they are to their definitions (fp8_block_reference.py)."""
import numpy as np
import pytest

import fp8_block_reference as block
from test_gpu_fp8 import _code, _dt, _gpu
from test_gpu_fp8_block import st  # noqa: F401  (fixture)

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


def test_activations_beside_their_argument(st):  # noqa: F811
    """The bounds that stamp.h states, over a million arguments."""
    rng = np.random.default_rng(0)
    z = np.concatenate([rng.uniform(-12, 12, 1 << 19), rng.uniform(-100, 100, 1 << 18), rng.uniform(-1, 1, 1 << 18)]).astype(np.float32)
    plan, X, Y, ws = _of_bias(st, z, "f32", 1)
    for act, bound in (("silu", 1.5e-7), ("gelu", 2.1e-7), ("gelu_tanh", 1.5e-7)):
        plan.linear_forward(X, Y, ws, activation=act)
        off = np.abs(Y[0].cpu().numpy() - block.activation(z.astype(np.float64), act))
        assert (off <= bound * np.abs(z) + 1e-37).all(), (act, np.max(off / np.abs(z)))
    plan.destroy()
