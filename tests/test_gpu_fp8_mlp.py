"""The dense MLP: every kernel of the up product with every one of the down product, whichever way h goes between them, against the definition in 64 bits
(fp8_block_reference.py), and rows that are no numbers."""
import numpy as np
import pytest

import fp8_block_reference as block
from test_gpu_fp8 import _activations, _code, _dt, _gpu, _strided, _weights
from test_gpu_fp8_block import _smaller, _values, st  # noqa: F401  (fixture)
from test_gpu_fp8_block import _held as _held_to

pytestmark = pytest.mark.gpu

_coded = block.coded


def coded(h, dh, pow2):
    """Where a block of h is tiny beside its error, its scale is anything up to that of the error: block.coded's relative bound overflows.  What h's codes stand for is within half
    a step of E4M3, 2^-4 relative, of a value that is dh off, so two of them differ by at most 1.07 times the largest magnitudes of both."""
    with np.errstate(over="ignore", invalid="ignore"):
        codes, scales, step = _coded(h, dh, pow2)

    def most(a):
        return np.repeat(np.pad(a, ((0, 0), (0, -a.shape[1] % 128))).reshape(len(a), -1, 128).max(-1), 128, 1)[:, :a.shape[1]]
    cap = 1.07 * (2 * most(np.abs(h)) + most(dh))
    return codes, scales, np.where(step < cap, step, cap)


@pytest.fixture(autouse=True)
def _bounds_that_are_numbers(monkeypatch):
    monkeypatch.setattr(block, "coded", coded)


def _held(got, want, tol, what):
    assert np.isfinite(tol).all()
    _held_to(got, want, tol, what)


def _case(st, rows, d, ff, n, gated, x, y, pow2):  # noqa: F811
    rng = np.random.default_rng(rows * 11 + d + gated)
    xv, X = _activations(rng, rows, d, x)
    w1, s1 = _weights(rng, (1, 2) if gated else (), ff, d, pow2)
    w2, s2 = _weights(rng, (), n, ff, pow2)
    s1 = _smaller(s1)
    b1, b2 = None if gated else rng.standard_normal(ff).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=gated, gated=gated, x_dtype=_code(st, x), scale_format=pow2), _gpu(w1), _gpu(s1), None if gated else _gpu(b1))
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=n, y_dtype=_code(st, y), scale_format=pow2), _gpu(w2), _gpu(s2), _gpu(b2))
    res, R, _ = _values(rng, rows, n, y, 1)

    def want(act, some):
        return block.mlp(xv[some], w1[0] if gated else w1, s1[0] if gated else s1, b1, w2, s2, b2, act, res[some], y, pow2)
    return X, up, down, R, want


@pytest.mark.parametrize("x,y,pow2", [("bf16", "bf16", 0), ("f32", "f32", 1), ("bf16", "f32", 0)])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("rows,d,ff,n", [(9, 300, 450, 200), (16, 1100, 257, 77), (17, 200, 385, 130), (50, 700, 260, 515), (200, 384, 641, 300), (1025, 130, 300, 70)])
def test_every_pair_of_kernels(st, rows, d, ff, n, gated, x, y, pow2):  # noqa: F811
    X, up, down, R, want = _case(st, rows, d, ff, n, gated, x, y, pow2)
    room = st.mlp_workspace(up, down, rows)
    Y, _ = _strided(rows, n, y, 3, 1)
    some = np.random.default_rng(1).permutation(rows)[:200]
    expected = want("gelu", some)
    for first in ("rows", "tiles_64", "tiles_128"):
        up.set_route(first)
        for second in ("rows", "tiles_64", "tiles_128") + (("tiles_256",) if y == "bf16" else ()):
            down.set_route(second)
            route = st.mlp_route(up, down, rows)
            if gated:
                assert route == (first, second, "rows" if first == "rows" and rows <= 16 else "codes")
            elif first == "rows" and rows > 1024:  # whose results are codes, which the kernel for few rows does not make
                assert route[0].startswith("tiles") and route[1:] == (second, "codes")
            else:
                assert route == (first, second, "rows" if first == "rows" else "codes")
            room.fill_(255)
            st.mlp_forward(up, down, X, Y, room, "gelu", residual=R)
            _held(Y[_gpu(some)], *expected, str(route))
    up.destroy()
    down.destroy()


def test_tiles_of_256_rows_are_no_choice_of_an_up_product(st):  # noqa: F811
    """Its sums are in fp32 whatever the type of its own rows: by rule there, as without the choice."""
    X, up, down, R, want = _case(st, 300, 256, 384, 256, 0, "bf16", "bf16", 0)
    by_rule = st.mlp_route(up, down, 300)
    up.set_route("tiles_256")
    down.set_route("tiles_256")
    assert st.mlp_route(up, down, 300) == (by_rule[0], "tiles_256", by_rule[2])
    Y, room = R.clone(), st.mlp_workspace(up, down, 300)
    st.mlp_forward(up, down, X, Y, room, "silu", residual=R)
    _held(Y, *want("silu", np.arange(300)), "")
    up.destroy()
    down.destroy()


RULES = [  # rows, d, ff, gated (d_out 200); kernels and h by rule on 256 CUs, for Y in fp32 and in bf16
    (4, 700, 900, 0, ("rows", "rows", "rows"), ("rows", "rows", "rows")), (50, 700, 900, 0, ("tiles_64", "rows", "codes"), ("tiles_64", "rows", "codes")),
    (50, 2048, 1536, 0, ("rows", "rows", "rows"), ("rows", "rows", "rows")), (100, 2048, 1536, 0, ("tiles_64", "rows", "rows"), ("tiles_64", "tiles_64", "rows")),
    (400, 700, 900, 0, ("tiles_64", "tiles_64", "codes"), ("tiles_64", "tiles_64", "codes")), (1025, 512, 4096, 0, ("tiles_128", "tiles_64", "codes"), ("tiles_128", "tiles_64", "codes")),
    (13, 700, 900, 1, ("rows", "rows", "rows"), ("rows", "rows", "rows")), (33, 700, 900, 1, ("rows", "rows", "codes"), ("rows", "rows", "codes")),
    (100, 2048, 1536, 1, ("rows", "rows", "codes"), ("rows", "tiles_64", "codes")), (200, 700, 900, 1, ("tiles_64", "tiles_64", "codes"), ("tiles_64", "tiles_64", "codes"))]


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,ff,gated,f32,bf16", RULES)
def test_what_runs_by_rule(st, rows, d, ff, gated, f32, bf16, y):  # noqa: F811
    X, up, down, R, want = _case(st, rows, d, ff, 200, gated, "bf16", y, 0)
    assert st.mlp_route(up, down, rows) == {"f32": f32, "bf16": bf16}[y]
    Y, room = R.clone(), st.mlp_workspace(up, down, rows)
    room.fill_(255)
    st.mlp_forward(up, down, X, Y, room, "silu", residual=R)
    some = np.random.default_rng(2).permutation(rows)[:60]
    _held(Y[_gpu(some)], *want("silu", some), "")
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("rows", [4, 16, 60, 300])
def test_rows_that_are_no_numbers(st, rows, gated, y):  # noqa: F811
    """A NaN or an infinity in a row of X makes that row of Y NaN and no other, whichever way h goes; the other rows keep their bits."""
    import torch
    X, up, down, R, _ = _case(st, rows, 300, 450, 200, gated, "bf16", y, 0)
    bad = X.clone()
    bad[1, 5], bad[2, 299], bad[rows - 1, 128] = float("nan"), float("inf"), -float("inf")
    lost = sorted({1, 2, rows - 1})
    keep = [i for i in range(rows) if i not in lost]
    room, Y, Z = st.mlp_workspace(up, down, rows), torch.empty_like(R), torch.empty_like(R)
    for first in ("", "rows", "tiles_64", "tiles_128"):
        up.set_route(first)
        for second in ("", "rows", "tiles_64", "tiles_128"):
            down.set_route(second)
            for act in ("relu", "gelu"):
                st.mlp_forward(up, down, X, Y, room, act, residual=R)
                st.mlp_forward(up, down, bad, Z, room, act, residual=R)
                assert torch.isfinite(Y).all() and torch.isnan(Z[lost]).all() and torch.equal(Y[keep], Z[keep]), (first, second, act)
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("rows", [3, 60])
def test_infinite_values_of_h(st, rows):  # noqa: F811
    """An infinity or NaN in h makes its row NaN (Q8); minus infinity through relu is a zero like any other."""
    import torch
    rng = np.random.default_rng(3)
    d, ff, n = 256, 300, 130
    w1, s1 = _weights(rng, (), ff, d, 0)
    w2, s2 = _weights(rng, (), n, ff, 0)
    xv, X = _activations(rng, rows, d, "bf16")
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=n, y_dtype=st.STAMP_F32), _gpu(w2), _gpu(s2))
    for value, act, number in ((np.inf, "relu", 0), (np.inf, "gelu", 0), (-np.inf, "relu", 1), (-np.inf, "silu", 0), (np.nan, "relu", 0)):
        b = rng.standard_normal(ff).astype(np.float32)
        b[290] = value
        up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff), _gpu(w1), _gpu(_smaller(s1)), _gpu(b))
        Y, room = torch.empty((rows, n), device="cuda"), st.mlp_workspace(up, down, rows)
        for route in ("rows", "tiles_64", "tiles_128"):
            up.set_route(route)
            st.mlp_forward(up, down, X, Y, room, act)
            if number:
                _held(Y, *block.mlp(xv, w1, _smaller(s1), np.where(np.isinf(b), -1e30, b).astype(np.float32), w2, s2, None, act, None, "f32", 0), f"{value} {act} {route}")
            else:
                assert torch.isnan(Y).all(), (value, act, route)
        up.destroy()
    down.destroy()


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("rows", [1, 13, 40, 300, 1100])
def test_rows_at_any_place_and_a_workspace_of_a_larger_call(st, rows, gated, x):  # noqa: F811
    """X in rows that lie apart and begin anywhere, a stream of its own, the workspace of 1500 rows before and after: the bits of the plain call."""
    import torch
    X, up, down, R, _ = _case(st, rows, 333, 450, 200, gated, x, "bf16", 0)
    Y, room = torch.empty_like(R), st.mlp_workspace(up, down, 1500)
    st.mlp_forward(up, down, X, Y, st.mlp_workspace(up, down, rows), "silu", residual=R)
    apart, _ = _strided(rows, 333, x, 4, 1)
    apart.copy_(X)
    more, Y1500 = torch.randn((1500, 333), device="cuda").to(X.dtype), torch.empty((1500, 200), dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()
    for _ in range(2):
        Z = torch.full_like(Y, -7.0)
        torch.cuda.synchronize()
        st.mlp_forward(up, down, more, Y1500, room, "silu", stream=stream)
        st.mlp_forward(up, down, apart, Z, room, "silu", residual=R, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(Y, Z)
    up.destroy()
    down.destroy()
