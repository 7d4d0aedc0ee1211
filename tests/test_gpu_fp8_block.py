"""What surrounds the 8-bit floating point layers: activation and residual in their epilogue, the dense MLP, the whole layer of experts, against
the definition in 64 bits (fp8_block_reference.py)."""
import numpy as np
import pytest

import fp8_block_reference as block
import fp8_reference as ref
from test_gpu_fp8 import _activations, _code, _dt, _gpu, _strided, _weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def st():
    import paper_2510_26771_amd as st
    st.load_library()
    return st


def _values(rng, rows, cols, dtype, pad=0, offset=0):
    """fp32 values that `dtype` holds, and the same on the GPU in rows that lie apart, and their buffer."""
    import torch
    t = torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32) * 3).to(_dt(dtype))
    view, buf = _strided(rows, cols, dtype, pad, offset)
    view.copy_(t)
    return t.float().numpy().astype(np.float64), view, buf


def _held(got, want, tol, what):
    got = got.float().cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all(), f"{what}: no numbers at {np.argwhere(~np.isfinite(got))[:2]}"
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the tolerance, worst {np.max(np.abs(got - want) / tol):.3g} times it, first at {np.argwhere(bad)[:1]}"


def _smaller(s):
    return (s * np.float32(2.0 ** -6)).astype(np.float32)  # sums of a size where the activations are curved


# ---- the epilogue ----

@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 40])
def test_activations_over_their_range(st, rows, y):
    """Weights of zero: Y is the activation of the bias, with infinities, NaN, zeros and the largest numbers among them."""
    import torch
    z = np.concatenate([np.linspace(-9, 9, 1201), [0.0, -0.0, 1e-30, -1e-30, 1e-4, -1e-4, 30, -30, 88, -88, 200, -200, 1e10, -1e10, 3e38, -3e38, np.inf, -np.inf, np.nan]])
    z = z.astype(np.float32)
    n, d = z.size, 128
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, y_dtype=_code(st, y)), _gpu(np.zeros((n, d), np.uint8)), _gpu(np.ones((-(-n // 128), 1), np.float32)), _gpu(z))
    X = torch.randn((rows, d), device="cuda").to(torch.bfloat16)
    Y, ws = torch.empty((rows, n), dtype=_dt(y), device="cuda"), plan.alloc_workspace(rows)
    for route in ("rows", "tiles_64", "tiles_128"):
        plan.set_route(route)
        for act in block.ACTIVATIONS[1:]:
            plan.linear_forward(X, Y, ws, activation=act)
            got = Y.float().cpu().numpy().astype(np.float64)
            fin = np.abs(z) < 1e9
            want, dv = block.activated(z[fin].astype(np.float64), 0.0, act)
            tol = dv + block.HALF[y] * (np.abs(want) + dv) * (1 + 2.0 ** -7) + 1e-37
            assert (np.abs(got[:, fin] - want) <= tol).all(), (route, act)
            assert np.isnan(got[:, -1]).all() and (got[:, -3] == np.inf).all(), (route, act)  # NaN, infinity
            big = np.flatnonzero(np.abs(z) > 1e9)[:4]
            want = torch.from_numpy(np.where(z[big] > 0, z[big], 0.0).astype(np.float32)).to(_dt(y)).float().numpy()
            assert np.array_equal(np.abs(got[:, big]), np.broadcast_to(want, (rows, 4))), (route, act)
    plan.destroy()


LAYERS = [  # rows, d_in, d_out
    (1, 128, 64), (1, 4096, 130), (3, 200, 75), (5, 1000, 200), (17, 257, 129), (40, 384, 333), (70, 600, 264), (130, 1111, 515), (300, 256, 1030), (513, 130, 384)]


@pytest.mark.parametrize("pow2", [0, 1])
@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,n", LAYERS)
def test_a_layer_with_activation_and_residual(st, rows, d, n, y, pow2):
    """Every activation and kernel; rows of X, Y and the residual that lie apart and begin anywhere; nothing beside Y is written."""
    import torch
    rng = np.random.default_rng(rows * 31 + d)
    x, xg = _activations(rng, rows, d, "bf16" if rows % 2 else "f32")
    w, ws = _weights(rng, (), n, d, pow2)
    ws = _smaller(ws)
    bias = rng.standard_normal(n).astype(np.float32)
    res, R, _ = _values(rng, rows, n, y, 5, 1)
    Y, buf = _strided(rows, n, y, 3, 1)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, x_dtype=_code(st, "bf16" if rows % 2 else "f32"), y_dtype=_code(st, y), scale_format=pow2), _gpu(w), _gpu(ws), _gpu(bias))
    room = plan.alloc_workspace(rows)
    for i, route in enumerate(("", "rows", "tiles_64", "tiles_128") + (("tiles_256",) if y == "bf16" else ())):
        plan.set_route(route)
        for j, act in enumerate(block.ACTIVATIONS):
            use = (i + j) % 3 != 0 or act == "none"
            room.fill_(255)
            plan.linear_forward(xg, Y, room, activation=act, residual=R if use else None)
            want, tol = block.layer(x, w, ws, bias, act, res if use else None, y, pow2, y == "f32")
            _held(Y, want, tol, f"{route} {act} residual {use}")
    plan.set_route("")
    codes, scales = plan.alloc_act_buffers(rows)
    plan.quantize_act(xg, codes, scales)
    plan.linear_forward_q(codes, scales, Y, room, activation="gelu", residual=R)
    _held(Y, *block.layer(x, w, ws, bias, "gelu", res, y, pow2, y == "f32"), "from codes")
    Y.fill_(-7.0)
    assert (buf == -7.0).all()
    plan.destroy()


@pytest.mark.parametrize("rows,d,n,what", [(130, 4096, 300, "parts"), (90, 7000, 515, "parts"), (3000, 520, 5700, "two launches"), (2900, 300, 5643, "two launches"),
                                            (300, 2048, 520, ""), (64, 1536, 300, ""), (2048, 256, 4400, ""), (8192, 128, 1152, "")])
@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_epilogue_where_the_depth_is_in_parts_and_columns_in_two_launches(st, rows, d, n, what, y):
    import torch
    rng = np.random.default_rng(rows + d)
    x, xg = _activations(rng, rows, d, "bf16")
    w, ws = _weights(rng, (), n, d, 0)
    ws = _smaller(ws)
    bias = rng.standard_normal(n).astype(np.float32)
    res, R, _ = _values(rng, rows, n, y, 1)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, y_dtype=_code(st, y)), _gpu(w), _gpu(ws), _gpu(bias))
    columns, parts, _ = plan.cut(rows)
    assert (columns > 0 or what != "two launches") and (parts > 1 or what != "parts")
    Y, room = torch.empty((rows, n), dtype=_dt(y), device="cuda"), plan.alloc_workspace(rows)
    some = rng.permutation(rows)[:300]
    for act in ("none", "gelu_tanh"):
        plan.linear_forward(xg, Y, room, activation=act, residual=R)
        want, tol = block.layer(x[some], w, ws, bias, act, res[some], y, 0, y == "f32")
        _held(Y[_gpu(some)], want, tol, act)
    plan.destroy()


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,n", [(1, 512, 512), (9, 300, 77), (260, 2048, 515), (600, 256, 301)])
def test_a_residual_that_is_y_itself(st, rows, d, n, y):
    import torch
    rng = np.random.default_rng(rows)
    _, xg = _activations(rng, rows, d, "bf16")
    w, ws = _weights(rng, (), n, d, 0)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, y_dtype=_code(st, y)), _gpu(w), _gpu(ws))
    room = plan.alloc_workspace(rows)
    _, R, buf = _values(rng, rows, n, y, 1, 1)
    for route in ("", "rows", "tiles_64", "tiles_128"):
        plan.set_route(route)
        Y, first = torch.empty((rows, n), dtype=_dt(y), device="cuda"), buf.clone()
        plan.linear_forward(xg, Y, room, activation="silu", residual=R)
        plan.linear_forward(xg, R, room, activation="silu", residual=R)
        assert torch.equal(R, Y), route
        R.copy_(first[1:1 + rows * (n + 1)].view(rows, n + 1)[:, :n])
        assert torch.equal(buf, first)
    plan.destroy()


@pytest.mark.parametrize("counts,d,n", [([3, 0, 1, 5], 256, 130), ([0, 0, 40], 300, 200), ([70, 1, 0, 130, 33], 512, 261), ([1] * 64 + [0] * 6, 128, 64)])
@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_rows_by_expert_with_activation_and_residual(st, counts, d, n, y):
    import torch
    rng = np.random.default_rng(sum(counts))
    used, E = sum(counts), len(counts)
    rows = used + 3  # rows behind the last expert's: left as they are
    x, xg = _activations(rng, rows, d, "bf16")
    w, ws = _weights(rng, (E,), n, d, 0)
    ws = _smaller(ws)
    bias = rng.standard_normal((E, n)).astype(np.float32)
    res, R, _ = _values(rng, rows, n, y, 2)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, experts=E, y_dtype=_code(st, y)), _gpu(w), _gpu(ws), _gpu(bias))
    Y, buf = _strided(rows, n, y, 1)
    room = plan.alloc_workspace(rows)
    for route in ("rows", "tiles_64", "tiles_128"):
        plan.set_route(route)
        for act in block.ACTIVATIONS:
            Y.fill_(-7.0)
            plan.grouped_forward(xg, _gpu(offsets), Y, room, activation=act, residual=R)
            for e in range(E):
                a, b = offsets[e], offsets[e + 1]
                if a < b:
                    want, tol = block.layer(x[a:b], w[e], ws[e], bias[e], act, res[a:b], y, 0, y == "f32")
                    _held(Y[a:b], want, tol, f"{route} {act} expert {e}")
            assert (Y[used:] == -7.0).all()
    Y[:used] = -7.0
    assert (buf == -7.0).all()
    plan.destroy()


# ---- the dense MLP ----

@pytest.mark.parametrize("rows,d,ff,n,gated,act,x,y,pow2", [
    (1, 128, 128, 128, 0, "gelu", "bf16", "bf16", 0), (1, 1, 1, 1, 0, "silu", "f32", "f32", 1), (1, 512, 1100, 512, 1, "silu", "bf16", "bf16", 0),
    (2, 1, 3, 2, 1, "gelu", "f32", "f32", 0), (5, 300, 257, 130, 0, "gelu_tanh", "f32", "bf16", 1), (16, 640, 384, 640, 1, "gelu_tanh", "bf16", "f32", 1),
    (33, 200, 65, 77, 0, "relu", "bf16", "f32", 0), (40, 257, 600, 257, 1, "relu", "bf16", "bf16", 0), (100, 590, 1185, 715, 0, "gelu", "f32", "f32", 1),
    (130, 384, 193, 384, 0, "gelu", "bf16", "bf16", 0), (260, 256, 512, 200, 1, "silu", "f32", "f32", 0), (700, 300, 450, 300, 0, "none", "bf16", "bf16", 1),
    (1500, 256, 900, 128, 0, "silu", "bf16", "bf16", 0), (1500, 256, 900, 128, 1, "gelu", "bf16", "bf16", 1)])
def test_mlp_against_the_definition(st, rows, d, ff, n, gated, act, x, y, pow2):
    import torch
    rng = np.random.default_rng(rows * 7 + d)
    xv, xg = _activations(rng, rows, d, x)
    w_up, s_up = _weights(rng, (1, 2) if gated else (), ff, d, pow2)
    w_down, s_down = _weights(rng, (), n, ff, pow2)
    s_up = _smaller(s_up)
    b_up = None if gated else rng.standard_normal(ff).astype(np.float32)
    b_down = rng.standard_normal(n).astype(np.float32)
    res, R, _ = _values(rng, rows, n, y, 1)
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=gated, gated=gated, x_dtype=_code(st, x), scale_format=pow2), _gpu(w_up), _gpu(s_up), None if gated else _gpu(b_up))
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=n, y_dtype=_code(st, y), scale_format=pow2), _gpu(w_down), _gpu(s_down), _gpu(b_down))
    room = st.mlp_workspace(up, down, rows)
    Y, buf = _strided(rows, n, y, 3, 1)
    some = rng.permutation(rows)[:200]
    for route in ("", "rows", "tiles_64", "tiles_128", "tiles_256"):
        if route == "tiles_256" and (gated or y == "f32"):
            continue
        up.set_route(route)
        down.set_route(route)
        for use in (0, 1):
            room.fill_(255)
            st.mlp_forward(up, down, xg, Y, room, act, residual=R if use else None)
            want, tol = block.mlp(xv[some], w_up[0] if gated else w_up, s_up[0] if gated else s_up, b_up, w_down, s_down, b_down, act, res[some] if use else None, y, pow2)
            _held(Y[_gpu(some)], want, tol, f"{route} residual {use}")
    first = Y.clone()
    room.fill_(0)
    st.mlp_forward(up, down, xg, Y, room, act, residual=R)
    assert torch.equal(first, Y)
    Y.fill_(-7.0)
    assert (buf == -7.0).all()
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("rows", [1, 50, 600])
@pytest.mark.parametrize("gated", [0, 1])
def test_mlp_in_place(st, rows, gated):
    """X, the residual and Y as one tensor: x += mlp(x)."""
    import torch
    rng = np.random.default_rng(rows)
    d, ff = 384, 700
    w_up, s_up = _weights(rng, (1, 2) if gated else (), ff, d, 0)
    w_down, s_down = _weights(rng, (), d, ff, 0)
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=gated, gated=gated), _gpu(w_up), _gpu(s_up))
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d, experts=gated), _gpu(w_down[None] if gated else w_down), _gpu(s_down[None] if gated else s_down))
    room = st.mlp_workspace(up, down, rows)
    X = torch.randn((rows, d), device="cuda").to(torch.bfloat16)
    Y = torch.empty_like(X)
    st.mlp_forward(up, down, X, Y, room, "silu", residual=X)
    st.mlp_forward(up, down, X, X, room, "silu", residual=X)
    assert torch.equal(X, Y)
    up.destroy()
    down.destroy()


# ---- the layer of experts ----

def _moe_case(st, rng, tokens, E, d, ff, x, y, router, pow2, bias):
    xv, xg = _activations(rng, tokens, d, x)
    xv = xv.astype(np.float64)
    w_up, s_up = _weights(rng, (E, 2), ff, d, pow2)
    w_down, s_down = _weights(rng, (E,), d, ff, pow2)
    s_up = _smaller(s_up)
    import torch
    rt = torch.from_numpy((rng.standard_normal((E, d)) / np.sqrt(30.0 * d)).astype(np.float32)).to(_dt(router))
    b = rng.standard_normal((E, d)).astype(np.float32) if bias else None
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=E, gated=1, x_dtype=_code(st, x), scale_format=pow2), _gpu(w_up), _gpu(s_up))
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d, experts=E, y_dtype=_code(st, y), scale_format=pow2), _gpu(w_down), _gpu(s_down), _gpu(b) if bias else None)
    return xv, xg, w_up, s_up, w_down, s_down, b, rt.float().numpy().astype(np.float64), rt.cuda(), up, down


MOES = [  # tokens, experts, top_k, d, ff, x, y, router, pow2, down bias, router bias, activation
    (1, 1, 1, 1, 1, "f32", "f32", "f32", 0, 0, 0, "silu"), (1, 4, 2, 128, 128, "bf16", "bf16", "bf16", 0, 0, 0, "silu"),
    (1, 64, 6, 512, 300, "bf16", "bf16", "bf16", 0, 1, 0, "silu"), (2, 3, 3, 40, 24, "f32", "f32", "bf16", 1, 1, 0, "gelu"),
    (3, 300, 8, 256, 129, "bf16", "f32", "f32", 0, 0, 1, "gelu_tanh"), (5, 2, 1, 1000, 700, "f32", "bf16", "f32", 0, 1, 0, "silu"),
    (7, 16, 16, 129, 257, "bf16", "bf16", "f32", 1, 0, 1, "relu"), (8, 1024, 4, 128, 64, "bf16", "bf16", "bf16", 0, 0, 0, "silu"),
    (16, 8, 2, 640, 384, "bf16", "bf16", "bf16", 0, 1, 0, "silu"), (16, 40, 32, 200, 200, "f32", "f32", "f32", 0, 0, 1, "silu"),
    (16, 4, 6, 384, 500, "bf16", "bf16", "f32", 1, 1, 0, "none"), (13, 70, 5, 300, 1100, "bf16", "bf16", "bf16", 0, 0, 0, "silu"),
    (17, 8, 2, 256, 200, "bf16", "bf16", "bf16", 0, 1, 0, "silu"), (40, 12, 3, 300, 384, "f32", "f32", "f32", 1, 0, 1, "gelu"),
    (200, 6, 2, 384, 256, "bf16", "bf16", "f32", 0, 1, 1, "silu"), (700, 5, 3, 257, 300, "bf16", "bf16", "bf16", 1, 0, 0, "gelu_tanh")]


@pytest.mark.parametrize("renormalize", [0, 1])
@pytest.mark.parametrize("tokens,E,top_k,d,ff,x,y,router,pow2,bias,rbias,act", MOES)
def test_layer_of_experts_against_the_definition(st, tokens, E, top_k, d, ff, x, y, router, pow2, bias, rbias, act, renormalize):
    import torch
    rng = np.random.default_rng(tokens * 7 + E)
    xv, xg, w_up, s_up, w_down, s_down, b, rt, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, x, y, router, pow2, bias)
    rb = None
    if rbias:  # some experts out of use
        rb = np.where(rng.random(E) < 0.4, -np.inf, rng.standard_normal(E)).astype(np.float32)
    res, R, _ = _values(rng, tokens, d, y, 1)
    r = st.Routing(tokens, E, top_k)
    room = st.moe_workspace(up, down, tokens, top_k)
    Y, buf = _strided(tokens, d, y, 3, 1)
    for use in (0, 1):
        room.fill_(255)  # NaN wherever something is read that was not written
        for t in (r.ids, r.offsets, r.token_of_row, r.row_of_slot):
            t.fill_(-9)
        r.weights.fill_(-9.0)
        st.moe_forward(rtg, up, down, xg, r, Y, room, router_bias=None if rb is None else _gpu(rb), renormalize=bool(renormalize), activation=act, residual=R if use else None)
        want, tol, ids, weights, offsets, token, row, dw = block.moe(xv, rt, rb, w_up, s_up, w_down, s_down, b, top_k, renormalize, act, res if use else None, y, pow2)
        assert np.array_equal(r.ids.cpu().numpy(), ids) and np.array_equal(r.offsets.cpu().numpy(), offsets)
        assert np.array_equal(r.token_of_row.cpu().numpy(), token) and np.array_equal(r.row_of_slot.cpu().numpy(), row)
        # the relative bound, and for weights below fp32's normal numbers (2^-126) those themselves: they may be flushed to zero
        assert (np.abs(r.weights.cpu().numpy() - weights) <= weights * dw + 2.0 ** -126).all()
        _held(Y, want, tol, f"residual {use}")
    first = Y.clone()
    room.fill_(0)
    st.moe_forward(rtg, up, down, xg, r, Y, room, router_bias=None if rb is None else _gpu(rb), renormalize=bool(renormalize), activation=act, residual=R)
    assert torch.equal(first, Y)
    Y.fill_(-7.0)
    assert (buf == -7.0).all()
    up.destroy()
    down.destroy()


# few tokens go through two kernels of their own; the same by the other calls' kernels, one after the other; and where the rows become too many or too long
@pytest.mark.parametrize("tokens,E,top_k,d,ff,two", [(1, 20, 4, 384, 300, 1), (16, 40, 8, 256, 140, 1), (16, 40, 9, 256, 140, 0), (4, 200, 32, 256, 64, 1), (16, 3, 2, 128, 6100, 0),
                                                     (3, 3, 2, 130, 5000, 1), (1, 2, 2, 128, 20000, 1), (17, 9, 2, 256, 256, 0), (16, 12, 1, 1600, 200, 1)])
def test_layer_of_experts_in_two_kernels_and_in_others(st, tokens, E, top_k, d, ff, two):
    import torch
    rng = np.random.default_rng(tokens * 100 + E)
    xv, xg, w_up, s_up, w_down, s_down, b, rt, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", "f32", "f32", 0, 1)
    res, R, _ = _values(rng, tokens, d, "f32", 1)
    want, tol, ids, weights, offsets, token, row, dw = block.moe(xv, rt, None, w_up, s_up, w_down, s_down, b, top_k, 1, "silu", res, "f32", 0)
    r, room = st.Routing(tokens, E, top_k), st.moe_workspace(up, down, tokens, top_k)
    got = []
    for route in ("", "rows", "tiles_64"):
        up.set_route(route)
        down.set_route(route)
        assert st.moe_route(up, down, tokens, top_k) == ("few" if two and not route else "many")
        Y = torch.full((tokens, d), -7.0, device="cuda")
        room.fill_(255)
        st.moe_forward(rtg, up, down, xg, r, Y, room, residual=R)
        _held(Y, want, tol, route)
        assert np.array_equal(r.ids.cpu().numpy(), ids) and np.array_equal(r.offsets.cpu().numpy(), offsets)
        assert np.array_equal(r.token_of_row.cpu().numpy(), token) and np.array_equal(r.row_of_slot.cpu().numpy(), row)
        got.append(Y)
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("tokens", [1, 4, 16, 33])
def test_tokens_without_an_expert_and_in_place(st, tokens):
    """All experts out of use: Y is the residual, or zeros.  X, the residual and Y as one tensor."""
    import torch
    rng = np.random.default_rng(tokens)
    E, k, d, ff = 9, 3, 256, 200
    *_, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", "bf16", "bf16", 0, 1)
    r, room = st.Routing(tokens, E, k), st.moe_workspace(up, down, tokens, k)
    X = torch.randn((tokens, d), device="cuda").to(torch.bfloat16)
    Y = torch.full_like(X, -7.0)
    none = torch.full((E,), -np.inf, device="cuda")
    st.moe_forward(rtg, up, down, X, r, Y, room, router_bias=none)
    assert (Y == 0).all() and (r.ids == -1).all() and (r.weights == 0).all() and (r.offsets == 0).all() and (r.token_of_row == -1).all() and (r.row_of_slot == -1).all()
    st.moe_forward(rtg, up, down, X, r, Y, room, router_bias=none, residual=X)
    assert torch.equal(X, Y)
    st.moe_forward(rtg, up, down, X, r, Y, room, residual=X)
    st.moe_forward(rtg, up, down, X, r, X, room, residual=X)
    assert torch.equal(X, Y)
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("tokens", [1, 7, 16, 50])
def test_experts_masked_by_the_lowest_number(st, tokens):
    """A bias of the type's lowest value instead of minus infinity: such experts are chosen behind all others, with weight 0, and change nothing."""
    import torch
    rng = np.random.default_rng(tokens)
    E, k, d, ff = 10, 6, 384, 256
    *_, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", "f32", "f32", 0, 1)
    X = torch.randn((tokens, d), device="cuda").to(torch.bfloat16)
    low = [1, 2, 5, 6, 8, 9]  # four are left
    outs = []
    for value in (-np.inf, float(np.finfo(np.float32).min)):
        b = torch.zeros(E, device="cuda")
        b[low] = value
        r, Y = st.Routing(tokens, E, k), torch.empty((tokens, d), device="cuda")
        st.moe_forward(rtg, up, down, X, r, Y, st.moe_workspace(up, down, tokens, k), router_bias=b)
        assert (r.weights[:, 4:] == 0).all() and not torch.isin(r.ids[:, :4], torch.tensor(low, dtype=torch.int32, device="cuda")).any()
        assert (r.ids[:, 4:] == (-1 if value == -np.inf else torch.tensor([1, 2], device="cuda"))).all()
        outs.append((Y, r.ids[:, :4].clone(), r.weights.clone()))
    assert torch.equal(outs[0][1], outs[1][1]) and torch.equal(outs[0][2], outs[1][2])
    a, b = outs[0][0], outs[1][0]
    assert float((a - b).abs().max()) <= 2.0 ** -18 * float(a.abs().max())  # the same terms, summed in another order
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("tokens", [3, 16, 40])
def test_tokens_that_are_no_numbers(st, tokens):
    """A token with a NaN or an infinity: its logits are NaN or infinite, no other token's row changes."""
    import torch
    rng = np.random.default_rng(tokens)
    E, k, d, ff = 12, 2, 384, 256
    *_, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", "bf16", "f32", 0, 0)
    r, room = st.Routing(tokens, E, k), st.moe_workspace(up, down, tokens, k)
    X = torch.randn((tokens, d), device="cuda").to(torch.bfloat16)
    Y, Z = torch.empty_like(X), torch.empty_like(X)
    st.moe_forward(rtg, up, down, X, r, Y, room)
    bad = X.clone()
    bad[1, 5] = float("nan")
    bad[2, 300] = float("inf")
    st.moe_forward(rtg, up, down, bad, r, Z, room)
    assert (r.ids[1] == -1).all() and (Z[1] == 0).all()       # every logit NaN: no expert
    assert r.ids[2, 0] >= 0 and torch.isnan(Z[2]).all()       # some logits infinite: experts, whose input is no number
    keep = [i for i in range(tokens) if i not in (1, 2)]
    if tokens > 16:
        assert torch.equal(Y[keep], Z[keep])
    else:  # sums may be dealt otherwise when other experts are hit
        assert torch.allclose(Y[keep].float(), Z[keep].float(), rtol=2.0 ** -6, atol=1e-3 * float(Y.float().abs().max()))
    up.destroy()
    down.destroy()


def test_all_tokens_alike_and_equal_logits(st):
    """Every token to the same experts; equal logits go to the lower index."""
    import torch
    rng = np.random.default_rng(1)
    E, k, d, ff = 20, 4, 256, 384
    *_, rtg, up, down = _moe_case(st, rng, 1, E, d, ff, "bf16", "bf16", "bf16", 0, 1)
    rtg = rtg[:1].expand(E, d).contiguous()
    x = torch.randn((1, d), device="cuda").to(torch.bfloat16)
    outs = []
    for tokens in (1, 2, 15, 16, 17, 50):
        X, r = x.expand(tokens, d).contiguous(), st.Routing(tokens, E, k)
        Y = torch.empty_like(X)
        st.moe_forward(rtg, up, down, X, r, Y, st.moe_workspace(up, down, tokens, k))
        assert (r.ids == torch.arange(k, device="cuda")).all() and (r.weights == 0.25).all()
        assert (Y == Y[:1]).all()
        outs.append(Y[0].float())
    for o in outs[1:]:
        assert float((o - outs[0]).norm() / outs[0].norm()) < 1e-2
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("tokens", [1, 4, 16, 60])
def test_captured_and_replayed(st, tokens):
    """Layer with epilogue, MLP and layer of experts in one graph, two graphs on the same workspaces, replayed on new inputs between eager calls."""
    import torch
    rng = np.random.default_rng(tokens)
    E, k, d, ff = 24, 3, 512, 300
    *_, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", "bf16", "bf16", 0, 1)
    w, s = _weights(rng, (), d, d, 0)
    lin = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=d), _gpu(w), _gpu(_smaller(s)))
    w1, s1 = _weights(rng, (1, 2), ff, d, 0)
    w2, s2 = _weights(rng, (), d, ff, 0)
    mup, mdown = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=1, gated=1), _gpu(w1), _gpu(_smaller(s1))), st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d), _gpu(w2), _gpu(s2))
    X = torch.empty((tokens, d), dtype=torch.bfloat16, device="cuda")

    def buffers():
        return [torch.empty_like(X) for _ in range(3)], st.Routing(tokens, E, k), lin.alloc_workspace(tokens), st.mlp_workspace(mup, mdown, tokens), st.moe_workspace(up, down, tokens, k)

    def step(b):
        (a, h, y), r, w_lin, w_mlp, w_moe = b
        lin.linear_forward(X, a, w_lin, activation="gelu_tanh", residual=X)
        st.mlp_forward(mup, mdown, a, h, w_mlp, "silu", residual=a)
        st.moe_forward(rtg, up, down, h, r, y, w_moe, residual=h)
    one, two = buffers(), buffers()
    X.normal_()
    step(one)
    step(two)
    torch.cuda.synchronize()
    assert torch.equal(one[0][2], two[0][2])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(one)
        graphs.append(g)
    for i in range(4):
        X.normal_()
        for t in one[0]:
            t.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        step(two)
        for a, b in zip(one[0], two[0]):
            assert torch.equal(a, b), i
        assert torch.equal(one[1].ids, two[1].ids)
    for p in (up, down, lin, mup, mdown):
        p.destroy()


def test_two_layers_of_experts_at_once(st):
    """Calls on two streams, each with buffers of its own, again and again: each gives what it gives alone."""
    import torch
    rng = np.random.default_rng(9)
    E, k, d, ff, tokens = 32, 4, 1024, 640, 8
    *_, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", "bf16", "bf16", 0, 0)
    X = [torch.randn((tokens, d), device="cuda").to(torch.bfloat16) for _ in range(2)]
    alone = []
    rooms = [(st.Routing(tokens, E, k), st.moe_workspace(up, down, tokens, k)) for _ in X]
    for x, (r, ws) in zip(X, rooms):
        Y = torch.empty_like(x)
        st.moe_forward(rtg, up, down, x, r, Y, ws, residual=x)
        alone.append(Y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in X]
    outs = [[torch.empty_like(x) for _ in range(20)] for x in X]
    torch.cuda.synchronize()
    for i in range(20):
        for s, x, (r, ws), o in zip(streams, X, rooms, outs):
            st.moe_forward(rtg, up, down, x, r, o[i], ws, residual=x, stream=s)
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(torch.equal(a, y) for y in o)
    up.destroy()
    down.destroy()


# ---- refusals that need plans ----

def test_refusals(st):
    import torch
    rng = np.random.default_rng(0)
    d, n = 256, 128

    def plan(d_in, d_out, experts=0, gated=0, **kw):
        lead = ((experts,) if experts else ()) + ((2,) if gated else ())
        w, ws = _weights(rng, lead, d_out, d_in, 1)
        return st.Fp8Plan(st.Fp8Desc(d_in=d_in, d_out=d_out, experts=experts, gated=gated, **kw), _gpu(w), _gpu(ws))

    def status(code, f):
        with pytest.raises(st.StampError) as e:
            f()
        assert e.value.status == code
    lin, sq, down, gated1, gated2, down2 = plan(d, n), plan(d, d), plan(n, d), plan(d, n, 1, 1), plan(d, n, 2, 1), plan(n, d, 2)
    X, Y, Z = (torch.zeros((4, c), dtype=torch.bfloat16, device="cuda") for c in (d, n, d))
    room = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    rt, r, r3 = torch.zeros((2, d), device="cuda"), st.Routing(4, 2, 1), st.Routing(4, 3, 1)
    status(2, lambda: sq.linear_forward(X, X, room, residual=X))                               # X is read while Y is written
    wide = torch.zeros((8, n), dtype=torch.bfloat16, device="cuda")
    status(2, lambda: lin.linear_forward(X, wide[:4], room, residual=torch.as_strided(wide, (4, n), (2 * n, 1))))  # from Y's address on, but other rows
    status(4, lambda: lin.linear_forward(X, Y, room[:64], activation="relu"))
    status(3, lambda: gated2.grouped_forward(X, torch.zeros(3, dtype=torch.int32, device="cuda"), Y, room, activation="relu"))
    status(3, lambda: st.mlp_forward(gated2, down2, X, Z, room, "silu"))                       # experts: moe_forward's
    status(3, lambda: st.mlp_forward(lin, down2, X, Z, room, "silu"))
    status(3, lambda: st.mlp_forward(lin, gated1, X, Y, room, "silu"))
    status(2, lambda: st.mlp_forward(lin, plan(n + 1, d), X, Z, room, "silu"))
    status(2, lambda: st.mlp_forward(lin, plan(n, d, scale_format=1), X, Z, room, "silu"))
    status(4, lambda: st.mlp_forward(lin, down, X, Z, room[:256], "silu"))
    assert st.mlp_workspace(gated2, down2, 4).numel() == 256                                   # nothing that the call would take
    status(3, lambda: st.moe_forward(rt, lin, down, X, r, Z, room))
    status(2, lambda: st.moe_forward(torch.zeros((3, d), device="cuda"), gated2, down2, X, r3, Z, room))
    status(4, lambda: st.moe_forward(rt, gated2, down2, X, r, Z, room[:256]))
    for bad in (lambda: lin.linear_forward(X, Y, room, activation="tanh"), lambda: lin.linear_forward(X, Y, room, residual=Z), lambda: lin.linear_forward(X, Y, room, residual=Y.float()),
                lambda: lin.linear_forward(X, Y, room, residual=Y.cpu()), lambda: st.mlp_forward(lin, down, X, Z, room, "swish"), lambda: st.mlp_forward(lin, down, X, Z, room, "gelu", residual=Y),
                lambda: st.moe_forward(rt.half(), gated2, down2, X, r, Z, room), lambda: st.moe_forward(rt[:, :-1], gated2, down2, X, r, Z, room),
                lambda: st.moe_forward(rt.t().contiguous().t(), gated2, down2, X, r, Z, room), lambda: st.moe_forward(rt.cpu(), gated2, down2, X, r, Z, room),
                lambda: st.moe_forward(rt, gated2, down2, X, r, Z, room, router_bias=torch.zeros(3, device="cuda")),
                lambda: st.moe_forward(rt, gated2, down2, X, r, Z, room, activation=2)):
        with pytest.raises(ValueError):
            bad()
    # nothing to do
    lin.linear_forward(X[:0], Y[:0], room, activation="gelu", residual=Y[:0])
    st.mlp_forward(lin, down, X[:0], Z[:0], room, "gelu", residual=Z[:0])
    r0 = st.Routing(0, 2, 1)
    r0.offsets.fill_(5)
    st.moe_forward(rt, gated2, down2, X[:0], r0, Z[:0], room)
    assert (r0.offsets == 0).all()
    for p in (lin, sq, down, gated1, gated2, down2):
        p.destroy()


# ---- large calls: places beyond 2^32 bytes ----

def test_rows_beyond_4_gib(st):
    """Y, the residual and the codes of h pass 2^32 bytes; rows from all over are held against the definition."""
    import torch
    rng = np.random.default_rng(11)
    rows, d, n = (1 << 20) + 77, 128, 4100
    w, ws = _weights(rng, (), n, d, 0)
    ws = _smaller(ws)
    X = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda").normal_()
    R = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda").normal_()
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n), _gpu(w), _gpu(ws))
    Y, room = torch.empty_like(R), plan.alloc_workspace(rows)
    some = np.concatenate([rng.integers(0, rows, 60), [0, 1, rows - 2, rows - 1]])
    at = _gpu(some)
    plan.linear_forward(X, Y, room, activation="gelu", residual=R)
    x, res = X[at].float().cpu().numpy(), R[at].float().cpu().numpy().astype(np.float64)
    _held(Y[at], *block.layer(x, w, ws, None, "gelu", res, "bf16", 0, False), "layer")
    plan.destroy()
    del R, Y, room
    ff, m = 4224, 64
    w1, s1 = _weights(rng, (), ff, d, 0)
    w2, s2 = _weights(rng, (), m, ff, 0)
    s1 = _smaller(s1)
    up, down = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff), _gpu(w1), _gpu(s1)), st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=m, y_dtype=st.STAMP_F32), _gpu(w2), _gpu(s2))
    room = st.mlp_workspace(up, down, rows)
    assert room.numel() > 1 << 32
    Y = torch.empty((rows, m), device="cuda")
    st.mlp_forward(up, down, X, Y, room, "silu")
    _held(Y[at], *block.mlp(x, w1, s1, None, w2, s2, None, "silu", None, "f32", 0), "mlp")
    up.destroy()
    down.destroy()


def test_many_tokens_through_the_layer_of_experts(st):
    import torch
    rng = np.random.default_rng(12)
    tokens, E, top_k, d, ff = 70000, 9, 3, 256, 200
    _, _, w_up, s_up, w_down, s_down, b, rt, rtg, up, down = _moe_case(st, rng, 1, E, d, ff, "bf16", "bf16", "bf16", 0, 1)
    X = torch.empty((tokens, d), dtype=torch.bfloat16, device="cuda").normal_()
    r, room, Y = st.Routing(tokens, E, top_k), st.moe_workspace(up, down, tokens, top_k), torch.empty_like(X)
    st.moe_forward(rtg, up, down, X, r, Y, room, residual=X)
    x = X.float().cpu().numpy().astype(np.float64)
    l, err = block.logits(x, rt, None)
    apart = [i for i in rng.integers(0, tokens, 400) if block.clear(l[i:i + 1], err[i:i + 1], top_k)][:150]
    assert len(apart) == 150
    want, tol, ids, weights, *_, dw = block.moe(x[apart], rt, None, w_up, s_up, w_down, s_down, b, top_k, 1, "silu", x[apart], "bf16", 0)
    at = _gpu(np.array(apart))
    assert np.array_equal(r.ids[at].cpu().numpy(), ids) and int(r.offsets[-1]) == tokens * top_k
    _held(Y[at], want, tol, "sampled tokens")
    up.destroy()
    down.destroy()
