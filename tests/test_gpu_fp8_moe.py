"""The two kernels of the layer of experts for few tokens where they can go wrong: waits that give up, widths and rows that take every loop round again, and what a
token's result depends on; against the definition in 64 bits (fp8_block_reference.py)."""
import numpy as np
import pytest

import fp8_block_reference as block
import fp8_reference as ref
from test_gpu_fp8 import _activations, _dt, _gpu, _strided
from test_gpu_fp8_block import _held, _moe_case, _values, st  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


# ---- waits ----

@pytest.mark.parametrize("tokens,E,top_k,d,ff", [(1, 1, 1, 256, 40000), (3, 8, 2, 384, 5000), (16, 40, 8, 256, 1400)])
@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_a_wait_that_gives_up_leaves_no_number(st, tokens, E, top_k, d, ff, y):  # noqa: F811
    """With no look behind the first, workgroups do not wait for the others' rows of h: every element of Y is the right one or NaN.  The first
    workgroup without a product comes to its columns while the products before are still worked on, so some are NaN."""
    import torch
    rng = np.random.default_rng(tokens)
    _, X, *_, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", y, "f32", 0, 1)
    r, room = st.Routing(tokens, E, top_k), st.moe_workspace(up, down, tokens, top_k)
    assert st.moe_route(up, down, tokens, top_k) == "few"
    want, Y = (torch.empty((tokens, d), dtype=_dt(y), device="cuda") for _ in range(2))
    st.moe_forward(rtg, up, down, X, r, want, room)
    assert torch.isfinite(want).all()
    ids, given_up = r.ids.clone(), 0
    up.set_looks(0)
    for value in (0, 63, 255) * 4:
        room.fill_(value)  # what a row of h holds that nobody has written
        Y.fill_(-7.0)
        st.moe_forward(rtg, up, down, X, r, Y, room)
        lost = torch.isnan(Y)
        assert torch.equal(Y[~lost], want[~lost]) and torch.equal(r.ids, ids)
        given_up += int(lost.any())
    assert given_up > 0
    up.set_looks()
    room.fill_(255)
    st.moe_forward(rtg, up, down, X, r, Y, room)
    assert torch.equal(Y, want)
    with pytest.raises(st.StampError) as e:
        up.set_looks(-2)
    assert e.value.status == 2
    up.destroy()
    down.destroy()


# ---- loops that go round again ----

def _rounds(tokens, offsets, top_k, d, ff):
    """What a call takes beyond the first round: blocks of channels that a wave of an up product asks for behind its first 4; sets of experts whose rows of h a part of the
    columns holds one after the other; units (128 rows of an expert's down matrix) of a wave beyond 60; columns beyond a workgroup's first 64."""
    import torch
    cus, E, groups, kb, kb_up = torch.cuda.get_device_properties(0).multi_processor_count, len(offsets) - 1, -(-d // 64), -(-ff // 128), -(-d // 128)
    parts = max(1, min(min(tokens * top_k, E) * kb // 8, max(1, min(16, cus // groups))))
    first = [0] + [int(b) for a, b in zip(offsets[:-1], offsets[1:]) if b > a]
    units, most, held, longest = (len(first) - 1) * kb, (96 << 10) // (132 * kb + 16), 0, 0
    for p in range(parts):
        a, b = units * p // parts, units * (p + 1) // parts
        i, end, sets = a // kb, (b - 1) // kb + 1, 0
        while a < b and i < end:
            j = i + 1
            while j < end and first[j + 1] - first[i] <= most:
                j += 1
            longest = max(longest, -(-(min(b, j * kb) - max(a, i * kb)) // 8))
            i, sets = j, sets + 1
        held = max(held, sets)
    return dict(channels=-(-kb_up // 8) > 4, rows=held > 1, units=longest > 64, columns=groups * parts > cus)


@pytest.mark.parametrize("tokens,E,top_k,d,ff,again", [
    (5, 6, 2, 5000, 200, "channels"), (16, 9, 3, 9001, 130, "channels"), (1, 2, 2, 4097, 77, "channels"), (16, 3, 3, 300, 5504, "rows"), (16, 5, 4, 4500, 2700, "channels rows"),
    (15, 7, 5, 200, 6000, "rows"), (2, 2, 1, 16700, 128, "channels columns"), (16, 4, 2, 16390, 300, "channels columns")])
@pytest.mark.parametrize("x,y,pow2", [("bf16", "f32", 0), ("f32", "bf16", 1)])
def test_few_tokens_where_loops_go_round_again(st, tokens, E, top_k, d, ff, again, x, y, pow2):  # noqa: F811
    import torch
    rng = np.random.default_rng(tokens * 1000 + d)
    xv, X, w_up, s_up, w_down, s_down, b, rt, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, x, y, "f32", pow2, 1)
    res, R, _ = _values(rng, tokens, d, y, 1)
    want, tol, ids, weights, offsets, token, row, dw = block.moe(xv, rt, None, w_up, s_up, w_down, s_down, b, top_k, 1, "silu", res, y, pow2)
    assert st.moe_route(up, down, tokens, top_k) == "few"
    assert [n for n, v in _rounds(tokens, offsets, top_k, d, ff).items() if v] == again.split()
    r, room = st.Routing(tokens, E, top_k), st.moe_workspace(up, down, tokens, top_k)
    Y = torch.full((tokens, d), -7.0, dtype=_dt(y), device="cuda")
    for value in (255, 0):
        room.fill_(value)
        first = Y.clone()
        st.moe_forward(rtg, up, down, X, r, Y, room, residual=R)
        _held(Y, want, tol, f"workspace of {value}")
        assert np.array_equal(r.ids.cpu().numpy(), ids) and np.array_equal(r.row_of_slot.cpu().numpy(), row)
    assert torch.equal(first, Y)
    up.destroy()
    down.destroy()


def test_few_tokens_where_a_wave_has_many_units(st):  # noqa: F811
    """More than 64 blocks of h a wave takes weights of 2 GB: the up matrices are zero behind their first 256 channels, Y is looked at in some blocks of columns."""
    import torch
    rng = np.random.default_rng(5)
    E, top_k, d, ff, used = 3, 3, 8256, 240 * 128 - 50, 256
    gen = torch.Generator(device="cuda").manual_seed(5)

    def codes(*shape):
        c = torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=gen)
        return c.masked_fill_((c & 0x7f) == 0x7f, 0x3a)

    def scales(low, *shape):
        return (2.0 ** rng.uniform(low - 8, low, shape)).astype(np.float32)
    nb, nf = -(-d // 128), -(-ff // 128)
    w_up = torch.zeros((E, 2, ff, d), dtype=torch.uint8, device="cuda")
    w_up[..., :used] = codes(E, 2, ff, used)
    w_down, s_up, s_down = codes(E, d, ff), scales(-10, E, 2, nf, nb), scales(-4, E, nb, nf)
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=E, gated=1), w_up, _gpu(s_up))
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d, experts=E, y_dtype=st.STAMP_F32), w_down, _gpu(s_down))
    xv, X = _activations(rng, 1, d, "bf16")
    rt = (rng.standard_normal((E, d)) / np.sqrt(30.0 * d)).astype(np.float32)
    assert st.moe_route(up, down, 1, top_k) == "few" and _rounds(1, [0, 1, 2, 3], top_k, d, ff)["units"]
    r, room, Y = st.Routing(1, E, top_k), st.moe_workspace(up, down, 1, top_k), torch.empty((1, d), device="cuda")
    room.fill_(255)
    st.moe_forward(_gpu(rt), up, down, X, r, Y, room)
    w_up = w_up[..., :used].cpu().numpy()
    for at in (0, 31, 63):  # blocks of 128 columns
        cols = slice(128 * at, 128 * at + 128)
        want, tol, ids, *_ = block.moe(xv.astype(np.float64), rt.astype(np.float64), None, w_up, s_up[..., :used // 128], w_down[:, cols].cpu().numpy(), s_down[:, at:at + 1], None, top_k, 1,
                                       "silu", None, "f32", 0)
        assert np.array_equal(r.ids.cpu().numpy(), ids)
        _held(Y[:, cols], want, tol, f"columns {cols}")
    up.destroy()
    down.destroy()


# ---- a token and the others of its call ----

@pytest.mark.parametrize("tokens,top_k", [(3, 2), (9, 5), (16, 8)])
def test_other_tokens_move_a_row_by_the_order_of_its_sums_alone(st, tokens, top_k):  # noqa: F811
    """Two tokens of a call stay, the others become NaN, infinite or other ones: the rows that stay have the same terms, one for each expert and 128 channels of h,
    and at most that many sums of theirs plus those of 8 waves, 16 parts, the bias of every slot; either call rounds each by at most 2^-24 of the magnitudes."""
    import torch
    rng = np.random.default_rng(tokens)
    E, d, ff = 20, 384, 700
    xv, X, w_up, s_up, w_down, s_down, b, rt, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, "bf16", "f32", "f32", 0, 1)
    keep = [0, tokens - 1]
    r, room, Y, Z = st.Routing(tokens, E, top_k), st.moe_workspace(up, down, tokens, top_k), *(torch.empty((tokens, d), device="cuda") for _ in range(2))
    st.moe_forward(rtg, up, down, X, r, Y, room)
    ids, weights = r.ids.cpu().numpy(), r.weights.cpu().numpy().astype(np.float64)
    size = np.zeros((len(keep), d))  # the terms' magnitudes
    codes, scales = ref.quantize(xv, 0)
    for i, t in enumerate(keep):
        for e, w in zip(ids[t], weights[t]):
            h, _ = block.hidden(codes[t:t + 1], scales[t:t + 1], w_up[e], s_up[e], None, "silu")
            size[i] += w * (ref.product(*ref.quantize(h.astype(np.float32), 0), w_down[e], s_down[e])[1][0] + np.abs(b[e]))
    sums = top_k * -(-ff // 128) + 8 + 16 + top_k
    others = X.clone()
    others[1, 5] = float("nan")
    if tokens > 3:
        others[2, 300] = float("inf")
        others[3:-1] = torch.randn_like(others[3:-1])
    room.fill_(255)
    st.moe_forward(rtg, up, down, others, r, Z, room)
    assert np.array_equal(r.ids.cpu().numpy()[keep], ids[keep]) and (r.ids[1] == -1).all() and (Z[1] == 0).all() and (tokens == 3 or torch.isnan(Z[2]).all())
    off = (Y[keep].double() - Z[keep].double()).abs().cpu().numpy()
    assert (off <= 2 * sums * 2.0 ** -24 * size * 1.01).all(), np.max(off / size) * 2.0 ** 24
    up.destroy()
    down.destroy()


# ---- where tensors lie ----

@pytest.mark.parametrize("tokens", [1, 5, 16, 30])
@pytest.mark.parametrize("x,router", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_rows_at_any_place_and_a_workspace_of_a_larger_call(st, tokens, x, router):  # noqa: F811
    """X in rows that lie apart and begin anywhere, the router's matrix too, a stream of its own, the workspace of 64 tokens before and after: the bits of
    the plain call."""
    import torch
    rng = np.random.default_rng(tokens)
    E, top_k, d, ff = 9, 3, 333, 200
    xv, X, *_, rtg, up, down = _moe_case(st, rng, tokens, E, d, ff, x, "bf16", router, 0, 1)
    r, Y = st.Routing(tokens, E, top_k), torch.empty((tokens, d), dtype=torch.bfloat16, device="cuda")
    st.moe_forward(rtg, up, down, X, r, Y, st.moe_workspace(up, down, tokens, top_k))
    apart, _ = _strided(tokens, d, x, 4, 1)
    apart.copy_(X)
    moved = torch.empty(E * d + 1, dtype=rtg.dtype, device="cuda")[1:].view(E, d)
    moved.copy_(rtg)
    room, more = st.moe_workspace(up, down, 64, top_k), torch.randn((64, d), device="cuda").to(X.dtype)
    r64, Y64 = st.Routing(64, E, top_k), torch.empty((64, d), dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):
        Z = torch.full_like(Y, -7.0)
        torch.cuda.synchronize()
        st.moe_forward(rtg, up, down, more, r64, Y64, room, stream=stream)
        st.moe_forward(moved, up, down, apart, r, Z, room, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(Y, Z)
    up.destroy()
    down.destroy()
