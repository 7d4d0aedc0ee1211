"""Calls of the 8-bit floating point layers, the router and the experts at the ends of their ranges, on the GPU."""
import numpy as np
import pytest

import fp8_calls_reference as calls
import fp8_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def st():
    import paper_2510_26771_amd as st
    st.load_library()
    return st


def _gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _needs(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of free GPU memory")


# ---- more units of work than one launch takes (2^32 threads) ----

def test_quantizer_and_widening_of_the_most_rows(st):
    """2^24 rows of 32 blocks: the first, the last, and the rows on both sides of every 2^31 units of 16 channels."""
    import torch
    _needs(214)
    rows, d = 1 << 24, 3969
    rng = np.random.default_rng(0)
    w, ws = rng.integers(0, 120, (1, d), dtype=np.uint8), np.ones((1, 32), np.float32)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=1, y_dtype=st.STAMP_F32), _gpu(w), _gpu(ws))
    X = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda")
    look = torch.tensor([0, 1, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, 12345678, rows - 2, rows - 1], device="cuda")
    x = torch.from_numpy(rng.standard_normal((look.numel(), d)).astype(np.float32)).to(torch.bfloat16)
    X[look] = x.cuda()
    codes, scales = plan.alloc_act_buffers(rows)
    codes[look] = 0xEE
    plan.quantize_act(X, codes, scales)
    want, wscale = ref.quantize(x.float().numpy(), 0)
    assert np.array_equal(codes[look].cpu().numpy(), want)
    assert np.array_equal(scales[:, look].cpu().numpy().T, wscale)
    del X
    torch.cuda.empty_cache()
    Y = torch.zeros((rows, 1), device="cuda")
    assert plan.route(rows) != "rows"  # tiles: the codes are widened first
    plan.linear_forward_q(codes, scales, Y, plan.alloc_workspace(rows))
    y, S, G = ref.product(want, wscale, w, ws)
    assert np.all(np.abs(Y[look].cpu().numpy() - y) <= ref.slack(S, G, d, True) + 2.0 ** -23 * np.abs(y))
    plan.destroy()
    del codes, scales, Y
    torch.cuda.empty_cache()


def test_weights_of_64_gib(st):
    """1024 experts of 8192 x 8192: codes of the first, the last and those in the middle."""
    import torch
    _needs(140)
    E, d, n = 1024, 8192, 8192
    rng = np.random.default_rng(1)
    w = torch.empty((E, n, d), dtype=torch.uint8, device="cuda")
    ws = torch.ones((E, 64, 64), device="cuda")
    look = [0, 511, 512, E - 1]
    for e in look:
        w[e] = torch.from_numpy(rng.integers(0, 120, (1, d), dtype=np.uint8)).cuda()  # every column of an expert alike
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, experts=E), w, ws)
    rows = len(look)
    x = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(torch.bfloat16)
    counts = np.zeros(E, int)
    counts[look] = 1
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    Y = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
    plan.grouped_forward(x.cuda(), _gpu(offsets), Y, plan.alloc_workspace(rows))
    codes, scales = ref.quantize(x.float().numpy(), 0)
    got = Y.float().cpu().numpy()
    for i, e in enumerate(look):
        y, S, G = ref.product(codes[i:i + 1], scales[i:i + 1], w[e, :1].cpu().numpy(), np.ones((1, 64), np.float32))
        assert np.all(np.abs(got[i] - y[0]) <= ref.slack(S, G, d, True)[0] + 2.0 ** -8 * np.abs(y[0]))
    plan.destroy()
    del w, ws
    torch.cuda.empty_cache()


def test_experts_of_the_most_slots(st):
    """2^24 slots, 64 tiles of columns each: every token has the outputs that it has among a few, by the same kernels."""
    import torch
    _needs(150)
    tokens, E, d, ff = 1 << 19, 32, 128, 8192
    g = torch.Generator(device="cuda").manual_seed(2)
    w_up = (torch.randn((E, 2, ff, d), device="cuda", generator=g) * d ** -0.5).to(torch.bfloat16)
    w_down = (torch.randn((E, d, ff), device="cuda", generator=g) * ff ** -0.5).to(torch.bfloat16)
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=E, gated=1, w_dtype=st.STAMP_BF16), w_up)
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d, experts=E, w_dtype=st.STAMP_BF16), w_down)
    up.set_route("tiles_128")
    down.set_route("tiles_256")
    X = torch.randn((tokens, d), device="cuda", generator=g).to(torch.bfloat16)
    L = torch.randn((tokens, E), device="cuda", generator=g)
    Y = torch.full((tokens, d), -7.0, dtype=torch.bfloat16, device="cuda")

    def run(x, l, y):
        r = st.Routing(x.shape[0], E, E)
        st.route_topk(l, r)
        st.experts_forward(up, down, x, r, y, st.experts_workspace(up, down, x.shape[0], E))
    run(X, L, Y)
    look = torch.tensor([0, 1, tokens // 2 - 1, tokens // 2, 400000, tokens - 2, tokens - 1], device="cuda")
    few = torch.empty((look.numel(), d), dtype=torch.bfloat16, device="cuda")
    run(X[look].contiguous(), L[look].contiguous(), few)
    assert torch.isfinite(few).all() and torch.equal(Y[look], few)
    # all tokens: from a second call on each quarter of them
    Q = torch.empty((tokens // 4, d), dtype=torch.bfloat16, device="cuda")
    for q in range(4):
        part = slice(q * (tokens // 4), (q + 1) * (tokens // 4))
        run(X[part], L[part], Q)
        assert torch.equal(Y[part], Q), q
    up.destroy()
    down.destroy()
    torch.cuda.empty_cache()


# ---- limits ----

@pytest.mark.parametrize("d", [1, 128, 385, 512])
def test_the_most_tokens_of_the_experts(st, d):
    """tokens * (d rounded up to 128) < 2^31: one token fewer gets as far as the missing workspace, nothing is launched."""
    import ctypes as C

    from paper_2510_26771_amd import fp8
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=8, experts=1, gated=1), _gpu(np.zeros((1, 2, 8, d), np.uint8)), _gpu(np.ones((2, -(-d // 128)), np.float32)))
    down = st.Fp8Plan(st.Fp8Desc(d_in=8, d_out=d, experts=1), _gpu(np.zeros((1, d, 8), np.uint8)), _gpu(np.ones((-(-d // 128), 1), np.float32)))
    most = min((2 ** 31 - 1) // (-(-d // 128) * 128), 1 << 22)

    def status(tokens):
        r = fp8._Routing(tokens, 1, 1, 256, 256, 256, 256, 256)
        return up.lib.stamp_experts_forward(up._h, down._h, C.byref(r), 256, d, 256, d, None, 0, None)
    assert status(most) == 4 and status(most + 1) == 3
    up.destroy()
    down.destroy()


# ---- fp32 results: sums of both products and the rows between them in fp32 ----

def _plans(st, w_up, s_up, w_down, s_down, y, pow2, up_route, down_route):
    E, _, ff, d = w_up.shape
    up = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=ff, experts=E, gated=1, x_dtype=st.STAMP_F32, scale_format=pow2), _gpu(w_up), _gpu(s_up))
    down = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=d, experts=E, y_dtype=y, scale_format=pow2), _gpu(w_down), _gpu(s_down))
    up.set_route(up_route)
    down.set_route(down_route)
    return up, down


@pytest.mark.parametrize("route", ["", "rows", "tiles_64", "tiles_128"])
@pytest.mark.parametrize("pow2", [0, 1])
@pytest.mark.parametrize("tokens,experts,top_k,d,ff", [(1, 3, 2, 130, 200), (40, 3, 2, 150, 270), (150, 6, 3, 300, 257), (300, 2, 1, 257, 640)])
def test_experts_in_fp32_against_the_definition(st, tokens, experts, top_k, d, ff, pow2, route):
    import torch
    rng = np.random.default_rng(tokens)
    x = rng.standard_normal((tokens, d)).astype(np.float32)
    w_up, w_down = (ref.encode(rng.standard_normal(s).astype(np.float32) * 40) for s in ((experts, 2, ff, d), (experts, d, ff)))
    s_up = np.exp2(rng.integers(-10, -8, (experts, 2, -(-ff // 128), -(-d // 128)))).astype(np.float32)
    s_down = np.exp2(rng.integers(-10, -8, (experts, -(-d // 128), -(-ff // 128)))).astype(np.float32)
    l = rng.standard_normal((tokens, experts)).astype(np.float32)
    up, down = _plans(st, w_up, s_up, w_down, s_down, st.STAMP_F32, pow2, route, route)
    r, Y = st.Routing(tokens, experts, top_k), torch.empty((tokens, d), device="cuda")
    st.route_topk(_gpu(l), r)
    st.experts_forward(up, down, _gpu(x), r, Y, st.experts_workspace(up, down, tokens, top_k))
    want, bound = calls.experts(x, l, w_up, s_up, w_down, s_down, top_k, 1, pow2, False)
    far = np.abs(Y.cpu().numpy() - want) / bound
    assert far.max() <= 1, f"{(far > 1).sum()} of {far.size} beyond the bound, worst {far.max():.3g} times it"
    up.destroy()
    down.destroy()


@pytest.mark.parametrize("route", ["", "rows", "tiles_64", "tiles_128"])
@pytest.mark.parametrize("rows", [3, 70, 300])
@pytest.mark.parametrize("ff", [128, 256, 520])
def test_fp32_results_hold_what_8_bit_sums_would_lose(st, rows, ff, route):
    """Small products between large ones that cancel: of a layer, of one by expert, and of the experts' down product."""
    import torch
    rng = np.random.default_rng(ff)
    n = 60
    h, w = calls.cancelling(rng, ff, n)
    blocks = -(-ff // 128)
    ones = np.ones((1, blocks), np.float32)
    x = ref.E4M3[h].astype(np.float32)[None].repeat(rows, 0)  # its codes are h: every block holds a 448
    codes, scales = ref.quantize(x, 0)
    assert (codes[:, :ff] == h).all() and (scales == 1).all()
    y, S, G = ref.product(codes, scales, w, ones)
    bound = ref.slack(S, G, ff, True)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=n, x_dtype=st.STAMP_F32, y_dtype=st.STAMP_F32), _gpu(w), _gpu(ones))
    two = st.Fp8Plan(st.Fp8Desc(d_in=ff, d_out=n, experts=2, x_dtype=st.STAMP_F32, y_dtype=st.STAMP_F32), _gpu(np.stack([w, w])), _gpu(np.stack([ones, ones])))
    Y = torch.empty((rows, n), device="cuda")
    for p, call in ((plan, lambda ws: plan.linear_forward(_gpu(x), Y, ws)), (two, lambda ws: two.grouped_forward(_gpu(x), _gpu(np.int32([0, 1, rows])), Y, ws))):
        p.set_route(route)
        Y.fill_(np.nan)
        call(p.alloc_workspace(rows))
        assert np.all(np.abs(Y.cpu().numpy() - y) <= bound + 2.0 ** -23 * np.abs(y))
        p.destroy()
    # experts of one channel: x = 1, gates of 16, up columns of h's values; h is 16 (1 - 1e-7) times those, its codes the same
    gate = np.full(ff, 16.0)
    w_up = ref.encode(np.stack([gate, ref.E4M3[h]])[None, :, :, None].repeat(2, 0).astype(np.float32))
    w_down = np.zeros((2, 1, ff), np.uint8)
    w_down[:] = w[:1]
    up, down = _plans(st, w_up, np.ones((2, 2, blocks, 1), np.float32), w_down, np.ones((2, 1, blocks), np.float32), st.STAMP_F32, 0, route, route)
    one = np.ones((rows, 1), np.float32)
    l = rng.standard_normal((rows, 2)).astype(np.float32)
    r, Y = st.Routing(rows, 2, 1), torch.empty((rows, 1), device="cuda")
    st.route_topk(_gpu(l), r)
    st.experts_forward(up, down, _gpu(one), r, Y, st.experts_workspace(up, down, rows, 1))
    want, bound = calls.experts(one, l, w_up, np.ones((2, 2, blocks, 1), np.float32), w_down, np.ones((2, 1, blocks), np.float32), 1, 1, 0, False)
    lost, _ = calls.experts(one, l, w_up, np.ones((2, 2, blocks, 1), np.float32), w_down, np.ones((2, 1, blocks), np.float32), 1, 1, 0, False,
                            sums=calls.eight_bit_sums)
    assert np.all(np.abs(lost - want) > bound), "the bound would let them pass"
    assert np.all(np.abs(Y.cpu().numpy() - want) <= bound)
    up.destroy()
    down.destroy()


# ---- the router where a lane has two of the chosen, a wave more than one round of tokens, and at 1024 experts ----

@pytest.mark.parametrize("kind", ["plain", "masked", "ties", "extreme"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,experts,top_k", [(130, 200, 32), (70, 40, 17), (65, 17, 32), (33, 1024, 32), (4096, 1024, 3), (4097, 1024, 3), (5000, 257, 20),
                                                  (16384, 20, 2), (16385, 20, 2), (17000, 256, 18), (40000, 100, 4)])
def test_router_over_many_tokens_and_choices(st, tokens, experts, top_k, dtype, kind):
    import torch
    rng = np.random.default_rng(tokens + experts)
    l = rng.standard_normal((tokens, experts)).astype(np.float32)
    if kind == "masked":
        l[rng.random(l.shape) < 0.7] = -np.inf
        l[rng.random(l.shape) < 0.1] = np.nan
        l[tokens // 2] = -np.inf
    if kind == "ties":
        l = rng.integers(-1, 2, l.shape).astype(np.float32) * np.where(rng.random(l.shape) < 0.5, -1, 1).astype(np.float32)
    if kind == "extreme":
        l[rng.random(l.shape) < 0.3] = np.finfo(np.float32).min
        l[tokens // 2, : experts // 2 + 1] = np.inf
    t = torch.from_numpy(l).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    r = st.Routing(tokens, experts, top_k)
    for renormalize in (0, 1):
        for a in (r.ids, r.offsets, r.token_of_row, r.row_of_slot):
            a.fill_(-77)
        st.route_topk(t.cuda(), r, renormalize=renormalize)
        ids, weights, offsets, token, row = calls.route(t.float().numpy(), top_k, renormalize)
        for name, want in (("ids", ids), ("offsets", offsets), ("token_of_row", token), ("row_of_slot", row)):
            assert np.array_equal(getattr(r, name).cpu().numpy(), want), name
        w = r.weights.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(w - weights) <= calls.weight_bound(experts) * weights + 1e-37)


# ---- loads far from even: one or two experts have nearly all rows, the rule knows only the average ----

@pytest.mark.parametrize("x,y,pow2", [("f32", "f32", 0), ("bf16", "bf16", 1)])
@pytest.mark.parametrize("experts,busy,d,n", [(64, {5: 200}, 256, 64), (64, {5: 700}, 256, 320), (128, {0: 740, 127: 760}, 300, 140), (40, {39: 352, 2: 1}, 520, 300),
                                              (256, {200: 2990, 3: 17}, 128, 70), (20, {7: 600, 8: 1, 9: 33}, 1152, 200)])
def test_grouped_with_uneven_loads(st, experts, busy, d, n, x, y, pow2):
    import torch
    rng = np.random.default_rng(experts + d)
    counts = np.zeros(experts, int)
    for e, c in busy.items():
        counts[e] = c
    rows = int(counts.sum())
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    types = {"f32": (torch.float32, st.STAMP_F32), "bf16": (torch.bfloat16, st.STAMP_BF16)}
    X = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(types[x][0])
    w = ref.encode(rng.standard_normal((experts, n, d)).astype(np.float32) * 40)
    ws = np.exp2(rng.integers(-10, -8, (experts, -(-n // 128), -(-d // 128)))).astype(np.float32)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, experts=experts, x_dtype=types[x][1], y_dtype=types[y][1], scale_format=pow2), _gpu(w), _gpu(ws))
    Y = torch.full((rows, n), np.nan, dtype=types[y][0], device="cuda")
    plan.grouped_forward(X.cuda(), _gpu(offsets), Y, plan.alloc_workspace(rows))
    codes, scales = ref.quantize(X.float().numpy(), pow2)
    got = Y.float().cpu().numpy()
    for e in busy:
        part = slice(offsets[e], offsets[e + 1])
        want, S, G = ref.product(codes[part], scales[part], w[e], ws[e])
        bound = ref.slack(S, G, d, y == "f32" or plan.route(rows) == "rows") + (2.0 ** -23 if y == "f32" else 2.0 ** -8) * np.abs(want)
        assert np.all(np.abs(got[part] - want) <= bound), e
    plan.destroy()


@pytest.mark.parametrize("tokens,experts,top_k,d,ff", [(300, 64, 2, 256, 128), (700, 64, 2, 130, 200), (90, 128, 3, 256, 300)])
def test_experts_with_one_that_every_token_chooses(st, tokens, experts, top_k, d, ff):
    import torch
    rng = np.random.default_rng(tokens)
    x = rng.standard_normal((tokens, d)).astype(np.float32)
    w_up, w_down = (ref.encode(rng.standard_normal(s).astype(np.float32) * 40) for s in ((experts, 2, ff, d), (experts, d, ff)))
    s_up, s_down = (np.full((*s[:-2], -(-s[-2] // 128), -(-s[-1] // 128)), 2.0 ** -9, np.float32) for s in (w_up.shape, w_down.shape))
    l = rng.standard_normal((tokens, experts)).astype(np.float32)
    l[:, 9] += 20
    up, down = _plans(st, w_up, s_up, w_down, s_down, st.STAMP_F32, 0, "", "")
    r, Y = st.Routing(tokens, experts, top_k), torch.empty((tokens, d), device="cuda")
    st.route_topk(_gpu(l), r, renormalize=False)
    st.experts_forward(up, down, _gpu(x), r, Y, st.experts_workspace(up, down, tokens, top_k))
    assert int(r.offsets.diff()[9]) == tokens
    want, bound = calls.experts(x, l, w_up, s_up, w_down, s_down, top_k, 0, 0, False)
    assert np.all(np.abs(Y.cpu().numpy() - want) <= bound)
    up.destroy()
    down.destroy()


# ---- tiles cut by depth and by columns: that the sizes which are meant to reach these launches do, by rule ----

PARTS = [(200, 1290, 2), (130, 1500, 3), (130, 2000, 4), (100, 2500, 5), (100, 3000, 6), (100, 3500, 7), (100, 4096, 8)]


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("experts", [0, 2])
@pytest.mark.parametrize("rows,d,parts", PARTS)
def test_every_number_of_parts_of_the_depth(st, rows, d, parts, experts, y):
    import torch
    rng = np.random.default_rng(d)
    n, wide = 130, y == "f32"
    lead = (experts,) if experts else ()
    x = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(torch.bfloat16)
    w = ref.encode(rng.standard_normal((*lead, n, d)).astype(np.float32) * 40)
    ws = np.exp2(rng.uniform(-10, -8, (*lead, 2, -(-d // 128)))).astype(np.float32)
    bias = rng.standard_normal((*lead, n)).astype(np.float32)
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, experts=experts, y_dtype=st.STAMP_F32 if wide else st.STAMP_BF16), _gpu(w), _gpu(ws), _gpu(bias))
    if experts:
        plan.set_route("tiles_64")
    assert plan.cut(rows) == (0, parts if wide or parts > 3 else 1, 0)  # 8-bit sums: short depths stay whole
    buf = torch.full((rows + 1, n + 3), -7.0, dtype=torch.float32 if wide else torch.bfloat16, device="cuda")
    Y = buf[:rows, 1:n + 1]
    workspace = plan.alloc_workspace(rows)
    workspace.fill_(255)
    offsets = [0, rows // 3, rows] if experts else [0, rows]
    if experts:
        plan.grouped_forward(x.cuda(), _gpu(np.int32(offsets)), Y, workspace)
    else:
        plan.linear_forward(x.cuda(), Y, workspace)
    codes, scales = ref.quantize(x.float().numpy(), 0)
    got = Y.float().cpu().numpy()
    for e in range(len(offsets) - 1):
        part = slice(offsets[e], offsets[e + 1])
        want, S, G = ref.product(codes[part], scales[part], *((w[e], ws[e]) if experts else (w, ws)))
        b = bias[e] if experts else bias
        bound = ref.slack(S + np.abs(b), G, d, wide) + (2.0 ** -23 if wide else 2.0 ** -8) * np.abs(want + b)
        assert np.all(np.abs(got[part] - (want + b)) <= bound)
    Y.fill_(-7.0)
    assert (buf == -7.0).all()
    plan.destroy()


@pytest.mark.parametrize("rows,d,n,y,two", [
    (200, 2000, 320, "bf16", 0), (200, 2000, 320, "f32", 0), (130, 4096, 300, "bf16", 0), (130, 4096, 300, "f32", 0), (90, 7000, 515, "bf16", 0),
    (90, 7000, 515, "f32", 0), (3000, 520, 5700, "bf16", 1), (3000, 520, 5700, "f32", 1), (2900, 300, 5643, "bf16", 1), (2900, 300, 5643, "f32", 1),
    (324, 4725, 10849, "bf16", 2), (323, 2998, 10965, "f32", 2)])
def test_the_sizes_of_the_product_tests_reach_their_launches(st, rows, d, n, y, two):
    """two: 0 the depth in parts, 1 columns in two launches, 2 the second of them in parts as well."""
    plan = st.Fp8Plan(st.Fp8Desc(d_in=d, d_out=n, y_dtype=st.STAMP_F32 if y == "f32" else st.STAMP_BF16), _gpu(np.zeros((n, d), np.uint8)),
                      _gpu(np.ones((-(-n // 128), -(-d // 128)), np.float32)))
    columns, first, second = plan.cut(rows)
    assert (columns > 0) == (two > 0) and (first if two == 0 else second) > (1 if two != 1 else 0)
    assert plan.cut(1) == (0, 0, 0)
    plan.destroy()
