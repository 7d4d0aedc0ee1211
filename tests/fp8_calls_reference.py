"""The router and the experts' MLP in 64 bits for larger calls and tighter bounds than fp8_reference.py: whole arrays at a time, and errors
that follow the types that Y is asked in."""
import numpy as np

import fp8_reference as ref


def route(logits, top_k, renormalize):
    """As ref.route, without a loop over tokens."""
    l = np.asarray(logits, np.float64)
    t, e = l.shape
    l = np.where(np.isnan(l), -np.inf, l)
    k = min(top_k, e)
    ids = np.full((t, top_k), -1, np.int32)
    value = np.full((t, top_k), -np.inf)
    order = np.argsort(-l, axis=1, kind="stable")[:, :k]  # equal ones stay in order of their index
    value[:, :k] = np.take_along_axis(l, order, 1)
    ids[:, :k] = np.where(value[:, :k] > -np.inf, order, -1)
    top = value[:, :1]

    def share(v):
        with np.errstate(invalid="ignore"):
            return np.where(v == -np.inf, 0.0, np.where(v == top, 1.0, np.exp(v - top)))
    total = share(value if renormalize else l).sum(1, keepdims=True)
    weights = np.where(ids >= 0, share(value) / np.where(total > 0, total, 1.0), 0.0)
    flat = ids.reshape(-1)
    slots = np.argsort(np.where(flat >= 0, flat, e), kind="stable")
    n = int((flat >= 0).sum())
    row, token = np.full(t * top_k, -1, np.int32), np.full(t * top_k, -1, np.int32)
    row[slots[:n]] = np.arange(n)
    token[:n] = slots[:n] // top_k
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=e))]).astype(np.int32)
    return ids, weights, offsets, token, row.reshape(t, top_k)


def weight_bound(experts):
    """Relative error of a router weight: exp of a difference of up to 16, its own error, the sum's roundings and the quotient's."""
    return (32 + experts / 64 + 8) * 2.0 ** -23


def experts(x, logits, w_up, s_up, w_down, s_down, top_k, renormalize, pow2, y_bf16, held=None, sums=None):
    """(Y, bound) of the gated MLP.  Roundings on the way: the sums in fp32 of both products (`ref.slack`; of the down product by the FP8
    instructions where Y is bf16), silu, a code of h that may be its neighbour, the rows in Y's type, the weights and the sum over a
    token's slots in fp32, Y's own.
    held, sums: what takes the place of the down product's rows, and of that product, where a test plants a mistake."""
    ids, weights, offsets, token, row = route(logits, top_k, renormalize)
    t, d, ff, E = x.shape[0], x.shape[1], w_up.shape[2], len(offsets) - 1
    codes, scales = ref.quantize(x, pow2)
    y, bound = np.zeros((t, w_down.shape[1])), np.zeros((t, w_down.shape[1]))
    for e in range(E):
        rows = np.arange(offsets[e], offsets[e + 1])
        if not rows.size:
            continue
        tk = token[rows]
        g, gS, gG = ref.product(codes[tk], scales[tk], w_up[e, 0], s_up[e, 0])
        u, uS, uG = ref.product(codes[tk], scales[tk], w_up[e, 1], s_up[e, 1])
        silu = g / (1 + np.exp(-np.clip(g, -700, 700)))
        h = silu * u
        # silu's slope is at most 1.1; exp(-g) is off by |g| 2^-23 and its own 2^-22, the sum, the quotient and the product by 2^-23 in all
        dh = 1.1 * ref.slack(gS, gG, d, True) * np.abs(u) + np.abs(silu) * ref.slack(uS, uG, d, True) + (2.0 ** -21 + np.abs(g) * 2.0 ** -23) * np.abs(h)
        hq, hs = ref.quantize(h.astype(np.float32), pow2)
        v, blocks = ref.values(hq, hs, ff), hs.shape[1]

        def by_block(a):
            return np.pad(a, ((0, 0), (0, -ff % 128))).reshape(len(h), blocks, 128)
        # the scale of a block is off as its largest magnitude is; a power of two is not, unless that is near to 448 times one
        at = by_block(np.abs(h)).argmax(-1)[..., None]
        most = np.take_along_axis(by_block(np.abs(h)), at, -1)[..., 0]
        off = np.take_along_axis(by_block(dh), at, -1)[..., 0] / np.where(most > 0, most, 1.0) + 2.0 ** -22
        ratio = most / (448 * hs.astype(np.float64))
        other = hs.astype(np.float64)
        if pow2:  # there the scale may be the next power of two on the other side, and the codes those at that scale
            other = np.where((most > 0) & (ratio > 1 - 2 * off), 2 * other, np.where((most > 0) & (ratio < 0.5 * (1 + 2 * off)), other / 2, other))
            off = 0 * off
        off, sc, other = (np.repeat(a.astype(np.float64), 128, 1)[:, :ff] for a in (off, hs, other))
        margin = dh + np.abs(h) * (off + 2.0 ** -22)
        lo, hi, lo2, hi2 = (ref.values(ref.quantize_like(h + m * margin, c), np.ones((len(h), blocks)), ff) * c for c in (sc, other) for m in (-1, 1))
        step = np.max([np.abs(a - v) for a in (lo, hi, lo2, hi2)], 0) + off * np.abs(v)
        r, S, G = ref.product(hq, hs, w_down[e], s_down[e])
        if sums is not None:
            r = sums(hq, hs, w_down[e], s_down[e])
        if held is not None:
            r = held(r)
        dr = ref.slack(S, G, ff, not y_bf16) + step @ np.abs(ref.weight_values(w_down[e], s_down[e])).T + (2.0 ** -8 if y_bf16 else 2.0 ** -23) * np.abs(r)
        slot = np.argmax(row[tk] == rows[:, None], 1)
        wt = weights[tk, slot][:, None]
        np.add.at(y, tk, wt * r)
        np.add.at(bound, tk, wt * dr + wt * np.abs(r) * (weight_bound(E) + (top_k + 1) * 2.0 ** -23))
    return y, bound + (2.0 ** -8 if y_bf16 else 2.0 ** -23) * np.abs(y) + 1e-37


def cancelling(rng, ff, n):
    """(codes of a row's h, weights [n, ff]): in each group of 8 channels two products of 448 * 448 of opposite sign and six of 1 to 8 between
    them.  The matrix instructions for 8-bit operands lose all of the six; fp32 sums hold them."""
    h, w = np.zeros(ff, np.uint8), np.zeros((n, ff), np.uint8)
    code = {abs(v): c for c, v in enumerate(ref.E4M3[:127])}
    for c in range(0, ff - ff % 8, 8):
        place = rng.permutation(8) + c
        h[place[:2]] = code[448.0]
        w[:, place[0]], w[:, place[1]] = code[448.0], code[448.0] | 0x80
        for p in place[2:]:
            h[p] = code[float(rng.choice([1, 2, 4]))]
            w[:, p] = rng.choice([code[1.0], code[2.0]], n)
    return h, w


def eight_bit_sums(codes, scales, wcodes, wscales):
    """The product by sums that drop, of every 8 neighbouring channels, what lies 2^-13 and less below the largest."""
    v, w = ref.values(codes, scales, wcodes.shape[1]), ref.weight_values(wcodes, wscales)
    pad = -v.shape[1] % 8
    p = np.pad(v[:, None, :] * w[None], ((0, 0), (0, 0), (0, pad))).reshape(len(v), len(w), -1, 8)
    unit = np.abs(p).max(-1, keepdims=True) * 2.0 ** -13
    return np.where(unit > 0, np.trunc(p / np.where(unit > 0, unit, 1.0)) * unit, 0.0).sum((-1, -2))
