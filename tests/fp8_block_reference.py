"""A layer's epilogue, the dense MLP and the whole layer of experts in 64 bits, each with how far fp32 kernels may be from it."""
import math

import numpy as np

import fp8_calls_reference as calls
import fp8_reference as ref

ACTIVATIONS = ("none", "relu", "silu", "gelu", "gelu_tanh")
U = 2.0 ** -23  # two roundings of an fp32 operation, or one and a function's last place
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, relative

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def sigmoid(v):
    return 0.5 * (1 + np.tanh(0.5 * v))


def activation(z, name):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "silu":
        return z * sigmoid(z)
    if name == "gelu":
        return z * 0.5 * _erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return z * sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def activated(z, dz, name):
    """(act(z), bound) of an argument that is dz off.  No activation is steeper than 1.13.  Of its own an fp32 evaluation is off by
    |z| times at most 4 U: the logistic's slope times its argument is at most 0.23 (of gelu's Phi: its density times a, 0.25), so an argument's relative
    error of 3 U counts less than U (Phi's argument is a polynomial's value, which is as much off); the exponential, 1 + it, the reciprocal and the product U
    each at most, halved where they are single roundings."""
    return activation(z, name), 1.13 * dz + (0.0 if name in ("none", "relu") else 4 * U * np.abs(z))


def finish(v, dv, residual, y):
    """(v + residual, bound) after the sum's and Y's rounding."""
    r = 0.0 if residual is None else residual
    want = v + r
    return want, dv + U * (np.abs(v) + np.abs(r)) + HALF[y] * (np.abs(want) + dv) * (1 + 2.0 ** -7) + 1e-37


def layer(x, w, ws, bias, act, residual, y, pow2, wide):
    """(Y, bound) of act(Q8(x) w + bias) + residual."""
    codes, scales = ref.quantize(x, pow2)
    z, S, G = ref.product(codes, scales, w, ws)
    dz = ref.slack(S, G, x.shape[1], wide)
    if bias is not None:
        z = z + bias
        dz = dz + U * (np.abs(z) + np.abs(bias))
    return finish(*activated(z, dz, act), residual, y)


def coded(h, dh, pow2):
    """Codes and scales of h, and by how much the values they stand for move when h is dh off: a code may be its neighbour, a block's scale
    follows its largest magnitude, a power of two may be the next one where the largest magnitude is near to 448 times one."""
    ff = h.shape[1]
    codes, scales = ref.quantize(h.astype(np.float32), pow2)
    blocks = scales.shape[1]
    v = ref.values(codes, scales, ff)

    def by_block(a):
        return np.pad(a, ((0, 0), (0, -ff % 128))).reshape(len(h), blocks, 128)
    most = by_block(np.abs(h)).max(-1)
    # the largest magnitude moves by at most the largest of all errors among those near to it
    near = by_block(np.abs(h)) + 2 * by_block(dh) >= most[..., None]
    off = np.where(near, by_block(dh), 0.0).max(-1) / np.where(most > 0, most, 1.0) + 2.0 ** -22
    ratio = most / (448 * scales.astype(np.float64))
    other = scales.astype(np.float64)
    if pow2:
        other = np.where((most > 0) & (ratio > 1 - 2 * off), 2 * other, np.where((most > 0) & (ratio < 0.5 * (1 + 2 * off)), other / 2, other))
        off = 0 * off
    off, sc, other = (np.repeat(a.astype(np.float64), 128, 1)[:, :ff] for a in (off, scales, other))
    margin = dh + np.abs(h) * (off + 2.0 ** -22)
    ends = [ref.values(ref.quantize_like(h + m * margin, c), np.ones((len(h), blocks)), ff) * c for c in (sc, other) for m in (-1, 1)]
    return codes, scales, np.max([np.abs(a - v) for a in ends], 0) + off * np.abs(v)


def hidden(codes, scales, w, ws, bias, act):
    """(h, bound) of an up product: w [ff, d] and bias, or gate and up matrices [2, ff, d]."""
    d = w.shape[-1]
    if w.ndim == 3:
        g, gS, gG = ref.product(codes, scales, w[0], ws[0])
        u, uS, uG = ref.product(codes, scales, w[1], ws[1])
        a, da = activated(g, ref.slack(gS, gG, d, True), act)
        du = ref.slack(uS, uG, d, True)
        return a * u, da * (np.abs(u) + du) + np.abs(a) * du + U * np.abs(a * u)
    z, S, G = ref.product(codes, scales, w, ws)
    dz = ref.slack(S, G, d, True)
    if bias is not None:
        z = z + bias
        dz = dz + U * (np.abs(z) + np.abs(bias))
    return activated(z, dz, act)


def mlp(x, w_up, s_up, b_up, w_down, s_down, b_down, act, residual, y, pow2):
    codes, scales = ref.quantize(x, pow2)
    h, dh = hidden(codes, scales, w_up, s_up, b_up, act)
    hq, hs, step = coded(h, dh, pow2)
    r, S, G = ref.product(hq, hs, w_down, s_down)
    dr = ref.slack(S, G, h.shape[1], y == "f32") + step @ np.abs(ref.weight_values(w_down, s_down)).T
    if b_down is not None:
        r = r + b_down
        dr = dr + U * (np.abs(r) + np.abs(b_down))
    return finish(r, dr, residual, y)


def logits(x, router, bias):
    """Router logits rounded to fp32 once, and a bound of their error before that: blocks of 32 channels in fp32, eight instructions of
    4 products one after the other: at most 4 + 8 roundings on a product's way, each U / 2 of the block's magnitudes."""
    l = x.astype(np.float64) @ router.astype(np.float64).T
    err = 12 * U / 2 * (np.abs(x.astype(np.float64)) @ np.abs(router.astype(np.float64)).T)
    if bias is not None:
        l = l + bias
    return l.astype(np.float32), err


def clear(l, err, top_k):
    """No two of a token's top_k + 1 largest logits are so near that their errors decide."""
    order = np.argsort(-l, axis=1, kind="stable")[:, :top_k + 1]
    v, e = np.take_along_axis(l.astype(np.float64), order, 1), np.take_along_axis(err, order, 1)
    finite = np.isfinite(v[:, 1:])
    with np.errstate(invalid="ignore"):
        gap = v[:, :-1] - v[:, 1:]
    return bool(np.all(~finite | (gap > e[:, :-1] + e[:, 1:] + 2 * U * np.abs(np.nan_to_num(v[:, :-1], neginf=0.0)))))


def moe(x, router, router_bias, w_up, s_up, w_down, s_down, b_down, top_k, renormalize, act, residual, y, pow2):
    """(Y, bound, ids, weights, offsets, token_of_row, row_of_slot, relative bound of a token's weights); the router's choice has to be `clear`."""
    l, err = logits(x, router, router_bias)
    assert clear(l, err, top_k), "inputs whose routing a rounding decides"
    ids, weights, offsets, token, row = calls.route(l, top_k, renormalize)
    E = len(offsets) - 1
    codes, scales = ref.quantize(x, pow2)
    out, bound = np.zeros((len(x), w_down.shape[1])), np.zeros((len(x), w_down.shape[1]))
    # a weight moves with its logits: relative error of exp of a difference
    ok = np.isfinite(l)
    dw = np.exp(2 * (np.where(ok, err, 0.0) + U * np.abs(np.where(ok, l, 0.0))).max(1, keepdims=True)) - 1 + calls.weight_bound(E)
    for e in range(E):
        rows = np.arange(offsets[e], offsets[e + 1])
        if not rows.size:
            continue
        tk = token[rows]
        h, dh = hidden(codes[tk], scales[tk], w_up[e], s_up[e], None, act)
        hq, hs, step = coded(h, dh, pow2)
        r, S, G = ref.product(hq, hs, w_down[e], s_down[e])
        dr = ref.slack(S, G, h.shape[1], y == "f32") + step @ np.abs(ref.weight_values(w_down[e], s_down[e])).T
        if b_down is not None:
            r = r + b_down[e]
            dr = dr + U * (np.abs(r) + np.abs(b_down[e]))
        wt = weights[tk, np.argmax(row[tk] == rows[:, None], 1)][:, None]
        np.add.at(out, tk, wt * r)
        # S: the terms' magnitudes; sums over a token's experts in any order, at most top_k + 16 of them
        np.add.at(bound, tk, wt * dr * (1 + dw[tk]) + wt * (S + np.abs(r)) * (dw[tk] + (top_k + 18) * U))
    want, tol = finish(out, bound, residual, y)
    return want, tol, ids, weights, offsets, token, row, dw
