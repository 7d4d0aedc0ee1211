"""The 8-bit floating point layers, the router and the experts' MLP in plain numpy: codes and scales in the individually rounded fp32
operations that define them, everything else in 64 bits."""
import numpy as np

BLOCK = 128
E4M3 = np.array([(-1.0 if c & 0x80 else 1.0) * ((c & 7) / 512.0 if (c >> 3 & 15) == 0 else (8 + (c & 7)) / 8.0 * 2.0 ** ((c >> 3 & 15) - 7))
                 for c in range(256)])
E4M3[[0x7F, 0xFF]] = np.nan
SMALLEST = np.float32(1.75 * 2.0 ** -118)


def encode(v):
    """fp32 -> E4M3 codes, nearest, ties to the even code; magnitudes up to 464 (beyond: not needed)."""
    v = np.asarray(v, np.float32)
    mag = np.abs(v.astype(np.float64))
    pos = E4M3[:127]
    i = np.clip(np.searchsorted(pos, mag), 1, 126)
    lo, hi = pos[i - 1], pos[i]
    down = (mag - lo < hi - mag) | ((mag - lo == hi - mag) & ((i - 1) % 2 == 0))
    code = np.where(down, i - 1, i).astype(np.uint8)
    code = np.where(np.signbit(v), code | 0x80, code)
    return np.where(np.isnan(v), 0x7F, code).astype(np.uint8)


def scale_of(amax, pow2):
    """fp32 (scale, multiplier) of blocks from their largest magnitudes."""
    a = np.maximum(np.asarray(amax, np.float32), SMALLEST)
    bad = ~np.isfinite(a)
    a = np.where(bad, np.float32(1), a).astype(np.float32)
    if pow2:
        m, e = np.frexp(a.astype(np.float64))  # m in [0.5, 1), 448 = 0.875 * 2^9
        e = e - 9 + (m > 0.875)
        scale, inv = np.ldexp(1.0, e).astype(np.float32), np.ldexp(1.0, -e).astype(np.float32)
    else:
        scale, inv = a / np.float32(448), np.float32(448) / a
    return np.where(bad, np.float32(np.nan), scale), np.where(bad, np.float32(np.nan), inv)


def quantize(x, pow2):
    """x [rows, d] fp32 -> codes [rows, Kp] and scales [rows, blocks] fp32."""
    x = np.asarray(x, np.float32)
    rows, d = x.shape
    kp = -(-d // BLOCK) * BLOCK
    p = np.zeros((rows, kp), np.float32)
    p[:, :d] = x
    p = p.reshape(rows, -1, BLOCK)
    amax = np.where(np.isnan(p).any(-1), np.float32(np.nan), np.abs(np.nan_to_num(p, nan=0.0, posinf=np.inf, neginf=-np.inf)).max(-1))
    amax = np.where(np.isnan(amax), np.inf, amax)
    scale, inv = scale_of(amax, pow2)
    with np.errstate(invalid="ignore", over="ignore"):
        codes = encode(p * inv[..., None])
    return codes.reshape(rows, kp), scale


def quantize_weights(w, pow2):
    """w [d_out, d_in] fp32 -> codes, scales [blocks of d_out, blocks of d_in]."""
    n, d = w.shape
    nb, kb = -(-n // BLOCK), -(-d // BLOCK)
    p = np.zeros((nb * BLOCK, kb * BLOCK), np.float32)
    p[:n, :d] = w
    p = p.reshape(nb, BLOCK, kb, BLOCK)
    scale, inv = scale_of(np.abs(p).max((1, 3)), pow2)
    codes = encode(p * inv[:, None, :, None])
    return codes.reshape(nb * BLOCK, kb * BLOCK)[:n, :d], scale


def values(codes, scales, d):
    """What codes [rows, Kp] and scales [rows, blocks] stand for, in 64 bits."""
    v = E4M3[codes].reshape(codes.shape[0], -1, BLOCK) * scales.astype(np.float64)[..., None]
    return v.reshape(codes.shape[0], -1)[:, :d]


def weight_values(codes, scales):
    n, d = codes.shape
    return E4M3[codes] * np.repeat(np.repeat(scales.astype(np.float64), BLOCK, 0)[:n], BLOCK, 1)[:, :d]


def product(codes, scales, wcodes, wscales):
    """(Y, S, G) in 64 bits: the product, the sum of its terms' magnitudes, and the sum over groups of 8 channels of the largest term's
    bound (largest factor of either side)."""
    d = wcodes.shape[1]
    x, w = values(codes, scales, d), weight_values(wcodes, wscales)
    pad = -d % 8
    gx = np.abs(np.pad(x, ((0, 0), (0, pad)))).reshape(x.shape[0], -1, 8).max(-1)
    gw = np.abs(np.pad(w, ((0, 0), (0, pad)))).reshape(w.shape[0], -1, 8).max(-1)
    return x @ w.T, np.abs(x) @ np.abs(w).T, gx @ gw.T


def slack(S, G, d_in, wide):
    """How far a kernel's fp32 sums may be from the product.  Wide sums: every one of the d_in / 32 + d_in / 128 + 16 roundings on a
    value's way (within an instruction, over the blocks and parts of the depth, the two scales) is at most 2^-23 of the terms'
    magnitudes.  FP8 instructions: each of a group's 8 products loses at most 2^-13 of the largest one as well."""
    s = (d_in / 32 + d_in / 128 + 16) * 2.0 ** -23 * S
    return s if wide else s + 8 * 2.0 ** -13 * G


def route(logits, top_k, renormalize):
    """ids, weights (64 bits), offsets, token_of_row, row_of_slot."""
    l = np.asarray(logits, np.float64)
    t, e = l.shape
    ids, weights = np.full((t, top_k), -1, np.int32), np.zeros((t, top_k))
    for i in range(t):
        open_ = [j for j in range(e) if l[i, j] > -np.inf]
        chosen = sorted(open_, key=lambda j: (-l[i, j], j))[:top_k]
        if not chosen:
            continue
        top = l[i, chosen[0]]

        def share(v):
            return 1.0 if v == top else (0.0 if top == np.inf else np.exp(v - top))
        total = sum(share(l[i, j]) for j in (chosen if renormalize else open_))
        ids[i, :len(chosen)] = chosen
        weights[i, :len(chosen)] = [share(l[i, j]) / total for j in chosen]
    flat = ids.reshape(-1)
    order = [s for x in range(e) for s in np.flatnonzero(flat == x)]
    row = np.full(t * top_k, -1, np.int32)
    token = np.full(t * top_k, -1, np.int32)
    for r, s in enumerate(order):
        row[s], token[r] = r, s // top_k
    offsets = np.concatenate([[0], np.cumsum([np.count_nonzero(flat == x) for x in range(e)])]).astype(np.int32)
    return ids, weights, offsets, token, row.reshape(t, top_k)


def quantize_like(x, scale):
    """Codes of x (64 bits) at given scales, element by element; beyond the largest code: that one.  Columns are padded to whole blocks."""
    with np.errstate(divide="ignore", invalid="ignore"):
        v = np.clip(np.asarray(x / scale), -448, 448).astype(np.float32)
    c = encode(v)
    return np.pad(c, ((0, 0), (0, -c.shape[1] % BLOCK)))
