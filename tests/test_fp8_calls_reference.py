"""The references of the GPU tests: against one another, and that their bounds see the mistakes that they are there for."""
import numpy as np
import pytest

import fp8_calls_reference as calls
import fp8_reference as ref


def _logits(rng, tokens, experts, kind):
    l = rng.standard_normal((tokens, experts)).astype(np.float32)
    if kind == "masked":
        l[rng.random(l.shape) < 0.7], l[rng.random(l.shape) < 0.1], l[0] = -np.inf, np.nan, -np.inf
    if kind == "ties":
        l = rng.integers(-1, 2, l.shape).astype(np.float32) * np.float32(-1)
    if kind == "extreme":
        l[rng.random(l.shape) < 0.3], l[tokens // 2, : experts // 2 + 1] = np.float32(np.finfo(np.float32).min), np.inf
    return l


@pytest.mark.parametrize("kind", ["plain", "masked", "ties", "extreme"])
@pytest.mark.parametrize("renormalize", [0, 1])
@pytest.mark.parametrize("tokens,experts,top_k", [(1, 1, 1), (3, 5, 8), (40, 33, 17), (64, 20, 2)])
def test_the_two_routers_agree(tokens, experts, top_k, renormalize, kind):
    l = _logits(np.random.default_rng(tokens), tokens, experts, kind)
    a, b = ref.route(l, top_k, renormalize), calls.route(l, top_k, renormalize)
    for i in (0, 2, 3, 4):
        assert np.array_equal(a[i], b[i])
    assert np.allclose(a[1], b[1], rtol=1e-12, atol=0)


def _bf16(v):
    import torch
    return torch.from_numpy(v).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("pow2", [0, 1])
def test_the_bound_of_an_fp32_result_sees_rows_held_in_bf16(pow2):
    rng = np.random.default_rng(pow2)
    t, E, k, d, ff = 40, 3, 2, 150, 270
    x = rng.standard_normal((t, d)).astype(np.float32)
    w_up, w_down = (ref.encode(rng.standard_normal(s).astype(np.float32) * 40) for s in ((E, 2, ff, d), (E, d, ff)))
    s_up, s_down = np.full((E, 2, 3, 2), 2.0 ** -9, np.float32), np.full((E, 2, 3), 2.0 ** -9, np.float32)
    l = rng.standard_normal((t, E)).astype(np.float32)
    y, bound = calls.experts(x, l, w_up, s_up, w_down, s_down, k, 1, pow2, False)
    wrong, _ = calls.experts(x, l, w_up, s_up, w_down, s_down, k, 1, pow2, False, held=_bf16)
    assert (np.abs(wrong - y) > bound).any()  # one element beyond it fails a test
    loose = calls.experts(x, l, w_up, s_up, w_down, s_down, k, 1, pow2, True)[1]
    assert not (np.abs(wrong - y) > loose).any()


@pytest.mark.parametrize("ff", [128, 256, 520])
def test_the_bound_of_an_fp32_result_sees_sums_of_8_bit_instructions(ff):
    rng = np.random.default_rng(ff)
    h, w = calls.cancelling(rng, ff, 60)
    hq, hs = np.zeros((1, -(-ff // 128) * 128), np.uint8), np.ones((1, -(-ff // 128)), np.float32)
    hq[0, :ff] = h
    ws = np.ones((1, hs.shape[1]), np.float32)
    y, S, G = ref.product(hq, hs, w, ws)
    wrong = calls.eight_bit_sums(hq, hs, w, ws)
    assert (np.abs(wrong - y) > ref.slack(S, G, ff, True)).all()
    assert not (np.abs(wrong - y) > ref.slack(S, G, ff, False)).any()
