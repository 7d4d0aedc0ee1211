"""The two kernels of the layer of experts for few tokens where they can go wrong: waits that give up."""
import numpy as np
import pytest

from test_gpu_fp8 import _dt
from test_gpu_fp8_block import _moe_case, st  # noqa: F401  (fixture)

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

