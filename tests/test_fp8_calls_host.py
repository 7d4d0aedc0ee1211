"""Calls of the 8-bit floating point layers and the router at their limits, without a GPU."""
import os

import pytest

import paper_2510_26771_amd as st


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(st.lib_path()):
        from paper_2510_26771_amd.build import build
        build(verbose=False)
    return st.load_library()


@pytest.mark.parametrize("experts", [1, 20, 64, 255, 256, 257, 1000, 1024])
def test_a_router_workspace_serves_every_smaller_call(lib, experts):
    """Around every step of the tokens of a workgroup (64 or 16 at once, 256 workgroups at most), up to the largest call."""
    tokens = sorted({t for m in range(1, 40) for t in (4096 * m - 1, 4096 * m, 4096 * m + 1)} | {0, 1, 15, 16, 17, 63, 64, 65, (1 << 22) - 1, 1 << 22})
    sizes = [lib.stamp_route_workspace_bytes(t, experts, 4) for t in tokens]
    falls = [(tokens[i], sizes[i], tokens[i + 1], sizes[i + 1]) for i in range(len(tokens) - 1) if sizes[i + 1] < sizes[i]]
    assert not falls, f"{len(falls)} steps down, the first (tokens, bytes): {falls[0]}"
