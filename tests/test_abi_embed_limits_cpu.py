"""The embedding's gradient near the largest V: ids are counted in 32 bits, with a workgroup's range on top (no GPU needed).

Every call here is refused before any HIP call: where the sizes are good, for its workspace.
"""
import pytest

from test_abi_trunk_cpu import E_SHAPE, E_WS, L, _embed_bwd, _embed_fwd          # noqa: F401

TOP = 2 ** 31 - 1024


@pytest.mark.parametrize("V", [TOP + 1, TOP + 512, 2 ** 31 - 9, 2 ** 31 - 2, 2 ** 31 - 1])
@pytest.mark.parametrize("T", [10, 5000])
@pytest.mark.parametrize("acc", [0, 1])
def test_ids_that_leave_32_bits_are_refused(L, V, T, acc):                       # noqa: F811
    assert L.agrl_token_embed_bwd_workspace_size(T, 1, V) == 0
    assert _embed_bwd(L, T=T, d=1, ldy=1, V=V, acc=acc, ws=None) == E_SHAPE


@pytest.mark.parametrize("T", [10, 5000])
def test_the_largest_is_taken(L, T):                                             # noqa: F811
    assert L.agrl_token_embed_bwd_workspace_size(T, 1, TOP) >= 4 * (TOP + 1) + 8 * T
    assert _embed_bwd(L, T=T, d=1, ldy=1, V=TOP, acc=1, ws=None) == E_WS


def test_the_forward_counts_no_ids(L):                                           # noqa: F811
    assert _embed_fwd(L, T=0, V=2 ** 31 - 2) == 0 and _embed_fwd(L, V=2 ** 31 - 1) == E_SHAPE
