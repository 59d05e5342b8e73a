"""Embedding gradient and attention refuse sizes whose launches have 2^32 lanes or more, which HIP does not launch (no GPU needed).

Every call here is refused before any HIP call: where the sizes are good, for its workspace.
"""
from test_abi_trunk_cpu import E_SHAPE, E_WS, L, _bwd, _embed_bwd, _fwd          # noqa: F401


def test_embedding_gradient(L):                                                  # noqa: F811
    size = L.agrl_token_embed_bwd_workspace_size
    # 8 rows to be cleared a workgroup of 256 lanes: 2^24 workgroups
    for T in (10, 5000):
        assert _embed_bwd(L, T=T, d=1, ldy=1, V=2 ** 27, acc=0, ws=None) == E_SHAPE
        assert _embed_bwd(L, T=T, d=1, ldy=1, V=2 ** 27 - 8 * T - 8, acc=0, ws=None) == E_WS
        assert _embed_bwd(L, T=T, d=1, ldy=1, V=2 ** 27, acc=1, ws=None) == E_WS
        assert size(T, 1, 2 ** 27) > 0
    # chunks of 32 tokens, 1024 columns a workgroup
    for T, d in ((2 ** 29, 1), (2 ** 29, 1024), (2 ** 28, 1025), (2 ** 19, 1 << 20)):
        assert size(T, d, 100) == 0
        assert _embed_bwd(L, T=T, d=d, ldy=d, acc=1, ws=None) == E_SHAPE
        assert size(T - 32, d, 100) > 0
        assert _embed_bwd(L, T=T - 32, d=d, ldy=d, acc=1, ws=None) == E_WS


def test_attention(L):                                                           # noqa: F811
    size = L.agrl_attention_bwd_workspace_size
    # 128 rows of a head a workgroup of 256 lanes
    for T, H in ((2 ** 27, 16), (2 ** 30, 2), (2 ** 24, 128)):
        assert size(T, H, 2, 64, 0) == 0
        assert _bwd(L, T=T, H=H, ws=None) == E_SHAPE and _fwd(L, T=T, H=H) == E_SHAPE
        assert size(T - 128, H, 2, 64, 0) > 0
        assert _bwd(L, T=T - 128, H=H, ws=None) == E_WS
