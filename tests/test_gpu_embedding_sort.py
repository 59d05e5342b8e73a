"""The embedding's gradient where its launches change: chunks of 32 sorted tokens, several batches of a wave's tokens, whole batches
without a mask, ids out of range among them.  Bounds as in test_gpu_embedding."""
import numpy as np
import pytest
import torch

from helpers import log
from test_gpu_embedding import BF, F32, U, _grad, _ids

pytestmark = pytest.mark.gpu


def _chunk(T, d, V):
    """Sorted tokens per chunk, from what the workspace holds: [T] (token, id), [V + 1] starts, a list of chunks, two sums of
    d a chunk; the first three rounded up to 256 bytes each."""
    import paper_2510_04206_amd as P
    up = lambda n: (n + 255) // 256 * 256                                          # noqa: E731
    size = P.agrl_token_embed_bwd_workspace_size(T, d, V)
    for chunk in (8, 32):
        n = -(-T // chunk)
        if size == up(8 * T) + up(4 * (V + 1)) + up(4 * (n + 1)) + 8 * n * d:
            return chunk
    raise AssertionError("the workspace is laid out in another way")


# tokens: past a batch of 64 x 16 a wave (16384 in all) the ids are read twice; whole batches without a mask have a loop
# of their own; rows: ceil(T / 32) ceil(d / 1024) >= 1024 makes chunks of 32
@pytest.mark.parametrize("T,d,V,chunk", [(8200, 5120, 300, 32), (32760, 64, 3000, 32), (33000, 1030, 40, 32),
                                         (16384, 65, 700, 8), (16449, 64, 700, 8), (20000, 96, 152064, 8),
                                         (40000, 40, 5, 32), (66000, 33, 1000, 32)])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("mask", ["none", "some"])
def test_gradient(T, d, V, chunk, accumulate, mask):
    assert _chunk(T, d, V) == chunk
    _grad(T, d, V, BF if d % 2 else F32, mask=mask, accumulate=accumulate, pitch=d % 3, scale=1.0 if d % 2 else d ** 0.5)


@pytest.mark.parametrize("kind", ["same", "all"])
@pytest.mark.parametrize("T,d,chunk", [(34000, 96, 32), (5000, 7000, 32), (17000, 48, 8)])
def test_gradient_runs(kind, T, d, chunk):
    """One id over all chunks (more pieces than four waves take at once), and ids that come back after 513 others."""
    assert _chunk(T, d, 513) == chunk
    _grad(T, d, 513, F32, kind=kind)
    _grad(T, d, 513, BF, kind=kind, accumulate=True, pitch=5)


@pytest.mark.parametrize("T,d", [(1000, 40), (20000, 64), (40000, 48)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_ids_out_of_range(T, d, accumulate):
    """In the sort: within a whole batch, in a wave's last one and in the last token; and one beside dead tokens."""
    import paper_2510_04206_amd as P
    V = 600
    dy = torch.randn(T, d, device="cuda")
    before = torch.randn(V, d, device="cuda")
    for bad in (-1, V, 2 ** 31 - 1, -2 ** 31):
        for at in (70, T // 2 + 3, T - 1):
            log(f"embed sort T={T} id {bad} at {at}")
            ids = _ids(T, V)
            ids[at] = bad
            op = P.TokenEmbedding(T, V, d, F32)
            op.dweight.copy_(before)
            got = op.backward(ids.cuda(), dy, accumulate=accumulate).clone()
            assert P.agrl_get_device_error() == 1
            mask = torch.ones(T, dtype=torch.uint8)
            mask[at] = 0
            op.dweight.copy_(before)
            assert torch.equal(got, op.backward(ids.cuda(), dy, mask.cuda(), accumulate=accumulate))
            assert P.agrl_get_device_error() == 0


@pytest.mark.parametrize("T,d,chunk", [(3000, 64, 8), (33000, 64, 32)])
def test_nan_stays_in_its_row(T, d, chunk):
    import paper_2510_04206_amd as P
    V = 90
    assert _chunk(T, d, V) == chunk
    ids, dy = _ids(T, V).cuda(), torch.randn(T, d, device="cuda")
    op = P.TokenEmbedding(T, V, d, F32)
    want = op.backward(ids, dy).clone()
    for at in (100, T - 2):
        hurt = dy.clone()
        hurt[at] = float("nan")
        got = op.backward(ids, hurt)
        hit = int(ids[at])
        keep = [v for v in range(V) if v != hit]
        assert torch.isnan(got[hit]).all() and torch.equal(got[keep], want[keep])


def test_repeats_and_replays():
    """Chunks of 32 and two reads of the ids: the bits do not change from call to call, nor in a graph."""
    import paper_2510_04206_amd as P
    T, V, d = 34000, 500, 96
    log("embed sort graph")
    assert _chunk(T, d, V) == 32
    ids, dy = _ids(T, V).cuda(), torch.randn(T, d, device="cuda").to(BF)
    op, eager = P.TokenEmbedding(T, V, d, BF), P.TokenEmbedding(T, V, d, BF)
    a = op.backward(ids, dy).clone()
    assert torch.equal(a, op.backward(ids, dy))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.backward(ids, dy)
    for seed in range(4):
        ids.copy_(_ids(T, V, seed))
        dy.copy_(torch.randn(T, d, device="cuda"))
        graph.replay()
        eager.backward(ids, dy)
        torch.cuda.synchronize()
        assert torch.equal(op.dweight, eager.dweight)


@pytest.mark.parametrize("T", [255, 256, 257, 511, 512, 513])
@pytest.mark.parametrize("kind", ["same", "all", "text"])
def test_around_the_one_launch(T, kind):
    """Up to 256 tokens go without the sort."""
    _grad(T, 300, 700, F32, kind=kind, mask="some")
    _grad(T, 1025, 90, BF, kind=kind, accumulate=True, pitch=5)
