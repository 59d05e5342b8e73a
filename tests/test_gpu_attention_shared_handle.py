"""One attention handle for several layers: the backward reads the o and lse that it is given."""
import pytest
import torch

from helpers import log
from test_gpu_attention import BF, F32, _make, _offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 33), (F32, 64)])
def test_layers_share_a_handle(dtype, d):
    import paper_2510_04206_amd as P
    T, H, G = 270, 4, 2
    log(f"attention shared handle {dtype} {d}")
    st = _offsets([0, 100, 260])
    layers = [[t.cuda() for t in _make(T, H, G, d, dtype, seed=s)] for s in range(3)]
    want = []
    for q, k, v, do in layers:
        own = P.PackedAttention(T, H, G, d, dtype)
        own.forward(q, k, v, st)
        want.append(torch.cat(own.backward(q, k, v, st, do), 1))
    op = P.PackedAttention(T, H, G, d, dtype)
    kept = [[t.clone() for t in op.forward(q, k, v, st)] for q, k, v, _ in layers]
    op.o.fill_(float("nan"))
    op.lse.fill_(float("nan"))
    # heads first in memory, as another layout of o
    kept = [(o.transpose(0, 1).contiguous().transpose(0, 1), lse) for o, lse in kept]
    for i in (2, 0, 1):
        q, k, v, do = layers[i]
        o, lse = kept[i]
        got = op.backward(q, k, v, st, do, o=o, lse=lse)
        assert torch.equal(torch.cat(got, 1), want[i])
