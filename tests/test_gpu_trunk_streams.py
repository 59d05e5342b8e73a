"""Handles of embedding, rotation and attention called from several streams; heads first in memory for the rotation."""
import pytest
import torch

from helpers import log
from test_gpu_attention import BF, F32, _make, _offsets
from test_gpu_handle_streams import WAIT, _both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [300, 3000])
def test_embedding(T):
    import paper_2510_04206_amd as P
    log(f"embedding on alternating streams T={T}")
    V, d = 700, 130
    g = torch.Generator().manual_seed(T)
    op = P.TokenEmbedding(T, V, d, BF)
    w = torch.randn(V, d, generator=g).to(BF).cuda()
    xs = [(torch.randint(0, V, (T,), generator=g).to(torch.int32).cuda(), torch.randn(T, d, generator=g).cuda())
          for _ in range(2)]

    def call(x, s):
        op.forward(w, x[0], stream=s)
        op.backward(x[0], x[1], stream=s)
    _both(call, [op.y, op.dweight], xs)


@pytest.mark.parametrize("inter", [False, True])
def test_rotation(inter):
    import paper_2510_04206_amd as P
    log(f"rotation on alternating streams {inter}")
    T, H, d = 500, 6, 64
    op = P.TokenRotation(T, H, d, F32, interleaved=inter)
    g = torch.Generator().manual_seed(1)
    xs = [torch.randn(T, H, d, generator=g).cuda() for _ in range(2)]
    _both(lambda x, s: op(x, stream=s), [op.out], xs)


@pytest.mark.parametrize("dtype,d,T", [(BF, 128, 900), (BF, 50, 200), (F32, 64, 500)])
def test_attention(dtype, d, T):
    import paper_2510_04206_amd as P
    log(f"attention on alternating streams {dtype} {d} {T}")
    op, st = P.PackedAttention(T, 4, 2, d, dtype), _offsets([0, T // 3, T - 5])
    xs = [[t.cuda() for t in _make(T, 4, 2, d, dtype, seed=s)] for s in range(2)]

    def call(x, s):
        op.forward(*x[:3], st, stream=s)
        op.backward(*x[:3], st, x[3], stream=s)
    _both(call, [op.o, op.lse, op.dqkv], xs)
    # a forward on one stream and its backward on another
    call(xs[0], None)
    want = op.dqkv.clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(WAIT)
    op.forward(*xs[0][:3], st, stream=s)
    op.backward(*xs[0][:3], st, xs[0][3])
    assert torch.equal(op.dqkv, want)


@pytest.mark.parametrize("d,rot", [(64, 64), (34, 20), (128, 64)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rotation_of_heads_first_in_memory(d, rot, inter, dtype):
    """The same bits as of tokens first, into either layout and in place."""
    import paper_2510_04206_amd as P
    T, H = 210, 5
    log(f"rotation heads first d={d} rot={rot} {inter} {dtype}")
    x = torch.randn(T, H, d, generator=torch.Generator().manual_seed(d)).to(dtype).cuda()
    pos = (torch.arange(T, dtype=torch.int32) * 37 % 1000).cuda()
    op = P.TokenRotation(T, H, d, dtype, rot=rot, interleaved=inter)
    want = op(x, pos).clone()
    y = x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(op(y, pos), want)
    z = torch.empty_like(y)
    assert z.stride() == y.stride() and torch.equal(op(x, pos, out=z), want)
    assert torch.equal(op(y, pos, out=y), want)
    back = op(want, pos, inverse=True).clone()
    assert torch.equal(op(y, pos, inverse=True), back)
