"""One handle called from several streams: each call's outputs are those of its own inputs."""
import pytest
import torch

from helpers import log

pytestmark = pytest.mark.gpu
WAIT = 20_000_000        # cycles of a stream that is behind


def _both(call, outputs, xs, rounds=4):
    """call(x, stream) in turn on the current stream, behind it on a side stream that is late, and
    back; the outputs copied on the stream of the call."""
    want = []
    for x in xs:
        call(x, None)
        want.append([t.clone() for t in outputs])
    torch.cuda.synchronize()
    late, other = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for k in range(rounds):
        for i, s in enumerate((late, None, other)):
            use = s if s is not None else torch.cuda.current_stream()
            if s is late:
                with torch.cuda.stream(s):
                    torch.cuda._sleep(WAIT)
            call(xs[(k + i) % len(xs)], s)
            with torch.cuda.stream(use):
                got.append((s, (k + i) % len(xs), [t.clone() for t in outputs]))
    torch.cuda.synchronize()
    for s, i, ts in got:
        for a, b in zip(ts, want[i]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("m,n", [(40, 90), (300, 500)])
def test_orthogonalize(m, n):
    import paper_2510_04206_amd as P
    log(f"orthogonalize {m} x {n} on alternating streams")
    op = P.Orthogonalize(m, n)
    g = torch.Generator().manual_seed(m)
    xs = [torch.randn(m, n, generator=g).cuda() for _ in range(2)]
    _both(lambda x, s: op(x, stream=s), [op.out], xs)


def test_norm_forward_and_backward():
    import paper_2510_04206_amd as P
    log("norm on alternating streams")
    T, d = 1500, 700
    op = P.TokenNorm(T, d, torch.bfloat16)
    g = torch.Generator().manual_seed(3)
    xs = [torch.randn(T, d, generator=g).bfloat16().cuda() for _ in range(2)]
    w, b, dy = (torch.randn(*n, generator=g).cuda() for n in ((d,), (d,), (T, d)))

    def call(x, s):
        op.forward(x, w, b, stream=s)
        op.backward(x, w, dy, stream=s)
    _both(call, [op.y, op.mean, op.rstd, op.dx, op.dweight, op.dbias], xs)
    # a forward on one stream and its backward on another
    op.forward(xs[0], w, b)
    op.backward(xs[0], w, dy)
    want = [op.dx.clone(), op.dweight.clone()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(WAIT)
    op.forward(xs[0], w, b, stream=s)
    op.backward(xs[0], w, dy)
    assert torch.equal(op.dx, want[0]) and torch.equal(op.dweight, want[1])


def test_muon_steps_follow_each_other():
    """Steps of two weights by one handle, the second's on another stream."""
    import paper_2510_04206_amd as P
    log("muon on alternating streams")
    g = torch.Generator().manual_seed(5)
    ws, gs = ([torch.randn(300, 200, generator=g).cuda() for _ in range(2)] for _ in range(2))
    def steps(op, streams):
        p, b = [w.clone() for w in ws], [torch.zeros_like(w) for w in ws]
        torch.cuda.synchronize()
        for k in range(4):
            for i in range(2):
                if streams[i] is not None and k % 2 == 0:
                    with torch.cuda.stream(streams[i]):
                        torch.cuda._sleep(WAIT)
                op(p[i], gs[i], b[i], 0.1, stream=streams[i])
        torch.cuda.synchronize()
        return p + b
    op = P.MuonStep(300, 200)
    want = steps(op, [None, None])
    got = steps(op, [torch.cuda.Stream(), None])
    for a, c in zip(got, want):
        assert torch.equal(a, c)
