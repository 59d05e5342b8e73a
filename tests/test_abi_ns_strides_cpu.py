"""Which strides of a written stack the orthogonalisation calls take: those whose rows do not overlap."""
import pytest

from test_abi_newton_schulz_cpu import E_SHAPE, E_WS, L, _muon, _orth  # noqa: F401

# (batch, m, n, row stride, matrix stride): accepted or not
CASES = [
    (2, 8, 16, 16, 128, True), (2, 8, 16, 16, 127, False),           # matrix after matrix
    (2, 8, 16, 20, 156, True), (2, 8, 16, 20, 155, False),           # the last row ends with the matrix
    (3, 8, 16, 48, 16, True), (3, 8, 16, 47, 16, False),             # row after row: [m, batch, n] seen as a stack
    (3, 8, 16, 60, 20, True), (3, 8, 16, 48, 15, False), (3, 8, 16, 48, 17, False),
    (3, 1, 16, 16, 16, True), (3, 1, 16, 16, 15, False),             # one row each
    (2, 8, 16, 16, 0, False), (2, 8, 16, 16, -128, False),           # one matrix over itself; backwards
    (1, 8, 16, 16, 0, True), (1, 8, 16, 16, -5, True),               # a single matrix: not read
    (2, 8, 16, 1 << 61, 1 << 62, False),                             # 8 rows of 2^61 are not 2^64 mod 2^64 = 0 apart
]


@pytest.mark.parametrize("batch,m,n,ld,stride,ok", CASES)
def test_rows_that_overlap_are_refused(L, batch, m, n, ld, stride, ok):  # noqa: F811
    want = E_WS if ok else E_SHAPE        # (the workspace is looked at next)
    assert _orth(L, batch=batch, m=m, n=n, sg=m * n, ldo=ld, so=stride, ws=None) == want
    assert _muon(L, batch=batch, m=m, n=n, sg=m * n, ldp=ld, sp=stride, ws=None) == want
