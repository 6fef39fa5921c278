"""What oz_orthogonalise refuses, found on the host before any CUDA call (the addresses are never dereferenced), and the size of its workspace."""
import math

import paper_2609_09095_b200 as oz

BASE = 0x7F0000000000
USUAL = (3.4445, -4.7750, 2.0315)


def call(m=8, n=16, count=2, dtype=oz.OZ_BF16, G=BASE, ldg=8, strideG=128, steps=5, coefficients=USUAL, eps=1e-7, otype=oz.OZ_F32, O=BASE + 4096, ldo=8,
         strideO=128, workspace=BASE + 8192, nbytes=1 << 30):
    return oz.oz_orthogonalise(m, n, count, dtype, G, ldg, strideG, steps, coefficients, eps, otype, O, ldo, strideO, workspace, nbytes, 0)


def test_refusals():
    for bad in (dict(m=-1), dict(n=-1), dict(count=-1), dict(steps=-1), dict(dtype=3), dict(otype=-1), dict(coefficients=None), dict(eps=-1.0),
                dict(eps=math.nan), dict(eps=math.inf), dict(G=None), dict(O=None), dict(G=BASE + 1), dict(O=BASE + 2), dict(ldg=7), dict(ldo=7),
                dict(strideG=-1), dict(strideO=127), dict(workspace=BASE + 8192 + 128), dict(coefficients=(math.nan, 0, 0)), dict(coefficients=(1, math.inf, 0))):
        assert call(**bad) == oz.OZ_ERR_INVALID_ARG, bad
    # singular values that leave the range of the planes on the way: 2^31 after a step, 10^5 after five, 0
    for bad in (dict(steps=101), dict(coefficients=(2.0 ** 31, 0, 0), steps=1), dict(coefficients=(100.0, 0, 0)), dict(coefficients=(0, 0, 0)),
                dict(coefficients=(3.0, 3.0, 3.0)), dict(m=1 << 20, n=1 << 20, ldg=1 << 20, ldo=1 << 20), dict(m=oz.OZ_EXTENT_MAX + 1, n=1, ldg=1 << 31, ldo=1 << 31)):
        assert call(**bad) == oz.OZ_ERR_UNSUPPORTED, bad
    assert call(workspace=None) == oz.OZ_ERR_WORKSPACE
    assert call(nbytes=oz.oz_orthogonalise_workspace_bytes(8, 16, 2) - 1) == oz.OZ_ERR_WORKSPACE


def test_nothing_to_do():
    for none in (dict(m=0), dict(n=0), dict(count=0)):
        assert call(workspace=None, G=None, O=None, **none) == oz.OZ_OK


def test_workspace():
    need = oz.oz_orthogonalise_workspace_bytes
    assert need(0, 5, 1) == need(5, 0, 1) == need(5, 5, 0) == need(-1, 5, 1) == 0
    assert need(1 << 20, 1 << 20, 1) == 0
    assert need(300, 700, 2) == need(700, 300, 2)
    # two copies of X, S and P, two 16-bit planes each
    assert 0 <= need(4096, 4096, 1) - 16 * 4096 * 4096 < 2048
    assert need(1000, 2000, 3) >= 3 * 8 * (1000 * 2000 + 1000 * 1000)
