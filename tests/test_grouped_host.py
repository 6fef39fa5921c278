"""What the grouped products refuse, found on the host before any CUDA call (so this runs without a GPU; the addresses are never
dereferenced), and what they take as nothing to do."""
import pytest

import paper_2609_09095_b200 as oz

BASE = 0x7F0000000000


def grouped(transA=0, m=8, n=16, k=24, groups=2, offsets=BASE, dtype=oz.OZ_BF16, A=BASE + 4096, lda=None, strideA=1024, B=BASE + 8192, ldb=24,
            ctype=oz.OZ_BF16, beta=0.0, C=BASE + 16384, ldc=8):
    lda = (k if transA else m) if lda is None else lda
    return oz.oz_gemm_grouped(transA, m, n, k, groups, offsets, dtype, A, lda, strideA, B, ldb, ctype, beta, C, ldc, 0)


def wgrad(m=8, n=16, tokens=24, groups=2, offsets=BASE, dtype=oz.OZ_BF16, A=BASE + 4096, lda=8, B=BASE + 8192, ldb=16, ctype=oz.OZ_F32, beta=0.0,
          C=BASE + 16384, ldc=8, strideC=128):
    return oz.oz_gemm_grouped_wgrad(m, n, tokens, groups, offsets, dtype, A, lda, B, ldb, ctype, beta, C, ldc, strideC, 0)


@pytest.mark.parametrize("call", [grouped, wgrad])
def test_shared_refusals(call):
    for bad in (dict(m=-1), dict(n=-1), dict(groups=-1), dict(dtype=oz.OZ_F32), dict(dtype=7), dict(ctype=oz.OZ_F16), dict(ctype=9),
                dict(offsets=None), dict(offsets=BASE + 4), dict(A=None), dict(B=None), dict(C=None), dict(A=BASE + 1), dict(B=BASE + 1),
                dict(C=BASE + 1), dict(ctype=oz.OZ_F32, C=BASE + 2), dict(lda=7), dict(ldb=15), dict(ldc=7)):
        assert call(**bad) == oz.OZ_ERR_INVALID_ARG, bad
    for bad in (dict(beta=0.5), dict(beta=float("nan")), dict(groups=oz.OZ_GROUPS_MAX + 1)):
        assert call(**bad) == oz.OZ_ERR_UNSUPPORTED, bad
    big = oz.OZ_EXTENT_MAX + 1
    assert call(m=big, lda=big, ldc=big) == oz.OZ_ERR_UNSUPPORTED


def test_refusals_of_one():
    assert grouped(transA=2) == oz.OZ_ERR_INVALID_ARG
    assert grouped(k=-1) == oz.OZ_ERR_INVALID_ARG
    assert grouped(strideA=-8) == oz.OZ_ERR_INVALID_ARG
    assert grouped(transA=1, lda=23) == oz.OZ_ERR_INVALID_ARG
    assert grouped(ldb=23) == oz.OZ_ERR_INVALID_ARG
    assert wgrad(tokens=-1) == oz.OZ_ERR_INVALID_ARG
    assert wgrad(strideC=127) == oz.OZ_ERR_INVALID_ARG            # the groups' results would overlap
    assert wgrad(strideC=-128) == oz.OZ_ERR_INVALID_ARG


def test_nothing_to_do():
    assert grouped(m=0) == oz.OZ_OK
    assert grouped(n=0) == oz.OZ_OK
    assert grouped(groups=0) == oz.OZ_OK
    assert grouped(k=0, beta=1.0, A=None, B=None) == oz.OZ_OK
    assert wgrad(m=0) == oz.OZ_OK
    assert wgrad(n=0) == oz.OZ_OK
    assert wgrad(groups=0) == oz.OZ_OK
