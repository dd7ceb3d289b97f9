"""The calls between a block's linears reject bad arguments on the host, before anything is launched.  Runs without a GPU."""
import os

import pytest

from paper_2402_02446_amd import binding

NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 5
P = 4096                                        # an aligned address that no call here gets to use


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2402_02446_amd import build
        build.build(verbose=False)
    return binding.lib()


def _norm(L, **kw):
    a = dict(x=P, xt=0, rows=4, cols=64, ldx=64, r=P, ldr=64, h=P, ldh=64, rt=0, w=P, wt=0, eps=1e-5, bits=8, codes=P, exps=P, values=P, ldv=64)
    a.update(kw)
    return L.lqer_rmsnorm_mx(*a.values(), None)


@pytest.mark.parametrize("status, bad", [
    (0, dict(rows=0)), (0, dict(cols=0)), (NULL, dict(x=None)), (NULL, dict(w=None)), (NULL, dict(codes=None)), (NULL, dict(exps=None)),
    (NULL, dict(r=None)), (NULL, dict(h=None)), (UNSUPPORTED, dict(xt=2)), (UNSUPPORTED, dict(rt=-1)), (UNSUPPORTED, dict(wt=7)),
    (UNSUPPORTED, dict(bits=4)), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=40)), (SHAPE, dict(cols=-16)), (SHAPE, dict(eps=-1.0)),
    (SHAPE, dict(eps=float("nan"))), (SHAPE, dict(ldx=48)), (SHAPE, dict(ldx=66)), (SHAPE, dict(xt=1, ldx=68)), (SHAPE, dict(ldr=60)),
    (SHAPE, dict(ldh=63)), (SHAPE, dict(rt=1, ldh=68)), (SHAPE, dict(ldv=68)), (SHAPE, dict(x=P + 4)), (SHAPE, dict(r=P + 8)),
    (SHAPE, dict(h=P + 8)), (SHAPE, dict(w=P + 4)), (SHAPE, dict(codes=P + 8)), (SHAPE, dict(values=P + 2))])
def test_norm(L, status, bad):
    assert _norm(L, **bad) == status
