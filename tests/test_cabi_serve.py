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


def _adapters(L, **kw):
    a = dict(X=P, M=4, K=64, ldx=64, ids=P, A=P, B=P, n=3, R=16, ranks=P, scales=P, yi=P, ldyi=40, yo=P, N=40, ldyo=40, ws=P, bytes=1 << 20)
    a.update(kw)
    return L.lqer_adapters_forward(*a.values(), None)


@pytest.mark.parametrize("status, bad", [
    (0, dict(M=0)), (0, dict(N=0)), (NULL, dict(X=None)), (NULL, dict(ids=None)), (NULL, dict(A=None)), (NULL, dict(B=None)),
    (NULL, dict(yi=None)), (NULL, dict(yo=None)), (UNSUPPORTED, dict(R=136)), (UNSUPPORTED, dict(n=8193)), (SHAPE, dict(M=-1)),
    (SHAPE, dict(K=0)), (SHAPE, dict(K=60)), (SHAPE, dict(N=-4)), (SHAPE, dict(R=12)), (SHAPE, dict(R=0)), (SHAPE, dict(n=0)),
    (SHAPE, dict(ldx=56)), (SHAPE, dict(ldx=68)), (SHAPE, dict(ldyi=36)), (SHAPE, dict(ldyi=42)), (SHAPE, dict(ldyo=44)),
    (SHAPE, dict(yo=P + 4096, ldyo=39)), (SHAPE, dict(N=4194304, ldyi=4194304, ldyo=4194304)), (SHAPE, dict(X=P + 2)), (SHAPE, dict(A=P + 8)),
    (SHAPE, dict(B=P + 4)), (SHAPE, dict(yi=P + 4)), (SHAPE, dict(yo=P + 8)), (SHAPE, dict(ids=P + 1)), (SHAPE, dict(ranks=P + 2)),
    (SHAPE, dict(scales=P + 3)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws=P + 128)), (WORKSPACE, dict(bytes=64))])
def test_adapters(L, status, bad):
    assert _adapters(L, **bad) == status


def test_adapters_workspace(L):
    need = L.lqer_adapters_workspace_bytes(4, 64, 40, 16, 3)
    assert need > 0 and _adapters(L, bytes=need - 1) == WORKSPACE
    assert L.lqer_adapters_workspace_bytes(0, 64, 40, 16, 3) == 0 and L.lqer_adapters_workspace_bytes(4, 60, 40, 16, 3) == 0
    # more than 64 tokens are sorted by adapter in the workspace
    assert L.lqer_adapters_workspace_bytes(65, 64, 40, 16, 3) > L.lqer_adapters_workspace_bytes(64, 64, 40, 16, 3)
