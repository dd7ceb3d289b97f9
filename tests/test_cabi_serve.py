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
    (SHAPE, dict(eps=float("nan"))), (SHAPE, dict(eps=float("inf"))), (SHAPE, dict(ldx=48)), (SHAPE, dict(ldx=66)), (SHAPE, dict(xt=1, ldx=68)), (SHAPE, dict(ldr=60)),
    (SHAPE, dict(ldh=63)), (SHAPE, dict(rt=1, ldh=68)), (SHAPE, dict(ldv=68)), (SHAPE, dict(x=P + 4)), (SHAPE, dict(r=P + 8)),
    (SHAPE, dict(h=P + 8)), (SHAPE, dict(w=P + 4)), (SHAPE, dict(codes=P + 8)), (SHAPE, dict(values=P + 2))])
def test_norm(L, status, bad):
    assert _norm(L, **bad) == status


# the residual updated in place is one array with one stride
@pytest.mark.parametrize("ldr, ldh", [(64, 128), (96, 64)])
def test_norm_in_place_strides(L, ldr, ldh):
    assert _norm(L, r=P, h=P, ldr=ldr, ldh=ldh) == SHAPE


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


def test_adapters_tokens(L):
    assert _adapters(L, M=(1 << 29) + 1) == SHAPE and L.lqer_adapters_workspace_bytes((1 << 29) + 1, 64, 40, 16, 3) == 0
    assert _adapters(L, M=1 << 29) == WORKSPACE and L.lqer_adapters_workspace_bytes(1 << 29, 64, 40, 16, 3) > 1 << 35


def test_adapters_workspace(L):
    need = L.lqer_adapters_workspace_bytes(4, 64, 40, 16, 3)
    assert need > 0 and _adapters(L, bytes=need - 1) == WORKSPACE
    assert L.lqer_adapters_workspace_bytes(0, 64, 40, 16, 3) == 0 and L.lqer_adapters_workspace_bytes(4, 60, 40, 16, 3) == 0
    # more than 64 tokens are sorted by adapter in the workspace
    assert L.lqer_adapters_workspace_bytes(65, 64, 40, 16, 3) > L.lqer_adapters_workspace_bytes(64, 64, 40, 16, 3)


def test_kv4_page_bytes(L):
    assert L.lqer_kv4_page_bytes(16, 128) == 16 * 128 * 9 // 8 and L.lqer_kv4_page_bytes(1024, 256) == 1024 * 288
    for P, D in ((8, 128), (24, 128), (2048, 128), (0, 64), (-16, 64), (16, 32), (16, 96), (16, 512)):
        assert L.lqer_kv4_page_bytes(P, D) == 0


def _append(L, **kw):
    a = dict(pool=P, pages=3, P=16, heads=2, D=64, k=P, ldk=128, v=P, ldv=128, t=1, T=5, slots=P)
    a.update(kw)
    return L.lqer_kv4_append(*a.values(), None)


@pytest.mark.parametrize("status, bad", [
    (0, dict(T=0)), (NULL, dict(pool=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(slots=None)), (UNSUPPORTED, dict(P=17)),
    (UNSUPPORTED, dict(D=80)), (UNSUPPORTED, dict(t=2)), (SHAPE, dict(T=-1)), (SHAPE, dict(pages=0)), (SHAPE, dict(pages=(1 << 26) + 1)),
    (SHAPE, dict(heads=0)), (SHAPE, dict(heads=1025)), (SHAPE, dict(ldk=120)), (SHAPE, dict(ldv=132)), (SHAPE, dict(k=P + 2)), (SHAPE, dict(v=P + 4)),
    (SHAPE, dict(pool=P + 8)), (SHAPE, dict(slots=P + 2))])
def test_kv4_append(L, status, bad):
    assert _append(L, **bad) == status


def _attend(L, ptrs=None, ws=P, ws_bytes=1 << 30, **kw):
    a = dict(n_requests=2, q_heads=8, kv_heads=2, head_dim=64, page_tokens=16, table_ld=400, pages=900, Tq=2, ldq=512, ldo=512, max_q=1, max_kv=6000,
             causal=1, window=0, scale=0.125, out_type=1)
    a.update(kw)
    p = dict(pool=P, q=P, cu=P, kv=P, table=P, out=P)
    p.update(ptrs or {})
    return L.lqer_kv4_attention(binding.C.byref(binding.Kv4Shape(*a.values())), *p.values(), ws, ws_bytes, None)


@pytest.mark.parametrize("status, bad", [
    (0, dict(Tq=0)), (0, dict(n_requests=0)), (UNSUPPORTED, dict(head_dim=96)), (UNSUPPORTED, dict(page_tokens=2048)), (UNSUPPORTED, dict(out_type=3)),
    (SHAPE, dict(q_heads=7)), (SHAPE, dict(q_heads=0)), (SHAPE, dict(kv_heads=0)), (SHAPE, dict(n_requests=-1)), (SHAPE, dict(n_requests=65536)),
    (SHAPE, dict(table_ld=0)), (SHAPE, dict(table_ld=(1 << 26) + 1)), (SHAPE, dict(Tq=-1)), (SHAPE, dict(Tq=1 << 31)), (SHAPE, dict(pages=0)),
    (SHAPE, dict(ldq=511)), (SHAPE, dict(ldq=516)), (SHAPE, dict(ldo=504)), (SHAPE, dict(max_q=-1)), (SHAPE, dict(max_kv=-1)), (SHAPE, dict(causal=2)),
    (SHAPE, dict(window=-1)), (SHAPE, dict(scale=float("nan"))), (NULL, dict(ptrs=dict(pool=None))), (NULL, dict(ptrs=dict(q=None))),
    (NULL, dict(ptrs=dict(cu=None))), (NULL, dict(ptrs=dict(kv=None))), (NULL, dict(ptrs=dict(table=None))), (NULL, dict(ptrs=dict(out=None))),
    (SHAPE, dict(ptrs=dict(pool=P + 8))), (SHAPE, dict(ptrs=dict(q=P + 2))), (SHAPE, dict(ptrs=dict(out=P + 4))), (SHAPE, dict(ptrs=dict(table=P + 1))),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws=P + 16)), (WORKSPACE, dict(ws_bytes=16))])
def test_kv4_attention(L, status, bad):
    assert _attend(L, **bad) == status


def test_kv4_attention_workspace(L):
    """Parts of a long axis, and of few tiles of many rows, are joined in the workspace; short caches need none."""
    def need(**kw):
        a = dict(n_requests=2, q_heads=8, kv_heads=2, head_dim=64, page_tokens=16, table_ld=400, pages=900, Tq=2, ldq=512, ldo=512, max_q=1,
                 max_kv=6000, causal=1, window=0, scale=0.125, out_type=1)
        a.update(kw)
        return L.lqer_kv4_attention_workspace_bytes(binding.C.byref(binding.Kv4Shape(*a.values())))
    assert need() > 0 and need(max_kv=600) == 0 and need(window=500) == 0 and need(q_heads=7) == 0 and need(Tq=0) == 0
    assert need(Tq=200, max_q=100) > 0
    assert need(n_requests=400, Tq=400 * 2000, max_q=2000, max_kv=100000) == 0          # enough tiles without parts
    assert need() % 256 == 0 and need(Tq=1001, n_requests=2, max_q=1000) < 600 << 20


def test_kv4_attention_without_a_shape(L):
    assert L.lqer_kv4_attention(None, P, P, P, P, P, P, P, 0, None) == NULL
    assert L.lqer_kv4_attention_workspace_bytes(None) == 0


@pytest.mark.parametrize("name", ["max_q", "max_kv", "window"])
def test_kv4_numbers_beyond_32_bits(L, name):
    """A caller's estimates and window are taken as the largest that the library takes, a negative one stays negative."""
    a = dict(n_requests=2, q_heads=8, kv_heads=2, head_dim=64, page_tokens=16, table_ld=400, pages=900, Tq=2, ldq=512, ldo=512, max_q=1, max_kv=6000,
             causal=True, window=0, scale=0.125, out_type=True)
    for value, taken in ((2 ** 31 - 1, 2 ** 31 - 1), (2 ** 32 + 1, 2 ** 31 - 1), (2 ** 63, 2 ** 31 - 1), (-2 ** 32 + 1, -1), (3, 3)):
        assert getattr(binding._kv4_sizes(*{**a, name: value}.values())[0]._obj, name) == taken


@pytest.mark.parametrize("rows", [0, 1])
def test_a_single_row_has_no_stride_of_its_own(rows):
    """What torch says of it, as a slice of a wider buffer or of an odd width, is not what a row has to keep to."""
    import torch
    for width, cols in ((4100, 4096), (4099, 4096), (203, 203), (8, 8), (1, 1)):
        got = binding._stride(torch.empty(3, width)[:rows, :cols], rows, cols)
        assert got >= cols and got % 8 == 0
    for heads, D, buffer in ((2, 64, (3, 2, 65)), (4, 128, (3, 7, 128)), (1, 64, (3, 1, 70)), (1, 256, (3, 5, 257))):
        t = torch.empty(buffer)[:rows, :heads, :D]
        if heads == 1 or t.stride(1) == D:
            assert binding._token_stride(t.stride(), rows, heads, D) == heads * D
        else:
            assert binding._token_stride(t.stride(), rows, heads, D) == 0
