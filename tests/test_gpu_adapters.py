"""lqer_adapters_forward against the 64-bit formula.

Tolerance, derived: every product is exact (bf16 by bf16), T enters the second product with its 24 bits, the sums over K and over the ranks are
fp32: elementwise |error| <= (C sqrt(K + R) + C0) u sum|x||a||b| |s| + 2 u |Y|, u = 2^-24, with the C and C0 that the
linear's tests use for such sums (helpers.py); rows without an adapter keep their bits."""
import numpy as np
import pytest

from helpers import ELEM_C, ELEM_C0, U32
from oracle import block

pytestmark = pytest.mark.gpu


def _data(M, K, N, R, n, seed=0, ids=None, ranks=None, ldx=None):
    import torch
    g = torch.Generator().manual_seed(seed * 7919 + M * 31 + N)
    d = dict(X=torch.randn(M, ldx or K, generator=g).bfloat16()[:, :K], A=(torch.randn(n, R, K, generator=g) / K ** 0.5).bfloat16(),
             B=(torch.randn(n, N, R, generator=g) * 0.3).bfloat16(), Y=torch.randn(M, (N + 3) // 4 * 4, generator=g)[:, :N],
             scales=torch.rand(n, generator=g) + 0.5, ids=torch.randint(-1, n, (M,), generator=g) if ids is None else torch.as_tensor(ids),
             ranks=torch.full((n,), R) if ranks is None else torch.as_tensor(ranks))
    d["ids"], d["ranks"] = d["ids"].to(torch.int32), d["ranks"].to(torch.int32)
    return d


def _check(d, out, ranks=True, scales=True):
    X, A, B, Y = (d[k].double().numpy() for k in ("X", "A", "B", "Y"))
    ref, mag = block.adapters(X, d["ids"].numpy(), A, B, Y, d["ranks"].numpy() if ranks else None, d["scales"].numpy() if scales else None)
    bound = (ELEM_C * np.sqrt(A.shape[2] + A.shape[1]) + ELEM_C0) * U32 * mag + 2 * U32 * np.abs(ref)
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - ref) <= bound), float(np.max(np.abs(got - ref) / np.maximum(bound, 1e-300)))
    alone = (d["ids"].numpy() < 0) | (d["ids"].numpy() >= A.shape[0])
    assert np.array_equal(got[alone], Y[alone])


def _run(d, inplace=False, **kw):
    import torch
    from paper_2402_02446_amd import binding
    X = torch.empty(d["X"].shape[0], d["X"].stride(0), dtype=torch.bfloat16, device="cuda")[:, : d["X"].shape[1]]
    X.copy_(d["X"])
    ldy = d["Y"].stride(0)
    Y = torch.empty(d["Y"].shape[0], ldy, device="cuda")[:, : d["Y"].shape[1]]
    Y.copy_(d["Y"])
    out = Y if inplace else torch.full((Y.shape[0], ldy + 8), float("nan"), device="cuda")[:, : Y.shape[1]]
    a = dict(ranks=d["ranks"].cuda(), scales=d["scales"].cuda())
    a.update(kw)
    got = binding.lqer_adapters_forward(X, d["ids"].cuda(), d["A"].cuda(), d["B"].cuda(), Y, out=out, **a)
    assert got.data_ptr() == out.data_ptr()
    return got


# one token to the last that needs no sorting, the first that does, tiles with a rest
@pytest.mark.parametrize("M", [1, 2, 15, 17, 33, 64, 65, 129, 300])
@pytest.mark.parametrize("R", [8, 16, 24, 40, 128])
def test_tokens_and_ranks(M, R):
    d = _data(M, 272, 203, R, 5)
    _check(d, _run(d))


@pytest.mark.parametrize("K", [8, 24, 64, 200, 256, 264, 1032, 4112])
def test_contractions(K):
    for M in (3, 70):
        d = _data(M, K, 132, 16, 3, ldx=K + 16)
        _check(d, _run(d))


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 63, 64, 65, 255, 257, 1000])
def test_columns(N):
    for M in (5, 90):
        d = _data(M, 64, N, 16, 4)
        _check(d, _run(d))


# beyond 1024 tokens: tiles of 64, K through LDS in stages of 128 (64 above 64 ranks)
@pytest.mark.parametrize("R", [8, 16, 24, 40, 72, 128])
@pytest.mark.parametrize("K", [8, 72, 136, 520, 1032])
def test_many_tokens(R, K):
    d = _data(1100, K, 61, R, 5, ldx=K + 8)
    _check(d, _run(d))


@pytest.mark.parametrize("N", [1, 3, 64, 255, 260, 1001])
def test_many_tokens_columns(N):
    d = _data(1300, 48, N, 24, 9, ids=[(i // 70) % 10 - 1 for i in range(1300)])
    _check(d, _run(d))
    _check(d, _run(d, inplace=True))


def test_many_tokens_low_ranks():
    ranks = [0, 1, 7, 8, 9, 31, 33, 40, 64, 128]
    d = _data(1500, 200, 90, 128, len(ranks), ranks=ranks)
    for a, r in enumerate(ranks):
        d["A"][a, r:] = float("nan")
        d["B"][a, :, r:] = float("inf")
    out = _run(d)
    for a, r in enumerate(ranks):
        d["A"][a, r:] = 0
        d["B"][a, :, r:] = 0
    _check(d, out)


def test_many_columns_few_tokens():
    d = _data(48, 128, 7001, 32, 40)             # enough workgroups for the wide instance
    _check(d, _run(d))


@pytest.mark.parametrize("M", [40, 500])
def test_in_place(M):
    d = _data(M, 192, 260, 16, 7)
    _check(d, _run(d, inplace=True))


@pytest.mark.parametrize("M", [64, 200])
def test_everyone_one_adapter_or_none(M):
    for ids in ([2] * M, [-1] * M, [3] * M, [2 ** 31 - 1] * M, [-2 ** 31] * M, [i % 3 for i in range(M)], [0] * (M - 1) + [2]):
        d = _data(M, 136, 77, 16, 3, ids=ids)
        _check(d, _run(d))
        _check(d, _run(d, inplace=True))


def test_as_many_adapters_as_tokens():
    for M, n in ((64, 64), (100, 150), (70, 8192)):
        d = _data(M, 64, 40, 8, n, ids=[(i * 37) % n for i in range(M)])
        _check(d, _run(d))


@pytest.mark.parametrize("M", [20, 150])
def test_beyond_an_adapters_rank_anything_may_stand(M):
    ranks = [0, 1, 7, 8, 9, 31, 33, 40, -5, 99]
    d = _data(M, 160, 90, 40, len(ranks), ranks=ranks)
    for a, r in enumerate(ranks):
        r = min(max(r, 0), 40)
        d["A"][a, r:] = float("nan")
        d["B"][a, :, r:] = float("inf")
    out = _run(d)
    for a, r in enumerate(ranks):
        d["A"][a, max(r, 0):] = 0
        d["B"][a, :, max(r, 0):] = 0
    _check(d, out)


def test_more_tokens_than_are_sorted_at_once():
    d = _data(8192 + 500, 16, 12, 8, 5)
    _check(d, _run(d))
    d = _data(8192, 16, 12, 8, 700)
    _check(d, _run(d))


def test_defaults():
    d = _data(30, 96, 64, 16, 3)
    _check(d, _run(d, ranks=None, scales=None), ranks=False, scales=False)


@pytest.mark.parametrize("M", [31, 333])
def test_the_same_bits_again_and_from_a_graph(M):
    import torch
    from paper_2402_02446_amd import binding
    d = _data(M, 520, 300, 24, 6)
    first = _run(d).clone()
    assert torch.equal(first, _run(d))
    X, ids, A, B, Y = (d[k].cuda() for k in ("X", "ids", "A", "B", "Y"))
    Y = Y.contiguous()
    out = torch.empty_like(Y)
    ws = torch.empty(binding.lqer_adapters_workspace_bytes(M, 520, 300, 24, 6), dtype=torch.uint8, device="cuda")
    call = lambda: binding.lqer_adapters_forward(X, ids, A, B, Y, out=out, ranks=ranks, scales=scales, workspace=ws)  # noqa: E731
    ranks, scales = d["ranks"].cuda(), d["scales"].cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        out.fill_(float("nan"))
        ids.copy_(ids.roll(1))
        X.copy_(X.roll(1, 0))
        Y.copy_(Y.roll(1, 0))
        first = first.roll(1, 0)
        ws.random_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_tensors_that_the_library_cannot_check():
    import torch
    from paper_2402_02446_amd import binding
    d = _data(4, 64, 32, 16, 2)
    a = {k: d[k].cuda() for k in ("X", "ids", "A", "B", "Y", "ranks", "scales")}
    for bad in (dict(X=a["X"].float()), dict(ids=a["ids"].long()), dict(ids=a["ids"][:3]), dict(A=a["A"].float()), dict(B=a["B"][:1]),
                dict(Y=a["Y"].bfloat16()), dict(out=a["Y"][:3]), dict(ranks=a["ranks"].long()), dict(scales=a["scales"].double()),
                dict(Y=a["Y"].cpu()), dict(X=a["X"][:, ::2])):
        with pytest.raises(ValueError):
            binding.lqer_adapters_forward(**{**a, **bad})


def test_a_workspace_of_its_own_is_contiguous_and_on_the_gpu():
    import torch
    from paper_2402_02446_amd import binding
    d = _data(4, 64, 32, 16, 2)
    a = {k: d[k].cuda() for k in ("X", "ids", "A", "B", "Y", "ranks", "scales")}
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(256, dtype=torch.uint8, device="cuda")[:, None].expand(256, 4096)):
        with pytest.raises(ValueError):
            binding.lqer_adapters_forward(**a, workspace=bad)


# Up to 64 tokens, more than 16 of them with one adapter, several blocks of columns to a workgroup and fewer to the last one or to its last
# wavefronts: B of the first block is read again for the next 16 tokens.  (ranks: 32, 64 and 128 at most)
@pytest.mark.parametrize("R", [16, 40, 128])
@pytest.mark.parametrize("N, groups, one", [(7001, 19, 46), (28672, 10, 55), (11008, 24, 41), (14336, 19, 30)])
def test_one_adapter_of_many_tokens_beside_others(R, N, groups, one):
    rng = np.random.default_rng(N + R)
    d = _data(one + groups - 1, 40, N, R, groups, ids=rng.permutation([groups - 1] * one + list(range(groups - 1))))
    _check(d, _run(d))
    _check(d, _run(d, inplace=True))


@pytest.mark.parametrize("M", [5, 100, 1100])
def test_numbers_that_are_not_finite_or_close_to_it(M):
    """T = X A^T infinite, NaN, or between the largest bf16 and the largest fp32 number: Y is what the formula gives."""
    d = _data(M, 64, 70, 16, 2, ids=[0] * M, ranks=[9, 16])
    d["A"][:], d["X"][:], d["B"][:] = 0, 0, 0
    for r in range(9):
        d["A"][0, r, r] = 1
        d["B"][0, :, r] = 1
    d["A"][0, :9, 20] = 2
    d["B"][0, 40:, 3] = 2.0 ** -100
    d["X"][:, 3] = 3.0
    d["X"][1, 20] = float("inf")                    # T infinite in every rank
    d["X"][2, 20] = -float("inf")
    d["X"][3, 20] = float("nan")
    big = 2.0 ** 127 * (2 - 2.0 ** -7)              # the largest bf16 number; half a unit more would round to infinity
    d["X"][4, 3], d["A"][0, 3, 30], d["X"][4, 30] = big, 1, 2.0 ** 119 * 1.5
    d["scales"][:] = 1
    out = _run(d).double().cpu().numpy()
    assert np.all(out[1] == np.inf) and np.all(out[2] == -np.inf) and np.all(np.isnan(out[3]))
    rest = [m for m in range(M) if m not in (1, 2, 3)]
    ref, mag = block.adapters(d["X"][rest].double().numpy(), np.zeros(len(rest)), d["A"].double().numpy(), d["B"].double().numpy(),
                              d["Y"][rest].double().numpy(), d["ranks"].numpy(), d["scales"].numpy())
    assert ref[4 - 3].max() > big                   # (token 4)
    assert np.all(np.abs(out[rest] - ref) <= 4 * U32 * (mag + np.abs(ref)))


# Every token's group is found by every workgroup alike, whatever the mix of adapters: no token is left out, none counted twice (in place).
@pytest.mark.parametrize("M", [2, 7, 16, 41, 64])
def test_mixes_of_adapters(M):
    rng = np.random.default_rng(M)
    for most in (1, 2, 3, 5, 9, 20, 64, 8192):
        ids = rng.integers(-1, most, M)
        ids[rng.integers(0, M, M // 3)] = ids[0]
        d = _data(M, 24, 140, 8, min(most, 300), ids=np.where(ids >= 300, ids % 300, ids))
        _check(d, _run(d, inplace=True))
