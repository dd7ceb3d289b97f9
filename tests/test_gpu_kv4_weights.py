"""How exactly the weights of lqer_kv4_attention enter the product with V: fp32 outputs, which no rounding of the output hides.

Tolerance, derived.  Keys, values and queries enter exactly.  Requests of up to 64 rows (queries times heads of a group): the weights enter as two bf16 terms, 2^-16
of each; the fp32 scores (up to about 100 in units of log 2, 2^-24 of that times a few), exponentials and sums add at most 2^-12.  Elementwise
|error| <= (2^-16 + 2^-12) sum_t w_t |V_t|, w the exact weights.  One bf16 term would be off by up to 2^-8 of each weight: every call
also asserts that weights rounded so leave the bound on the same data."""
import numpy as np
import pytest

from oracle import block
from test_gpu_kv4 import _cache

pytestmark = pytest.mark.gpu
BOUND = 2.0 ** -16 + 2.0 ** -12


def _bf16(x):
    """fp64 -> the nearest bf16 (8 significant bits), ties to even"""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256), e - 8)


def _few(q_lens, lens, q_heads, kv_heads, D, P, causal=True, window=0, max_q=None, spare_rows=0):
    """The requests of up to 64 rows of a call against the bound; the others may be any."""
    import torch
    from paper_2402_02446_amd import binding
    rng = np.random.default_rng(101 * D + P + sum(lens))
    pool, table, K, V = _cache(rng, lens, kv_heads, D, P)
    T = sum(q_lens) + spare_rows
    q = torch.from_numpy(rng.standard_normal((T, q_heads, D)).astype(np.float32)).bfloat16()
    cu = np.cumsum([0] + list(q_lens)).astype(np.int32)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    out = torch.full((T, q_heads, D), 7.0, device="cuda")
    got = binding.lqer_kv4_attention(dev(pool), q.cuda(), dev(cu), dev(np.array(lens, np.int32)), dev(table), max(q_lens) if max_q is None else max_q,
                                     max(lens), D ** -0.5, causal=causal, window=window, out=out).double().cpu().numpy()
    G, scale, seen_by_one_term = q_heads // kv_heads, float(np.float32(D ** -0.5)), False
    for b, n in enumerate(q_lens):
        if n * G > 64:
            continue
        pos = lens[b] - n + np.arange(n)
        end = pos + 1 if causal else np.full(n, lens[b])
        begin = np.maximum(pos - window + 1, 0) if window else np.zeros(n, int)
        for h in range(q_heads):
            qq = q[cu[b]: cu[b + 1], h].double().numpy()
            o, mag = block.attention(qq, K[b][:, h // G], V[b][:, h // G], scale, begin, end)
            err = np.abs(got[cu[b]: cu[b + 1], h] - o)
            assert np.all(err <= BOUND * mag), (b, h, float(np.max(err / np.maximum(mag, 1e-300))))
            for i in range(n):
                if end[i] > begin[i]:
                    s = (K[b][begin[i]: end[i], h // G] @ qq[i]) * scale
                    w = np.exp(s - s.max())
                    seen_by_one_term |= bool(np.any(np.abs((_bf16(w) / w.sum()) @ V[b][begin[i]: end[i], h // G] - o[i]) > BOUND * mag[i]))
    assert seen_by_one_term
    assert np.all(got[cu[-1]:] == 7.0)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_single_tokens(D):
    _few([1] * 6, [2, 3, 7, 19, 130, 300], 8, 2, D, 16)
    _few([1, 1], [3000, 5], 4, 1, D, 64)                # parts of the axis, joined


@pytest.mark.parametrize("D", [64, 128, 256])
def test_several_tokens(D):
    _few([5, 1, 16, 0], [5, 9, 40, 12], 8, 2, D, 16)
    _few([7, 3], [50, 8], 4, 2, D, 16, causal=False)
    _few([7, 9], [50, 800], 4, 2, D, 16, window=6)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_beside_a_prompt(D):
    _few([130, 1, 4], [130, 9, 20], 4, 1, D, 16)


# Rows of q that no request covers, and estimates of the longest request that are too small or too large, say nothing about the other requests.
@pytest.mark.parametrize("D", [64, 128, 256])
def test_beside_a_prompt_with_spare_rows(D):
    _few([300, 1], [300, 6], 1, 1, D, 16, spare_rows=723)
    _few([70, 2, 3], [90, 5, 9], 2, 1, D, 16, spare_rows=200)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_beside_a_prompt_that_is_longer_than_estimated(D):
    _few([150, 1], [150, 6], 1, 1, D, 16, max_q=75)
    _few([290, 3, 7], [290, 6, 20], 1, 1, D, 16, max_q=100)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_one_request_that_is_shorter_than_estimated(D):
    _few([3], [9], 4, 1, D, 16, max_q=4000)
