"""lqer_kv4_append and lqer_kv4_attention against the oracle.

Appending: the pool's bytes are the oracle's, and no other byte changes.
Attention, tolerance derived: keys, values and queries enter exactly (codes times powers of two, bf16); scores are fp32; the weights enter the
product with V as two bf16 terms (relative 2^-16); the exponentials and the fp32 scores behind them (arguments of up to about 100, relative 2^-24
times a few) add at most 2^-12; a bf16 output is rounded by 2^-8 of itself at most, and |o| <= sum_t w_t |V_t|.  Elementwise, within
|error| <= (2^-9 + 2^-12) sum_t w_t |V_t| + 2^-9 |o| (the last term for bf16 outputs), w the exact weights.
Where a request has more than 64 rows (queries times heads of a group) the weights enter as one bf16 term, rounded by 2^-8 at most, their sum in
fp32: |error| <= (2^-8 + 2^-12) sum_t w_t |V_t| + 2^-8 |o|."""
import numpy as np
import pytest

from oracle import block

pytestmark = pytest.mark.gpu


def _cache(rng, lens, heads, D, P, spare=2, fill=0xFF):
    """Pool, table and the exact keys and values [request][t][head][D]; what no length covers is filled with `fill`."""
    pages = [-(-t // P) for t in lens]
    n = sum(pages) + spare
    pool = np.full((n, heads, P * D * 9 // 8), fill, np.uint8)
    order = rng.permutation(n)
    table = np.full((len(lens), max(max(pages), 1)), -1, np.int32)
    K, V, at = [], [], 0
    for b, t in enumerate(lens):
        table[b, : pages[b]] = order[at: at + pages[b]]
        at += pages[b]
        got = []
        for which in range(2):
            x = rng.standard_normal((t, heads, D)) * (4.0 if which == 0 else 1.0) ** rng.integers(0, 2, (1, heads, D))
            c, e = block.kv4_quantize(x.astype(np.float32))
            for i in range(t):
                for h in range(heads):
                    block.kv4_store(pool, P, D, table[b, i // P], h, i % P, which, c[i, h], e[i, h])
            got.append(block.kv4_values(c, e).reshape(t, heads, D))
        K.append(got[0])
        V.append(got[1])
    return pool, table, K, V


def _attend(q_lens, lens, q_heads, kv_heads, D, P, causal=True, window=0, scale=None, f32=False, max_q=None, max_kv=None, seed=0, pad=0, edit=None,
            spare_rows=0, fill=0xFF):
    import torch
    from paper_2402_02446_amd import binding
    rng = np.random.default_rng(seed + 13 * D + P)
    pool, table, K, V = _cache(rng, lens, kv_heads, D, P, fill=fill)
    seen = [np.ones(t, bool) for t in lens]
    kv_len = list(lens)
    if edit:
        edit(pool, table, seen, kv_len)
    T = sum(q_lens) + spare_rows
    scale = D ** -0.5 if scale is None else scale
    q = torch.from_numpy(rng.standard_normal((T, q_heads, D)).astype(np.float32)).bfloat16()
    qd = torch.empty(T, q_heads * D + pad, dtype=torch.bfloat16, device="cuda")[:, : q_heads * D].view(T, q_heads, D) if pad == 0 else \
        torch.empty(T, q_heads + pad, D, dtype=torch.bfloat16, device="cuda")[:, :q_heads]
    qd.copy_(q)
    cu = np.cumsum([0] + list(q_lens)).astype(np.int32)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    out = torch.full((T, q_heads + pad, D), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")[:, :q_heads]
    got = binding.lqer_kv4_attention(dev(pool), qd, dev(cu), dev(np.array(kv_len, np.int32)), dev(table), max(q_lens) if max_q is None else max_q,
                                     max(lens) if max_kv is None else max_kv, scale, causal=causal, window=window, out=out).double().cpu().numpy()
    G = q_heads // kv_heads
    scale = float(np.float32(scale))
    for b, n in enumerate(q_lens):
        t = min(kv_len[b], table.shape[1] * P)
        pos = t - n + np.arange(n)
        end = pos + 1 if causal else np.full(n, t)
        begin = pos - window + 1 if window else np.zeros(n, int)
        for h in range(q_heads):
            qq = q[cu[b]: cu[b + 1], h].double().numpy()
            o, mag = block.attention(qq, K[b][:t, h // G], V[b][:t, h // G], scale, begin, end, seen[b])
            unit = 2.0 ** -8 if n * G > 64 else 2.0 ** -9
            bound = (unit + 2.0 ** -12) * mag + (0 if f32 else unit) * np.abs(o)
            err = np.abs(got[cu[b]: cu[b + 1], h] - o)
            assert np.all(err <= bound), (b, h, np.argwhere(~(err <= bound))[:3].tolist(), float(np.nanmax(err)))
    assert np.all(got[cu[-1]:] == 7.0)
    return got


# ---- appending ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("heads, P", [(1, 16), (3, 64), (8, 32)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append(D, heads, P, dtype):
    import torch
    from paper_2402_02446_amd import binding
    rng = np.random.default_rng(D + heads)
    pages, T = 4, 37
    old = rng.integers(0, 256, (pages, heads, P * D * 9 // 8), dtype=np.uint8)
    slots = rng.permutation(pages * P)[:T].astype(np.int32) if pages * P >= T else None
    slots[5], slots[17], slots[20] = -1, pages * P, 2 ** 31 - 1       # not stored
    k = torch.from_numpy(rng.standard_normal((T, heads + 2, D)).astype(np.float32))
    v = torch.from_numpy(rng.standard_normal((T, heads, D)).astype(np.float32)) * 1e-3
    k[3, :, 16:32] = 0
    k[4, 0, 0], v[6, 0, 5] = 3e38, -1.9
    v[7] *= 1e30
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    k, v = k.to(t), v.to(t)
    pool = torch.from_numpy(old).cuda()
    binding.lqer_kv4_append(pool, k.cuda()[:, :heads], v.cuda(), torch.from_numpy(slots).cuda())
    want = old.copy()
    for which, x in enumerate((k[:, :heads], v)):
        c, e = block.kv4_quantize(x.double().numpy())
        for i in range(T):
            if 0 <= slots[i] < pages * P:
                for h in range(heads):
                    block.kv4_store(want, P, D, slots[i] // P, h, slots[i] % P, which, c[i, h], e[i, h])
    assert np.array_equal(pool.cpu().numpy(), want)


def test_append_many_tokens_and_none():
    import torch
    from paper_2402_02446_amd import binding
    T, heads, D, P = 70000, 1, 64, 1024            # more tokens than a grid's second axis has workgroups
    pool = binding.lqer_kv4_pool(69, heads, P, D)
    k, v = (torch.randn(T, heads, D, device="cuda") for _ in range(2))
    slots = torch.randperm(69 * P, device="cuda")[:T].to(torch.int32)
    binding.lqer_kv4_append(pool, k, v, slots)
    rows = [0, 1, 4095, 65535, 65536, 69999]
    for which, x in enumerate((k, v)):
        c, e = block.kv4_quantize(x[rows].double().cpu().numpy())
        want = np.zeros((69, heads, P * D * 9 // 8), np.uint8)
        for j, i in enumerate(rows):
            s = int(slots[i])
            block.kv4_store(want, P, D, s // P, 0, s % P, which, c[j, 0], e[j, 0])
            mask = np.zeros_like(want)
            block.kv4_store(mask, P, D, s // P, 0, s % P, which, np.full(D, -7, np.int8), np.full(D // 16, 255, np.uint8))
            rec = mask[s // P, 0] > 0
            assert np.array_equal(pool[s // P, 0].cpu().numpy()[rec], want[s // P, 0][rec])
    binding.lqer_kv4_append(pool, k[:0], v[:0], slots[:0])


# ---- attention: single tokens ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads, kv_heads", [(1, 1), (8, 2), (5, 1), (32, 2), (40, 1)])
def test_one_token(D, q_heads, kv_heads):
    _attend([1] * 6, [1, 16, 17, 33, 130, 300], q_heads, kv_heads, D, 16)


@pytest.mark.parametrize("P", [16, 32, 64, 256, 1024])
def test_pages(P):
    _attend([1, 1, 1], [P - 1, P + 1, 2 * P], 4, 2, 64, P)
    _attend([1, 1], [40, 1], 4, 2, 128, P, f32=True)


@pytest.mark.parametrize("length", [0, 1, 2, 3, 4, 5, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1100])
def test_lengths(length):
    _attend([1, 1], [length, 40], 4, 1, 128, 16)
    _attend([1], [length], 2, 2, 64, 32)


def test_long_and_split():
    _attend([1, 1], [5000, 37], 8, 1, 128, 64)
    _attend([1, 0, 1], [3000, 0, 1], 4, 1, 256, 128, f32=True)


# ---- several tokens: tiles of 16 and of 128 rows, requests of either kind in one call -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_len", [2, 5, 17, 40])
def test_several_tokens(D, q_len):
    _attend([q_len, 1, 0, q_len - 1], [q_len, 150, 9, 77], 6, 2, D, 16)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads, kv_heads", [(1, 1), (3, 1), (8, 2), (40, 1)])
def test_prompts(D, q_heads, kv_heads):
    _attend([130, 33, 64], [130, 200, 64], q_heads, kv_heads, D, 32)


@pytest.mark.parametrize("length", [33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 191, 193, 257])
def test_prompt_lengths(length):
    _attend([length, 40], [length, length], 1, 1, 128, 16)
    _attend([length], [length + 70], 1, 1, 64, 64, f32=True)
    _attend([length], [length + 3], 1, 1, 256, 16)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_chunk_on_a_long_cache(D):
    """Few tiles of rows over many tokens: the axis is cut into parts."""
    _attend([20], [3000], 4, 2, D, 64)
    _attend([40, 35], [1500, 2100], 2, 1, D, 16, f32=True, window=900)


def test_prompts_and_single_tokens_in_one_call():
    _attend([1, 200, 1, 3, 0, 33], [900, 260, 1, 70, 0, 400], 8, 2, 128, 16)
    _attend([300, 1, 1], [300, 2500, 700], 4, 1, 64, 64, f32=True)
    _attend([5, 100, 8, 9], [50, 100, 64, 300], 4, 1, 256, 16, causal=False)


@pytest.mark.parametrize("window", [1, 2, 16, 33, 100, 1000])
@pytest.mark.parametrize("q_len", [1, 4, 50])
def test_window(window, q_len):
    _attend([q_len, q_len], [200, 60], 4, 2, 64, 16, window=window)


def test_not_causal():
    _attend([3, 1, 30], [50, 7, 80], 4, 2, 128, 16, causal=False)
    _attend([3, 1, 30], [50, 7, 80], 4, 2, 64, 16, causal=False, window=20)


def test_queries_that_see_nothing():
    """More queries than cached tokens: the first stand before the cache's beginning; empty requests."""
    out = _attend([5, 3, 20], [2, 0, 18], 4, 2, 64, 16)
    assert np.all(out[:3] == 0) and np.all(out[5:8] == 0)


def test_rows_of_no_request_are_left_alone():
    _attend([1, 2], [30, 40], 4, 2, 64, 16, spare_rows=3)


def test_estimates_too_small():
    _attend([9, 33, 1], [700, 90, 2500], 8, 2, 64, 16, max_q=1, max_kv=1)
    _attend([9, 1], [90, 400], 4, 2, 128, 16, max_q=0, max_kv=0)
    _attend([1, 5], [90, 400], 4, 2, 128, 16, max_q=4000, max_kv=100000)


def test_strided_and_scaled():
    _attend([2, 1], [70, 33], 4, 2, 128, 16, pad=3)
    _attend([2, 1], [70, 33], 4, 2, 64, 16, scale=-0.3, f32=True)
    _attend([2, 1], [70, 33], 4, 2, 64, 16, scale=0.0)
    _attend([1, 1], [70, 330], 4, 2, 64, 16, scale=3.0)


@pytest.mark.parametrize("fill", [0x00, 0x7F, 0xFF])
def test_what_lies_beyond_the_lengths(fill):
    _attend([1, 4, 40], [5, 100, 77], 4, 2, 128, 64, fill=fill)
    _attend([1, 4, 40], [5, 100, 77], 4, 2, 64, 64, fill=fill, window=30)


def test_pages_outside_the_pool_are_not_seen():
    def edit(pool, table, seen, kv_len):
        for b, i, bad in ((0, 1, -1), (0, 3, pool.shape[0]), (1, 0, -2 ** 31), (1, 2, 2 ** 31 - 1)):
            table[b, i] = bad
            seen[b][16 * i: 16 * i + 16] = False
        table[2, :] = -7
        seen[2][:] = False
    out = _attend([1, 20, 3], [90, 80, 40], 4, 2, 64, 16, edit=edit)
    assert np.all(out[21:] == 0)


def test_lengths_beyond_the_table():
    def edit(pool, table, seen, kv_len):
        kv_len[0] += 1000                        # taken as what the table holds
        kv_len[1] = -5                           # taken as 0
    _attend([1, 1], [64, 20], 4, 2, 64, 16, edit=edit)


def test_a_cache_beyond_four_gigabytes():
    """The last pages of a large pool: offsets of more than 32 bits."""
    import torch
    from paper_2402_02446_amd import binding
    heads, D, P, pages = 8, 128, 64, 70000                              # 5.2 GB
    pool = binding.lqer_kv4_pool(pages, heads, P, D)
    rng = np.random.default_rng(3)
    n = 200
    table = np.array([[69999, 12, 69000, 60000]], np.int32)
    k, v = (torch.from_numpy(rng.standard_normal((n, heads, D)).astype(np.float32)) for _ in range(2))
    slots = np.array([table[0, i // P] * P + i % P for i in range(n)], np.int32)
    binding.lqer_kv4_append(pool, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda())
    q = torch.from_numpy(rng.standard_normal((1, heads, D)).astype(np.float32)).bfloat16()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = binding.lqer_kv4_attention(pool, q.cuda(), i32(0, 1), i32(n), torch.from_numpy(table).cuda(), 1, n, D ** -0.5).double().cpu().numpy()
    K, V = (block.kv4_values(*block.kv4_quantize(x.numpy())) for x in (k, v))
    for h in range(heads):
        o, mag = block.attention(q[:, h].double().numpy(), K[:, h], V[:, h], float(np.float32(D ** -0.5)), [0], [n])
        assert np.all(np.abs(out[:, h] - o) <= (2.0 ** -9 + 2.0 ** -12) * mag + 2.0 ** -9 * np.abs(o))


@pytest.mark.parametrize("q_lens, lens", [([1, 1, 1], [700, 33, 1500]), ([40, 1], [300, 80])])
def test_a_step_captured_in_a_graph(q_lens, lens):
    """Append and attention in one graph: every replay has the bits of the eager calls on the same data."""
    import torch
    from paper_2402_02446_amd import binding
    rng = np.random.default_rng(11)
    heads, G, D, P = 2, 4, 128, 16
    pool_np, table, _, _ = _cache(rng, lens, heads, D, P)
    T = sum(q_lens)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    pool, table_d, cu, kv = dev(pool_np), dev(table), dev(np.cumsum([0] + q_lens).astype(np.int32)), dev(np.array(lens, np.int32))
    slots = dev(np.array([table[b, p // P] * P + p % P for b, n in enumerate(q_lens) for p in range(lens[b] - n, lens[b])], np.int32))
    q = torch.randn(T, heads * G, D, device="cuda").bfloat16()
    k, v = (torch.randn(T, heads, D, device="cuda") for _ in range(2))
    out = torch.empty_like(q)
    ws = torch.empty(max(binding.lqer_kv4_attention_workspace_bytes(pool, q, table_d, max(q_lens), max(lens)), 256), dtype=torch.uint8, device="cuda")

    def step():
        binding.lqer_kv4_append(pool, k, v, slots)
        binding.lqer_kv4_attention(pool, q, cu, kv, table_d, max(q_lens), max(lens), D ** -0.5, out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        q.normal_()
        k.normal_()
        v.normal_()
        ws.random_()
        step()
        want, bytes_ = out.clone(), pool.clone()
        pool.copy_(dev(pool_np))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(pool, bytes_)


def test_tensors_that_the_library_cannot_check():
    import torch
    from paper_2402_02446_amd import binding
    pool = binding.lqer_kv4_pool(4, 2, 16, 64)
    k = torch.zeros(3, 2, 64, device="cuda")
    slots = torch.arange(3, dtype=torch.int32, device="cuda")
    for bad in (dict(k=k.half()), dict(v=k.bfloat16()), dict(v=k[:2]), dict(slots=slots.long()), dict(slots=slots[:2]), dict(pool=pool.cpu()),
                dict(pool=pool[:, :1]), dict(k=k[:, :1], v=k[:, :1]), dict(k=k[..., ::2])):
        with pytest.raises(ValueError):
            binding.lqer_kv4_append(**{**dict(pool=pool, k=k, v=k, slots=slots), **bad})
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    i = torch.ones(2, dtype=torch.int32, device="cuda")
    a = dict(pool=pool, q=q, cu_q=i, kv_len=i[:1], table=i[None], max_q=1, max_kv=1, scale=1.0)
    for bad in (dict(q=q.float()), dict(cu_q=i[:1]), dict(kv_len=i), dict(table=i), dict(table=i[None].long()), dict(out=q[:, :2]),
                dict(out=q.half()), dict(pool=pool.to(torch.int8))):
        with pytest.raises(ValueError):
            binding.lqer_kv4_attention(**{**a, **bad})
    with pytest.raises(binding.LqerError):
        binding.lqer_kv4_attention(**{**a, "q": torch.zeros(1, 3, 64, dtype=torch.bfloat16, device="cuda")})
    with pytest.raises(binding.LqerError):
        binding.lqer_kv4_pool(4, 2, 24, 64)


def test_a_workspace_of_its_own_is_contiguous_and_on_the_gpu():
    import torch
    from paper_2402_02446_amd import binding
    pool = binding.lqer_kv4_pool(4, 2, 16, 64)
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    i = torch.ones(2, dtype=torch.int32, device="cuda")
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(256, dtype=torch.uint8, device="cuda")[:, None].expand(256, 4096)):
        with pytest.raises(ValueError):
            binding.lqer_kv4_attention(pool, q, i, i[:1], i[None], 1, 4000, 1.0, workspace=bad)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 12])
def test_windows_as_wide_as_the_type(window):
    """A query before the cache's beginning: its window begins below -2^31."""
    _attend([21, 1], [18, 30], 4, 2, 64, 16, window=window)
    _attend([25, 90], [3, 40], 4, 2, 128, 16, causal=False, window=window)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("tokens, n", [(40, 1), (700, 2), (4000, 1), (300, 40), (3000, 40)])
def test_a_query_that_is_not_finite_spoils_itself_only(bad, tokens, n):
    """Its scores are NaN wherever a key has a zero there, and so is the softmax over them; the other rows keep their bits."""
    import torch
    from paper_2402_02446_amd import binding
    D, P, heads, G = 128, 16, 2, 4
    g = torch.Generator().manual_seed(tokens + n)
    pages = -(-tokens // P)
    pool = binding.lqer_kv4_pool(pages, heads, P, D)
    k, v = (torch.randn(tokens, heads, D, generator=g) for _ in range(2))
    k[:, :, 5] = 0
    v[::3] = 0                                      # (NaN times 0)
    binding.lqer_kv4_append(pool, k.cuda(), v.cuda(), torch.arange(tokens, dtype=torch.int32, device="cuda"))
    q = torch.randn(n, heads * G, D, generator=g).bfloat16().cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    call = lambda: binding.lqer_kv4_attention(pool, q, i32(0, n), i32(tokens), table, n, tokens, D ** -0.5)  # noqa: E731
    want = call()
    q[n // 2, 6, 5] = bad
    got = call()
    assert bool(torch.isnan(got[n // 2, 6]).all())
    got[n // 2, 6] = want[n // 2, 6]
    assert torch.equal(got, want)
