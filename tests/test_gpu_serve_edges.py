"""The calls between a block's linears on numbers below the smallest normal one, and on a stream other than the default.

Blocks whose largest magnitude is below 2^-127 have the exponent byte 0 (the oracle's lower limit): codes, bytes and values are asserted equal.
Attention over such values: what is below 2^-126 may be lost, on top of the bound of tests/test_gpu_kv4_weights.py."""
import numpy as np
import pytest

from oracle import block, mxint

pytestmark = pytest.mark.gpu
# magnitudes of a block's values: normal, around the smallest normal number, the smallest ones of either type
GAINS = [1.0, 2.0 ** -120, 2.0 ** -126, 2.0 ** -127, 2.0 ** -130, 2.0 ** -133, 2.0 ** -140, 2.0 ** -148]


def _gains(n):
    return np.repeat(np.resize(GAINS, n // 16), 16).astype(np.float64)


@pytest.mark.parametrize("bits", [8, 6])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm(bits, dtype):
    import torch
    from paper_2402_02446_amd import binding
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(bits)
    x = torch.randn(5, 256, generator=g)
    x[1:3] *= 2.0 ** -120
    x[3, 1:] = 0
    x[3, 0] = 2.0 ** -130
    r = (torch.randn(5, 256, generator=g) * torch.from_numpy(_gains(256)).float()).to(t)
    x = x.to(t)
    w = (torch.randn(256, generator=g).double() * torch.from_numpy(_gains(256))).to(t)
    for residual in (None, r):
        h = x.float() if residual is None else x.float() + r.float()
        for eps in (0.0, 1e-5):
            codes, exps, _, values = binding.lqer_rmsnorm_mx(x.cuda(), w.cuda(), eps, residual=None if residual is None else r.cuda(), elem_bits=bits, values=True)
            oc, oe = mxint.mx_quantize(block.rmsnorm(h.double().numpy(), w.double().numpy(), float(np.float32(eps))), bits)
            assert np.array_equal(exps.cpu().numpy(), oe) and np.array_equal(codes.cpu().numpy(), oc)
            assert np.array_equal(values.double().cpu().numpy(), mxint.mx_dequantize(oc, oe, bits))
            assert oe.min() == 0


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cache(D, dtype):
    import torch
    from paper_2402_02446_amd import binding
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    T, heads, P = 40, 2, 16
    rng = np.random.default_rng(D)
    k, v = (torch.from_numpy(rng.standard_normal((T, heads, D))) for _ in range(2))
    k[7] *= torch.from_numpy(_gains(D))
    v *= torch.from_numpy(_gains(D))
    v[3] = 2.0 ** -149
    k, v = k.to(t), v.to(t)
    pool = torch.full((3, heads, P * D * 9 // 8), 0, dtype=torch.uint8, device="cuda")
    binding.lqer_kv4_append(pool, k.cuda(), v.cuda(), torch.arange(T, dtype=torch.int32, device="cuda"))
    want = np.zeros(pool.shape, np.uint8)
    kv = []
    for which, x in enumerate((k, v)):
        c, e = block.kv4_quantize(x.double().numpy())
        for i in range(T):
            for h in range(heads):
                block.kv4_store(want, P, D, i // P, h, i % P, which, c[i, h], e[i, h])
        kv.append(block.kv4_values(c, e).reshape(x.shape))
    assert np.array_equal(pool.cpu().numpy(), want)
    for n in (1, 40):                               # few rows and many
        q = torch.from_numpy(rng.standard_normal((n, heads * 2, D)).astype(np.float32)).bfloat16()
        i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        out = torch.empty(n, heads * 2, D, device="cuda")
        binding.lqer_kv4_attention(pool, q.cuda(), i32(0, n), i32(T), i32(0, 1, 2)[None], n, T, D ** -0.5, out=out)
        for h in range(heads * 2):
            o, mag = block.attention(q[:, h].double().numpy(), kv[0][:, h // 2], kv[1][:, h // 2], float(np.float32(D ** -0.5)), np.zeros(n, int), T - n + 1 + np.arange(n))
            bound = ((2.0 ** -16 if n * 2 <= 64 else 2.0 ** -8) + 2.0 ** -12) * mag + 2.0 ** -126
            assert np.all(np.abs(out[:, h].double().cpu().numpy() - o) <= bound)


def test_on_another_stream():
    """Inputs made, calls made and results used on a stream of their own, beside other work on the default one."""
    import torch
    from paper_2402_02446_amd import binding as lqer
    D, P, heads, G, T = 64, 16, 2, 2, 150
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    w, A, B = torch.rand(512, device="cuda"), torch.randn(3, 8, 512, device="cuda").bfloat16(), torch.randn(3, 256, 8, device="cuda").bfloat16()
    table, slots, cu, kv = torch.arange(10, dtype=torch.int32, device="cuda")[None], torch.arange(T, dtype=torch.int32, device="cuda"), i32(0, T), i32(T)
    ids = slots % 4 - 1
    base = torch.randn(T, 512, device="cuda")
    busy = torch.randn(4096, 4096, device="cuda")

    def program():
        x = base
        for _ in range(30):                         # (what the calls read is still on its way when they are made)
            x = torch.sin(x + busy[0, :512])
        codes, exps, h, values = lqer.lqer_rmsnorm_mx(x, w, residual=base, values=True)
        y = lqer.lqer_adapters_forward(values, ids, A, B, h[:, :256].contiguous())
        pool = lqer.lqer_kv4_pool(10, heads, P, D)
        pool.zero_()
        lqer.lqer_kv4_append(pool, y[:, :128].unflatten(1, (2, 64)), y[:, 128:].unflatten(1, (2, 64)), slots)
        out = lqer.lqer_kv4_attention(pool, y.bfloat16().view(T, heads * G, D), cu, kv, table, T, T, 0.125)
        return codes, exps, h, values, y, pool, out
    torch.cuda.synchronize()
    want = program()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        for _ in range(4):
            busy @ busy                             # (the default stream is busy; the other does not wait for it)
        with torch.cuda.stream(side):
            got = program()
        side.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
