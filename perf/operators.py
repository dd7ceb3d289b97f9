"""What the operators between two linear calls of a served decoder block are judged by: one pass of a call on new data.

A case's `op`:

  norm       residual addition, root-mean-square norm, MXINT codes of the result (lqer_rmsnorm_mx): what the linears of
             a block are handed.  Comes back: the new residual stream and the values that the codes stand for.
  adapters   the low-rank adapters of many requests on the output of a shared linear (lqer_adapters_forward)
  attention  one step of a paged cache held in MXINT4: the step's keys and values are appended, then its queries attend
             (lqer_kv4_append, lqer_kv4_attention).  Comes back: the attention's output and the cache's bytes, which two
             right programs write alike, bit for bit.

The plain forms are elementary torch operations in fp32 on whole tensors: every request padded to the longest, every
adapter applied to every token and masked.
"""
import math
import random

import torch

DEV = "cuda"
own = False


# ---- the cases --------------------------------------------------------------------------------------------------------
def _norm(name, rows, cols, x="f32", residual="f32", bits=8, pad=0):
    """x and residual: their types ("none": no residual); pad: values between x's rows"""
    return dict(name=name, op="norm", rows=rows, cols=cols, x=x, residual=residual, bits=bits, pad=pad)


def _adapters(name, M, K, N, R, adapters, ids="mixed", none=0.0, ragged=False):
    """R: the rank that the stacked adapters have room for, ragged: they have lower ones of their own; ids: each token's
    adapter by itself, or runs of tokens (prompts) with one; none: the share of tokens (or runs) that have none"""
    return dict(name=name, op="adapters", M=M, K=K, N=N, R=R, adapters=adapters, ids=ids, none=none, ragged=ragged)


def _attention(name, requests, q_len, ctx, q_heads, kv_heads, dim, page, window=0, ragged=False, kv="bf16"):
    """ctx: cached tokens of the longest request, this step's among them; ragged: requests of other lengths, empty ones
    among them; window: how many tokens back a query sees (0: all); kv: the type that new keys and values come in"""
    return dict(name=name, op="attention", requests=requests, q_len=q_len, ctx=ctx, q_heads=q_heads, kv_heads=kv_heads,
                dim=dim, page=page, window=window, ragged=ragged, kv=kv)


def listed():
    return [
        # one token of one chat in front of the q/k/v of a 7B-shaped block: latency
        _norm("norm_7b_m1", 1, 4096),
        # a short prompt of 6-bit activations, x a slice of a wider buffer, on a size that no tile divides
        _norm("norm_ragged_m203", 203, 4112, x="bf16", bits=6, pad=24),
        # prefill of a batch of prompts on the 70B-shaped block, the residual stream in bf16
        _norm("norm_70b_m8192", 8192, 8192, residual="bf16"),
        # 16 chats decoded together, each with an adapter of its own or a neighbour's, beside a 7B-shaped linear
        _adapters("adapters_7b_m16", 16, 4096, 4096, 16, 32),
        # a verification batch on odd sizes: low ranks, some tokens without an adapter
        _adapters("adapters_ragged_m203", 203, 4112, 11000, 24, 9, none=0.2, ragged=True),
        # 64 chats beside the 70B-shaped MLP up projection, adapters of up to 64 ranks: the stream of their weights
        _adapters("adapters_70b_m64", 64, 8192, 28672, 64, 48, none=0.1, ragged=True),
        # prefill of prompts with an adapter each beside the same linear: the largest Y
        _adapters("adapters_70b_m4096", 4096, 8192, 28672, 32, 6, ids="runs"),
        # the next token of one chat on a 7B-shaped block (every query head its own cache): latency
        _attention("attend_7b_m1", 1, 1, 517, 32, 32, 128, 16, kv="f32"),
        # 16 chats of mixed lengths decoded together on a 70B-shaped block (8 query heads to a cached one)
        _attention("attend_70b_m16", 16, 1, 4096, 64, 8, 128, 64, ragged=True),
        # four long documents: the cache's stream is what counts
        _attention("attend_70b_long", 4, 1, 100003, 64, 8, 128, 64),
        # verification of up to five proposed tokens under a sliding window, small heads, odd sizes
        _attention("attend_verify_window", 37, 5, 1501, 14, 2, 64, 16, window=1000, ragged=True),
        # a chunk of two prompts on what is cached of them, 70B-shaped: matrix products
        _attention("attend_70b_chunk", 2, 2048, 6144, 64, 8, 128, 64, ragged=True),
    ]


def _log(rng, lo, hi, step=1):
    """log-uniform in [lo, hi], a multiple of step"""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step
    return min(max(v, -(-lo // step) * step), hi // step * step)


def draw(rng):
    op = rng.choice(["norm", "adapters", "attention", "attention"])
    if op == "norm":
        cols = _log(rng, 256, 11008, 16)
        c = _norm("", min(_log(rng, 1, 16384), 8192 * 8192 // cols), cols, x=rng.choice(["f32", "f32", "bf16"]),
                  residual=rng.choice(["f32", "f32", "bf16", "none"]), bits=rng.choice([8, 8, 6]), pad=rng.choice([0, 0, 8, 104]))
    elif op == "adapters":
        K, N, n = _log(rng, 512, 8192, 16), _log(rng, 512, 11008, rng.choice([1, 4, 16, 128])), _log(rng, 1, 64)
        R = rng.choice([8, 16, 16, 24, 32, 64, 128])
        n = max(1, min(n, int(48 * 64 * (8192 + 28672) / (R * (K + N)))))
        # (the plain form applies every adapter to every token)
        M = max(1, min(_log(rng, 1, 8192), int(4096 * 6 * 32 * (8192 + 28672) / (n * R * (K + N)))))
        c = _adapters("", M, K, N, R, n, ids=rng.choice(["mixed", "runs"]), none=rng.choice([0.0, 0.0, 0.3]), ragged=rng.random() < 0.5)
    else:
        kv_heads, group, dim = rng.choice([1, 2, 8, 8, 32]), rng.choice([1, 1, 4, 7, 8, 16]), rng.choice([64, 128, 128, 256])
        group = min(group, 64 // kv_heads)
        group = max(group, 1)
        kind = rng.choice(["decode", "decode", "verify", "chunk"])
        q_len = {"decode": 1, "verify": rng.randint(2, 9), "chunk": _log(rng, 10, 4096)}[kind]
        requests = _log(rng, 1, 4 if kind == "chunk" else 128)
        ctx = max(q_len, _log(rng, 1, 8192 if kind == "chunk" else 65536))
        q_heads = kv_heads * group
        # no more cache, and no more pairs of query and key, than the listed ones have
        ctx = max(1, min(ctx, 4 * 100003 * 8 * 128 // (requests * kv_heads * dim)))
        q_len = max(1, min(q_len, ctx, 2 * 2048 * 6144 * 64 * 128 // (requests * ctx * q_heads * dim)))
        window = rng.choice([0, 0, 0, _log(rng, 1, 4096)])
        c = _attention("", requests, q_len, ctx, q_heads, kv_heads, dim, rng.choice([16, 16, 32, 64, 128, 256]), window=window,
                       ragged=rng.random() < 0.7, kv=rng.choice(["bf16", "bf16", "f32"]))
    del c["name"]
    return c


# ---- inputs, from the seed alone ------------------------------------------------------------------------------------------
def _gen(seed, *what):
    g = torch.Generator(device=DEV)
    s = int(seed) & 0x7FFFFFFF
    for w in what:
        s = (s * 1000003 + int(w) + 17) % (1 << 61)
    g.manual_seed(s)
    return g


def _randn(seed, what, *shape, type="f32"):
    return torch.randn(*shape, generator=_gen(seed, what), device=DEV).to(torch.bfloat16 if type == "bf16" else torch.float32)


def _lengths(c):
    """(new tokens, cached tokens with them) of every request: the case's own"""
    r = random.Random("%d %d %d %d" % (c["requests"], c["q_len"], c["ctx"], c["page"]))
    got = [(c["q_len"], c["ctx"])]
    for _ in range(c["requests"] - 1):
        if not c["ragged"]:
            got.append(got[0])
            continue
        n = c["q_len"] if c["q_len"] == 1 else r.randint(1, c["q_len"])
        t = r.randint(max(n, c["ctx"] // 8), max(n, c["ctx"]))
        got.append((0, 0) if r.random() < 0.05 else (n, t))
    r.shuffle(got)
    return got


def _ids(c):
    """every token's adapter (-1: none): the case's own"""
    r = random.Random("%d %d %d %d %s" % (c["M"], c["K"], c["N"], c["adapters"], c["ids"]))
    got = []
    while len(got) < c["M"]:
        a = -1 if r.random() < c["none"] else r.randrange(c["adapters"])
        got += [a] * (1 if c["ids"] == "mixed" else r.randint(1, max(1, c["M"] // 4)))
    return got[: c["M"]]


def _ranks(c):
    r = random.Random("%d %d" % (c["R"], c["adapters"]))
    return [r.randint(1, c["R"]) if c["ragged"] and i else c["R"] for i in range(c["adapters"])]


def _words(v):
    """fp32 [.., D] -> MXINT4 in blocks of 16 along D: code words [.., D / 8][4 bytes] and exponent bytes [.., D / 16].
    Byte i of a word: |e_i| in bits 0-2, the sign of e_(4 + (i + 3) % 4) in bit 3, |e_(4 + i)| in bits 4-6, the sign of e_i in bit 7."""
    b = v.reshape(*v.shape[:-1], -1, 16)
    amax = b.abs().amax(-1)
    e = torch.where(amax > 0, torch.frexp(amax)[1] - 1, torch.full_like(amax, -127, dtype=torch.int32)).clamp(max=120)
    codes = torch.round(torch.ldexp(b, torch.where(amax > 0, 2 - e, 0).unsqueeze(-1))).clamp(-7, 7).to(torch.int8)
    codes = codes.reshape(*v.shape[:-1], -1, 2, 4)
    size, sign = codes.abs(), (codes < 0).to(torch.int8)
    low, high = size[..., 0, :], size[..., 1, :]
    words = low | (sign[..., 1, :].roll(1, -1) << 3) | (high << 4)
    return words.view(torch.uint8) | (sign[..., 0, :].view(torch.uint8) << 7), (e + 127).to(torch.uint8)


def _parts(pool, P, D):
    """The four parts of every page's record, as views [pages][heads] ..: keys' words [P][D / 8][4], values' words
    [P / 4][D / 8][4 tokens][4], keys' exponents [P][D / 16], values' exponents [P / 4][D / 16][4 tokens]."""
    n, h = pool.shape[:2]
    at = [0, P * D // 2, P * D, P * D * 17 // 16, P * D * 9 // 8]
    kw, vw, ke, ve = (pool[:, :, a:b] for a, b in zip(at, at[1:]))
    return (kw.unflatten(2, (P, D // 8, 4)), vw.unflatten(2, (P // 4, D // 8, 4, 4)),
            ke.unflatten(2, (P, D // 16)), ve.unflatten(2, (P // 4, D // 16, 4)))


def _keys(seed, what, heads, n, D):
    """keys with the few large channels that keys have"""
    k = _randn(seed, what, n, heads, D)
    big = torch.randint(0, D, (heads, 4), generator=_gen(seed, 41), device=DEV)
    gain = torch.ones(heads, D, device=DEV).scatter_(1, big, 4.0)
    return k * gain


def prepare(case, seed):
    c = case
    if c["op"] == "norm":
        x = _randn(seed, 1, c["rows"], c["cols"] + c["pad"], type=c["x"])[:, : c["cols"]]
        x[:, :: 97] *= 20.0                              # outlier channels
        s = dict(c, X=x, weight=1.0 + 0.1 * _randn(seed, 2, c["cols"]), eps=1e-5, h=None)
        if c["residual"] != "none":
            s["R"] = _randn(seed, 3, c["rows"], c["cols"], type=c["residual"]) * 3.0
            s["h"] = torch.empty_like(s["R"])
        return s
    if c["op"] == "adapters":
        M, K, N, R, n = (c[k] for k in ("M", "K", "N", "R", "adapters"))
        ranks = torch.tensor(_ranks(c), dtype=torch.int32, device=DEV)
        room = torch.arange(R, device=DEV) < ranks[:, None]                        # [n][R]
        A = (_randn(seed, 1, n, R, K) * room[:, :, None] / math.sqrt(K)).bfloat16()
        B = (_randn(seed, 2, n, N, R) * room[:, None, :] * 0.2).bfloat16()
        ldy = (N + 3) // 4 * 4
        return dict(c, X=_randn(seed, 3, M, K, type="bf16"), A=A, B=B, ranks=ranks,
                    scales=0.5 + torch.rand(n, generator=_gen(seed, 4), device=DEV),
                    ids=torch.tensor(_ids(c), dtype=torch.int32, device=DEV),
                    Y=torch.randn(M, ldy, generator=_gen(seed, 5), device=DEV)[:, :N],
                    out=torch.empty(M, ldy, device=DEV)[:, :N])
    H, G, D, P = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["page"]
    lens = _lengths(c)
    pages = [-(-t // P) for _, t in lens]
    used = sum(pages)
    order = torch.randperm(used + 3, generator=_gen(seed, 6), device=DEV).to(torch.int32)
    table = torch.full((len(lens), max(max(pages), 1)), -1, dtype=torch.int32)
    at, order_h, slots, request, position = 0, order.cpu(), [], [], []
    for b, (n, t) in enumerate(lens):
        table[b, : pages[b]] = order_h[at: at + pages[b]]
        at += pages[b]
        pos = torch.arange(t - n, t)
        slots.append(table[b][pos // P] * P + pos % P)
        request.append(torch.full((n,), b))
        position.append(torch.arange(n))
    pool = torch.empty(used + 3, H, P * D * 9 // 8, dtype=torch.uint8, device=DEV)
    kw, vw, ke, ve = _parts(pool, P, D)
    for lo in range(0, used + 3, max(1, (1 << 27) // (H * P * D))):
        hi = min(used + 3, lo + max(1, (1 << 27) // (H * P * D)))
        w, e = _words(_keys(seed, 100 + lo, H, (hi - lo) * P, D).view(hi - lo, P, H, D).transpose(1, 2))
        kw[lo:hi], ke[lo:hi] = w, e
        w, e = _words(_randn(seed, 100000000 + lo, hi - lo, H, P, D))
        vw[lo:hi] = w.unflatten(2, (P // 4, 4)).transpose(3, 4)
        ve[lo:hi] = e.unflatten(2, (P // 4, 4)).transpose(3, 4)
    T = sum(n for n, _ in lens)
    t = torch.bfloat16 if c["kv"] == "bf16" else torch.float32
    if c["kv"] == "bf16":                                # one buffer of q, k and v, as a fused projection leaves it
        qkv = torch.empty(T, H * G + 2 * H, D, dtype=t, device=DEV)
        q, k, v = qkv[:, : H * G], qkv[:, H * G: H * G + H], qkv[:, H * G + H:]
    else:
        q = torch.empty(T, H * G, D, dtype=torch.bfloat16, device=DEV)
        k, v = (torch.empty(T, H, D, device=DEV) for _ in range(2))
    q.copy_(_randn(seed, 7, T, H * G, D))
    k.copy_(_keys(seed, 8, H, T, D))
    v.copy_(_randn(seed, 9, T, H, D))
    dev = lambda x, dt=torch.int32: x.to(dt).to(DEV)  # noqa: E731
    return dict(c, pool=pool, q=q, k=k, v=v, table=dev(table), slots=dev(torch.cat(slots)),
                cu_q=dev(torch.tensor([0] + [n for n, _ in lens]).cumsum(0)), kv_len=dev(torch.tensor([t for _, t in lens])),
                q_lens=dev(torch.tensor([n for n, _ in lens])), request=dev(torch.cat(request), torch.int64),
                position=dev(torch.cat(position), torch.int64), scale=1.0 / math.sqrt(D))


# ---- the plain forms --------------------------------------------------------------------------------------------------------
def _plain_norm(s):
    h = s["X"].float()
    if s["h"] is not None:
        h = h + s["R"].float()
    v = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * s["weight"]
    b = v.unflatten(-1, (-1, 16))
    amax = b.abs().amax(-1, keepdim=True)
    f = s["bits"] - 2
    e = torch.where(amax > 0, torch.frexp(amax)[1] - 1, torch.zeros_like(amax, dtype=torch.int32))
    top = 2 ** (s["bits"] - 1) - 1
    values = torch.ldexp(torch.round(torch.ldexp(b, f - e)).clamp(-top, top), e - f).flatten(-2).bfloat16()
    return values if s["h"] is None else (h.to(s["h"].dtype), values)


def _plain_adapters(s):
    n, R, K = s["A"].shape
    N = s["N"]
    X, A, Bt = s["X"].float(), s["A"].float().view(n * R, K), s["B"].float().transpose(0, 1).reshape(N, n * R)
    mine = (s["ids"][:, None] == torch.arange(n, dtype=torch.int32, device=DEV)) * s["scales"]        # [M][n]
    T = (X @ A.t()).view(-1, n, R) * mine[:, :, None]
    return s["Y"] + T.view(-1, n * R) @ Bt.t()


def _plain_values(words, exps):
    """code words [.., tokens, D / 8, 4] and exponent bytes [.., tokens, D / 16] -> fp32 [.., tokens, D]"""
    w = words.to(torch.int8)                             # (bit 7 is the sign)
    low, high = (w & 7), ((w >> 4) & 7)
    low = torch.where(w < 0, -low, low)
    high = torch.where((w.roll(-1, -1) & 8) > 0, -high, high)
    codes = torch.stack([low, high], -2).flatten(-3).float()                     # [.., tokens, D]
    return torch.ldexp(codes.unflatten(-1, (-1, 16)), exps.to(torch.int32).unsqueeze(-1) - 129).flatten(-2)


def _plain_attention(s):
    P, D, H, G = s["page"], s["dim"], s["kv_heads"], s["q_heads"] // s["kv_heads"]
    kw, vw, ke, ve = _parts(s["pool"], P, D)
    page, off = (s["slots"] // P).long(), (s["slots"] % P).long()
    kw[page, :, off], ke[page, :, off] = _words(s["k"].float())
    vw[page, :, off // 4, :, off % 4], ve[page, :, off // 4, :, off % 4] = _words(s["v"].float())

    table = s["table"].clamp(min=0).long()               # [B][pages]: its records, then tokens in order
    n = table.shape[0]
    order = lambda x: x[table].transpose(1, 2).flatten(2, 3)  # noqa: E731  [B][pages][H][P] .. -> [B][H][pages * P] ..
    K = _plain_values(order(kw), order(ke))
    V = _plain_values(order(vw.transpose(3, 4).reshape(*vw.shape[:2], P, D // 8, 4)),
                      order(ve.transpose(3, 4).reshape(*ve.shape[:2], P, D // 16)))
    L = s["q_len"]
    q = torch.zeros(n, L, H, G, D, device=DEV)
    q[s["request"], s["position"]] = s["q"].float().unflatten(1, (H, G))
    S = (q.permute(0, 2, 1, 3, 4).reshape(n, H, L * G, D) @ K.transpose(2, 3)) * s["scale"]
    at = (s["kv_len"] - s["q_lens"])[:, None] + torch.arange(L, device=DEV)       # [B][L]: the queries' own positions
    t = torch.arange(K.shape[2], device=DEV)
    seen = t <= at[..., None]                            # [B][L][tokens]
    if s["window"]:
        seen = seen & (t > at[..., None] - s["window"])
    S = S.unflatten(2, (L, G)).masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = S.amax(-1, keepdim=True)
    p = torch.exp(S - torch.where(top == -math.inf, 0.0, top))
    O = (p.flatten(2, 3) @ V).unflatten(2, (L, G)) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = O.permute(0, 2, 1, 3, 4)[s["request"], s["position"]].flatten(1, 2)     # [tokens][heads][D]
    return out.bfloat16(), s["pool"]


def run(state):
    s = state
    if not own:
        return {"norm": _plain_norm, "adapters": _plain_adapters, "attention": _plain_attention}[s["op"]](s)
    from paper_2402_02446_amd import binding
    if s["op"] == "norm":
        _, _, h, values = binding.lqer_rmsnorm_mx(s["X"], s["weight"], s["eps"], residual=s.get("R"), h_out=s["h"],
                                                  elem_bits=s["bits"], values=True)
        return values if h is None else (h, values)
    if s["op"] == "adapters":
        return binding.lqer_adapters_forward(s["X"], s["ids"], s["A"], s["B"], s["Y"], out=s["out"],
                                             ranks=s["ranks"], scales=s["scales"])
    binding.lqer_kv4_append(s["pool"], s["k"], s["v"], s["slots"])
    out = binding.lqer_kv4_attention(s["pool"], s["q"], s["cu_q"], s["kv_len"], s["table"], max_q=s["q_len"],
                                     max_kv=s["ctx"], scale=s["scale"], window=s["window"])
    return out, s["pool"]


# ---- what a pass cannot do without, and how exact it is ---------------------------------------------------------------------
def work(case):
    c = case
    size = {"f32": 4, "bf16": 2, "none": 0}
    if c["op"] == "norm":
        n = c["rows"] * c["cols"]
        # x, the residual in and out, codes, exponent bytes, values
        return {"bytes": n * (size[c["x"]] + 2 * size[c["residual"]] + 1 + 1 / 16 + 2) + 4 * c["cols"], "flops": 8 * n}
    if c["op"] == "adapters":
        ids, ranks = _ids(c), _ranks(c)
        used = sum(ranks[a] for a in set(ids) if a >= 0)
        fl = sum(2 * ranks[a] * (c["K"] + c["N"]) for a in ids if a >= 0)
        with_one = sum(a >= 0 for a in ids)
        return {"bytes": with_one * c["K"] * 2 + used * (c["K"] + c["N"]) * 2 + 8 * c["M"] * c["N"], "flops": fl}
    D, H, W = c["dim"], c["kv_heads"], c["window"]
    read, pairs, new = 0, 0, 0
    for n, t in _lengths(c):
        new += n
        read += min(t, W + n - 1) if W else t            # tokens that any of the request's queries sees
        pairs += sum(min(t - n + i + 1, W) if W else t - n + i + 1 for i in range(n))
    return {"bytes": read * H * D * 9 / 8 + new * D * (4 * c["q_heads"] + 2 * H * (size[c["kv"]] + 9 / 16)),
            "flops": 4 * D * c["q_heads"] * pairs}


def _exact_cells(pool, P, D, which, table, t):
    """fp64 [t][heads][D] of one request's keys (which = 0) or values (1), token by token from the record's bytes"""
    at = torch.arange(t, device=DEV)
    page, off = table[at // P].long(), at % P
    rec = pool[page]                                     # [t][heads][bytes]
    d = torch.arange(D, device=DEV)
    word = off[:, None] * (D // 8) + d // 8 if which == 0 else ((off // 4)[:, None] * (D // 8) + d // 8) * 4 + (off % 4)[:, None]
    block = off[:, None] * (D // 16) + d // 16 if which == 0 else ((off // 4)[:, None] * (D // 16) + d // 16) * 4 + (off % 4)[:, None]
    base, ebase = (0, P * D) if which == 0 else (P * D // 2, P * D * 17 // 16)
    j = d % 8
    pick = lambda i: torch.gather(rec, 2, i[:, None, :].expand(-1, rec.shape[1], -1)).long()  # noqa: E731
    size = (pick(base + word * 4 + j % 4) >> torch.where(j < 4, 0, 4)) & 7
    sign = (pick(base + word * 4 + torch.where(j < 4, j, (j + 1) % 4)) >> torch.where(j < 4, 7, 3)) & 1
    return torch.ldexp((size * (1 - 2 * sign)).double(), pick(ebase + block) - 129)


def _exact_mx(v, bits):
    """The values of MXINT codes of fp64 numbers, blocks of 16 along the last axis"""
    b = v.reshape(-1, 16)
    top = b.abs().max(1, keepdim=True).values
    unit = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - (bits - 2))
    m = 2 ** (bits - 1) - 1
    return (torch.round(b / unit).clamp(-m, m) * unit).reshape(v.shape)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm":
        h = s["X"].double() + (s["R"].double() if s["h"] is not None else 0.0)
        v = h / torch.sqrt(h.square().sum(1, keepdim=True) / c["cols"] + s["eps"]) * s["weight"].double()
        values = _exact_mx(v, c["bits"])
        return values if s["h"] is None else (h, values)
    if c["op"] == "adapters":
        out, ids = s["Y"].double(), s["ids"].long()
        for a in range(c["adapters"]):
            rows = (ids == a).nonzero().flatten()
            if rows.numel():
                t = s["X"][rows].double() @ s["A"][a].double().t()
                out[rows] += float(s["scales"][a]) * (t @ s["B"][a].double().t())
        return out
    P, D, H, G = c["page"], c["dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, t) in enumerate(_lengths(c)):
        if n == 0:
            continue
        K, V = (_exact_cells(s["pool"], P, D, w, s["table"][b], t) for w in (0, 1))
        K[t - n:] = _exact_mx(s["k"][first: first + n].double(), 4)
        V[t - n:] = _exact_mx(s["v"][first: first + n].double(), 4)
        at, pos = torch.arange(t - n, t, device=DEV), torch.arange(t, device=DEV)
        seen = pos <= at[:, None]
        if c["window"]:
            seen &= pos > at[:, None] - c["window"]
        for h in range(H * G):
            S = (s["q"][first: first + n, h].double() @ K[:, h // G].t()) * s["scale"]
            out[first: first + n, h] = torch.softmax(S.masked_fill(~seen, -math.inf), -1) @ V[:, h // G]
        first += n
    return out, None
