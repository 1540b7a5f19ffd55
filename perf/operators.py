"""The paged cache's calls and the FEM read over it, for timing and comparison.

A case is a plain dict.  ``kind`` names what a serving program does:

  write  fem_cache_append of a batch's new keys and values, then fem_cache_gather
         of its sequences: storing (quantised or not) and reading back
  back   fem_cache_gather alone
  read   fem_paged_fwd: new tokens of every sequence read the cache, causally;
         one token a sequence is a decoding step
  cross  fem_paged_fwd without the causal mask: a decoder's tokens read an
         encoder's states

Sequences are ragged: ``n`` new tokens at most and ``L`` cached tokens at most
(the new ones included), spread by ``spread``; the pages of a sequence are
scattered over the pool.  q, k, v ~ N(0, 1) are slices of one projection's
output, beta is log-uniform.  ``own`` selects the library's calls; else the same
results come from elementary torch operations in 32 bits.
"""

import math
import random

import torch

own = False

DEV = "cuda"
MOST = {"e4m3": 448.0, "int8": 127.0}  # the largest code of a type
LEAST_EXP = -100                       # of a scale
BETA = dict(beta_lo=0.1, beta_hi=8.0)


def listed():
    return [
        # A decoding step's new rows of eight short sequences: the smallest write.
        dict(name="write_step_e4m3", kind="write", kv="e4m3", B=8, Hkv=8, H=8, d=128, dv=128,
             page=16, n=1, L=200, spread="ragged"),
        # Prompts of a batch stored as 8-bit integers.
        dict(name="write_prompt_int8", kind="write", kv="int8", B=6, Hkv=16, H=16, d=128, dv=128,
             page=64, n=4096, L=4096, spread="ragged"),
        # A chunk of each prompt in bf16, half-width values, small pages.
        dict(name="write_chunk_bf16", kind="write", kv="bf16", B=5, Hkv=12, H=12, d=64, dv=32,
             page=32, n=333, L=1777, spread="ragged"),
        # Long contexts handed to a dense read.
        dict(name="back_long_e4m3", kind="back", kv="e4m3", B=4, Hkv=8, H=8, d=128, dv=128,
             page=64, n=1, L=32768, spread="ragged"),
        # One user, one token, a short context: the smallest read.
        dict(name="token_one", kind="read", kv="bf16", B=1, Hkv=8, H=8, d=64, dv=64, page=16,
             n=1, L=701, spread="same", **BETA),
        # An ordinary decoding batch.
        dict(name="token_batch", kind="read", kv="bf16", B=8, Hkv=16, H=16, d=128, dv=128,
             page=64, n=1, L=4096, spread="ragged", **BETA),
        # Long contexts in 8 bits, four query heads to a cached head.
        dict(name="token_long_e4m3", kind="read", kv="e4m3", B=16, Hkv=8, H=32, d=128, dv=128,
             page=64, n=1, L=32768, spread="ragged", **BETA),
        # Eight drafted tokens a sequence checked in one call.
        dict(name="draft_int8", kind="read", kv="int8", B=13, Hkv=8, H=16, d=64, dv=64, page=32,
             n=8, L=8192, spread="ragged", **BETA),
        # Prompts and decoding steps in one call.
        dict(name="mixed_e4m3", kind="read", kv="e4m3", B=12, Hkv=8, H=32, d=128, dv=128, page=64,
             n=700, L=8192, spread="ragged", **BETA),
        # A prompt's next chunk behind a long context.
        dict(name="chunk_large", kind="read", kv="bf16", B=1, Hkv=16, H=16, d=128, dv=128,
             page=64, n=4096, L=16384, spread="same", **BETA),
        # A decoder's tokens over an encoder's states.
        dict(name="cross_ragged", kind="cross", kv="bf16", B=8, Hkv=12, H=12, d=64, dv=64,
             page=64, n=448, L=1500, spread="ragged", **BETA),
        # One decoder token a sequence over the same kind of states, half-width values.
        dict(name="cross_token", kind="cross", kv="int8", B=24, Hkv=8, H=16, d=128, dv=64,
             page=128, n=1, L=1500, spread="ragged", **BETA),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "back", "read", "read", "read", "cross"])
    d, dv = rng.choice([(32, 32), (64, 64), (64, 32), (128, 128), (128, 128), (128, 64)])
    Hkv = _logint(rng, 1, 16)
    G = rng.choice([1, 1, 2, 3, 4, 8])
    case = dict(kind=kind, kv=rng.choice(["bf16", "e4m3", "int8"]), Hkv=Hkv, H=Hkv * G, d=d, dv=dv,
                page=rng.choice([16, 32, 64, 128, 256]), spread=rng.choice(["ragged", "ragged", "same"]))
    if kind in ("write", "back"):
        B = _logint(rng, 1, 32)
        L = _logint(rng, 1, max(2, min(32768, int(3e8 / (B * Hkv * (d + dv))))))
        n = 1 if rng.random() < 0.3 else _logint(rng, 1, L)
        return dict(case, B=B, L=L, n=n)
    B = _logint(rng, 1, 64)
    shape = rng.choice(["token", "draft", "chunk"])
    n = 1 if shape == "token" else rng.randint(2, 16) if shape == "draft" else _logint(rng, 17, 2048)
    # bounds of the work: pairs of a query row and a key, and cached values
    most = min(32768, 5e11 / (B * n * Hkv * G * 2 * (d + dv)), 3e8 / (B * Hkv * (d + dv)))
    L = _logint(rng, 1, max(2, int(most)))
    return dict(case, B=B, n=min(n, L) if kind == "read" else n, L=L, **BETA)


# ---- inputs ------------------------------------------------------------------

def _lengths(case):
    """New tokens and lengths (new tokens included) of the case's sequences."""
    B, n, L, cross = case["B"], case["n"], case["L"], case["kind"] == "cross"
    if case["spread"] == "same":
        return [n] * B, [L] * B
    r = random.Random("%d %d %d" % (B, n, L))
    news = [max(1, int(n * r.random() ** 2)) for _ in range(B)]
    lens = [r.randint((L + 3) // 4, L) for _ in range(B)]
    k = r.randrange(B)
    news[k], lens[k] = n, L  # the largest is there
    return (news, lens) if cross else ([min(a, b) for a, b in zip(news, lens)], lens)


def _quantise(x, kv):
    """Codes [.., d] and scale bytes [.., d / 32] of x [.., d], 32 channels a scale."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    m, e = torch.frexp(top / MOST[kv])
    e = torch.where(m == 0.5, e - 1, e).clamp(min=LEAST_EXP)
    fine = torch.isfinite(top)
    y = torch.ldexp(b, -e.unsqueeze(-1)).masked_fill(~fine.unsqueeze(-1), 0.0).flatten(-2)
    codes = y.to(torch.float8_e4m3fn) if kv == "e4m3" else torch.round(y).to(torch.int8)
    return codes, torch.where(fine, e + 127, 255).to(torch.uint8)


def _dequantise(codes, scale):
    """float32 values of codes [.., d] and scale bytes [.., d / 32]."""
    s = torch.ldexp(torch.ones((), device=codes.device), scale.int() - 127)
    return (codes.float().unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    host = random.Random(int(seed))

    def normal(*shape):
        return torch.randn(shape, device=DEV, dtype=torch.float32, generator=gen)

    B, H, Hkv, d, dv = (case[x] for x in ("B", "H", "Hkv", "d", "dv"))
    page, kv = case["page"], case["kv"]
    news, lens = _lengths(case)
    N = sum(news)
    used = [-(-n // page) for n in lens]
    width = max(used)
    pages = sum(used) + 3
    ids = list(range(pages))
    host.shuffle(ids)
    table, at = [], 0
    for u in used:  # entries past a sequence's pages hold no page
        table.append(ids[at:at + u] + [-1] * (width - u))
        at += u
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    st = dict(case=case, N=N, width=width, n_max=max(news), L=max(lens))
    for name, x in (("table", table), ("q_start", starts), ("lens", lens)):
        st[name] = torch.tensor(x, dtype=torch.int32, device=DEV)
    for name, w in (("k", d), ("v", dv)):
        x = normal(pages, Hkv, page, w)
        if kv == "bf16":
            st[name + "_pool"], st[name + "_scale"] = x.bfloat16(), None
        else:
            st[name + "_pool"], st[name + "_scale"] = _quantise(x.bfloat16(), kv)
    # one projection's output: queries, keys and values of a token side by side
    qkv = normal(N, H * d + Hkv * (d + dv)).bfloat16()
    st["q"] = qkv[:, :H * d].unflatten(1, (H, d))
    st["new_k"] = qkv[:, H * d:H * d + Hkv * d].unflatten(1, (Hkv, d))
    st["new_v"] = qkv[:, H * d + Hkv * d:].unflatten(1, (Hkv, dv))
    if "beta_lo" in case:
        u = torch.rand((Hkv, dv), device=DEV, dtype=torch.float64, generator=gen)
        lo, hi = math.log(case["beta_lo"]), math.log(case["beta_hi"])
        st["beta"] = torch.exp(lo + (hi - lo) * u).float()
        st["out"] = torch.empty((N, H, dv), device=DEV, dtype=torch.bfloat16)
    else:
        st["k_out"] = torch.zeros((B, Hkv, st["L"], d), device=DEV, dtype=torch.bfloat16)
        st["v_out"] = torch.zeros((B, Hkv, st["L"], dv), device=DEV, dtype=torch.bfloat16)
    return st


# ---- one pass ----------------------------------------------------------------

def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        return _run_own(s, kind)
    if kind == "write":
        _plain_append(s)
    return _plain_gather(s) if kind in ("write", "back") else _plain_read(s, kind == "cross")


def _run_own(s, kind):
    from paper_2602_07160_amd import binding

    if "cache" not in s:  # descriptions of the program's buffers, kept as the buffers are
        s["cache"] = binding.PagedCache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
        s["batch"] = binding.PagedBatch(s["q_start"], s["lens"], s["table"], s["N"], s["n_max"])
        if "out" in s:
            need = binding.fem_paged_workspace_bytes(s["cache"], s["batch"], s["case"]["H"])
            s["ws"] = torch.empty(need, device=DEV, dtype=torch.uint8) if need else None
    if kind == "write":
        binding.fem_cache_append(s["cache"], s["batch"], s["new_k"], s["new_v"])
    if kind in ("write", "back"):
        return binding.fem_cache_gather(s["cache"], s["batch"], s["k_out"], s["v_out"])
    return binding.fem_paged_fwd(s["cache"], s["batch"], s["q"], s["beta"], causal=kind != "cross",
                                 out=s["out"], ws=s["ws"])


def _tokens(s):
    """Sequence of each new token and its index among the sequence's."""
    t = torch.arange(s["N"], device=DEV)
    ends = s["q_start"][1:].long()
    b = torch.searchsorted(ends, t, right=True)
    return b, t - s["q_start"].long()[b]


def _plain_append(s):
    page = s["case"]["page"]
    b, i = _tokens(s)
    news = (s["q_start"][1:] - s["q_start"][:-1]).long()
    pos = s["lens"].long()[b] - news[b] + i
    pg, at = s["table"].long()[b, pos // page], pos % page
    for name in ("k", "v"):
        x, scale = s["new_" + name], s[name + "_scale"]
        if scale is None:
            s[name + "_pool"][pg, :, at] = x
        else:
            codes, e = _quantise(x, s["case"]["kv"])
            s[name + "_pool"].view(torch.uint8)[pg, :, at] = codes.view(torch.uint8)
            scale[pg, :, at] = e


def _rows(s, name):
    """float32 rows [B, Hkv, width * page, w] of every sequence, in order."""
    ids = s["table"].long().clamp(min=0)
    x = s[name + "_pool"]
    if s[name + "_scale"] is not None:
        x = x.view(torch.uint8)[ids].view(x.dtype)
        x = _dequantise(x, s[name + "_scale"][ids])
    else:
        x = x[ids].float()
    return x.transpose(1, 2).flatten(2, 3)


def _plain_gather(s):
    L = s["L"]
    for name in ("k", "v"):
        x, out = _rows(s, name)[:, :, :L], s[name + "_out"]
        valid = torch.arange(L, device=DEV) < s["lens"][:, None]
        out.copy_(torch.where(valid[:, None, :, None], x.to(out.dtype), out))
    return s["k_out"], s["v_out"]


def _plain_read(s, cross):
    """softmax, exp(beta v - c) with c a channel's largest, their product, its log."""
    d, H, Hkv = s["case"]["d"], s["case"]["H"], s["case"]["Hkv"]
    k, v = _rows(s, "k"), _rows(s, "v")
    B, n, S = k.shape[0], s["n_max"], k.shape[2]
    b, i = _tokens(s)
    starts, lens = s["q_start"].long(), s["lens"].long()
    news = starts[1:] - starts[:-1]
    at = (starts[:-1, None] + torch.arange(n, device=DEV)).clamp(max=s["N"] - 1)
    q = s["q"][at].float().unflatten(2, (Hkv, H // Hkv))       # [B, n, Hkv, G, d]
    q = q.permute(0, 2, 1, 3, 4).flatten(2, 3)                 # [B, Hkv, n G, d]
    key = torch.arange(S, device=DEV)
    live = key < lens[:, None]                                 # [B, S]
    if cross:
        seen = live[:, None, :].expand(B, n, S)
    else:
        last = (lens - news)[:, None] + torch.arange(n, device=DEV)
        seen = (key <= last[:, :, None]) & live[:, None, :]
    hidden = ~seen.repeat_interleave(H // Hkv, 1)[:, None]     # [B, 1, n G, S]
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d))
    p.masked_fill_(hidden, -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    norm = p.sum(-1, keepdim=True)
    beta = s["beta"][None, :, None, :]
    x = (v * beta).masked_fill_(~live[:, None, :, None], -math.inf)
    c = x.amax(2, keepdim=True)
    e = x.sub_(c).exp_()
    o = (torch.log(torch.matmul(p, e) / norm) + c) / beta      # [B, Hkv, n G, dv]
    o = o.unflatten(2, (n, H // Hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s["out"].copy_(o[b, i])
    return s["out"]


def work(case):
    """Bytes and operations of the pass: inputs read once, outputs written once;
    multiply-adds counted as two, exponentials not at all."""
    news, lens = _lengths(case)
    N, rows = sum(news), sum(lens) * case["Hkv"]
    Hkv, H, d, dv = case["Hkv"], case["H"], case["d"], case["dv"]
    w = d + dv
    held = 2 * w if case["kv"] == "bf16" else w + w // 32       # bytes of a cached row
    if case["kind"] in ("write", "back"):
        new = N * Hkv if case["kind"] == "write" else 0
        # reading back takes the rows just written from the cache again
        return {"bytes": new * (2 * w + held) + rows * (held + 2 * w), "flops": rows * w}
    if case["kind"] == "cross":
        pairs = sum(a * b for a, b in zip(news, lens))
    else:
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(news, lens))
    return {"bytes": rows * held + N * H * 2 * w, "flops": pairs * H * 2 * w}


# ---- the same results in 64 bits -------------------------------------------------

def _value64(codes, scale, kv):
    """float64 values of a pool, from the meaning of its bits."""
    if scale is None:
        return codes.double()
    if kv == "int8":
        x = codes.double()
    else:  # e4m3: sign, four bits of exponent (bias 7), three of fraction
        u = codes.view(torch.uint8).int()
        exp, frac = (u >> 3) & 15, (u & 7).double()
        x = torch.where(exp == 0, frac / 512, (1 + frac / 8) * torch.exp2((exp - 7).double()))
        x = torch.where(u >= 128, -x, x)
    return x * torch.exp2(scale.double() - 127).repeat_interleave(32, -1)


def _store64(x, kv):
    """The values that float64 x [.., w] has once stored: per 32 channels the
    smallest step whose codes reach the largest value, ties to even."""
    if kv == "bf16":
        return x
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True).clamp(min=1e-300)
    e = torch.ceil(torch.log2(top / MOST[kv]) - 1e-12).clamp(min=LEAST_EXP)
    y = b / torch.exp2(e)
    if kv == "int8":
        step = torch.ones_like(y)
    else:  # three bits below the leading one, the smallest step 2^-9
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    news, lens = _lengths(case)
    kv, page, kind = case["kv"], case["page"], case["kind"]
    B, H, Hkv, d, dv = (case[x] for x in ("B", "H", "Hkv", "d", "dv"))
    G, starts, pages = H // Hkv, s["q_start"].tolist(), s["table"].tolist()

    def sequence(b, name):
        ids = pages[b][:-(-lens[b] // page)]
        pool, scale = s[name + "_pool"], s[name + "_scale"]
        x = _value64(pool.view(torch.uint8)[ids].view(pool.dtype) if scale is not None else pool[ids],
                     None if scale is None else scale[ids], kv)
        x = x.transpose(0, 1).flatten(1, 2)[:, :lens[b]].clone()
        if kind == "write":
            new = s["new_" + name][starts[b]:starts[b + 1]].double().transpose(0, 1)
            x[:, lens[b] - news[b]:] = _store64(new, kv)
        return x

    if kind in ("write", "back"):
        outs = []
        for name, w in (("k", d), ("v", dv)):
            o = torch.zeros((B, Hkv, s["L"], w), device=DEV, dtype=torch.float64)
            for b in range(B):
                o[b, :, :lens[b]] = sequence(b, name)
            outs.append(o)
        return tuple(outs)
    out = torch.empty((s["N"], H, dv), device=DEV, dtype=torch.float64)
    beta = s["beta"].double()
    for b in range(B):
        k, v = sequence(b, "k"), sequence(b, "v")
        q = s["q"][starts[b]:starts[b + 1]].double()
        n = news[b]
        first = lens[b] - n
        for g in range(Hkv):
            x = v[g] * beta[g]
            c = x.amax(0)
            e = torch.exp(x - c)
            for t0 in range(0, n, 1024):  # bounds the [rows, keys] matrices
                t1 = min(n, t0 + 1024)
                a = torch.matmul(q[t0:t1, g * G:(g + 1) * G].reshape(-1, d), k[g].t()) / math.sqrt(d)
                if kind == "read":
                    last = first + torch.arange(t0, t1, device=DEV).repeat_interleave(G)
                    a.masked_fill_(torch.arange(lens[b], device=DEV) > last[:, None], -math.inf)
                p = torch.softmax(a, -1)
                o = (torch.log(torch.matmul(p, e)) + c) / beta[g]
                out[starts[b] + t0:starts[b] + t1, g * G:(g + 1) * G] = o.reshape(t1 - t0, G, dv)
    return out
