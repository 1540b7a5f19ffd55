"""GPU checks of the read over a paged cache (fem_paged_fwd) against the float64
oracle, through the binding.

Tolerance, per element of channel j with value range R_j over its sequence
(u = 2^-8, the largest relative rounding of a bf16):

  u R_j / 2            probabilities enter the product rounded to bf16, and their
                       sum adds the same rounded numbers: the read moves by at most
                       (1/beta) u |q - p|_1 (q the posterior), and |q - p|_1 is at
                       most beta R / 2
  u / beta             exponentials rounded to bf16, channels with beta >= 0.5
  2^-15 / beta         their hi + lo parts otherwise
  2e-5 / beta + 2e-5   float32 sums, scores and logarithms (log2 of a partial sum
                       has magnitude up to 128: half a step is 4e-6)
  u |o|                a bf16 output

A quantised cache holds bf16 numbers, so its read is compared with the same bits:
the read over a bf16 cache that holds them.
"""

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


class Call:
    """A filled cache, a batch and queries."""

    def __init__(self, fem, news, lens, Hkv, G, d, dv, page, kv="bf16", seed=0, beta=(0.1, 8.0), tail=0,
                 qs=1.0, vs=1.0, causal=True, stale=float("nan"), extra=1, q_pad=0):
        self.fem, self.news, self.lens, self.Hkv, self.G, self.causal = fem, news, lens, Hkv, G, causal
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        used = [-(-n // page) for n in lens]
        pages, width = sum(used) + extra, max(max(used), 1)
        ids = rng.permutation(pages)
        table, at = np.full((len(lens), width), 1 << 30, dtype=np.int32), 0
        for b, u in enumerate(used):
            table[b, :u] = ids[at:at + u]
            at += u
        self.starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        N = int(self.starts[-1]) + tail
        self.table, self.page = table, page
        src = fem.PagedCache.empty(pages, Hkv, d, dv, page)
        src.k.normal_(generator=g)
        src.v.normal_(generator=g).mul_(vs)
        if kv != "bf16":  # store every row, then hold its values in bf16 too
            rows = pages * page
            all_ = fem.PagedBatch(torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                                  torch.tensor([rows], dtype=torch.int32, device="cuda"),
                                  torch.arange(pages, dtype=torch.int32, device="cuda")[None], rows)
            self.cache = fem.PagedCache.empty(pages, Hkv, d, dv, page, DT[kv])
            flat = [x.transpose(1, 2).reshape(rows, Hkv, -1).contiguous() for x in (src.k, src.v)]
            fem.fem_cache_append(self.cache, all_, *flat)
            back = fem.fem_cache_gather(self.cache, all_)
            for x, o in zip((src.k, src.v), back):
                x.copy_(o[0].unflatten(1, (pages, page)).transpose(0, 1))
            self.same = src
        else:
            self.cache = src
        for b, n in enumerate(lens):  # what lies behind a sequence is anything
            if n % page and kv == "bf16":
                p = int(table[b, n // page])
                src.k[p, :, n % page:] = stale
                src.v[p, :, n % page:] = stale
            elif n % page:
                p = int(table[b, n // page])
                for x in (self.cache.k, self.cache.v):
                    x.view(torch.uint8)[p, :, n % page:] = 0x7f
                for x in (self.cache.k_scale, self.cache.v_scale):
                    x[p, :, n % page:] = 255
        self.batch = fem.PagedBatch(*[torch.from_numpy(x.copy()).cuda() for x in
                                      (self.starts, np.asarray(lens, np.int32), table)],
                                    n_tok=N, max_q=max(max(news), 1))
        wide = torch.randn((N, Hkv * G * d + q_pad), device="cuda", generator=g).mul_(qs).bfloat16()
        self.q = wide[:, :Hkv * G * d].unflatten(1, (Hkv * G, d))
        u = torch.rand((Hkv, dv), device="cuda", generator=g, dtype=torch.float64)
        self.beta = (beta[0] * (beta[1] / beta[0]) ** u).float()

    def read(self, cache=None, **kw):
        out = self.fem.fem_paged_fwd(cache or self.cache, self.batch, self.q, self.beta,
                                     causal=self.causal, **kw)
        torch.cuda.synchronize()
        return out

    def rows(self, name):
        """float64 [Hkv, n, w] of every sequence, from the bf16 pool of its values."""
        pool = getattr(getattr(self, "same", self.cache), name)
        got = []
        for b, n in enumerate(self.lens):
            x = pool[self.table[b, :-(-n // self.page)].tolist()].double().transpose(0, 1).flatten(1, 2)
            got.append(x[:, :n].cpu().numpy())
        return got

    def check(self, out):
        ks, vs = self.rows("k"), self.rows("v")
        beta = self.beta.double().cpu().numpy()
        want = oracle.fem_paged(self.q.double().cpu().numpy(), ks, vs, beta, self.starts, self.causal)
        got = out.double().cpu().numpy()
        worst = 0.0
        for b in range(len(self.lens)):
            t0, t1 = int(self.starts[b]), int(self.starts[b + 1])
            if t1 == t0:
                continue
            if self.lens[b] == 0:
                assert np.isnan(got[t0:t1]).all()
                continue
            R = (vs[b].max(1) - vs[b].min(1)).repeat(self.G, 0)
            bt = beta.repeat(self.G, 0)
            tol = 2.0 ** -9 * R + np.where(bt >= 0.5, 2.0 ** -8, 2.0 ** -15) / bt + 2e-5 / bt + 2e-5
            tol = tol[None] + (2.0 ** -8 * np.abs(want[t0:t1]) if out.dtype == torch.bfloat16 else 0.0)
            err = np.abs(got[t0:t1] - want[t0:t1])
            assert np.isfinite(got[t0:t1]).all()
            assert (err <= tol).all(), (b, float((err / tol).max()), float(err.max()))
            worst = max(worst, float((err / tol).max()))
        print(f"   worst error over its tolerance {worst:.2f}", flush=True)
        return want


def say(*a):
    print("[case]", *a, flush=True)


@pytest.mark.parametrize("d,dv", [(32, 32), (64, 64), (64, 32), (128, 128), (128, 64)])
@pytest.mark.parametrize("kv", list(DT))
@pytest.mark.parametrize("page,news,lens", [
    (16, [1], [1]),
    (16, [1, 1, 1, 1], [1, 31, 32, 500]),
    (64, [3, 1, 9, 0, 2], [3, 130, 64, 70, 33]),
    (32, [40, 2], [41, 900]),
])
def test_widths_and_types(fem, d, dv, kv, page, news, lens):
    say(d, dv, kv, page, news, lens)
    c = Call(fem, news, lens, 2, 2, d, dv, page, kv)
    out = c.read()
    c.check(out)
    if kv != "bf16":
        assert torch.equal(out, c.read(cache=c.same))


@pytest.mark.parametrize("G", [1, 3, 4, 8, 16, 17, 33])
@pytest.mark.parametrize("n", [1, 2, 5])
def test_groups(fem, G, n):
    say("groups", G, n)
    c = Call(fem, [n, 1, n], [n, 77, 300], 2, G, 64, 64, 16, seed=G)
    c.check(c.read())


@pytest.mark.parametrize("news,lens", [
    ([15], [15]), ([16], [16]), ([17], [17]), ([31], [95]), ([32], [64]), ([33], [33]),
    ([63, 64, 65], [63, 128, 200]), ([127, 128, 129, 1], [127, 300, 129, 600]),
    ([255, 257, 300], [255, 257, 1111]), ([700], [1500]),
])
@pytest.mark.parametrize("causal", [True, False])
def test_chunks(fem, news, lens, causal):
    say("chunks", news, lens, causal)
    c = Call(fem, news, lens, 2, 1, 64, 64, 64, causal=causal, seed=len(news))
    c.check(c.read())


@pytest.mark.parametrize("kv", list(DT))
@pytest.mark.parametrize("d,dv", [(128, 128), (64, 32), (32, 32), (128, 64)])
def test_chunk_types(fem, kv, d, dv):
    say("chunk", kv, d, dv)
    c = Call(fem, [150, 1, 70, 300], [400, 333, 70, 301], 2, 2, d, dv, 32, kv, seed=7)
    out = c.read()
    c.check(out)
    if kv != "bf16":
        assert torch.equal(out, c.read(cache=c.same))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
def test_pages(fem, page):
    say("page", page)
    c = Call(fem, [1, 70, 5], [1030, 333, 5], 3, 1, 64, 64, page, seed=page)
    c.check(c.read())


def test_encoder_lengths(fem):
    """Lengths that have nothing to do with the tokens', an empty one among them."""
    say("encoder lengths")
    c = Call(fem, [3, 50, 2, 1, 0, 200], [1, 0, 700, 33, 9, 64], 2, 3, 64, 64, 16, causal=False)
    c.check(c.read())


def test_long_context_splits(fem):
    say("long contexts, one token and a few")
    c = Call(fem, [1, 4, 1], [20000, 9001, 1], 2, 1, 64, 64, 256)
    c.check(c.read())


def test_many_sequences(fem):
    """More sequences than a wave has lanes, some without tokens."""
    say("many sequences")
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(1, 200, 150)]
    news = [int(min(n, rng.integers(0, 4))) for n in lens]
    c = Call(fem, news, lens, 2, 2, 32, 32, 16)
    c.check(c.read())


@pytest.mark.parametrize("causal", [True, False])
def test_many_sequences_of_all_sizes(fem, causal):
    """More sequences than lanes, chunks and single tokens mixed."""
    say("many sequences of all sizes", causal)
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(1, 900, 90)]
    news = [int(min(n, rng.choice([0, 1, 1, 1, 33, 150]))) for n in lens]
    c = Call(fem, news, lens, 2, 1, 64, 64, 16, "int8", causal=causal, seed=4, tail=3)
    out = c.read()
    c.check(out)
    assert torch.equal(out[:-3], c.read(cache=c.same)[:-3])


@pytest.mark.parametrize("kv", list(DT))
def test_chunks_and_tokens_with_long_contexts(fem, kv):
    """Both kinds of rows split over their keys in one call."""
    say("chunks and tokens", kv)
    c = Call(fem, [1, 70, 1, 300, 2], [9000, 5000, 1, 6100, 3000], 2, 2, 64, 64, 64, kv, seed=6)
    c.check(c.read())


def test_shared_pages(fem):
    """Two sequences whose first pages are the same ones."""
    say("shared pages")
    for n in (1, 50):
        c = Call(fem, [n, n], [320, 320], 2, 1, 64, 64, 64, seed=n)
        c.table[1, :4] = c.table[0, :4]
        c.batch.table.copy_(torch.from_numpy(c.table))
        c.check(c.read())


@pytest.mark.parametrize("beta", [(1e-3, 1e-3), (0.499, 0.501), (16.0, 64.0)])
def test_temperatures(fem, beta):
    say("beta", beta)
    c = Call(fem, [1, 40], [300, 500], 2, 1, 64, 64, 64, beta=beta)
    c.check(c.read())


@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (32, 32)])
@pytest.mark.parametrize("news", [[1, 2], [140, 300]])
def test_wide_ranges(fem, news, d, dv):
    """Scores spread over hundreds of octaves and values too: sums that fall out of
    the kernels' common frames are formed again."""
    say("wide ranges", news, d, dv)
    c = Call(fem, news, [700, 300], 1, 1, d, dv, 64, qs=40.0, vs=12.0, beta=(1.0, 16.0), seed=11)
    c.check(c.read())


@pytest.mark.parametrize("n", [1, 90, 200])
def test_opposed_ranges(fem, n):
    """The likeliest key holds the smallest value of every channel."""
    say("opposed", n)
    c = Call(fem, [n], [n + 200], 1, 1, 64, 64, 64, beta=(16.0, 16.0), seed=12)
    pg = c.table[0]
    c.cache.v[pg[0], 0, 3] = -12.0
    c.cache.k[pg[0], 0, 3] = 60.0
    c.cache.v[pg[0], 0, 40] = 12.0
    c.cache.k[pg[0], 0, 40] = -60.0
    c.q.abs_()
    c.check(c.read())


@pytest.mark.parametrize("n", [1, 3, 60, 200])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size(fem, n, sign):
    """Scores near the ends of float32, all of one sign: one key has all the weight."""
    say("huge scores", n, sign)
    c = Call(fem, [n], [n + 300], 1, 2, 64, 64, 64, seed=13, stale=0.0)
    c.cache.k.abs_().mul_(sign * 1e15)
    c.q.abs_().mul_(1e20)
    c.check(c.read())


@pytest.mark.parametrize("kv", ["bf16", "int8"])
@pytest.mark.parametrize("news,lens", [([1], [9000]), ([3, 1], [700, 5000]), ([40], [3000]), ([70], [70])])
def test_large_scores_that_differ_little(fem, news, lens, kv):
    """Every score is 126976 and a small part, exactly; only the small parts count."""
    say("offset scores", news, lens, kv)
    c = Call(fem, news, lens, 1, 4, 64, 64, 64, kv=kv, seed=14, stale=0.0)
    c.q[:] = 64.0
    c.q[..., 1], c.q[..., 32:] = 0.125, 0.0  # 31 x 64 x 512 / sqrt(64), and j / 8
    rows = getattr(c, "same", c.cache).k
    j = torch.arange(rows.shape[0] * rows.shape[2], device="cuda").view(-1, 1, rows.shape[2]) * 7 % 33
    rows[:], rows[..., 1] = 512.0, (8 * j).bfloat16()
    if kv != "bf16":
        c.cache.k[:], c.cache.k[..., 1] = 64, j.to(torch.int8)
        c.cache.k_scale[:] = 127 + 3
    c.check(c.read())


def test_beta_anywhere(fem):
    """beta needs no alignment of its own."""
    say("beta")
    c = Call(fem, [1, 40], [3000, 500], 2, 1, 64, 64, 64)
    want = c.read()
    c.beta = torch.cat((c.beta.new_zeros(1), c.beta.flatten()))[1:].view(2, 64)
    assert c.beta.data_ptr() % 16 and torch.equal(c.read(), want)


def test_outputs_and_padding(fem):
    """bf16 output; rows behind the last sequence and sequences without tokens."""
    say("outputs")
    for news, lens in (([2, 0, 3], [50, 10, 3]), ([80, 0, 100], [90, 10, 333])):
        c = Call(fem, news, lens, 2, 2, 64, 64, 16, tail=5)
        f = torch.full((sum(news) + 5, 4, 64), 9.0, device="cuda")
        h = f.bfloat16()
        c.read(out=f)
        c.read(out=h)
        c.check(f)
        c.check(h)
        assert (f[sum(news):] == 9.0).all() and (h[sum(news):] == 9.0).all()
        assert torch.equal(f.bfloat16(), h)


def test_strided_queries_and_streams(fem):
    say("strided")
    c = Call(fem, [5, 60], [100, 60], 2, 2, 64, 64, 16, q_pad=72)
    assert not c.q.is_contiguous()
    a = c.read()
    c.check(a)
    assert torch.equal(a, c.read())  # the same bits
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    assert torch.equal(a, c.read(stream=s))
    need = fem.fem_paged_workspace_bytes(c.cache, c.batch, 4)
    ws = torch.full((need + 512,), 0xa5, dtype=torch.uint8, device="cuda")
    assert torch.equal(a, c.read(ws=ws[:need]))
    assert (ws[need:] == 0xa5).all()


def test_two_workspaces_at_once(fem):
    say("two streams")
    c = [Call(fem, [1, 3, 100], [900, 800, 700], 2, 1, 64, 64, 16, seed=s) for s in (1, 2)]
    want = [x.read() for x in c]
    streams = [torch.cuda.Stream() for _ in c]
    outs = []
    for x, s in zip(c, streams):
        s.wait_stream(torch.cuda.current_stream())
        outs.append(fem.fem_paged_fwd(x.cache, x.batch, x.q, x.beta, stream=s))
    torch.cuda.synchronize()
    for a, b in zip(want, outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("wide", [False, True])
def test_contradictions_read_nan(fem, wide):
    """Lengths and pages that cannot be: those sequences are NaN, the others whole."""
    say("contradictions", wide)
    n = 90 if wide else 2
    news, lens = [n] * 6, [n + 40] * 6
    c = Call(fem, news, lens, 2, 1, 64, 64, 16)
    want = c.read().clone()
    c.check(want)
    c.batch.lens[1] = n - 1                         # shorter than the new tokens
    c.batch.lens[2] = c.batch.table.shape[1] * 16 + 1
    c.batch.table[3, 1] = c.cache.c.pages
    c.batch.table[4, 0] = -1
    out = c.read()
    for b in range(6):
        part = out[b * n:(b + 1) * n]
        if b in (0, 5):
            assert torch.equal(part, want[b * n:(b + 1) * n])
        elif b in (1, 2, 4):
            assert part.isnan().all(), b
        else:  # page 1 holds keys that every row of these sizes sees
            assert part.isnan().all(), b
    few = fem.PagedBatch(c.batch.q_start, torch.tensor(lens, dtype=torch.int32).cuda(),
                         torch.from_numpy(c.table).cuda(), 6 * n, n - 1)
    assert fem.fem_paged_fwd(c.cache, few, c.q, c.beta).isnan().all()


def test_starts_that_do_not_ascend(fem):
    """Nothing outside the buffers is touched; the call ends."""
    say("starts")
    c = Call(fem, [4, 4, 4], [40, 50, 60], 2, 1, 64, 64, 16)
    for bad in ([0, 9, 3, 12], [-5, 4, 8, 12], [0, 4, 8, 10 ** 9], [12, 8, 4, 0]):
        b = fem.PagedBatch(torch.tensor(bad, dtype=torch.int32).cuda(), c.batch.lens, c.batch.table, 12, 4)
        guard = torch.full((16, 2, 64), 5.0, device="cuda")
        fem.fem_paged_fwd(c.cache, b, c.q, c.beta, out=guard[2:14])
        fem.fem_cache_append(c.cache, b, c.q, c.q)
        torch.cuda.synchronize()
        assert (guard[:2] == 5.0).all() and (guard[14:] == 5.0).all()


def test_offsets_past_32_bits(fem):
    """A pool of more than 4 GiB whose last pages are in use."""
    say("large pool")
    pages, page = 70000, 256  # K and V: 70000 * 1 * 256 * 128 * 2 bytes = 4.6e9 each
    cache = fem.PagedCache.empty(pages, 1, 128, 128, page)
    g = torch.Generator(device="cuda").manual_seed(5)
    small = Call(fem, [1, 70], [600, 500], 1, 1, 128, 128, page, seed=5)
    table = small.table.copy()
    for b, n in enumerate(small.lens):
        for i in range(-(-n // page)):
            far = pages - 1 - 7 * b - i
            cache.k[far], cache.v[far] = small.cache.k[int(table[b, i])], small.cache.v[int(table[b, i])]
            table[b, i] = far
    batch = fem.PagedBatch(small.batch.q_start, small.batch.lens, torch.from_numpy(table).cuda(), 71, 70)
    out = fem.fem_paged_fwd(cache, batch, small.q, small.beta)
    torch.cuda.synchronize()
    assert torch.equal(out, small.read())
    k = torch.randn((71, 1, 128), device="cuda", generator=g).bfloat16()
    fem.fem_cache_append(cache, batch, k, k)
    ko, vo = fem.fem_cache_gather(cache, batch)
    torch.cuda.synchronize()
    assert torch.equal(ko[0, 0, 599], k[0, 0]) and torch.equal(vo[1, 0, 430:500], k[1:, 0])


def test_capture_replays(fem):
    """A decoding loop's step captured once: append, then read, with tokens, lengths
    and tables changing between replays, each replay against the eager call."""
    say("capture")
    for G, n in ((2, 1), (1, 40)):
        c = Call(fem, [n, n, n], [900, 300, 700], 2, G, 64, 64, 16, kv="e4m3")
        k, v = (torch.randn((3 * n, 2, 64), device="cuda").bfloat16() for _ in range(2))
        out = torch.empty((3 * n, 2 * G, 64), device="cuda", dtype=torch.bfloat16)
        ws = torch.empty(max(fem.fem_paged_workspace_bytes(c.cache, c.batch, 2 * G), 1),
                         dtype=torch.uint8, device="cuda")

        def step():
            fem.fem_cache_append(c.cache, c.batch, k, v)
            fem.fem_paged_fwd(c.cache, c.batch, c.q, c.beta, out=out, ws=ws)

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for i in range(4):
            c.batch.lens.sub_(torch.tensor([3, 50, 1], dtype=torch.int32, device="cuda") * i)
            k.normal_()
            c.q.normal_()
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            got = out.clone()
            step()
            torch.cuda.synchronize()
            # sequence 1 ends with no length left (300 - 50 - 100 - 150): NaN
            live = (c.batch.lens >= n).repeat_interleave(n)
            assert live.sum() == (3 * n if i < 3 else 2 * n)
            assert torch.equal(got[live], out[live]) and torch.isfinite(got[live]).all(), (G, i)
            assert got[~live].isnan().all() and out[~live].isnan().all()


def test_with_the_dense_reads(fem):
    """A prompt stored in chunks and read as it is stored, then decoded, against the
    dense read of the whole and the dense decoding step over the gathered rows."""
    say("dense")
    H, d, T, page = 4, 64, 200, 16
    g = torch.Generator(device="cuda").manual_seed(9)
    q, k, v = (torch.randn((T, H, d), device="cuda", generator=g).bfloat16() for _ in range(3))
    beta = (0.2 + 4 * torch.rand((H, d), device="cuda", generator=g))
    dense = fem.fem_softmax_fwd(*(x.transpose(0, 1).contiguous()[None] for x in (q, k, v)), beta)[0]
    cache = fem.PagedCache.empty(20, H, d, page=page)
    table = torch.randperm(20, device="cuda", generator=g)[:13].int()[None].contiguous()
    at, parts = 0, []
    for n in (70, 1, 1, 100, 27, 1):
        at += n
        batch = fem.PagedBatch(torch.tensor([0, n], dtype=torch.int32).cuda(),
                               torch.tensor([at], dtype=torch.int32).cuda(), table, n)
        fem.fem_cache_append(cache, batch, k[at - n:at], v[at - n:at])
        parts.append(fem.fem_paged_fwd(cache, batch, q[at - n:at], beta))
    got = torch.cat(parts).transpose(0, 1)
    assert at == T and (got - dense).abs().max() <= 4e-2  # two reads of 2e-2 each
    kc, vc = fem.fem_cache_gather(cache, batch)
    assert torch.equal(kc[0, :, :T], k.transpose(0, 1)) and torch.equal(vc[0, :, :T], v.transpose(0, 1))
    step = fem.fem_softmax_decode(q[-1:].contiguous(), kc, vc, beta, lens=batch.lens)
    assert (step[0] - got[:, -1]).abs().max() <= 2e-2


def test_binding_checks(fem):
    c = Call(fem, [2], [9], 2, 2, 64, 64, 16)
    for kw in (dict(q=c.q.float()), dict(q=c.q[:1]), dict(q=c.q[:, :, :32]), dict(q=c.q.cpu()),
               dict(beta=c.beta[:1]), dict(beta=c.beta.double()),
               dict(out=torch.empty(2, 4, 32, device="cuda")), dict(out_dtype=torch.float16),
               dict(out=torch.empty(2, 4, 64, dtype=torch.float16, device="cuda"))):
        args = dict(q=c.q, beta=c.beta)
        args.update(kw)
        with pytest.raises(ValueError):
            fem.fem_paged_fwd(c.cache, c.batch, **args)
    with pytest.raises(fem.FemError) as e:
        fem.fem_paged_fwd(c.cache, c.batch, c.q[:, :3], c.beta)
    assert e.value.status == 2
