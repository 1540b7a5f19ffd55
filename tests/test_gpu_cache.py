"""GPU checks of storing into the paged cache and reading it back
(fem_cache_append, fem_cache_gather) against the float64 oracle, through the
binding.  Stored codes, scales and values are exact, so every comparison is for
equality, over the whole pools: slots that no new token has keep their bytes."""

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def setup(fem, kv, heads, d, dv, page, news, lens, seed=0, extra=2, tail=0, fill=0x55):
    """A cache whose bytes are all `fill`, and a batch with scattered pages."""
    rng = np.random.default_rng(seed)
    used = [-(-n // page) for n in lens]
    width = max(max(used), 1)
    ids = rng.permutation(sum(used) + extra)
    table, at = np.full((len(lens), width), -7, dtype=np.int32), 0
    for b, u in enumerate(used):
        table[b, :u] = ids[at:at + u]
        at += u
    cache = fem.PagedCache.empty(sum(used) + extra, heads, d, dv, page, DT[kv])
    for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        if x is not None:
            x.view(torch.uint8).fill_(fill)
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    n_tok = int(starts[-1]) + tail
    dev = [torch.from_numpy(x.copy()).cuda() for x in (starts, np.asarray(lens, np.int32), table)]
    batch = fem.PagedBatch(*dev, n_tok=n_tok, max_q=max(max(news), 1))
    return cache, batch, starts, table, n_tok


def bits(x):
    return x.contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16).cpu().numpy()


def expected(cache_bits, scale_bits, x, kv, table, news, lens, starts, page):
    """The pools' bits after the rows x [N, heads, w] are stored."""
    pool = cache_bits.copy()
    scale = None if scale_bits is None else scale_bits.copy()
    if kv != "bf16":
        codes, byte = oracle.codes_of(x.double().numpy(), kv)
    for b in range(len(news)):
        for i in range(news[b]):
            pos, t = lens[b] - news[b] + i, starts[b] + i
            pg, at = table[b][pos // page], pos % page
            if kv == "bf16":
                pool[pg, :, at] = x[t].view(torch.int16).numpy()
            else:
                pool[pg, :, at], scale[pg, :, at] = codes[t], byte[t]
    return pool, scale


def check(cache, batch, k, v, kv, table, news, lens, starts, fem, stream=None):
    page = cache.c.page
    before = [None if x is None else bits(x) for x in (cache.k, cache.k_scale, cache.v, cache.v_scale)]
    fem.fem_cache_append(cache, batch, k, v, stream=stream)
    torch.cuda.synchronize()
    for i, (x, pool, scale) in enumerate(((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale))):
        want = expected(before[2 * i], before[2 * i + 1], x.cpu().contiguous(), kv, table, news, lens,
                        starts, page)
        assert np.array_equal(bits(pool), want[0])
        if scale is not None:
            assert np.array_equal(bits(scale), want[1])


def draw(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-12, 12, shape[:1] + (1,) * (len(shape) - 1),
                                                                  generator=g).float())
    return x.bfloat16()


@pytest.mark.parametrize("kv", list(DT))
@pytest.mark.parametrize("heads,d,dv,page,news,lens", [
    (1, 32, 32, 16, [1], [1]),
    (3, 64, 64, 16, [1, 1, 1, 1], [1, 16, 17, 33]),
    (2, 64, 32, 32, [5, 0, 33, 64], [5, 9, 100, 64]),
    (5, 128, 64, 64, [7, 130], [70, 131]),
    (16, 128, 128, 256, [40, 1, 3], [600, 257, 256]),
])
def test_append_and_gather(fem, kv, heads, d, dv, page, news, lens):
    print("[case]", kv, heads, d, dv, page, news, lens, flush=True)
    cache, batch, starts, table, n = setup(fem, kv, heads, d, dv, page, news, lens, tail=2)
    k, v = draw(1, n, heads, d), draw(2, n, heads, dv)
    check(cache, batch, k.cuda(), v.cuda(), kv, table, news, lens, starts, fem)
    L = max(lens) + 3
    outs = [torch.full((len(lens), heads, L, w), 7.0, dtype=torch.bfloat16, device="cuda")
            for w in (d, dv)]
    got = fem.fem_cache_gather(cache, batch, *outs)
    torch.cuda.synchronize()
    assert got[0] is outs[0] and got[1] is outs[1]
    for x, pool, scale, o in ((k, cache.k, cache.k_scale, outs[0]), (v, cache.v, cache.v_scale, outs[1])):
        p = bits(pool)
        if kv == "bf16":
            vals = pool.float().cpu().numpy().astype(np.float64)
        else:
            vals = oracle.values_of(p, bits(scale), kv)
        want = np.full(o.shape, 7.0)
        for b, ln in enumerate(lens):
            for i in range(ln):
                want[b, :, i] = vals[table[b][i // page], :, i % page]
        assert np.array_equal(o.double().cpu().numpy(), want, equal_nan=True)
        new = oracle.stored(x.double().numpy(), kv)  # the rows just written, by value
        for b, ln in enumerate(lens):
            for i in range(news[b]):
                assert np.array_equal(want[b, :, ln - news[b] + i], new[starts[b] + i])


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_borders(fem, kv):
    """Zeros, the least scale, ties, the largest bf16, inf and NaN."""
    top = oracle.paged.LARGEST[kv]
    cache, batch, starts, table, n = setup(fem, kv, 2, 64, 64, 16, [9], [9])
    x = torch.zeros(9, 2, 64)
    x[1, 0, 3] = 2.0 ** -126
    x[2, 0, 5], x[2, 1, 40] = float("inf"), float("-inf")
    x[3, 1, 63] = float("nan")
    x[4, 0, :32] = torch.tensor([top] + [0.5, 1.5, -2.5, 3.5, -0.5] + [0.0] * 26)
    x[5, :, 7] = 3.3895313892515355e38
    x[6, 0, 0], x[6, 0, 1] = top * 2.0 ** -100, 2.0 ** -109
    x[7, 1] = -torch.arange(64) / 8.0
    x[8, 0] = torch.tensor([224.0, 17.0, 18.0, 19.0, 20.0, 21.0, 22.0, 23.0] * 8)
    x = x.bfloat16()
    check(cache, batch, x.cuda(), (-x).cuda(), kv, table, [9], [9], starts, fem)


@pytest.mark.parametrize("kv", list(DT))
def test_strided_slices(fem, kv):
    """Keys and values as slices of one projection's output."""
    news, lens = [3, 1, 20], [30, 1, 20]
    cache, batch, starts, table, n = setup(fem, kv, 4, 64, 32, 16, news, lens)
    x = draw(3, n, 8 + 4 * 64 + 16 + 4 * 32).cuda()
    k, v = x[:, 8:8 + 256].unflatten(1, (4, 64)), x[:, -128:].unflatten(1, (4, 32))
    assert not k.is_contiguous() and not v.is_contiguous()
    check(cache, batch, k, v, kv, table, news, lens, starts, fem)


@pytest.mark.parametrize("kv", list(DT))
def test_another_stream(fem, kv):
    news, lens = [17], [40]
    cache, batch, starts, table, n = setup(fem, kv, 2, 128, 128, 32, news, lens)
    k, v = draw(4, n, 2, 128).cuda(), draw(5, n, 2, 128).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check(cache, batch, k, v, kv, table, news, lens, starts, fem, stream=s)


def test_nothing_without_a_slot(fem):
    """Bad pages, lengths past the table, more new tokens than max_q's range or the
    length: such rows are not stored, the other sequences' are."""
    news, lens = [2, 3, 4, 2], [18, 9, 20, 33]
    cache, batch, starts, table, n = setup(fem, "e4m3", 2, 32, 32, 16, news, lens)
    k, v = draw(6, n, 2, 32).cuda(), draw(7, n, 2, 32).cuda()
    t = batch.table.clone()
    pages = cache.c.pages
    t[0, 1], t[2, 1] = pages, -1          # their new tokens' page (0: both; 2: positions 16..19)
    bad_lens = batch.lens.clone()
    bad_lens[3] = t.shape[1] * 16 + 1     # past the table
    bad = fem.PagedBatch(batch.q_start, bad_lens, t, n, 4)
    before = [bits(x) for x in (cache.k, cache.k_scale, cache.v, cache.v_scale)]
    fem.fem_cache_append(cache, bad, k, v)
    torch.cuda.synchronize()
    for i, (x, pool, scale) in enumerate(((k, cache.k, cache.k_scale), (v, cache.v, cache.v_scale))):
        want = expected(before[2 * i], before[2 * i + 1], x.cpu(), "e4m3", table, [0, 3, 0, 0], lens,
                        starts, 16)
        # sequence 1's rows start at token 2
        assert np.array_equal(bits(pool), want[0]) and np.array_equal(bits(scale), want[1])
    short = fem.PagedBatch(batch.q_start, torch.tensor([1, -1, 3, 1], dtype=torch.int32).cuda(),
                           batch.table, n, 4)  # each shorter than its new tokens
    now = [bits(x) for x in (cache.k, cache.k_scale, cache.v, cache.v_scale)]
    fem.fem_cache_append(cache, short, k, v)
    torch.cuda.synchronize()
    assert all(np.array_equal(a, bits(x)) for a, x in
               zip(now, (cache.k, cache.k_scale, cache.v, cache.v_scale)))


def test_gather_of_bad_pages_and_lengths(fem):
    cache, batch, starts, table, n = setup(fem, "int8", 2, 32, 64 // 2, 16, [0] * 4, [40, 16, 5, 30],
                                           fill=0x70)
    t = batch.table.clone()
    t[0, 1] = cache.c.pages + 5
    lens = torch.tensor([40, -3, 0, 16 * t.shape[1] + 1], dtype=torch.int32).cuda()
    b2 = fem.PagedBatch(None, lens, t)
    k = torch.full((4, 2, 33, 32), 3.0, dtype=torch.bfloat16, device="cuda")  # L below a length
    got, v = fem.fem_cache_gather(cache, b2, k=k)
    torch.cuda.synchronize()
    val = 0x70 * 2.0 ** (0x70 - 127)
    g = got.float().cpu()
    assert (g[0, :, :16] == val).all() and g[0, :, 16:32].isnan().all() and (g[0, :, 32] == val).all()
    assert (g[1:] == 3.0).all()
    assert (v[1:] == 0).all() and v.shape == (4, 2, 33, 32)


def test_capture_replays(fem):
    """Append and read-back captured once, replayed with other tokens, lengths and
    pages, beside eager work."""
    news, lens = [1, 1, 1], [5, 16, 33]
    cache, batch, starts, table, n = setup(fem, "e4m3", 2, 64, 64, 16, news, [48, 48, 48], fill=0)
    batch.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    batch.q_start.copy_(torch.tensor([0, 1, 2, 3], dtype=torch.int32))
    k, v = draw(8, 3, 2, 64).cuda(), draw(9, 3, 2, 64).cuda()
    ko, vo = (torch.zeros((3, 2, 48, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fem.fem_cache_append(cache, batch, k, v)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fem.fem_cache_append(cache, batch, k, v)
        fem.fem_cache_gather(cache, batch, ko, vo)
    held = [{}, {}, {}]
    for step in range(4):
        k.copy_(draw(20 + step, 3, 2, 64))
        v.copy_(draw(30 + step, 3, 2, 64))
        batch.lens.add_(1)
        g.replay()
        torch.cuda.synchronize()
        for b in range(3):
            held[b][int(batch.lens[b]) - 1] = (k[b].clone(), v[b].clone())
            for pos, (kk, vv) in held[b].items():
                for o, x in ((ko, kk), (vo, vv)):
                    want = oracle.stored(x.double().cpu().numpy(), "e4m3")
                    assert np.array_equal(o[b, :, pos].double().cpu().numpy(), want), (step, b, pos)


def test_binding_checks(fem):
    cache, batch, starts, table, n = setup(fem, "bf16", 2, 64, 64, 16, [4], [4])
    k = draw(10, 4, 2, 64).cuda()
    for bad in (k[:3], k.float(), k[:, :1], k.transpose(0, 1).contiguous().transpose(0, 1),
                k.cpu(), draw(11, 4, 2, 32).cuda()):
        with pytest.raises(ValueError):
            fem.fem_cache_append(cache, batch, bad, k)
    with pytest.raises(ValueError):
        fem.fem_cache_gather(cache, batch, torch.zeros(1, 2, 9, 32, dtype=torch.bfloat16).cuda())
    with pytest.raises(fem.FemError) as e:
        fem.fem_cache_append(cache, fem.PagedBatch(None, batch.lens, batch.table, 4), k, k)
    assert e.value.status == 1
