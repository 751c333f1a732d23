"""The paged cache on the GPU against the oracle in 64 bits: writing, reading, and attention over the pages.

Tolerances.  A product of two bf16 is exact in fp32; a score is a sum of d of them in fp32, times the scale: off by at most
(d + 4) 2^-24 reach, with reach = scale sum |q k|, and the exponential adds 2^-21 (hardware exp2, and its argument near 2^7 rounded to 2^-17).  So a
probability is off by E = (d + 4) 2^-24 reach + 2^-17 relative, lse by E + 2^-23 |lse| + 2^-17 (a few hundred fp32 additions).  P goes into the second
product in bf16: half a step is 2^-8 of a value, and 2^-8 again for the sum that it is divided by; the output is rounded once more, to bf16
(2^-8 of it).  With size = sum p |v|: |out error| <= (2 E + 2^-7) size + 2^-8 |out| + 2^-17 size."""
import math

import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tb():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2509_26541_amd import binding
    return binding


def _cache(tb, n_pages, page, hkv, d, kind, seed):
    """A cache full of values of about one (e4m3: with scales from 2^-9 to 2^-3), on the device, and what it stands for in 64 bits."""
    gen = torch.Generator().manual_seed(seed)
    got, values = [], []
    for _ in range(2):
        x = torch.randn((n_pages, hkv, page, d), generator=gen)
        if kind == "bf16":
            x = x.to(torch.bfloat16)
            got.append(x.cuda())
            values.append(x.double().numpy())
        else:
            lift = torch.randint(3, 10, (n_pages, hkv, page), generator=gen)
            x = (x * torch.exp2(lift.float() - 3)[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
            byte = (127 - lift).to(torch.uint8)
            got += [x.cuda(), byte.view(torch.float8_e8m0fnu).cuda()]
            values.append(x.double().numpy() * np.exp2(-lift.double().numpy())[..., None])
    cache = tb.PagedCache(*got) if kind == "bf16" else tb.PagedCache(got[0], got[2], got[1], got[3])
    return cache, values


def _table(kvs, page, n_pages, seed, width=None):
    """Scattered pages, -1 behind the last."""
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    width = width or max(1, max(-(-x // page) for x in kvs))
    rows = []
    for x in kvs:
        n = -(-x // page)
        rows.append([order.pop() for _ in range(n)] + [-1] * (width - n))
    return rows


def _batch(tb, table, kv, starts, n_rows, max_rows=0):
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return tb.PagedBatch(ints(table), ints(kv), ints(starts), n_rows, max_rows)


def _check(out, lse, want, d, fp32=False):
    o, l, size, reach = want
    e = (d + 4) * 2.0**-24 * reach + 2.0**-17
    nan = np.isnan(l)                                       # rows of no sequence (and rows whose result is NaN) are compared elsewhere
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    none = np.isneginf(l)
    assert np.array_equal(none, np.isneginf(lse) & ~nan)
    assert not out[none].any()
    live = ~nan & ~none
    lerr = np.abs(lse[live] - l[live]) - (e[live] + 2.0**-23 * np.abs(l[live]) + 2.0**-17)
    assert lerr.size == 0 or lerr.max() <= 0, lerr.max()
    bound = (2 * e[..., None] + 2.0**-7 + 2.0**-17) * size + (0 if fp32 else 2.0**-8) * np.abs(o)
    oerr = (np.abs(out - o) - bound)[live]
    assert np.isfinite(out[live]).all() and (oerr.size == 0 or oerr.max() <= 0), oerr.max()


# lengths: one token; around a stage, a tile and a page; sequences without rows, without keys, with more rows than tokens
BATCHES = {
    "one": ([1], [1]), "few": ([1, 1, 1], [17, 130, 33]), "edges": ([1, 2, 1, 3, 1, 1], [15, 16, 31, 64, 127, 129]),
    "empty": ([0, 1, 0, 2, 0], [5, 0, 0, 40, 9]), "short": ([5, 1], [2, 1]), "chunk": ([37, 1, 50], [37, 200, 131]), "long": ([2, 1], [1500, 2111]),
    "prompt": ([200, 129, 1], [200, 700, 77]), "tiles": ([64, 65, 63, 33], [64, 129, 1023, 1025]),
    "many": ([1] * 70 + [3], [3 * i % 97 for i in range(70)] + [301]),
}
HEADS = [(4, 4, 128), (8, 2, 64), (6, 2, 128), (16, 1, 64), (5, 5, 64), (24, 1, 128)]
MASKS = [("causal", 0, 0), ("causal", 1, 0), ("causal", 40, 0), ("causal", 64, 4), ("causal", 100, 70), ("full", 0, 0)]
CASES = [(b, h, m, kind, page) for i, b in enumerate(BATCHES) for j, m in enumerate(MASKS)
         for h, kind, page in [(HEADS[(i + j) % 6], ("bf16", "e4m3")[(i + j) % 2], (16, 64, 32, 256)[(i + 2 * j) % 4]),
                               (HEADS[(i + 2 * j + 3) % 6], ("e4m3", "bf16")[(i + j) % 2], (32, 16, 128, 64)[(3 * i + j) % 4])]]


@pytest.mark.parametrize("name,heads,mask,kind,page", CASES, ids=lambda x: str(x).replace(" ", ""))
def test_attention(tb, name, heads, mask, kind, page):
    hq, hkv, d = heads
    new, kv = BATCHES[name]
    starts = np.concatenate([[0], np.cumsum(new)]).tolist()
    n_pages = sum(-(-x // page) for x in kv) + 3
    cache, (k, v) = _cache(tb, n_pages, page, hkv, d, kind, 11)
    table = _table(kv, page, n_pages, 5)
    q = torch.randn((starts[-1], hq, d), generator=torch.Generator().manual_seed(7)).to(torch.bfloat16)
    batch = _batch(tb, table, kv, starts, starts[-1], max(new))
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, batch, tb.MASK_CAUSAL if mask[0] == "causal" else tb.MASK_FULL, mask[1], mask[2])
    want = paged.attention(q.double().numpy(), k, v, table, kv, starts, mask[0] == "causal", mask[1], mask[2])
    _check(out, lse, want, d)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq,hkv,d", [(12, 4, 128), (4, 4, 64)])
def test_rows_of_no_sequence_are_left_and_strides_and_types(tb, kind, hq, hkv, d):
    new, kv, page = [4, 0, 19], [77, 3, 64], 16
    starts = [3, 7, 7, 26]
    n_rows = 31
    cache, (k, v) = _cache(tb, 14, page, hkv, d, kind, 3)
    table = _table(kv, page, 14, 2)
    fused = torch.randn((n_rows, hq * d + 72), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    q = fused.cuda()[:, 64 : 64 + hq * d].view(n_rows, hq, d)
    want = paged.attention(fused[:, 64 : 64 + hq * d].reshape(n_rows, hq, d).double().numpy(), k, v, table, kv, starts, scale=0.3)
    for dtype in (torch.bfloat16, torch.float32):
        plan = tb.PagedAttnPlan(q, cache, _batch(tb, table, kv, starts, n_rows), softmax_scale=0.3, out_dtype=dtype)
        plan.out.fill_(7.0)
        plan.lse.fill_(9.0)
        out, lse = plan.run()
        _check(out, lse, want, d, fp32=dtype == torch.float32)
        for rows in (slice(0, 3), slice(26, None)):
            assert (out[rows] == 7).all() and (lse[rows] == 9).all()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pages_that_name_none_are_not_visible(tb, kind):
    new, kv, page, n_pages = [3, 1, 20], [70, 100, 90], 16, 12
    starts = [0, 3, 4, 24]
    cache, (k, v) = _cache(tb, n_pages, page, 2, 128, kind, 3)
    table = [[1, -1, 3, 12, 5, 0, 7], [-7, 2**31 - 1, -(2**31), 99, -1, 12, -1], [0, 1, 2, 3, 4, 5, -1]]
    q = torch.randn((24, 6, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    for args in ((tb.MASK_CAUSAL, 0, 0), (tb.MASK_CAUSAL, 33, 5), (tb.MASK_FULL, 0, 0)):
        out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, starts, 24), *args)
        _check(out, lse, paged.attention(q.double().numpy(), k, v, table, kv, starts, args[0] == tb.MASK_CAUSAL, args[1], args[2]), 128)
        assert torch.isneginf(lse[3]).all() and not out[3].any()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [3, 60])
def test_a_sequence_that_outgrew_its_table(tb, kind, new):
    """Tokens behind the table's last page are neither written nor seen, and what is in the pages stays."""
    page, n_pages, kv = 16, 6, [100, 40]
    cache, (k, v) = _cache(tb, n_pages, page, 2, 64, kind, 3)
    table, starts = [[1, 4, 2], [0, 3, 5]], [0, new, 2 * new]
    before = [x.view(torch.uint8).clone() for x in (cache.k, cache.v)]
    batch = _batch(tb, table, kv, starts, 2 * new)
    q = torch.randn((2 * new, 4, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    for args in ((tb.MASK_CAUSAL, 0, 0), (tb.MASK_CAUSAL, 70, 3), (tb.MASK_FULL, 0, 0)):
        out, lse = tb.tasp_paged_attn(q.cuda(), cache, batch, *args)
        _check(out, lse, paged.attention(q.double().numpy(), k, v, table, kv, starts, args[0] == tb.MASK_CAUSAL, args[1], args[2]), 64)
    rows = torch.ones((2 * new, 2, 64), dtype=torch.bfloat16, device="cuda")
    tb.tasp_cache_write(rows, rows, cache, batch)
    for x, old in zip((cache.k, cache.v), before):
        same = (x.view(torch.uint8) == old).all(-1)[:, 0].cpu()                        # [pages, slots]
        kept = [min(48, kv[b] - new) if kv[b] - new > 0 else 0 for b in range(2)]
        assert same[table[0]].flatten()[: kept[0]].all() and same[table[1]].flatten()[: kept[1]].all()
        assert same[table[0]].flatten().sum() == kept[0] and same[table[1]].flatten()[: 40].sum() == kept[1]


def test_many_sequences(tb):
    """More sequences than lanes, and than lanes of lanes: each with one row, a few with none."""
    for n_seqs in (65, 200, 4200):
        gen = torch.Generator().manual_seed(n_seqs)
        kv = torch.randint(0, 40, (n_seqs,), generator=gen).tolist()
        new = [0 if i % 7 == 3 else 1 for i in range(n_seqs)]
        starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        table = torch.randint(0, 50, (n_seqs, 3), generator=gen).tolist()
        cache, (k, v) = _cache(tb, 50, 16, 1, 64, "bf16", 5)
        for g in (2, 20):
            q = torch.randn((starts[-1], g, 64), generator=gen).to(torch.bfloat16)
            out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, starts, starts[-1], 1 if g == 2 else 8))
            _check(out, lse, paged.attention(q.double().numpy(), k, v, table, kv, starts), 64)


@pytest.mark.parametrize("new", [1, 40])
def test_scores_far_below_zero(tb, new):
    kv, page, d = 70, 16, 64
    k = torch.full((5, 1, page, d), -(2.0**55), dtype=torch.bfloat16, device="cuda")
    v = torch.randn((5, 1, page, d), device="cuda").to(torch.bfloat16)
    q = torch.full((new, 2, d), 2.0**60, dtype=torch.bfloat16, device="cuda")
    table = [[0, 1, 2, 3, 4]]
    out, lse = tb.tasp_paged_attn(q, tb.PagedCache(k, v), _batch(tb, table, [kv], [0, new], new))
    want = paged.attention(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(), table, [kv], [0, new])
    assert np.allclose(lse.double().cpu().numpy(), want[1], rtol=1e-6) and (want[1] < -1e34).all()
    _check(out, torch.from_numpy(want[1]), (want[0], want[1], want[2], np.zeros_like(want[3])), d)       # (equal scores are equal exactly)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [6, 40])
def test_what_is_not_seen_does_not_reach_a_row(tb, kind, d, new):
    """NaN and infinities behind the last token, in later tokens of the chunk and outside the window; and those that are seen."""
    kv, page, n_pages, hkv, hq = 150, 32, 8, 2, 4
    cache, (k, v) = _cache(tb, n_pages, page, hkv, d, kind, 21)
    table = _table([kv], page, n_pages, 9)
    t = torch.tensor(table[0], device="cuda")
    q = torch.randn((new, hq, d), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    byte = lambda x: x.view(torch.uint8)  # noqa: E731

    def put(pos, column, infinite):
        for pages, host in ((cache.k, k), (cache.v, v)):
            p, s = table[0][pos // page], pos % page
            if kind == "bf16":
                pages[p, :, s, column] = math.inf if infinite else math.nan
                host[p, :, s, column] = math.inf if infinite else math.nan
            else:
                byte(pages)[p, :, s, column] = 0x7F
                host[p, :, s, column] = math.nan

    # everything behind the last token, scales too
    last = t[kv // page]
    if kind == "bf16":
        cache.k[last, :, kv % page :] = math.nan
        cache.v[last, :, kv % page :] = math.inf
    else:
        for x in (cache.k, cache.v, cache.k_scale, cache.v_scale):
            byte(x)[last, :, kv % page :] = 0xFF
    batch = _batch(tb, table, [kv], [0, new], new)
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, batch, tb.MASK_FULL)
    _check(out, lse, paged.attention(q.double().numpy(), k, v, table, [kv], [0, new], causal=False), d)
    # a late token of the chunk and one left of the window: rows that see neither are as they were, the others are not finite where V is not
    put(kv - 3, 5, True)
    put(kv - new - 17, 3, False)
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, batch, tb.MASK_CAUSAL, 16, 0)
    want = paged.attention(q.double().numpy(), k, v, table, [kv], [0, new], True, 16, 0)
    clean = np.isfinite(want[0]).all(-1) & np.isfinite(want[1])
    assert clean[: new - 3].all() and not clean[new - 3 :].any()
    good = tuple(np.where(clean.reshape(clean.shape + (1,) * (x.ndim - 2)), x, np.nan) for x in want)
    _check(out, lse, good, d)
    # a key with an infinity has the score inf or, where q is negative, -inf: there it has no weight, and lse is that of the others
    l, got = want[1][new - 3 :], lse[new - 3 :].double().cpu().numpy()
    assert np.isnan(l).any() and np.array_equal(np.isnan(got), np.isnan(l)) and np.allclose(got, l, atol=1e-4, equal_nan=True)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [1, 30])
def test_an_infinite_value_that_is_seen_stays_in_its_column(tb, kind, new):
    kv, page, hkv, hq, d = 90, 16, 1, 3, 128
    cache, (k, v) = _cache(tb, 6, page, hkv, d, kind, 5)
    table = _table([kv], page, 6, 4)
    p, s = table[0][50 // page], 50 % page
    if kind == "bf16":
        cache.v[p, :, s, 17] = math.inf
    else:
        cache.v.view(torch.uint8)[p, :, s, 17] = 0x7F
    v[p, :, s, 17] = math.inf if kind == "bf16" else math.nan
    q = torch.randn((new, hq, d), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, [kv], [0, new], new))
    want = paged.attention(q.double().numpy(), k, v, table, [kv], [0, new])
    assert (torch.isposinf(out[:, :, 17]) if kind == "bf16" else torch.isnan(out[:, :, 17])).all()
    rest = [i for i in range(d) if i != 17]
    _check(out[:, :, rest], lse, (want[0][..., rest], want[1], want[2][..., rest], want[3]), d)


def test_large_scores_and_one_dominant_key(tb):
    """Scores of hundreds, rising along the keys, and an early key that outweighs a long row: the sum keeps the others (lse to 1e-4)."""
    kv, page, d = 40000, 64, 64
    n = -(-kv // page)
    x = torch.zeros((n, 1, page, d), dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n * page, device="cuda").view(n, 1, page)
    x[..., 0] = (pos // 200).to(torch.bfloat16)              # steps that bf16 holds
    v = torch.randn((n, 1, page, d), device="cuda").to(torch.bfloat16)
    q = torch.zeros((1, 1, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 8.0
    table = [list(range(n))]
    batch = _batch(tb, table, [kv], [0, 1], 1)
    out, lse = tb.tasp_paged_attn(q, tb.PagedCache(x, v), batch)
    want = paged.attention(q.double().cpu().numpy(), x.double().cpu().numpy(), v.double().cpu().numpy(), table, [kv], [0, 1])
    _check(out, lse, want, d)
    x.zero_()
    x[0, 0, 0, 0] = 13.0                                     # score 13: e^13 against 40 000 times 1
    out, lse = tb.tasp_paged_attn(q, tb.PagedCache(x, v), batch)
    assert abs(float(lse) - math.log(math.exp(13.0) + kv - 1)) < 1e-4
    

def _same(a, b):
    off = int(((a != b) & ~(torch.isnan(a) & torch.isnan(b))).sum())
    assert off == 0, "%d values differ" % off


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hkv,page", [(1, 16), (3, 64)])
def test_write_and_read(tb, kind, d, dtype, hkv, page):
    new, kv = [1, 0, 40, 3, 150, 2], [1, 7, 90, 2, 151, 33]             # the fourth has more rows than tokens
    starts = [2] + (2 + np.cumsum(new)).tolist()
    n_rows, n_pages = starts[-1] + 3, 40
    table = _table([max(a, b) for a, b in zip(new, kv)], page, n_pages - 1, 8)
    table[5][0] = n_pages + 3 if page == 64 else -5                     # names no page
    gen = torch.Generator().manual_seed(4)
    wide = torch.randn((n_rows, 2, hkv, d), generator=gen) * torch.exp2(torch.randint(-30, 30, (n_rows, 2, hkv, 1), generator=gen).float())
    wide[5, 0, 0, 3], wide[6, 1, 0, 0], wide[7, :, 0], wide[8, 0, 0, 1] = math.inf, math.nan, 0.0, 448.0
    wide[9, 0], wide[10, 0], wide[11, 1] = 1e-38, 3e38, 2.0**-118
    wide = wide.to(dtype)
    k, v = wide.cuda()[:, 0], wide.cuda()[:, 1]                         # tokens two rows apart
    cache = tb.PagedCache.empty(n_pages, page, hkv, d, torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn)
    held = [x for x in (cache.k, cache.v, cache.k_scale, cache.v_scale) if x is not None]
    for x in held:
        x.view(torch.uint8).fill_(0x55)
    batch = _batch(tb, table, kv, starts, n_rows)
    assert tb.tasp_cache_write(k, v, cache, batch) is cache
    got = [x.view(torch.uint8).cpu() for x in held]
    want = [torch.full_like(x, 0x55) for x in got]
    back = [torch.full((n_rows, hkv, d), 0.0, dtype=torch.float64) for _ in range(2)]
    for row, page_i, slot in paged.places(table, kv, starts, page, n_pages):
        for s in range(2):
            x = wide[row, s]
            if page_i is None:
                continue
            if kind == "bf16":
                want[s].view(torch.bfloat16)[page_i, :, slot] = x.to(torch.bfloat16)
                back[s][row] = x.to(torch.bfloat16).double()
            else:
                values, exps = paged.quantise(x.double().numpy())
                want[s].view(torch.float8_e4m3fn)[page_i, :, slot] = torch.from_numpy(values).float().to(torch.float8_e4m3fn)
                want[2 + s][page_i, :, slot] = torch.from_numpy(exps + 127).to(torch.uint8)
                back[s][row] = torch.from_numpy(values * np.exp2(exps.astype(np.float64))[:, None])
    for g, w, x in zip(got, want, held):
        if x.dtype == torch.float8_e8m0fnu:
            assert torch.equal(g, w)
        else:
            _same(g.view(x.dtype).float(), w.view(x.dtype).float())
    for out_type in (torch.bfloat16, torch.float32):
        plan = tb.CacheReadPlan(cache, batch, out_type)
        plan.k.fill_(7.0)
        plan.v.fill_(7.0)
        for x, w in zip(plan.run(), back):
            x = x.double().cpu()
            assert (x[:2] == 7).all() and (x[starts[-1] :] == 7).all()
            _same(x[2 : starts[-1]], w[2 : starts[-1]].to(out_type).double())


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pages_behind_4_gib(tb, kind):
    """Pages at the far end of pools whose byte offsets need 33 bits."""
    page, hkv, d = 64, 8, 128
    per = page * hkv * d * (2 if kind == "bf16" else 1)
    n_pages = (5 << 30) // per
    cache = tb.PagedCache.empty(n_pages, page, hkv, d, torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn)
    kv, new = [100, 30], [100, 30]
    table = [[n_pages - 1, n_pages - 5], [n_pages - 3, -1]]
    gen = torch.Generator().manual_seed(3)
    k, v = (torch.randn((130, hkv, d), generator=gen).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((130, hkv, d), generator=gen).to(torch.bfloat16)
    batch = _batch(tb, table, kv, [0, 100, 130], 130)
    tb.tasp_cache_write(k.cuda(), v.cuda(), cache, batch)
    kr, vr = tb.tasp_cache_read(cache, batch, torch.float32)
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, batch)
    kp, vp = np.zeros((4, hkv, page, d)), np.zeros((4, hkv, page, d))
    for row, p, slot in paged.places([[0, 1], [2, -1]], kv, [0, 100, 130], page, 4):
        for src, pages in ((k, kp), (v, vp)):
            x = src[row].double().numpy()
            if kind == "e4m3":
                values, exps = paged.quantise(x)
                x = values * np.exp2(exps.astype(np.float64))[:, None]
            pages[p, :, slot] = x
    want = paged.attention(q.double().numpy(), kp, vp, [[0, 1], [2, -1]], kv, [0, 100, 130])
    _check(out, lse, want, d)
    for got, pages in ((kr, kp), (vr, vp)):
        for row, p, slot in paged.places([[0, 1], [2, -1]], kv, [0, 100, 130], page, 4):
            assert np.array_equal(got[row].double().cpu().numpy(), pages[p, :, slot])


def _serve(tb, cache, steps, k, v, q, kv_len, batch, write, attn, bufs):
    outs = []
    for i in range(steps):
        bufs["k"].copy_(k[i])
        bufs["v"].copy_(v[i])
        bufs["q"].copy_(q[i])
        kv_len += 1
        outs.append(tuple(x.clone() for x in (write.run() and attn.run())))
    return outs


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_prompt_then_tokens_as_served(tb, kind):
    """A prompt written in chunks and attended to, then tokens one by one, eagerly and from a captured graph that reads the lengths as they grow;
    the last one against the oracle over everything written."""
    page, hkv, hq, d, n_pages = 16, 2, 8, 128, 40
    cache = tb.PagedCache.empty(n_pages, page, hkv, d, torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn)
    gen = torch.Generator().manual_seed(12)
    prompt, steps = [70, 33], 6
    table = _table([x + steps for x in prompt], page, n_pages, 6)
    ks, vs, qs = ([torch.randn((x + steps, h, d), generator=gen).to(torch.bfloat16).cuda() for x in prompt] for h in (hkv, hkv, hq))
    done = [0, 0]
    outs = [[], []]
    for take in ((40, 1), (30, 32)):                                     # the prompt in two chunks
        done = [a + b for a, b in zip(done, take)]
        cut = lambda xs: torch.cat([x[e - n : e] for x, e, n in zip(xs, done, take)])  # noqa: E731
        batch = _batch(tb, table, done, [0, take[0], sum(take)], sum(take))
        tb.tasp_cache_write(cut(ks), cut(vs), cache, batch)
        o, _ = tb.tasp_paged_attn(cut(qs), cache, batch)
        outs[0].append(o[: take[0]])
        outs[1].append(o[take[0] :])
    kv_len = torch.tensor(done, dtype=torch.int32, device="cuda")
    batch = tb.PagedBatch(torch.tensor(table, dtype=torch.int32, device="cuda"), kv_len, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), 2, 1)
    bufs = {n: torch.empty((2, h, d), dtype=torch.bfloat16, device="cuda") for n, h in (("k", hkv), ("v", hkv), ("q", hq))}
    write, attn = tb.CacheWritePlan(bufs["k"], bufs["v"], cache, batch), tb.PagedAttnPlan(bufs["q"], cache, batch)
    at = lambda xs, i: torch.stack([x[p + i] for x, p in zip(xs, prompt)])  # noqa: E731
    k_new, v_new, q_new = ([at(xs, i) for i in range(steps)] for xs in (ks, vs, qs))
    eager = _serve(tb, cache, steps, k_new, v_new, q_new, kv_len, batch, write, attn, bufs)
    kv_len.copy_(torch.tensor(done, dtype=torch.int32))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        kv_len.add_(1)
        write.run()
        attn.run()
    kv_len.copy_(torch.tensor(done, dtype=torch.int32))
    for i in range(steps):
        bufs["k"].copy_(k_new[i])
        bufs["v"].copy_(v_new[i])
        bufs["q"].copy_(q_new[i])
        graph.replay()
        assert torch.equal(attn.out, eager[i][0]) and torch.equal(attn.lse, eager[i][1]), i
        torch.cuda.synchronize()
        torch.randn(1000, device="cuda").sum()
    # everything written, by the oracle
    kp, vp = np.zeros((n_pages, hkv, page, d)), np.zeros((n_pages, hkv, page, d))
    for b, n in enumerate(prompt):
        for t in range(n + steps):
            for src, pages in ((ks, kp), (vs, vp)):
                x = src[b][t].double().cpu().numpy()
                if kind == "e4m3":
                    values, exps = paged.quantise(x)
                    x = values * np.exp2(exps.astype(np.float64))[:, None]
                pages[table[b][t // page], :, t % page] = x
    full = torch.cat(qs).double().cpu().numpy()
    ends = [n + steps for n in prompt]
    want = paged.attention(full, kp, vp, table, ends, [0, ends[0], sum(ends)])
    got = torch.cat([torch.cat(outs[b] + [o[b : b + 1] for o, _ in eager]) for b in range(2)])
    lse = torch.cat([torch.cat([torch.full((prompt[b], hq), math.nan, device="cuda")] + [l[b : b + 1] for _, l in eager]) for b in range(2)])
    o, l, size, reach = want
    bound = (2 * ((d + 4) * 2.0**-24 * reach + 2.0**-17)[..., None] + 2.0**-7 + 2.0**-17) * size + 2.0**-8 * np.abs(o)
    assert (np.abs(got.double().cpu().numpy() - o) <= bound).all()
    fed = ~np.isnan(lse.cpu().numpy())
    assert np.abs(lse.double().cpu().numpy()[fed] - l[fed]).max() < 1e-4


def test_a_cache_spread_over_ranks_is_joined_by_the_merge(tb):
    """Each rank holds a third of a sequence's pages and attends without a mask; the fp32 pairs merge to the whole."""
    page, hkv, hq, d, new = 32, 2, 8, 64, 5
    cuts = [100, 0, 77]
    gen = torch.Generator().manual_seed(2)
    q = torch.randn((new, hq, d), generator=gen).to(torch.bfloat16)
    parts, ks, vs = [], [], []
    for i, kv in enumerate(cuts):
        cache, (k, v) = _cache(tb, 6, page, hkv, d, ("bf16", "e4m3")[i % 2], 30 + i)
        table = _table([kv], page, 6, i, width=4)
        parts.append(tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, [kv], [0, new], new), tb.MASK_FULL, out_dtype=torch.float32))
        for t in range(kv):
            ks.append(k[table[0][t // page], :, t % page])
            vs.append(v[table[0][t // page], :, t % page])
    total = len(ks)
    pad = -total % page
    as_pages = lambda x: np.concatenate([np.stack(x), np.zeros((pad,) + x[0].shape)]).reshape(-1, page, hkv, d).transpose(0, 2, 1, 3)  # noqa: E731
    want = paged.attention(q.double().numpy(), as_pages(ks), as_pages(vs), [list(range((total + pad) // page))], [total], [0, new], causal=False)
    out, lse = tb.tasp_lse_merge_many([o for o, _ in parts], [l for _, l in parts])
    _check(out, lse, want, d, fp32=True)
    o, l = parts[0]
    for po, pl in parts[1:]:
        tb.tasp_lse_merge(o, l, po, pl)
    _check(o, l, want, d, fp32=True)


@pytest.mark.parametrize("new", [1, 64])
def test_cached_prompt_read_back_feeds_chunk_attention(tb, new):
    """Pages -> dense K and V -> tasp_chunk_attn over the whole sequence gives what the pages give."""
    n_ranks, S, hkv, hq, d, page = 4, 256, 2, 4, 128, 32
    cache, _ = _cache(tb, 10, page, hkv, d, "e4m3", 9)
    table = _table([S], page, 10, 1)
    batch = _batch(tb, table, [S], [0, S], S)
    k, v = tb.tasp_cache_read(cache, batch)
    q = torch.randn((S // n_ranks, hq, d), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    a, al = tb.tasp_chunk_attn(q, k, v, tb.tasp_schedule(n_ranks, 0), tb.MASK_FULL)
    b, bl = tb.tasp_paged_attn(q[:new], cache, _batch(tb, table, [S], [0, new], new), tb.MASK_FULL)
    assert (a[:new].float() - b.float()).abs().max() <= 2e-2 and (al[:new] - bl).abs().max() <= 1e-3


def test_two_streams_with_their_own_plans(tb):
    cache, (k, v) = _cache(tb, 20, 16, 2, 64, "bf16", 3)
    table = _table([130, 90], 16, 20, 1)
    gen = torch.Generator().manual_seed(1)
    q = [torch.randn((2, 8, 64), generator=gen).to(torch.bfloat16) for _ in range(2)]
    batch = _batch(tb, table, [130, 90], [0, 1, 2], 2)
    plans = [tb.PagedAttnPlan(x.cuda(), cache, batch) for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for s, p in zip(streams, plans):
            with torch.cuda.stream(s):
                p.run()
    torch.cuda.synchronize()
    for x, p in zip(q, plans):
        _check(p.out, p.lse, paged.attention(x.double().numpy(), k, v, table, [130, 90], [0, 1, 2]), 64)


@pytest.mark.parametrize("max_rows", [0, 1])
def test_lists_that_fall_stay_inside(tb, max_rows):
    """Sequences that share their rows, against the documented order, with more work than 32 bits count: the call ends, its buffers' surroundings and the
    cache stay as they were, and so does a row behind the last one."""
    seqs, rows, page = 300, 2048, 1024
    cache, _ = _cache(tb, 1, page, 8, 128, "bf16", 5)
    before = [t.clone() for t in (cache.k, cache.v)]
    batch = _batch(tb, [[-1] * 64] * seqs, [64 * page] * seqs, [rows * (b % 2) for b in range(seqs + 1)], rows, max_rows)
    plan = tb.PagedAttnPlan(torch.zeros((rows, 32, 128), dtype=torch.bfloat16, device="cuda"), cache, batch)
    out, lse = torch.full((rows + 1, 32, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((rows + 1, 32), 7.0, device="cuda")
    workspace = torch.full((plan.args.workspace_bytes + 65536,), 7, dtype=torch.uint8, device="cuda")
    plan.args.out, plan.args.lse, plan.args.workspace = out.data_ptr(), lse.data_ptr(), workspace.data_ptr()
    plan.run()
    torch.cuda.synchronize()
    assert (out[rows] == 7).all() and (lse[rows] == 7).all() and (workspace[plan.args.workspace_bytes:] == 7).all()
    assert torch.equal(before[0], cache.k) and torch.equal(before[1], cache.v)
