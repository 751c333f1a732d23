"""The paged cache on the GPU at the far ends of what its arguments may hold, against the oracle in 64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import paged
from tests.test_gpu_paged import _batch, _cache, _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tb():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2509_26541_amd import binding
    return binding


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("starts", [[0, 20], [0, 5, 30], [2, 9, 12, 40]])
def test_lists_that_reach_beyond_the_rows(tb, kind, starts):
    """row_start counts as at most n_rows, for the write, the read and the attention alike: the last sequence has fewer rows, and they are its last ones."""
    page, hkv, hq, d, n_rows = 16, 2, 4, 64, 12
    kv = [60, 45, 100][: len(starts) - 1]
    table = [[7 * b + i for i in range(7)] for b in range(len(kv))]
    cache, (k, v) = _cache(tb, 21, page, hkv, d, kind, 4)
    gen = torch.Generator().manual_seed(8)
    rows = [torch.randn((n_rows, hkv, d), generator=gen).to(torch.bfloat16) for _ in range(2)]
    before = [x.view(torch.uint8).cpu() for x in (cache.k, cache.v)]
    batch = _batch(tb, table, kv, starts, n_rows)
    tb.tasp_cache_write(rows[0].cuda(), rows[1].cuda(), cache, batch)
    changed = torch.zeros((21, page), dtype=torch.bool)
    for row, p, slot in paged.places(table, kv, starts, page, 21, n_rows):
        changed[p, slot] = True
        for x, values in zip(rows, (k, v)):
            y = x[row].double().numpy()
            if kind == "e4m3":
                y, exps = paged.quantise(y)
                y = y * np.exp2(exps.astype(np.float64))[:, None]
            values[p, :, slot] = y
    for x, old in zip((cache.k, cache.v), before):
        assert torch.equal((x.view(torch.uint8).cpu() != old).any(-1).any(1), changed)
    plan = tb.CacheReadPlan(cache, batch, torch.float32)
    for x, values in zip(plan.run(), (k, v)):
        for row, p, slot in paged.places(table, kv, starts, page, 21, n_rows):
            assert np.array_equal(x[row].double().cpu().numpy(), values[p, :, slot])
    q = torch.randn((n_rows, hq, d), generator=gen).to(torch.bfloat16)
    for hint in (1, 40):                                       # both kernels
        out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, starts, n_rows, hint))
        _check(out, lse, paged.attention(q.double().numpy(), k, v, table, kv, starts), d)


@pytest.mark.parametrize("hint", [1, 64])
@pytest.mark.parametrize("kv,low,high", [(64, 5, 40), (64, 40, 5), (2000, 5, 1900), (9000, 8900, 100), (9000, 100, 8900)])
def test_large_scores_that_differ(tb, kv, low, high, hint):
    """Scores 3 2^31 + 1 024 and + 1 536 (times 1/8), exact in fp32: they differ by 64, though their products with log2(e) round to the same float.  The keys lie
    with two wavefronts, or with two workgroups; the larger one takes all the weight."""
    page, d, hq = 64, 64, 2
    c = np.float32(1.4426950408889634) / np.float32(8)
    assert np.float32(3 * 2**31 + 1024) * c == np.float32(3 * 2**31 + 1536) * c
    n = -(-kv // page)
    k = torch.zeros((n, 1, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.randn((n, 1, page, d), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    for t, x in ((low, 32.0), (high, 48.0)):
        k[t // page, 0, t % page, 0], k[t // page, 0, t % page, 1] = 1.5 * 2.0**16, x
    q = torch.zeros((1, hq, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0], q[..., 1] = 2.0**16, 32.0
    table = [list(range(n))]
    out, lse = tb.tasp_paged_attn(q, tb.PagedCache(k, v), _batch(tb, table, [kv], [0, 1], 1, hint), out_dtype=torch.float32)
    want = v[high // page, 0, high % page].float()
    assert (out[0] - want).abs().max() <= 2.0**-20 * want.abs().max()                  # the other key's weight is 2^-92
    assert ((lse.double() - (3 * 2.0**31 + 1536) / 8).abs() <= 2.0**-22 * 2.0**30).all()


@pytest.mark.parametrize("hint", [1, 64])
@pytest.mark.parametrize("kv,one,other", [(64, 5, 40), (64, 40, 5), (2000, 5, 1900), (9000, 8900, 100)])
def test_equal_scores_beside_an_infinity(tb, kv, one, other, hint):
    """Two keys of the same score, about 2^28 (base 2), of which one has a neighbour with an infinite value: only that one's wavefront or workgroup takes the
    scores off its maximum before they are multiplied.  Both weigh the same, although rounding takes more than 2^3 from the product."""
    page, d = 64, 64
    c = np.float32(1.4426950408889634) / np.float32(8)
    j = next(j for j in range(32) if abs(float(np.float32(2**31 + 256 * j) * c) - (2**31 + 256 * j) * float(c)) > 8)
    n = -(-kv // page)
    k = torch.zeros((n, 1, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.randn((n, 1, page, d), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    for t in (one, other):
        k[t // page, 0, t % page, 0], k[t // page, 0, t % page, 1] = 2.0**15, 8.0 * j
    v[(one + 1) // page, 0, (one + 1) % page, 9] = math.inf
    q = torch.zeros((1, 2, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0], q[..., 1] = 2.0**16, 32.0
    out, _ = tb.tasp_paged_attn(q, tb.PagedCache(k, v), _batch(tb, [list(range(n))], [kv], [0, 1], 1, hint), out_dtype=torch.float32)
    rest = [x for x in range(d) if x != 9]
    a, b = (v[t // page, 0, t % page].float() for t in (one, other))
    assert ((out - (a + b) / 2).abs() <= 2.0**-18 * (a.abs() + b.abs()))[..., rest].all()


@pytest.mark.parametrize("hint", [1, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_scale_bytes_from_0_to_26(tb, d, hint):
    """Factors that the write never makes.  Byte 0 stands for 0 and the others for 2^(b - 127): read back exactly where the type holds the product; what they
    add to an output is right to 2^-110 (64 keys, each off by at most 2^-134 times 448)."""
    page, n_pages = 16, 4
    gen = torch.Generator().manual_seed(6)
    x = torch.randn((2, n_pages, 1, page, d), generator=gen).clamp(-4, 4).mul(64).to(torch.float8_e4m3fn)
    for name in ("zero", "small"):
        byte = torch.zeros((n_pages, 1, page), dtype=torch.uint8) if name == "zero" else torch.randint(0, 27, (n_pages, 1, page), generator=gen).to(torch.uint8)
        factor = torch.where(byte == 0, 0.0, torch.exp2(byte.double() - 127))[..., None]
        cache = tb.PagedCache(x[0].cuda(), x[1].cuda(), *(byte.view(torch.float8_e8m0fnu).cuda() for _ in range(2)))
        table, kv = [[2, 0, 3, 1]], [64]
        batch = _batch(tb, table, kv, [0, 64], 64, 64)
        for dtype in (torch.float32, torch.bfloat16):
            for got, pages in zip(tb.tasp_cache_read(cache, batch, dtype), x):
                want = (pages.double() * factor)[table[0]].transpose(1, 2).reshape(64, 1, d)
                assert torch.equal(got.double().cpu(), want.to(dtype).double())
        q = torch.randn((1, 3, d), generator=gen).to(torch.bfloat16)
        out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, [0, 1], 1, hint), out_dtype=torch.float32)
        want = paged.attention(q.double().numpy(), (x[0].double() * factor).numpy(), (x[1].double() * factor).numpy(), table, kv, [0, 1])
        assert np.abs(lse.double().cpu().numpy() - math.log(64)).max() <= 2.0**-20
        err = np.abs(out.double().cpu().numpy() - want[0])
        assert (err <= (0 if name == "zero" else 2.0**-110 + 2.0**-6 * want[2])).all(), float(err.max())
        # the same bytes for K alone: scores of 0, ordinary values
        cache = tb.PagedCache(x[0].cuda(), x[1].cuda(), byte.view(torch.float8_e8m0fnu).cuda(), torch.full_like(byte, 121).view(torch.float8_e8m0fnu).cuda())
        out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, [0, 1], 1, hint))
        _check(out, lse, paged.attention(q.double().numpy(), (x[0].double() * factor).numpy(), (x[1].double() / 64).numpy(), table, kv, [0, 1]), d)
        # 0 times NaN is NaN, in its column alone
        if name == "zero":
            pages = x[1].clone()
            pages.view(torch.uint8)[3, 0, 7, 11] = 0x7F
            cache = tb.PagedCache(x[0].cuda(), pages.cuda(), *(byte.view(torch.float8_e8m0fnu).cuda() for _ in range(2)))
            out, _ = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, [0, 1], 1, hint))
            assert torch.isnan(out[..., 11]).all() and not out[..., [i for i in range(d) if i != 11]].any()


@pytest.mark.parametrize("hint", [1, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_a_score_of_minus_infinity_is_seen(tb, d, hint):
    """A key of -inf has weight 0 for rows with a positive product, and 0 times an infinite value is NaN, as in the formula; a row behind which the key lies
    has neither."""
    page, new, kv, at = 16, 3, 40, 38
    cache, (k, v) = _cache(tb, 3, page, 1, d, "bf16", 4)
    for pages, host, x in ((cache.k, k, -math.inf), (cache.v, v, math.inf)):
        pages[at // page, 0, at % page, 9] = x
        host[at // page, 0, at % page, 9] = x
    q = torch.randn((new, 2, d), generator=torch.Generator().manual_seed(5)).abs().to(torch.bfloat16)
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, [[0, 1, 2]], [kv], [0, new], new, hint))
    want = paged.attention(q.double().numpy(), k, v, [[0, 1, 2]], [kv], [0, new])
    assert np.isnan(want[0][1:, :, 9]).all() and np.isfinite(want[0][0]).all() and np.isfinite(want[1]).all()
    assert torch.isnan(out[1:, :, 9]).all()
    rest = [i for i in range(d) if i != 9]
    reach = np.where(np.isfinite(want[3]), want[3], 32.0)
    size = np.where(np.isfinite(want[2]), want[2], 4.0)
    _check(out[..., rest], lse, (want[0][..., rest], want[1], size[..., rest], reach), d)
    _check(out[:1], lse[:1], tuple(x[:1] for x in want), d)


@pytest.mark.parametrize("hint", [1, 64])
@pytest.mark.parametrize("window", [2**30, 2**30 + 7, 2**31 - 1])
def test_windows_and_lengths_near_2_31(tb, window, hint):
    """Sequences that have outgrown their table by far: what a wide window still reaches of the pages is seen."""
    page, d, new = 16, 64, 3
    cache, (k, v) = _cache(tb, 4, page, 1, d, "bf16", 9)
    q = torch.randn((2 * new, 2, d), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    kv = [min(window + 23, 2**31 - 1), min(window + 40, 2**31 - 1)]
    table, starts = [[0, 1, 2, 3], [3, 1, 0, 2]], [0, new, 2 * new]
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, starts, 2 * new, hint), tb.MASK_CAUSAL, window, 2)
    want = [np.full((2 * new, 2, d), np.nan), np.full((2 * new, 2), np.nan), np.full((2 * new, 2, d), np.nan), np.zeros((2 * new, 2))]
    for b in range(2):
        for j in range(new):
            pos = kv[b] - new + j
            seen = [t for t in range(4 * page) if t > pos - window or t < 2]
            # one row at a time: the oracle, without a mask, over the keys that it sees
            kk, vv = (np.stack([x[p, :, s] for p, s in ((table[b][t // page], t % page) for t in seen)]) for x in (k, v))
            row = starts[b] + j
            pad = -len(kk) % page
            as_pages = lambda x: np.concatenate([x, np.zeros((pad, 1, d))]).reshape(-1, page, 1, d).transpose(0, 2, 1, 3)  # noqa: E731
            got = paged.attention(q[row : row + 1].double().numpy(), as_pages(kk), as_pages(vv), [list(range((len(kk) + pad) // page))], [len(kk)], [0, 1], causal=False)
            for dst, src in zip(want, got):
                dst[row] = src[0]
    _check(out, lse, want, d)
