"""Attention over a paged cache where every workgroup walks many key tiles, and the precision of the kernel for few rows, against 64 bits.

Tolerances.  With reach = scale max sum |q k| and size = sum p |v|: a score is off by (d + 4) 2^-24 reach.  Its exponential is taken by
the hardware (2^-22) of an argument that lies within 2^5 of 0 wherever the weight counts (rounded: 2^-20), so a probability is off by
E = (d + 4) 2^-24 reach + 2^-19 relative.  Up to 32 rows, P goes into the product as two bf16: the second one is at most 2^-8 of the value and off by
half a step of its binade, 2^-17 of the value.  A matrix instruction adds 32 products to a sum; what it cuts off is taken to be at most 2^-22 of the sum's size,
and there are two of them to a stage of 32 keys, T stages to a wavefront.  Joining partial results: two roundings each (2^-23), and the quotient's (2^-22).
  fp32 outputs, up to 32 rows: |error| <= (2 E + 2^-17 + 2 T 2^-22 + 2^-20) size
  more rows, P once in bf16 (2^-8, and 2^-8 of the largest again in the sum it is divided by): 2^-7 size beside that
  lse: E + 2^-23 |lse| + 2^-19 (the sums have two levels of at most 64 and T / 64 terms, each rounded by 2^-24)"""
import numpy as np
import pytest
import torch

from tests import paged_shapes
from tests.test_gpu_paged import _batch, _cache, _table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tb():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2509_26541_amd import binding
    return binding


def _exact(q, k, v, table, kv, starts, causal=True, window=0, sinks=0):
    """The oracle's formula in torch operations in 64 bits on the device: q [rows, Hq, d], k and v [n_pages, Hkv, page, d] (what the pages stand for).
    Returns out, lse, size, reach as the oracle does."""
    n_pages, hkv, ps, d = k.shape
    g = q.shape[1] // hkv
    out, size = torch.full_like(q, np.nan), torch.full_like(q, np.nan)
    lse, reach = torch.full_like(q[..., 0], np.nan), torch.zeros_like(q[..., 0])
    for b, length in enumerate(kv):
        n = starts[b + 1] - starts[b]
        if n == 0:
            continue
        pages = torch.tensor(table[b], device=q.device)
        t = torch.arange(min(length, len(table[b]) * ps), device=q.device)
        t = t[(pages[t // ps] >= 0) & (pages[t // ps] < n_pages)]
        pos = torch.arange(length - n, length, device=q.device)[:, None]
        seen = torch.ones((n, len(t)), dtype=torch.bool, device=q.device)
        if causal:
            seen = t[None, :] <= pos
            if window:
                seen &= (t[None, :] > pos - window) | (t[None, :] < sinks)
        at = slice(starts[b], starts[b + 1])
        for h in range(hkv):
            kh, vh = k[pages[t // ps], h, t % ps], v[pages[t // ps], h, t % ps]
            qh = q[at, h * g : (h + 1) * g].reshape(n * g, d) / d**0.5
            s = (qh @ kh.t().contiguous()).masked_fill(~seen.repeat_interleave(g, 0), -np.inf)
            none = ~seen.any(1).repeat_interleave(g)
            l = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(none, torch.zeros_like(l), l)[:, None])
            put = lambda dst, x: dst[at, h * g : (h + 1) * g].copy_(x.view(n, g, *x.shape[1:]))  # noqa: E731
            put(out, p @ vh)
            put(size, p @ vh.abs())
            put(lse, torch.where(none, torch.full_like(l, -np.inf), l))
            put(reach, (qh.abs() @ kh.abs().t().contiguous()).amax(1) if len(t) else torch.zeros(n * g, dtype=q.dtype, device=q.device))
    return out, lse, size, reach


def _bounds(want, d, stages, few):
    o, l, size, reach = want
    e = (d + 4) * 2.0**-24 * reach + 2.0**-19
    return (2 * e[..., None] + 2.0**-17 + 2 * stages * 2.0**-22 + 2.0**-20 + (0 if few else 2.0**-7)) * size, e + 2.0**-23 * l.abs() + 2.0**-19


def _compare(out, lse, want, bounds, columns=slice(None)):
    o, l = want[0], want[1]
    none = torch.isneginf(l)
    assert torch.equal(none, torch.isneginf(lse)) and not out[none].any()
    oerr = ((out.double() - o).abs() / bounds[0].clamp(min=1e-300))[~none][..., columns]
    lerr = ((lse.double() - l).abs() / bounds[1])[~none]
    assert torch.isfinite(oerr).all() and float(oerr.max()) <= 1, float(oerr.max())
    assert torch.isfinite(lerr).all() and float(lerr.max()) <= 1, float(lerr.max())


def _queries(k, table, kv, starts, hq, seed):
    """Rows of three kinds: of about one (weights spread over all keys), 2.5 times that (some dozens of keys), and rows that point at one key."""
    n_pages, hkv, ps, d = k.shape
    gen = torch.Generator().manual_seed(seed)
    q = torch.randn((starts[-1], hq, d), generator=gen)
    q[:, 1::3] *= 2.5
    for b, length in enumerate(kv):
        live = [t for t in range(0, min(length, len(table[b]) * ps), ps) if 0 <= table[b][t // ps] < n_pages]
        for row in range(starts[b], starts[b + 1]):
            for h in range(2, hq, 3):
                if not live:
                    continue
                t = live[int(torch.randint(len(live), (1,), generator=gen))] + int(torch.randint(ps, (1,), generator=gen))
                key = k[table[b][t // ps], h * hkv // hq, t % ps]
                q[row, h] = key * float(24 * d**0.5 / (key * key).sum())
    return q.to(torch.bfloat16)


@pytest.mark.parametrize("windowed", [False, True])
@pytest.mark.parametrize("kind,d,tokens", list(paged_shapes.ROWS) + list(paged_shapes.TILES))
def test_long_runs(tb, kind, d, tokens, windowed):
    """Pieces of more than 256 key tiles (few rows) and 128 (many); then with a column of V that is not finite in a few pages, so that sums are formed again by
    the pass for such values, over all tiles."""
    new, kv = paged_shapes.batch(kind, d, tokens)
    starts = np.concatenate([[0], np.cumsum(new)]).tolist()
    table = paged_shapes.table(kv, d + tokens)
    hkv, hq = paged_shapes.HKV, paged_shapes.HKV * paged_shapes.GROUP
    cache, (k, v) = _cache(tb, paged_shapes.POOL, paged_shapes.PAGE, hkv, d, kind, 17)
    k, v = torch.from_numpy(k), torch.from_numpy(v)
    q = _queries(k, table, kv, starts, hq, 3)
    # the oracle's column 7 says whether a row sees a key that will not be finite there
    v[..., 7] = 0.0
    for page in (3, 77, 250):
        v[page, :, 5::11, 7] = 1.0
    columns = [c for c in range(d) if c != 7]
    few = (kind, d, tokens) in paged_shapes.ROWS
    plan = tb.PagedAttnPlan(q.cuda(), cache, _batch(tb, table, kv, starts, starts[-1], max(new)), tb.MASK_CAUSAL if windowed else tb.MASK_FULL,
                            paged_shapes.WINDOW if windowed else 0, paged_shapes.SINKS if windowed else 0, out_dtype=torch.float32)
    want = _exact(q.cuda().double(), k.cuda(), v.cuda(), table, kv, starts, windowed, plan.args.window, plan.args.sinks)
    sees = want[0][..., 7] > 0
    assert 0.5 < float(sees.double().mean()) < 1
    for odd in (False, True):
        if odd:
            for page in (3, 77, 250):
                if kind == "bf16":
                    cache.v[page, :, 5::11, 7] = np.inf
                else:
                    cache.v.view(torch.uint8)[page, :, 5::11, 7] = 0x7F
        out, lse = (x.clone() for x in plan.run())
        _compare(out, lse, want, _bounds(want, d, 300, few), columns)
        assert torch.equal(~torch.isfinite(out[..., 7]), sees & odd)
        # the same call gives the same bits
        for _ in range(2):
            plan.out.fill_(7.0)
            again, lse_again = plan.run()
            assert torch.equal(again.view(torch.int32), out.view(torch.int32)) and torch.equal(lse_again, lse)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq,hkv,d,new", [(4, 4, 128, 1), (16, 2, 128, 2), (8, 1, 64, 4), (6, 2, 64, 3)])
def test_few_rows_keep_probabilities_to_17_bits(tb, kind, hq, hkv, d, new):
    """fp32 outputs of up to 32 rows over up to 64 keys, of which each of two wavefronts has one stage; the bound is one that P in one bf16 does not keep."""
    kv, page = [64, 3, 33, 17, 50, 64, 7, 5], 16
    starts = [new * i for i in range(len(kv) + 1)]
    kv = [max(x, new) for x in kv]
    cache, (k, v) = _cache(tb, 40, page, hkv, d, kind, 23)
    table = _table(kv, page, 40, 2)
    q = (torch.randn((starts[-1], hq, d), generator=torch.Generator().manual_seed(5)) / 4).to(torch.bfloat16)
    out, lse = tb.tasp_paged_attn(q.cuda(), cache, _batch(tb, table, kv, starts, starts[-1], new), out_dtype=torch.float32)
    want = _exact(q.double(), torch.from_numpy(k), torch.from_numpy(v), table, kv, starts)
    bounds = _bounds(want, d, 1, True)
    coarse = torch.full_like(want[0], np.nan)                  # P rounded to bf16, everything else exact
    for b in range(len(kv)):
        for row in range(starts[b], starts[b + 1]):
            t = np.arange(kv[b] - new + row - starts[b] + 1)
            for h in range(hq):
                at = (np.asarray(table[b])[t // page], h * hkv // hq, t % page)
                s = torch.from_numpy(k[at]) @ q[row, h].double() / d**0.5
                coarse[row, h] = torch.exp(s - s.max()).to(torch.bfloat16).double() @ torch.from_numpy(v[at]) / torch.exp(s - s.max()).sum()
    assert float(((coarse - want[0]).abs() / bounds[0]).max()) > 4
    _compare(out.cpu(), lse.cpu(), want, bounds)
