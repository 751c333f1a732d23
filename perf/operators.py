"""A paged cache of K and V, and the attention of new tokens over it, as measurable cases.

A serving program keeps the K and V of its sequences in pages of a few dozen tokens.  For every step of a model's layer it
has the new tokens' q, k and v: it writes k and v into the cache and attends from q to all of the sequence.

  op      "write"   CacheWritePlan.run: the new tokens' K and V into the pages
          "read"    CacheReadPlan.run: the last rows of every sequence back as dense K and V
          "attn"    PagedAttnPlan.run: the new tokens' attention over the pages
          "step"    the write and the attention behind it, as a layer calls them
  hq, hkv, d, page  heads, head dimension, tokens to a page
  cache             "bf16", or "e4m3" with a scale per token and head
  rows              type of the dense k and v that are written or read: "bf16" or "fp32"
  n_seqs, new_lo, new_hi, kv_lo, kv_hi, lens
                    sequences, new tokens and tokens in all of each (evenly over the logarithm, from the generator `lens`)
  mask, window, sinks
                    "causal" (with a window of that many tokens and a few first tokens that stay visible, or 0) or "full"
"""
import math
import random

import torch

own = False

_BASE = {"op": "attn", "hq": 32, "hkv": 8, "d": 128, "page": 64, "cache": "bf16", "rows": "bf16", "n_seqs": 1, "new_lo": 1, "new_hi": 1,
         "kv_lo": 1024, "kv_hi": 1024, "lens": 1, "mask": "causal", "window": 0, "sinks": 0}


def _case(name=None, **kw):
    c = dict(_BASE, **kw)
    return dict({"name": name}, **c) if name else c


def listed():
    return [
        # One user, one new token of a small model: what a step costs where only latency counts.
        _case("write 1 token", op="write", hkv=2, d=64, page=16, kv_lo=700, kv_hi=700),
        _case("attn 1 token of 700", hq=8, hkv=2, d=64, page=16, kv_lo=700, kv_hi=700),
        # A prompt batch's K and V into an 8-bit cache: ragged lengths, pages of 16 tokens.
        _case("write prompts e4m3", op="write", cache="e4m3", page=16, n_seqs=7, new_lo=4000, new_hi=20000, kv_lo=4000, kv_hi=30000),
        # Cached prefixes back as dense tensors, for a pass over the whole sequence.
        _case("read e4m3", op="read", cache="e4m3", n_seqs=3, new_lo=9000, new_hi=33000, kv_lo=9000, kv_hi=33000, lens=2),
        _case("read bf16 short", op="read", hkv=20, d=64, page=32, rows="fp32", n_seqs=5, new_lo=17, new_hi=300, kv_lo=300, kv_hi=900),
        # The serving loop of a grouped-query model: a batch of requests of all lengths, one new token each, written and attended.
        _case("step batch 64 e4m3", op="step", cache="e4m3", n_seqs=64, kv_lo=1000, kv_hi=32000),
        # The same for multi-head attention with heads of 64, a 16-bit cache and small pages.
        _case("step batch 33 mha d64", op="step", hq=20, hkv=20, d=64, page=16, n_seqs=33, kv_lo=200, kv_hi=12000),
        # One request with a very long context; a rank's share of it, all of which the new token sees.
        _case("attn 1 token of 500k", mask="full", kv_lo=500003, kv_hi=500003, page=128),
        # A few tokens a sequence, as when a draft is checked, over windows of a long cache.
        _case("attn draft window e4m3", cache="e4m3", hq=64, n_seqs=48, new_lo=2, new_hi=6, kv_lo=3500, kv_hi=60000, window=8192, sinks=4),
        # A long prompt taken in chunks: the last chunk attends to everything before it.
        _case("chunk 2048 of 64k", new_lo=2048, new_hi=2048, kv_lo=65536, kv_hi=65536),
        # A chunk of a model with sliding windows, 8-bit cache, heads of 64.
        _case("chunk window e4m3 d64", cache="e4m3", hq=20, hkv=20, d=64, page=32, new_lo=4003, new_hi=4003, kv_lo=16001, kv_hi=16001, window=2048, sinks=4),
        # What a scheduler makes of many users: chunks of prompts of all sizes in one call.
        _case("chunks ragged", hq=16, hkv=4, page=16, n_seqs=12, new_lo=1, new_hi=1500, kv_lo=300, kv_hi=9000, lens=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above: sizes over their logarithm, lengths of no particular divisor."""
    while True:
        op = rng.choice(["write", "read", "attn", "attn", "attn", "step", "step"])
        c = _case(op=op, cache=rng.choice(["bf16", "e4m3"]), page=rng.choice([16, 32, 64, 128, 256]), lens=rng.randrange(1 << 20))
        if rng.random() < 0.35:
            h = rng.choice([4, 12, 20])
            c.update(hq=h, hkv=h, d=64)
        else:
            hkv = rng.choice([1, 2, 4, 8])
            c.update(hq=hkv * rng.choice([1, 3, 4, 8]), hkv=hkv, d=rng.choice([64, 128, 128]))
        c["n_seqs"] = _log_int(rng, 1, 128)
        kind = rng.choice(["token", "token", "draft", "chunk"])
        if op in ("write", "read"):
            c["rows"] = rng.choice(["bf16", "bf16", "fp32"])
            kind = rng.choice(["token", "chunk", "chunk"])
        if kind == "token":
            kv = (1, 500000)
        elif kind == "draft":
            c.update(new_lo=1, new_hi=rng.randint(2, 8))
            kv = (1, 200000)
        else:
            c["new_hi"] = _log_int(rng, 16, 4000)
            c["new_lo"] = max(1, int(c["new_hi"] * rng.uniform(0.05, 1.0)))
            kv = (16, 65536)
        c["kv_lo"] = _log_int(rng, *kv)
        c["kv_hi"] = _log_int(rng, c["kv_lo"], kv[1])
        if op in ("attn", "step"):
            c["mask"] = rng.choice(["causal", "causal", "causal", "full"])
            if c["mask"] == "causal" and rng.random() < 0.4:
                c.update(window=_log_int(rng, 16, 16384), sinks=rng.choice([0, 1, 4, 64]))
        new, kvs = _lengths(c)
        padded = c["n_seqs"] * max(kvs)
        w = work(c)
        if (w["flops"] <= 2.2e12 and w["bytes"] <= 2e9 and padded * c["hkv"] * c["d"] <= 2.2e9
                and (op in ("write", "read") or padded * max(new) * c["hq"] <= 4.3e9)):
            return c


def _lengths(c):
    """New tokens and tokens in all of every sequence."""
    rng = random.Random(c["lens"])
    new = [_log_int(rng, c["new_lo"], c["new_hi"]) for _ in range(c["n_seqs"])]
    kv = [_log_int(rng, c["kv_lo"], c["kv_hi"]) for _ in range(c["n_seqs"])]
    return new, [max(a, b) for a, b in zip(new, kv)]


def _type(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}[name]


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    new, kv = _lengths(c)
    ps, hkv, d = c["page"], c["hkv"], c["d"]
    pages = [-(-x // ps) for x in kv]
    total = sum(pages)
    # The pool is shared: a sequence's pages lie anywhere in it, and entries behind its last one name none.
    order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
    at = torch.arange(max(pages), device=dev)[None, :]
    count = torch.tensor(pages, device=dev)
    table = torch.where(at < count[:, None], order[((count.cumsum(0) - count)[:, None] + at).clamp(max=total - 1)], -1).to(torch.int32)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    rows = starts[-1]
    s = dict(c, table=table, kv_len=torch.tensor(kv, dtype=torch.int32, device=dev), starts=torch.tensor(starts, dtype=torch.int32, device=dev),
             n_rows=rows, max_new=max(new), max_kv=max(kv))
    shape = (total, hkv, ps, d)
    fill = c["op"] != "write"

    def pool():
        """The cache as earlier steps left it: values of about one; e4m3 with scales that differ from row to row."""
        if not fill:
            return torch.zeros(shape, dtype=_type(c["cache"]), device=dev), torch.zeros(shape[:3], dtype=torch.uint8, device=dev)
        if c["cache"] == "bf16":
            return torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen), None
        lift = torch.randint(5, 8, shape[:3], generator=gen, device=dev)
        x = torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen) * torch.exp2(lift.float())[..., None].to(torch.bfloat16)
        return x.clamp_(-448, 448).to(torch.float8_e4m3fn), (127 - lift).to(torch.uint8)

    for name in ("k", "v"):
        x, scale = pool()
        s[name + "_pages"] = x
        s[name + "_scale"] = scale.view(torch.float8_e8m0fnu) if c["cache"] == "e4m3" else None
    if c["op"] in ("write", "step"):
        for name in ("k", "v"):
            x = torch.empty((rows, hkv, d), dtype=torch.float32, device=dev).normal_(generator=gen)
            if name == "k":
                x[..., :: d // 4] *= 6.0                          # a few channels of K are large, whatever the token
            else:
                x *= torch.exp2(torch.randint(-3, 3, (rows, hkv, 1), generator=gen, device=dev).float())
            s[name] = x.to(_type(c["rows"]))
    if c["op"] in ("attn", "step"):
        s["q"] = torch.empty((rows, c["hq"], d), dtype=torch.bfloat16, device=dev).normal_(generator=gen)
    if own:
        _plans(s)
    return s


def _plans(s):
    """What a program sets up once for its buffers."""
    from paper_2509_26541_amd import binding as tb
    cache = tb.PagedCache(s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"])
    batch = tb.PagedBatch(s["table"], s["kv_len"], s["starts"], s["n_rows"], s["max_new"])
    if s["op"] in ("write", "step"):
        s["write"] = tb.CacheWritePlan(s["k"], s["v"], cache, batch)
    if s["op"] == "read":
        s["read"] = tb.CacheReadPlan(cache, batch, _type(s["rows"]))
    if s["op"] in ("attn", "step"):
        s["attn"] = tb.PagedAttnPlan(s["q"], cache, batch, tb.MASK_CAUSAL if s["mask"] == "causal" else tb.MASK_FULL, s["window"], s["sinks"])


def run(s):
    if own:
        got = {}
        if "write" in s:
            s["write"].run()
            got = _pages(s)
        if "read" in s:
            got["k"], got["v"] = s["read"].run()
        if "attn" in s:
            got["out"], got["lse"] = s["attn"].run()
        return got
    got = {}
    if s["op"] in ("write", "step"):
        _plain_write(s)
        got = _pages(s)
    if s["op"] == "read":
        got["k"], got["v"] = _plain_read(s)
    if s["op"] in ("attn", "step"):
        got["out"], got["lse"] = _plain_attn(s)
    return got


def _pages(s):
    got = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if s["cache"] == "e4m3":
        got.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    return got


def _places(s):
    """Sequence and position of every new row, and the page and the slot it has."""
    row = torch.arange(s["n_rows"], device=s["table"].device)
    b = torch.searchsorted(s["starts"], row, right=True, out_int32=True).long() - 1
    pos = s["kv_len"][b].long() - s["starts"][b + 1].long() + row
    return b, pos, s["table"][b, pos // s["page"]].long(), pos % s["page"]


def _plain_write(s):
    _, _, page, slot = _places(s)
    for x, pages, scales in ((s["k"], s["k_pages"], s["k_scale"]), (s["v"], s["v_pages"], s["v_scale"])):
        if s["cache"] == "bf16":
            pages[page, :, slot] = x.to(torch.bfloat16)
            continue
        f = x.float()
        f = torch.where(torch.isfinite(f), f, math.nan)
        top = torch.nan_to_num(f).abs().amax(-1)
        m, e = torch.frexp(top)                                   # m in [1/2, 1): the row fits 448 = 7/8 2^9 times 2^(e - 9), or twice that
        byte = torch.where(top > 0, e + 118 + (m > 0.875), 27).clamp(min=27)
        f = f.clamp(-(2.0**127) * 1.875, 2.0**127 * 1.875) * torch.exp2(127.0 - byte)[..., None]
        pages.view(torch.uint8)[page, :, slot] = f.to(torch.float8_e4m3fn).view(torch.uint8)
        scales.view(torch.uint8)[page, :, slot] = byte.to(torch.uint8)


def _values(pages, scale, index):
    """The values that the pages at `index` stand for, in 32 bits."""
    if scale is None:
        return pages[index].float()
    return pages.view(torch.uint8)[index].view(torch.float8_e4m3fn).float() * torch.exp2(scale.view(torch.uint8)[index].float() - 127.0)[..., None]


def _plain_read(s):
    _, _, page, slot = _places(s)
    got = []
    for pages, scale in ((s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"])):
        head = torch.arange(s["hkv"], device=page.device)
        got.append(_values(pages, scale, (page[:, None], head[None, :], slot[:, None])).to(_type(s["rows"])))
    return got


def _plain_attn(s):
    """Every sequence padded to the longest, all scores at once."""
    n_seqs, hkv, d, n, kv = s["n_seqs"], s["hkv"], s["d"], s["max_new"], s["max_kv"]
    g = s["hq"] // hkv
    table = s["table"].long().clamp(min=0)
    k = _values(s["k_pages"], s["k_scale"], table).permute(0, 2, 4, 1, 3).reshape(n_seqs, hkv, d, -1)[..., :kv].contiguous()
    v = _values(s["v_pages"], s["v_scale"], table).permute(0, 2, 1, 3, 4).reshape(n_seqs, hkv, -1, d)[:, :, :kv].contiguous()
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    j = torch.arange(n, device=k.device)
    q = s["q"].float()[(s["starts"][:-1, None] + j).clamp(max=s["n_rows"] - 1)]                      # [sequences, n, hq, d]
    q = q.reshape(n_seqs, n, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n_seqs, hkv, g * n, d)
    p = torch.matmul(q * d**-0.5, k).reshape(n_seqs, hkv, g, n, kv)
    t = torch.arange(kv, device=k.device)
    length = s["kv_len"].long()[:, None, None]
    pos = (s["kv_len"].long() - new)[:, None, None] + j[:, None]
    seen = (t < length).expand(n_seqs, n, kv)
    if s["mask"] == "causal":
        seen = seen & (t <= pos)
        if s["window"]:
            seen = seen & ((t > pos - s["window"]) | (t < s["sinks"]))
    p.masked_fill_(~seen[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True).clamp(min=-1e30)
    p.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n_seqs, hkv, g * n, kv), v).reshape(n_seqs, hkv, g, n, d) / total.clamp(min=1e-30)
    lse = (m + total.log()).squeeze(-1)
    b, at, _, _ = _places(s)
    at = at - (s["kv_len"].long() - new)[b]
    return (o.permute(0, 3, 1, 2, 4).reshape(n_seqs, n, s["hq"], d)[b, at].to(torch.bfloat16), lse.permute(0, 3, 1, 2).reshape(n_seqs, n, s["hq"])[b, at])


def _seen(c, n, kv):
    """(pairs of row and key, keys that some row sees) of one head of a sequence with n new tokens of kv."""
    if c["mask"] == "full":
        return n * kv, kv
    w = c["window"]
    if not w:
        return n * (kv - n) + n * (n + 1) // 2, kv
    pairs = 0
    for p in range(kv - n, kv):
        low = max(0, p - w + 1)
        pairs += p + 1 - low + min(c["sinks"], low)
    low = max(0, kv - n - w + 1)
    return pairs, kv - low + min(c["sinks"], low)


def work(case):
    """Rows read and written, the cache's rows that some new token sees, and two products for each pair."""
    c = case
    new, kv = _lengths(c)
    row = c["hkv"] * (c["d"] * 2 if c["cache"] == "bf16" else c["d"] + 1)            # bytes of a token's K (or V) in the cache
    dense = c["hkv"] * c["d"] * (4 if c["rows"] == "fp32" else 2)
    total, flops = 0.0, 0.0
    if c["op"] in ("write", "read", "step"):
        total += 2.0 * sum(new) * (row + dense)
    if c["op"] in ("attn", "step"):
        for n, t in zip(new, kv):
            pairs, keys = _seen(c, n, t)
            flops += 4.0 * c["d"] * c["hq"] * pairs
            total += 2.0 * keys * row + n * c["hq"] * (4.0 * c["d"] + 4)
            if c["op"] == "step":
                total -= 2.0 * n * row                            # the new tokens' rows are written, and need not be read again
    return {"bytes": total, "flops": flops}


def _exact_quantised(x):
    """x [rows, heads, d] in 64 bits -> (x over its scale, scale): the scale is the smallest power of two, from 2^-100 on, that keeps the row within 448."""
    x = torch.where(torch.isfinite(x), x, math.nan)
    top = torch.nan_to_num(x).abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2((top / 448.0).clamp(min=2.0**-120)))
    e = torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e)
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e).clamp(min=-100.0)
    return x / torch.exp2(e), torch.exp2(e)


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    new, kv = _lengths(c)
    dev = s["table"].device
    table = s["table"].cpu().tolist()
    starts = s["starts"].cpu().tolist()
    ps = c["page"]
    small = c["cache"] == "e4m3"

    def rows_of(name, b):
        """All tokens of sequence b, as the cache holds them, in 64 bits: [tokens, heads, d]."""
        index = torch.tensor([x for x in table[b] if x >= 0], device=dev)
        x = s[name + "_pages"].view(torch.uint8)[index].view(torch.float8_e4m3fn).double() if small else s[name + "_pages"][index].double()
        if small:
            x = x * s[name + "_scale"].view(torch.uint8)[index].double().sub(127.0).exp2()[..., None]
        x = x.transpose(1, 2).reshape(-1, c["hkv"], c["d"])[: kv[b]]
        if c["op"] == "step":
            y = s[name][starts[b]: starts[b + 1]].double()
            if small:
                y, scale = _exact_quantised(y)
                y = y.float().to(torch.float8_e4m3fn).double() * scale
            else:
                y = y.to(torch.bfloat16).double()
            x = torch.cat([x[: kv[b] - new[b]], y])
        return x

    got = {}
    if c["op"] in ("write", "step"):
        got = dict.fromkeys(_pages(s))
    if c["op"] == "write":
        for name in ("k", "v"):
            y = s[name].double()
            y = _exact_quantised(y)[0] if small else y
            full = s[name + "_pages"].to(torch.float64)
            for b in range(c["n_seqs"]):
                at = torch.arange(kv[b] - new[b], kv[b], device=dev)
                full[s["table"][b].long()[at // ps], :, at % ps] = y[starts[b]: starts[b + 1]]
            got[name + "_pages"] = full
    if c["op"] == "read":
        for name in ("k", "v"):
            got[name] = torch.cat([rows_of(name, b)[kv[b] - new[b]:] for b in range(c["n_seqs"])])
    if c["op"] in ("attn", "step"):
        g = c["hq"] // c["hkv"]
        outs, lses = [], []
        for b in range(c["n_seqs"]):
            k, v = rows_of("k", b), rows_of("v", b)
            q = s["q"][starts[b]: starts[b + 1]].double() / math.sqrt(c["d"])
            t = torch.arange(kv[b], device=dev)[None, :]
            pos = torch.arange(kv[b] - new[b], kv[b], device=dev)[:, None]
            hide = torch.zeros((new[b], kv[b]), dtype=torch.bool, device=dev)
            if c["mask"] == "causal":
                hide = t > pos
                if c["window"]:
                    hide = hide | ((pos - t >= c["window"]) & (t >= c["sinks"]))
            out = torch.empty((new[b], c["hq"], c["d"]), dtype=torch.float64, device=dev)
            lse = torch.empty((new[b], c["hq"]), dtype=torch.float64, device=dev)
            for h in range(c["hq"]):
                x = (q[:, h] @ k[:, h // g].t().contiguous()).masked_fill(hide, -math.inf)
                lse[:, h] = torch.logsumexp(x, -1)
                out[:, h] = torch.softmax(x, -1) @ v[:, h // g].contiguous()
            outs.append(out)
            lses.append(lse)
        got["out"], got["lse"] = torch.cat(outs), torch.cat(lses)
    return got
