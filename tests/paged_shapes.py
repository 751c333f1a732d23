"""Batches of a paged cache whose runs are long: what the loops over keys do once they have left their first tiles behind.

A workgroup of the kernel for up to 32 rows looks its pages up 128 tiles of 64 keys at a time, one of the kernel for more 8 tiles at a time, and its
sums go through a second level every 64 tiles.  Work is cut into equal runs for all workgroups, so long pieces need much work: many sequences that
share a pool of pages.  tests/test_paged_runs.py works out on the host how long the pieces of these batches are."""
import random

HKV, GROUP, PAGE, POOL = 2, 8, 32, 400
WINDOW, SINKS = 28001, 70
# (kind, d, tokens to a sequence): workgroups that share the work, as test_paged_runs.py checks
ROWS = {("bf16", 128, 2): 512, ("bf16", 128, 4): 512, ("e4m3", 128, 2): 1024, ("e4m3", 128, 4): 1024, ("bf16", 64, 2): 1024, ("bf16", 64, 4): 1024,
        ("e4m3", 64, 2): 1536, ("e4m3", 64, 4): 1024}
TILES = {("bf16", 128, 5): 512, ("e4m3", 128, 5): 512, ("bf16", 64, 5): 768, ("e4m3", 64, 5): 512}


def batch(kind, d, tokens):
    """(new tokens, tokens in all) of every sequence: long ones, so many that a workgroup's share is some 270 tiles (kernel for few rows) or 140, and,
    for the kernel for many rows, shorter ones that are not split."""
    rng = random.Random(1000 * d + 10 * tokens + (kind == "e4m3"))
    few = (kind, d, tokens) in ROWS
    workers = (ROWS if few else TILES)[kind, d, tokens]
    keys = (17600 if few else 8500) * workers
    kv = []
    while sum(kv) * HKV < keys:
        kv.append(rng.randint(28100, 31000))
    new = [tokens] * len(kv)
    if few:
        kv += [1, 40, 0, 3000]
        new += [1, tokens, 0, tokens]
    else:
        kv += [rng.randint(1000, 4500) for _ in range(24)] + [rng.randint(1, 200) for _ in range(4)]
        new += [tokens] * 23 + [17] + [1, tokens, 0, 3]
    return new, [max(a, b) for a, b in zip(new, kv)]


def table(kv, seed):
    """Pages of a shared pool, in any order and more than once; one entry in 50 names none."""
    rng = random.Random(seed)
    width = max(-(-x // PAGE) for x in kv)
    none = [-1, POOL, -(2**31), 2**31 - 1]
    return [[rng.choice(none) if i >= -(-x // PAGE) or rng.random() < 0.02 else rng.randrange(POOL) for i in range(width)] for x in kv]
