"""The 8-bit key/value cache on the GPU (foe_cache_append, foe_cache_attention,
foe_cache_evict) against the fp64 oracle, through the binding."""

import sys

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2605_06206_amd import foe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA, SCALE = 500000.0, 16.0


def say(*a):
    print("[cache]", *a, file=sys.stderr, flush=True)


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    foe.lib()


# ---- moving pools between the oracle's form and the library's ---------------------

def to_dev(pool):
    f8 = torch.float8_e4m3fn
    return {"k": torch.from_numpy(pool["k"]).to(DEV).view(f8),
            "v": torch.from_numpy(pool["v"]).to(DEV).view(f8),
            "kv_scale": torch.from_numpy(pool["kv_scale"].astype(np.float32)).to(DEV),
            "mass": torch.from_numpy(pool["mass"]).to(DEV)}


def to_host(dev):
    return {"k": dev["k"].view(torch.uint8).cpu().numpy(),
            "v": dev["v"].view(torch.uint8).cpu().numpy(),
            "kv_scale": dev["kv_scale"].double().cpu().numpy(),
            "mass": dev["mass"].cpu().numpy()}


def same(got, want):
    """Two pools' codes, scales and masses bit for bit; tells how the first differ."""
    for name in ("kv_scale", "k", "v", "mass"):
        g, w = got[name], want[name]
        at = np.nonzero((g != w) & ~((g != g) & (w != w)))
        assert at[0].size == 0, (name, at[0].size, [(tuple(int(i[j]) for i in at), g[at][j],
                                                     w[at][j]) for j in range(min(6, at[0].size))])


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def bf16(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DEV).to(torch.bfloat16)


def host(t):
    return t.double().cpu().numpy()


def random_pool(rng, pages, H, hd):
    """A pool as earlier steps leave it: finite codes everywhere a token may be."""
    k = rng.integers(0, 256, (pages, H, 64, hd), dtype=np.uint8)
    v = rng.integers(0, 256, (pages, H, 4, hd, 16), dtype=np.uint8)
    # magnitudes up to 2 in units of the scale's 2^-8: codes 0 .. 0x40
    k, v = (np.where(c & 127 > 0x40, c & 0xBF, c) for c in (k, v))
    s = 2.0 ** rng.integers(-2, 1, (pages, H, 2))
    return {"k": k, "v": v, "kv_scale": s,
            "mass": rng.exponential(size=(pages, H, 64)).astype(np.float32)}


def batch(rng, seqs, extra=0):
    """(ctx, row_start, table, pages) of sequences [(ctx, rows), ...]"""
    ctx = [c for c, _ in seqs]
    rs = np.concatenate([[0], np.cumsum([n for _, n in seqs])])
    blocks = max(1, max((c + n + 63) // 64 for c, n in seqs)) + extra
    pages = len(seqs) * blocks + 3
    table = rng.permutation(pages)[:len(seqs) * blocks].reshape(len(seqs), blocks)
    return ctx, rs, table.astype(np.int32), pages


# ---- append ---------------------------------------------------------------------

def check_append(pool, dev, qkv, table, ctx, rs, q, pos=None, theta=THETA, scale=SCALE):
    """The library's pool after the call against the oracle's from the same start."""
    want = {n: a.copy() for n, a in pool.items()}
    q_ref, raw = co.append(want, qkv, table, ctx, rs, theta, scale, pos)
    got = to_host(dev)
    rows = np.concatenate([np.arange(rs[b], rs[b + 1]) for b in range(len(ctx))]).astype(int)
    # the angle (reduced in fp64, then fp32: 2^-23), its sine and cosine (2^-22) and two
    # products and a sum (3 * 2^-24), each relative to the pair: 2^-20 of |x| covers them; q is
    # then rounded to bf16 once (2^-8)
    x = np.abs(qkv[:, rows, :-2].astype(np.float64))
    half = x.shape[-1] // 2
    pair = np.concatenate([x[..., :half] + x[..., half:]] * 2, -1)
    err = np.abs(host(q)[:, rows] - q_ref[:, rows])
    with np.errstate(invalid="ignore"):
        ok = (err <= 2.0 ** -8 * np.abs(q_ref[:, rows]) + 2.0 ** -20 * pair + 1e-37)
    assert (ok | ~np.isfinite(q_ref[:, rows])).all()
    assert np.array_equal(got["kv_scale"], want["kv_scale"])
    assert np.array_equal(got["mass"], want["mass"])
    kd, vd = got["k"] != want["k"], got["v"] != want["v"]
    # values are quantised from their own bits: every code is the oracle's
    assert not vd.any()
    # a key's code may be the next one where its fp32 value lies on the other side of a border
    n = 0
    for p, h, t, d in zip(*np.nonzero(kd)):
        k, _, ok = raw[(p, h, t)]
        assert ok
        s = want["kv_scale"][p, h, 0]
        a, b = co.decode(got["k"][p, h, t, d]) * s, co.decode(want["k"][p, h, t, d]) * s
        row_max = np.abs(k).max()
        assert abs(abs(a - k[d]) - abs(b - k[d])) <= 2.0 ** -18 * row_max, (p, h, t, d)
        n += 1
    assert n <= 1e-3 * sum(1 for _ in raw) * qkv.shape[-1] + 2
    return got


APPENDS = [
    # H, nq, hd, [(ctx, rows)]
    (1, 1, 96, [(0, 1)]),
    (2, 2, 128, [(0, 1), (63, 1), (64, 1), (65, 1), (127, 1)]),
    (2, 1, 128, [(0, 64), (64, 64), (1, 63), (1, 64)]),
    (3, 2, 96, [(10, 130), (0, 0), (5, 3), (60, 8), (200, 1)]),
    (1, 4, 128, [(1000, 300)]),
    (8, 3, 96, [(0, 17), (15, 1), (16, 1), (17, 30)]),
    (2, 64, 128, [(3, 2)]),
]


@pytest.mark.parametrize("H,nq,hd,seqs", APPENDS)
def test_append_parity(H, nq, hd, seqs):
    say("append", H, nq, hd, seqs)
    rng = np.random.default_rng([3, H, nq, hd, len(seqs)])
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    dev = to_dev(pool)
    qkv = bf16(rng.normal(size=(H, rs[-1], nq + 2, hd)))
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                         ints(rs), THETA, SCALE)
    torch.cuda.synchronize()
    check_append(pool, dev, host(qkv), table, ctx, rs, q)


def test_append_many_sequences():
    """More sequences than a workgroup has threads, most with one row or none."""
    rng = np.random.default_rng(5)
    seqs = [(int(c), int(n)) for c, n in zip(rng.integers(0, 130, 700), rng.integers(0, 3, 700))]
    seqs[650] = (30, 90)
    say("append many", len(seqs))
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, 1, 96)
    dev = to_dev(pool)
    qkv = bf16(rng.normal(size=(1, rs[-1], 3, 96)))
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                         ints(rs), THETA, SCALE)
    torch.cuda.synchronize()
    check_append(pool, dev, host(qkv), table, ctx, rs, q)


def test_append_positions_and_far_angles():
    """Positions of the caller's own (after an eviction), some of them large."""
    rng = np.random.default_rng(6)
    seqs, pos = [(10, 3), (70, 5), (0, 2)], [130000, 70, 1 << 20]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, 2, 128)
    dev = to_dev(pool)
    qkv = bf16(rng.normal(size=(2, rs[-1], 3, 128)))
    say("append positions")
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                         ints(rs), 10000.0, 1.0, pos=ints(pos))
    torch.cuda.synchronize()
    check_append(pool, dev, host(qkv), table, ctx, rs, q, pos, 10000.0, 1.0)


@pytest.mark.parametrize("hd", [96, 128])
def test_append_scales_grow_and_fall(hd):
    """Magnitudes from the smallest scale to the largest, token by token in one page:
    the codes before are rescaled, a smaller token keeps the scale."""
    rng = np.random.default_rng(7)
    H, table = 2, np.array([[1]], dtype=np.int32)
    dev = to_dev(random_pool(rng, 3, H, hd))
    mags = [0.0, 1e-36, 1e-30, 3e-5, 1.0, 1.75, 448.0, 449.0, 2.0, 1e5, 1e38, 1e-3]
    for t, m in enumerate(mags):
        say("append magnitude", hd, m)
        pool = to_host(dev)
        qkv = bf16(rng.uniform(-1, 1, (H, 1, 3, hd)) * m)
        if m:
            qkv[:, 0, 2, 3] = m  # the largest value is m itself
        q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints([t]),
                             ints([0, 1]), THETA, SCALE)
        torch.cuda.synchronize()
        check_append(pool, dev, host(qkv), table, [t], [0, 1], q)


def test_append_non_finite_rows():
    rng = np.random.default_rng(8)
    H, nq, hd = 2, 1, 128
    ctx, rs, table, pages = batch(rng, [(5, 40), (0, 3)])
    pool = random_pool(rng, pages, H, hd)
    dev = to_dev(pool)
    x = rng.normal(size=(H, rs[-1], nq + 2, hd))
    x[0, 3, 1, 7] = np.nan       # a key
    x[1, 9, 2, 100] = -np.inf    # a value
    x[1, 41, 1:, :] = np.inf     # both, whole rows
    x[0, 20, 0, 0] = np.nan      # a query: no concern of the cache
    qkv = bf16(x)
    say("append non-finite")
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                         ints(rs), THETA, SCALE)
    torch.cuda.synchronize()
    got = check_append(pool, dev, host(qkv), table, ctx, rs, q)
    assert (got["k"][table[0, 0], 0, 8] == 0x7F).all()
    # the queries that see such a token give NaN, the others are finite
    o = host(foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                                 ints(rs), 40))
    want = np.zeros((rs[-1], H), dtype=bool)
    want[3:40, 0] = want[9:40, 1] = want[41:, 1] = want[20, 0] = True
    assert np.array_equal(np.isnan(o).all((2, 3)), want)
    assert np.isfinite(o[~want]).all()


def test_append_absent_pages_and_bad_batches():
    """Table entries outside the pool, contexts outside the table and row ranges
    outside the batch: what can be done is done, nothing else is written."""
    rng = np.random.default_rng(9)
    H, hd = 1, 96
    pool = random_pool(rng, 4, H, hd)
    dev = to_dev(pool)
    table = np.array([[-1, 0], [4, 1], [2, 3], [2, 3]], dtype=np.int32)
    ctx, rs = [60, 60, -5, 1 << 30], [0, 8, 16, 17, 99]
    qkv = bf16(rng.normal(size=(H, 18, 3, hd)))
    say("append absent pages")
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                         ints(rs), THETA, SCALE)
    torch.cuda.synchronize()
    # the same as with lengths and ranges cut to what there is; row 17 has no slot
    check_append(pool, dev, host(qkv), table, [60, 60, 0, 128], [0, 8, 16, 17, 18], q)


# ---- attention --------------------------------------------------------------------

def attention_bound(o, spread):
    """Each probability is rounded to bf16 once (2^-8 of it), the output once (2^-8); the fp32
    scores, exponentials and sums add 2^-12 of sum p |v| (scores below 2^6 in log2 units
    with 2^-22 relative: 2^-16, 128-term sums 2^-17, two exponentials)."""
    return (2.0 ** -8 + 2.0 ** -12) * spread + 2.0 ** -8 * np.abs(o)


def mass_bound(got, before, big, hd, n_cols):
    """A probability's relative error: its score's (hd + 8 roundings of 2^-24 of at most
    `big` * log2 e), twice for the maximum and the sum, and the sums' own (2^-24 a term)."""
    rel = 2 * (hd + 8) * 2.0 ** -24 * big * 1.45 + 2.0 ** -20 + n_cols * 2.0 ** -24
    return rel * got + 2.0 ** -23 * np.abs(before + got)


def run_attention(rng, H, nq, hd, seqs, with_mass, q_sigma=1.5, max_rows=None, pool=None):
    ctx, rs, table, pages = batch(rng, seqs)
    pool = pool or random_pool(rng, pages, H, hd)
    dev = to_dev(pool)
    N = int(rs[-1])
    q = bf16(q_sigma * rng.normal(size=(H, N, nq, hd)))
    mass_out = torch.full_like(dev["mass"], -7.0) if with_mass else None
    out = torch.full((N, H, nq, hd), -3.0, dtype=torch.bfloat16, device=DEV)
    foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx), ints(rs),
                        max_rows or max(n for _, n in seqs), out=out,
                        mass_in=dev["mass"] if with_mass else None, mass_out=mass_out)
    torch.cuda.synchronize()
    return pool, table, ctx, rs, q, out, mass_out


def check_attention(pool, table, ctx, rs, q, out, mass_out, rows=None):
    ref = co.attend(pool, host(q), table, ctx, rs, rows=rows, mass=mass_out is not None)
    o, spread = ref[0], ref[1]
    got = host(out)
    mine = ~np.isnan(spread)
    err = np.abs(got - o)[mine]
    lim = attention_bound(o, spread)[mine]
    say(f"error {float((err / np.maximum(lim, 1e-30)).max()):.3f} of the bound")
    assert (err <= lim).all()
    if mass_out is None:
        return
    m, touched = host(mass_out), np.zeros(mass_out.shape, dtype=bool)
    for (b, h), w in ref[3].items():
        cols = (rs[b + 1] - rs[b]) * q.shape[2]
        for t, x in enumerate(w):
            p = table[b, t // 64]
            if not 0 <= p < len(m):
                continue
            touched[p, h, t % 64] = True
            before = float(pool["mass"][p, h, t % 64]) if t < ctx[b] else 0.0
            assert abs(m[p, h, t % 64] - before - x) <= mass_bound(x, before, ref[2],
                                                                   q.shape[3], cols), (b, h, t)
    assert (m[~touched] == -7.0).all()


ATTENTIONS = [
    # H, nq, hd, [(ctx, rows)]
    (1, 1, 96, [(0, 1)]),                                  # one token that sees itself
    (2, 2, 128, [(0, 1), (62, 1), (63, 1), (64, 1), (65, 1)]),
    (1, 2, 128, [(1500, 1)]),
    (2, 1, 96, [(700, 1), (3, 1), (0, 0), (255, 1), (256, 1)]),
    (2, 8, 128, [(300, 1), (10, 2)]),                      # 8 and 16 columns
    (1, 16, 96, [(200, 1)]),
    (1, 17, 128, [(100, 1), (77, 1)]),                     # one head past a tile
    (1, 64, 96, [(130, 1)]),
    (2, 1, 128, [(500, 16)]),                              # a few rows of one sequence
    (1, 3, 96, [(90, 5), (0, 6), (1000, 2)]),
    (2, 2, 128, [(0, 33)]),                                # a prompt from the start
    (1, 2, 96, [(100, 128), (40, 1), (0, 129), (333, 7)]), # chunks beside single tokens
    (2, 1, 128, [(0, 256)]),
    (1, 3, 128, [(61, 200)]),
    (1, 2, 128, [(1000, 257)]),
    (1, 5, 96, [(64, 100), (0, 64), (63, 65)]),
]


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("H,nq,hd,seqs", ATTENTIONS)
def test_attention_parity(H, nq, hd, seqs, mass):
    say("attention", H, nq, hd, seqs, mass)
    rng = np.random.default_rng([11, H, nq, hd, len(seqs), seqs[0][0]])
    check_attention(*run_attention(rng, H, nq, hd, seqs, mass))


@pytest.mark.parametrize("i", range(12))
def test_attention_random_batches(i):
    rng = np.random.default_rng([12, i])
    H, nq = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 4, 7]))
    hd, top = int(rng.choice([96, 128])), int(rng.choice([1, 4, 40, 300]))
    B = int(rng.integers(1, 6 if top > 4 else 20))
    seqs = [(int(2 ** rng.uniform(0, 11)) - 1, int(rng.integers(0, top + 1))) for _ in range(B)]
    seqs[int(rng.integers(B))] = (int(rng.integers(0, 300)), top)
    say("random batch", i, H, nq, hd, seqs)
    check_attention(*run_attention(rng, H, nq, hd, seqs, bool(i % 2)))


@pytest.mark.parametrize("nq,top", [(1, 1), (2, 20)])
def test_attention_many_sequences(nq, top):
    """More sequences than a workgroup has threads, many of them without rows, one long."""
    rng = np.random.default_rng([18, nq])
    seqs = [(int(c), int(n)) for c, n in zip(rng.integers(0, 150, 1100),
                                             rng.integers(0, top + 1, 1100))]
    seqs[3], seqs[900], seqs[1099] = (2000, 1), (1000, top), (70, top)
    say("many sequences", nq, top)
    check_attention(*run_attention(rng, 1, nq, 96, seqs, True))


@pytest.mark.parametrize("rows", [1, 150])
def test_attention_sharp_and_rising_scores(rows):
    """Scores over hundreds of log2 units, rising along the keys, so that the running
    maximum moves in every page."""
    rng = np.random.default_rng(13)
    H, nq, hd, ctx = 1, 2, 128, 1000
    ctx_l, rs, table, pages = batch(rng, [(ctx, rows)])
    pool = random_pool(rng, pages, H, hd)
    for t in range(ctx + rows):  # key t: (t / 1000) in every dim, in codes of scale 1/4
        pool["k"][table[0, t // 64], :, t % 64] = co.encode(np.full(hd, t / 1000.0) * 4)
    pool["kv_scale"][..., 0] = 0.25
    dev = to_dev(pool)
    q = bf16(np.abs(rng.normal(size=(H, rows, nq, hd))) + 8.0)
    say("sharp scores", rows)
    mass = torch.full_like(dev["mass"], -7.0)
    out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints([ctx]),
                              ints(rs), rows, mass_in=dev["mass"], mass_out=mass)
    torch.cuda.synchronize()
    check_attention(pool, table, [ctx], rs, q, out, mass)


@pytest.mark.parametrize("rows", [1, 70])
def test_attention_absent_pages_and_garbage_behind_the_end(rows):
    """Pages that are not there are not seen, a row whose pages are all absent gives
    zeros, and the slots behind a sequence's end may hold NaN codes."""
    rng = np.random.default_rng(14)
    H, nq, hd = 2, 2, 96
    seqs = [(200, rows), (0, 1), (130, 1)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    for b, (c, n) in enumerate(seqs):
        end = c + n
        for t in range(end, table.shape[1] * 64):
            p = table[b, t // 64]
            pool["k"][p, :, t % 64] = 0x7F
            pool["v"][p, :, (t % 64) // 16, :, t % 16] = 0xFF
    table[0, 1] = pages + 5
    table[0, 0] = -1
    table[2, :] = -3
    dev = to_dev(pool)
    q = bf16(rng.normal(size=(H, rs[-1], nq, hd)))
    say("absent pages", rows)
    mass = torch.full_like(dev["mass"], -7.0)
    out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                              ints(rs), rows, mass_in=dev["mass"], mass_out=mass)
    torch.cuda.synchronize()
    check_attention(pool, table, ctx, rs, q, out, mass)
    assert (host(out)[rs[2]:] == 0).all()


def test_attention_wide_table():
    """A table with room for far more pages than there are (the scores of so many are not
    kept for the mass) and a narrow one, whose pages are dealt out otherwise: each within
    the bounds (another order of the sums, so not bit for bit)."""
    rng = np.random.default_rng(19)
    H, nq, hd, seqs = 2, 8, 128, [(300, 2), (0, 1), (700, 1)]
    ctx, rs, table, pages = batch(rng, seqs)
    dev = to_dev(random_pool(rng, pages, H, hd))
    wide = np.full((3, 50000), -1, dtype=np.int32)
    wide[:, :table.shape[1]] = table
    q = bf16(rng.normal(size=(H, rs[-1], nq, hd)))
    say("wide table")
    outs = []
    for t in (table, wide):
        m = torch.full_like(dev["mass"], -7.0)
        outs.append((foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(t), ints(ctx),
                                         ints(rs), 2, mass_in=dev["mass"], mass_out=m), m))
    torch.cuda.synchronize()
    pool = to_host(dev)
    for o, m in outs:
        check_attention(pool, table, ctx, rs, q, o, m)


def test_attention_rows_past_max_rows_are_left():
    rng = np.random.default_rng(15)
    pool, table, ctx, rs, q, out, mass = run_attention(rng, 1, 2, 128, [(100, 3), (50, 1)], True,
                                                       max_rows=1)
    got = host(out)
    assert (got[1:3] == -3.0).all() and (got[0] != -3.0).any() and (got[3] != -3.0).any()
    # the same as with those rows taken out of the batch
    keep = [0, 3]
    dev = to_dev(pool)
    again = foe.cache_attention(q[:, keep].contiguous(), dev["k"], dev["v"], dev["kv_scale"],
                                ints(table), ints(ctx), ints([0, 1, 2]), 1)
    assert torch.equal(out[keep], again)


def test_attention_past_the_tables_end():
    """Rows behind the last slot see what the table holds."""
    rng = np.random.default_rng(16)
    H, nq, hd = 1, 1, 96
    pool = random_pool(rng, 4, H, hd)
    dev, table = to_dev(pool), np.array([[2, 0]], dtype=np.int32)
    q = bf16(rng.normal(size=(H, 12, nq, hd)))
    say("past the table's end")
    mass = torch.full_like(dev["mass"], -7.0)
    out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints([120]),
                              ints([0, 12]), 12, mass_in=dev["mass"], mass_out=mass)
    torch.cuda.synchronize()
    check_attention(pool, table, [120], np.array([0, 12]), q, out, mass)


def test_attention_full_tables():
    """Sequences that fill their tables, or would pass them, beside one another: what is
    kept for the mass stays within the workspace."""
    rng = np.random.default_rng(20)
    H, nq, hd, B = 2, 4, 96, 5
    pool = random_pool(rng, 12, H, hd)
    dev, table = to_dev(pool), rng.permutation(12)[:10].reshape(5, 2).astype(np.int32)
    ctx, rs = [128, 127, 128, 300, 126], np.array([0, 1, 3, 4, 6, 9])
    q = bf16(rng.normal(size=(H, 9, nq, hd)))
    n = foe.cache_attention_workspace_bytes(q, ints(table), 3, True)
    ws = torch.zeros(n + (1 << 20), dtype=torch.uint8, device=DEV)
    ws[n:] = 0xA5
    say("full tables")
    mass = torch.full_like(dev["mass"], -7.0)
    out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                              ints(rs), 3, mass_in=dev["mass"], mass_out=mass, ws=ws)
    torch.cuda.synchronize()
    assert (ws[n:] == 0xA5).all()
    check_attention(pool, table, [min(c, 128) for c in ctx], rs, q, out, mass)


def test_attention_large_decode_batch():
    """A batch whose pages are dealt to more workgroups than the card holds at a time, with
    the mass; three of its sequences against the oracle, in a pool of their pages."""
    H, nq, hd, B, blocks = 2, 2, 96, 72, 110
    rng = np.random.default_rng(19)
    g = torch.Generator(DEV).manual_seed(19)
    dev = foe.cache_empty(B * blocks, H, hd, DEV)
    for n in ("k", "v"):
        dev[n].copy_(torch.randn(dev[n].shape, generator=g, device=DEV))
    dev["kv_scale"].copy_(2.0 ** torch.randint(-2, 2, dev["kv_scale"].shape, generator=g,
                                               device=DEV))
    dev["mass"].uniform_(generator=g)
    table = rng.permutation(B * blocks).astype(np.int32).reshape(B, blocks)
    ctx = rng.integers(5500, 64 * blocks, B)
    q = bf16(rng.normal(size=(H, B, nq, hd)))
    mass = torch.full_like(dev["mass"], -7.0)
    say("large decode batch")
    out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                              ints(range(B + 1)), 1, mass_in=dev["mass"], mass_out=mass)
    torch.cuda.synchronize()
    picked = [0, 41, B - 1]
    pages = torch.from_numpy(table[picked].reshape(-1)).long().to(DEV)
    pool = to_host({n: t.view(torch.uint8)[pages].view(t.dtype) if n in "kv" else t[pages]
                    for n, t in dev.items()})
    check_attention(pool, np.arange(len(pages), dtype=np.int32).reshape(3, blocks), ctx[picked],
                    np.arange(4), q[:, picked].contiguous(), out[picked], mass[pages])


@pytest.mark.parametrize("H,nq,hd,ctx,rows,picked", [
    (1, 2, 128, 131071, 1, [0]),
    (1, 1, 96, 40000, 300, [0, 1, 63, 64, 255, 256, 299]),
])
def test_attention_long_contexts(H, nq, hd, ctx, rows, picked):
    rng = np.random.default_rng(17)
    say("long", ctx, rows)
    a = run_attention(rng, H, nq, hd, [(ctx, rows)], False)
    check_attention(*a, rows=picked)


def test_pool_past_four_gib():
    """Pages whose offsets in the pool pass 32 bits, in every entry point."""
    H, hd, pages = 8, 128, 70000  # 4.6 GB of keys, as much of values
    rng = np.random.default_rng(18)
    dev = foe.cache_empty(pages, H, hd, DEV)
    table = np.array([[69999, 3], [66000, 68000]], dtype=np.int32)
    dst = np.array([[69000], [65999]], dtype=np.int32)
    rs = [0, 100, 170]
    qkv = bf16(rng.normal(size=(H, 170, 3, hd)))
    say("large pool")
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints([0, 0]),
                         ints(rs), THETA, SCALE)
    out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints([0, 0]),
                              ints(rs), 100, mass_in=dev["mass"], mass_out=dev["mass"])
    kept, n = foe.cache_evict(dev["k"], dev["v"], dev["kv_scale"], dev["mass"], ints(table),
                              ints([100, 70]), 40, 10, ints(dst))
    torch.cuda.synchronize()
    # the same in a small pool
    small = foe.cache_empty(6, H, hd, DEV)
    t2, d2 = np.array([[0, 1], [2, 3]], dtype=np.int32), np.array([[4], [5]], dtype=np.int32)
    q2 = foe.cache_append(qkv, small["k"], small["v"], small["kv_scale"], ints(t2), ints([0, 0]),
                          ints(rs), THETA, SCALE)
    out2 = foe.cache_attention(q2, small["k"], small["v"], small["kv_scale"], ints(t2),
                               ints([0, 0]), ints(rs), 100, mass_in=small["mass"],
                               mass_out=small["mass"])
    kept2, n2 = foe.cache_evict(small["k"], small["v"], small["kv_scale"], small["mass"],
                                ints(t2), ints([100, 70]), 40, 10, ints(d2))
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(out, out2) and torch.equal(kept, kept2)
    assert torch.equal(n, n2)
    for a, b in ((table[0, 0], 0), (table[1, 0], 2)):  # full pages (others end before slot 64)
        for name in ("k", "v"):
            assert torch.equal(dev[name][a].view(torch.uint8), small[name][b].view(torch.uint8))
    for a, b in ((dst[0, 0], 4), (dst[1, 0], 5)):
        assert torch.equal(dev["k"][a, :, :40].view(torch.uint8),
                           small["k"][b, :, :40].view(torch.uint8))
        assert torch.equal(dev["mass"][a, :, :40], small["mass"][b, :, :40])
        assert torch.equal(dev["kv_scale"][a], small["kv_scale"][b])


# ---- eviction -----------------------------------------------------------------------

def check_evict(rng, H, hd, lengths, keep, recent, blocks=None, mass=None, table=None, pool=None,
                absent=(), dst=None):
    B = len(lengths)
    blocks = blocks or max(1, max((n + 63) // 64 for n in lengths))
    D = (keep + 63) // 64
    pages = B * (blocks + D) + 2
    order = rng.permutation(pages).astype(np.int32)
    table = order[:B * blocks].reshape(B, blocks) if table is None else table
    for at in absent:
        table[at] = -1
    dst = order[B * blocks:B * (blocks + D)].reshape(B, D) if dst is None else dst
    pool = pool or random_pool(rng, pages, H, hd)
    if mass is not None:
        pool["mass"] = mass(pool["mass"]).astype(np.float32)
    dev = to_dev(pool)
    kept, new_len = foe.cache_evict(dev["k"], dev["v"], dev["kv_scale"], dev["mass"], ints(table),
                                    ints(lengths), keep, recent, ints(dst))
    torch.cuda.synchronize()
    want = {n: a.copy() for n, a in pool.items()}
    k_ref, n_ref = co.evict(want, table, np.clip(lengths, 0, blocks * 64), keep, recent, dst)
    assert np.array_equal(new_len.cpu().numpy(), n_ref)
    assert np.array_equal(kept.cpu().numpy(), k_ref)
    same(to_host(dev), want)


EVICTS = [
    # H, hd, lengths, keep, recent
    (1, 96, [1], 1, 0),
    (2, 128, [65, 64, 63, 0, 200], 64, 16),
    (2, 96, [300, 10, 129], 100, 100),       # the recent tokens only
    (1, 128, [1000], 1, 0),
    (3, 96, [257, 1500, 64], 200, 0),
    (2, 128, [2000, 1024, 1025], 777, 33),
    (1, 96, [5000], 4999, 1),
]


@pytest.mark.parametrize("H,hd,lengths,keep,recent", EVICTS)
def test_evict_parity(H, hd, lengths, keep, recent):
    say("evict", H, hd, lengths, keep, recent)
    check_evict(np.random.default_rng([21, H, hd, keep]), H, hd, lengths, keep, recent)


@pytest.mark.parametrize("hd", [96, 128])
@pytest.mark.parametrize("keep", [1900, 1000, 500, 250, 60])
def test_evict_thick_and_sparse(hd, keep):
    """16 kept tokens out of two to more than four of the source's 16-token groups, absent
    pages among them."""
    rng = np.random.default_rng([27, hd, keep])
    say("evict thick and sparse", hd, keep)
    check_evict(rng, 2, hd, [1984, 1951], keep, 20, absent=[(0, 3), (1, 0), (1, 17)])


@pytest.mark.parametrize("first", [48, 57, 63])
def test_evict_into_the_pools_first_page(first):
    """Kept tokens that pass from the end of another page into page 0."""
    rng = np.random.default_rng([28, first])
    n, keep = 128, 128 - first

    def mass(m):
        m[1], m[0] = np.arange(64) >= first, 1.0
        return m

    say("evict into page 0", first)
    check_evict(rng, 1, 128, [n], keep, 0, mass=mass, table=np.array([[1, 0]], dtype=np.int32),
                dst=np.array([[3, 2]], dtype=np.int32))


@pytest.mark.parametrize("what", ["equal", "two", "neighbours", "special", "infinite",
                                  "negative"])
def test_evict_masses_near_each_other(what):
    rng = np.random.default_rng(22)

    def mass(m):
        if what == "equal":
            return np.zeros_like(m)
        if what == "two":
            return (rng.random(m.shape) < 0.3) * 0.25
        if what == "neighbours":  # within four steps of each other
            return np.float32(1.0) + rng.integers(0, 4, m.shape) * np.float32(2.0 ** -23)
        if what == "infinite":  # NaN ranks above infinity
            return rng.choice(np.float32([np.nan, -np.nan, np.inf, -np.inf, 0.5]), m.shape)
        if what == "special":
            m = m.copy()
            m[rng.random(m.shape) < 0.05] = np.nan
            m[rng.random(m.shape) < 0.3] = 0.0
            m[rng.random(m.shape) < 0.3] = -0.0
            return m
        return -m

    say("evict", what)
    check_evict(rng, 2, 96, [700, 100, 1500], 333, 20, mass=mass)


@pytest.mark.parametrize("what", ["equal", "two", "spread"])
def test_evict_long_sequences(what):
    """Sequences of more tokens than a workgroup of the selection holds, beside shorter
    ones of the same call, ties across the workgroups' borders included."""
    rng = np.random.default_rng(25)

    def mass(m):
        if what == "equal":
            return np.full_like(m, 0.5)
        return (rng.random(m.shape) < 0.4) * 0.25 if what == "two" else m

    say("evict long sequences", what)
    check_evict(rng, 1, 96, [70001, 32768, 33000, 150, 65536], 20000, 300, mass=mass)


def test_evict_spread_scales_and_nan_keys():
    """Tokens of pages with scales far apart in one new page (the small ones fall
    among its subnormals or to zero), keys of NaN codes, and absent pages."""
    rng = np.random.default_rng(23)
    H, hd, B, blocks = 2, 128, 1, 8
    pages = 20
    pool = random_pool(rng, pages, H, hd)
    pool["kv_scale"] = 2.0 ** rng.integers(-100, 60, (pages, H, 2)).astype(np.float64)
    pool["kv_scale"][1::2] = 2.0 ** rng.integers(-9, 4, (pages // 2, H, 2))
    pool["k"][:, :, 7] = 0x7F
    table = np.arange(8, dtype=np.int32)[None]
    table[0, 3] = -1
    pool["mass"][...] = rng.random(pool["mass"].shape)
    say("evict spread scales")
    dst = np.array([[10, 12, 14]], dtype=np.int32)
    dev = to_dev(pool)
    kept, _ = foe.cache_evict(dev["k"], dev["v"], dev["kv_scale"], dev["mass"], ints(table),
                              ints([blocks * 64]), 170, 5, ints(dst))
    torch.cuda.synchronize()
    want = {n: a.copy() for n, a in pool.items()}
    k_ref, _ = co.evict(want, table, [blocks * 64], 170, 5, dst)
    assert np.array_equal(kept.cpu().numpy(), k_ref)
    same(to_host(dev), want)


def test_evict_long_and_bad_lengths():
    rng = np.random.default_rng(24)
    say("evict long")
    check_evict(rng, 1, 96, [40000, -3, 1 << 30], 3001, 64, blocks=640)


# ---- together, and how the calls may be made ---------------------------------------

def serve(H, nq, hd, steps, keep, recent, stream=None):
    """Two sequences through prompt chunks, decode steps and evictions; everything that
    the calls return, and a check of each call against the oracle."""
    rng = np.random.default_rng(31)
    pages, blocks, D = 40, 8, (keep + 63) // 64
    free = list(range(pages))
    table = np.full((2, blocks), -1, dtype=np.int32)
    pool = random_pool(rng, pages, H, hd)
    dev = to_dev(pool)
    ctx, pos = [0, 0], [0, 0]
    for n in steps:
        rs = np.concatenate([[0], np.cumsum(n)])
        for b in range(2):
            for blk in range((ctx[b] + n[b] + 63) // 64):
                if table[b, blk] < 0:
                    table[b, blk] = free.pop()
        qkv = bf16(rng.normal(size=(H, rs[-1], nq + 2, hd)))
        pool = to_host(dev)
        q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                             ints(rs), THETA, SCALE, pos=ints(pos), stream=stream)
        torch.cuda.synchronize()
        check_append(pool, dev, host(qkv), table, ctx, rs, q, pos)
        pool = to_host(dev)
        out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                                  ints(rs), int(max(n)), mass_in=dev["mass"],
                                  mass_out=dev["mass"], stream=stream)
        torch.cuda.synchronize()
        o, spread, big, got = co.attend(pool, host(q), table, ctx, rs, mass=True)
        assert (np.abs(host(out) - o) <= attention_bound(o, spread)).all()
        m = dev["mass"].double().cpu().numpy()
        for (b, h), w in got.items():
            for t, x in enumerate(w):
                p = table[b, t // 64]
                before = float(pool["mass"][p, h, t % 64]) if t < ctx[b] else 0.0
                assert abs(m[p, h, t % 64] - before - x) <= mass_bound(x, before, big, hd,
                                                                       int(n[b]) * nq)
        ctx = [c + k for c, k in zip(ctx, n)]
        pos = [c + k for c, k in zip(pos, n)]
        if max(ctx) > keep:
            dst = np.array([[free.pop() for _ in range(D)] for _ in range(2)], dtype=np.int32)
            pool = to_host(dev)
            kept, new_len = foe.cache_evict(dev["k"], dev["v"], dev["kv_scale"], dev["mass"],
                                            ints(table), ints(ctx), keep, recent, ints(dst),
                                            stream=stream)
            torch.cuda.synchronize()
            k_ref, n_ref = co.evict(pool, table, ctx, keep, recent, dst)
            assert np.array_equal(kept.cpu().numpy(), k_ref)
            same(to_host(dev), pool)
            free += [int(p) for p in table.flatten() if p >= 0]
            table[:] = -1
            for b in range(2):
                used = (n_ref[b] + 63) // 64
                table[b, :used] = dst[b, :used]
                free += [int(p) for p in dst[b, used:]]
            ctx = [int(x) for x in n_ref]


def test_serving_loop():
    say("serving loop")
    serve(2, 2, 128, [(100, 30), (1, 1), (40, 1), (1, 1), (1, 130), (1, 1), (1, 1), (60, 60)],
          128, 24)


def test_serving_loop_small_head_on_another_stream():
    say("serving loop, stream")
    serve(3, 1, 96, [(10, 200), (1, 1), (1, 1)], 150, 150, stream=torch.cuda.Stream())


def _decode_inputs(seed, mass=True, seqs=((700, 1), (90, 1), (64, 1))):
    rng = np.random.default_rng(seed)
    H, nq, hd = 2, 2, 128
    ctx, rs, table, pages = batch(rng, seqs, extra=1)
    dev = to_dev(random_pool(rng, pages + 20, H, hd))
    dst = ints(np.arange(pages, pages + 3 * len(seqs)).reshape(len(seqs), 3))
    qkv = bf16(rng.normal(size=(H, rs[-1], nq + 2, hd)))
    return dev, ints(table), ints(ctx), ints(rs), qkv, dst


@pytest.mark.parametrize("seqs", [((700, 1), (90, 1), (64, 1)), ((300, 90), (64, 200))],
                         ids=["step", "chunk"])
def test_calls_repeat_bit_for_bit(seqs):
    dev, table, ctx, rs, qkv, _ = _decode_inputs(41, seqs=seqs)
    say("determinism", seqs)
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], table, ctx, rs, THETA)
    outs = []
    for _ in range(3):
        m = torch.zeros_like(dev["mass"])
        outs.append((foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], table, ctx, rs,
                                         200, mass_in=dev["mass"], mass_out=m), m))
    torch.cuda.synchronize()
    for o, m in outs[1:]:
        assert torch.equal(o, outs[0][0]) and torch.equal(m, outs[0][1])


@pytest.mark.parametrize("seqs", [((700, 1), (90, 1), (64, 1)), ((300, 90), (64, 200))],
                         ids=["step", "chunk"])
def test_graph_replay(seqs):
    """A step of all three calls captured once and replayed, eager work between the
    replays, gives the eager result each time; two graphs share one workspace."""
    dev, table, ctx, rs, qkv, dst = _decode_inputs(42, seqs=seqs)
    rows = max(n for _, n in seqs)
    length = ctx + (rs[1:] - rs[:-1])
    B, H = table.shape[0], 2
    q = torch.empty((H, qkv.shape[1], 2, 128), dtype=torch.bfloat16, device=DEV)
    out = torch.empty((qkv.shape[1], H, 2, 128), dtype=torch.bfloat16, device=DEV)
    kept = torch.empty((B, H, 150), dtype=torch.int32, device=DEV)
    new_len = torch.empty((B,), dtype=torch.int32, device=DEV)
    ws = torch.empty(max(1, foe.cache_attention_workspace_bytes(q, table, rows, True)),
                     dtype=torch.uint8, device=DEV)
    mass0 = dev["mass"].clone()
    pool = {n: dev[n].clone() for n in ("k", "v", "kv_scale")}

    def step(stream=None):
        foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], table, ctx, rs, THETA, q=q,
                         stream=stream)
        foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], table, ctx, rs, rows,
                            mass_in=dev["mass"], mass_out=dev["mass"], out=out, ws=ws,
                            stream=stream)
        foe.cache_evict(dev["k"], dev["v"], dev["kv_scale"], dev["mass"], table, length, 150, 30,
                        dst, kept=kept, new_len=new_len, stream=stream)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (q.view(torch.int16), out.view(torch.int16), kept, new_len,
                                    dev["mass"], dev["kv_scale"], dev["k"].view(torch.uint8),
                                    dev["v"].view(torch.uint8))]

    def reset():
        dev["mass"].copy_(mass0)
        for n in pool:
            dev[n].view(torch.uint8).copy_(pool[n].view(torch.uint8))
        for t in (q, out, kept, new_len):
            t.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()

    step()
    want = results()
    side = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    say("graph replay", seqs)
    for g in graphs:
        with torch.cuda.graph(g, stream=side):
            step(side)
    for rep in range(4):
        reset()
        graphs[rep % 2].replay()
        for a, b in zip(results(), want):
            assert torch.equal(a, b), rep
        reset()
        step()
        for a, b in zip(results(), want):
            assert torch.equal(a, b), rep


def test_calls_on_two_streams_at_once():
    """Two batches on streams of their own, in flight together, give what each gives alone."""
    batches = [_decode_inputs(seed, seqs=seqs) for seed, seqs in (
        (50, ((700, 1), (3000, 1), (64, 1))), (51, ((900, 60), (5, 1), (64, 90))))]

    for x in batches:
        x[0]["mass_out"] = torch.zeros_like(x[0]["mass"])

    def call(x, stream=None):
        dev, table, ctx, rs, qkv, dst = x
        rows = 1 if qkv.shape[1] == table.shape[0] else 90
        q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], table, ctx, rs, THETA,
                             stream=stream)
        out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], table, ctx, rs, rows,
                                  mass_in=dev["mass"], mass_out=dev["mass_out"], stream=stream)
        kept, n = foe.cache_evict(dev["k"], dev["v"], dev["kv_scale"], dev["mass"], table, ctx,
                                  150, 30, dst, stream=stream)
        return out.view(torch.int16), dev["mass_out"], kept, n

    say("two streams")
    want = [[t.clone() for t in call(x)] for x in batches]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for _ in range(8):
        got = [call(x, s) for x, s in zip(batches, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_shared_prefix_pages():
    """Sequences that read the same pages: a common prefix, and one table twice."""
    rng = np.random.default_rng(52)
    pool = random_pool(rng, 24, 2, 96)
    table = rng.permutation(12).astype(np.int32).reshape(3, 4)
    table[1, :3] = table[0, :3]
    table[2] = table[0]
    ctx, rs = [200, 230, 200], np.array([0, 1, 41, 42])
    dev, q = to_dev(pool), bf16(rng.normal(size=(2, 42, 2, 96)))
    say("shared prefix")
    out = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                              ints(rs), 40)
    torch.cuda.synchronize()
    check_attention(pool, table, ctx, rs, q, out, None)
    check_evict(rng, 2, 96, [200, 230, 200], 90, 10, table=table, pool=pool,
                dst=np.arange(12, 18, dtype=np.int32).reshape(3, 2))


def test_empty_batches():
    dev = foe.cache_empty(2, 1, 96, DEV)
    table, none = ints([[0, 1]]), ints([0])
    q = foe.cache_append(torch.empty((1, 0, 3, 96), dtype=torch.bfloat16, device=DEV), dev["k"],
                         dev["v"], dev["kv_scale"], table, none, ints([0, 0]), THETA)
    assert q.shape == (1, 0, 1, 96)
    o = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], table, none, ints([0, 0]), 1)
    assert o.shape == (0, 1, 1, 96)
    empty = torch.empty((0, 2), dtype=torch.int32, device=DEV)
    kept, n = foe.cache_evict(dev["k"], dev["v"], dev["kv_scale"], dev["mass"], empty,
                              ints(np.zeros(0)), 4, 1, torch.empty((0, 1), dtype=torch.int32,
                                                                   device=DEV))
    assert kept.shape == (0, 1, 4) and n.shape == (0,)


def test_binding_refuses():
    dev = foe.cache_empty(2, 2, 96, DEV)
    table, ctx, rs = ints([[0, 1]]), ints([0]), ints([0, 1])
    qkv = torch.zeros((2, 1, 3, 96), dtype=torch.bfloat16, device=DEV)
    pool = (dev["k"], dev["v"], dev["kv_scale"])
    with pytest.raises(foe.FoeError, match="bf16"):
        foe.cache_append(qkv.float(), *pool, table, ctx, rs, THETA)
    with pytest.raises(foe.FoeError, match="row_start"):
        foe.cache_append(qkv, *pool, table, ctx, ctx, THETA)
    with pytest.raises(foe.FoeError, match="v must be"):
        foe.cache_append(qkv, dev["k"], dev["v"][:1], dev["kv_scale"], table, ctx, rs, THETA)
    with pytest.raises(TypeError, match="block_table"):
        foe.cache_append(qkv, *pool, table.long(), ctx, rs, THETA)
    with pytest.raises(ValueError, match="contiguous"):
        foe.cache_append(torch.zeros((2, 2, 3, 96), dtype=torch.bfloat16, device=DEV)[:, ::2],
                         *pool, table, ctx, rs, THETA)
    q = qkv[:, :, :1].contiguous()
    with pytest.raises(ValueError, match="tensors on"):
        foe.cache_attention(q, *pool, table, ctx.cpu(), rs, 1)
    with pytest.raises(foe.FoeError, match="max_rows"):
        foe.cache_attention(q, *pool, table, ctx, rs, 0)
    with pytest.raises(foe.FoeError, match="go together"):
        foe.cache_attention(q, *pool, table, ctx, rs, 1, mass_in=dev["mass"])
    with pytest.raises(foe.FoeError, match="dst_blocks"):
        foe.cache_evict(*pool, dev["mass"], table, ctx, 65, 1, ints([[1]]))
    with pytest.raises(foe.FoeError, match="recent"):
        foe.cache_evict(*pool, dev["mass"], table, ctx, 4, 5, ints([[1]]))
