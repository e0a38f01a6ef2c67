"""The 8-bit key/value cache at the ends of its range."""

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2605_06206_amd import foe
from test_gpu_cache import (DEV, SCALE, THETA, attention_bound, batch, bf16, check_append,
                            check_evict, host, ints, mass_bound, random_pool, say, to_dev, to_host)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    foe.lib()


# ---- eviction ---------------------------------------------------------------------

def zero_tokens(pool, table, which, what):
    """Codes 0 (either sign) for the tokens `which` of the first sequence."""
    for t in which:
        p, s = table[0, t // 64], t % 64
        if what != "v":
            pool["k"][p, :, s] &= 0x80
        if what != "k":
            pool["v"][p, :, s // 16, :, s % 16] &= 0x80
        pool["mass"][p, :, s] = 2.0


@pytest.mark.parametrize("hd", [96, 128])
@pytest.mark.parametrize("what", ["k", "v", "both"])
@pytest.mark.parametrize("which", ["thick", "sparse"])
def test_evict_zero_tokens_of_large_scales(hd, what, which):
    """The kept tokens of a new page are all zero, in pages whose scale passes the smallest
    one by more than fp32 holds: they stay zero."""
    rng = np.random.default_rng([61, hd])
    pool = random_pool(rng, 12, 2, hd)
    pool["mass"][...] = 1.0
    pool["kv_scale"][:6] = 2.0 ** np.array([27, 28, 30, 60, 100, 120])[:, None, None]
    table = np.arange(6, dtype=np.int32)[None]
    tokens = range(10, 384, 5) if which == "sparse" else [t for t in range(384) if t % 64 >= 20]
    zero_tokens(pool, table, tokens, what)
    say("evict zero tokens", hd, what, which)
    check_evict(rng, 2, hd, [384], len(tokens), 0, pool=pool, table=table,
                dst=np.arange(6, 6 + (len(tokens) + 63) // 64, dtype=np.int32)[None])


@pytest.mark.parametrize("hd", [96, 128])
def test_evict_zero_tokens_beside_small_ones(hd):
    """Zero tokens of a page of large scale, and NaN keys there, beside tokens of a page of
    small scale: the ratio of the scales passes fp32."""
    rng = np.random.default_rng([62, hd])
    pool = random_pool(rng, 4, 1, hd)
    pool["mass"][...] = 1.0
    pool["kv_scale"][:2] = 2.0 ** np.array([60, -90])[:, None, None]
    pool["kv_scale"][0, 0] = 2.0 ** 60, 2.0 ** 100
    pool["k"][0, :, 8] = 0x7F
    table = np.array([[0, 1]], dtype=np.int32)
    zero_tokens(pool, table, [t for t in range(0, 64, 3) if t != 8], "both")
    pool["v"][0, :, 0, :, 8] = 0
    pool["mass"][0, :, 8] = pool["mass"][1, :, 5:20] = 2.0
    say("evict zero tokens beside small ones", hd)
    check_evict(rng, 1, hd, [128], 22 + 1 + 15, 0, pool=pool, table=table,
                dst=np.array([[3]], dtype=np.int32))


def test_evict_the_neighbours_of_an_outlier():
    """A token of 1e12 makes its page's ordinary tokens zero codes; it is evicted, and what
    sees the others afterwards is finite."""
    rng = np.random.default_rng(63)
    H, nq, hd = 2, 2, 128
    dev = foe.cache_empty(4, H, hd, DEV)
    x = rng.normal(size=(H, 40, nq + 2, hd))
    x[:, 3, nq:] = 1e12
    table, rs = ints([[0]]), ints([0, 40])
    pool = (dev["k"], dev["v"], dev["kv_scale"])
    say("evict an outlier")
    foe.cache_append(bf16(x), *pool, table, ints([0]), rs, THETA, SCALE)
    dev["mass"].fill_(1.0)
    dev["mass"][:, :, 3] = 0.5
    before = to_host(dev)
    kept, n = foe.cache_evict(*pool, dev["mass"], table, ints([40]), 30, 4, ints([[2]]))
    q = foe.cache_append(bf16(rng.normal(size=(H, 1, nq + 2, hd))), *pool, ints([[2]]), n,
                         ints([0, 1]), THETA, SCALE, pos=ints([40]))
    o = foe.cache_attention(q, *pool, ints([[2]]), n, ints([0, 1]), 1)
    torch.cuda.synchronize()
    assert not (kept == 3).any()
    k_ref, _ = co.evict(before, np.array([[0]]), [40], 30, 4, np.array([[2]]))
    assert np.array_equal(kept.cpu().numpy(), k_ref)
    assert (before["kv_scale"][2] == 2.0 ** -100).all()
    assert (to_host(dev)["k"][2, :, :30] & 0x7F == 0).all()
    assert torch.isfinite(o).all()


# ---- mass beside rows that are not finite ----------------------------------------------

def check_mass(pool, table, ctx, rs, q, mass_out, far=False):
    """Masses against the oracle's, NaN where it has NaN.  (far: the probabilities are 0 or
    equal, of scores that are exact)"""
    m = host(mass_out)
    nq, hd = q.shape[2:]
    ref = co.attend(pool, host(q), table, ctx, rs, mass=True)
    finite = np.nan_to_num(host(q), nan=0.0, posinf=0.0, neginf=0.0)
    big = 0.0 if far else co.attend(pool, finite, table, ctx, rs)[2]
    for (b, h), w in ref[3].items():
        slot = np.arange(len(w))
        p = table[b, slot // 64]
        there = (p >= 0) & (p < len(m))
        slot, p, w = slot[there], p[there], w[there]
        got = m[p, h, slot % 64]
        before = np.where(slot < ctx[b], pool["mass"][p, h, slot % 64], 0.0).astype(np.float64)
        assert np.array_equal(np.isnan(got), np.isnan(w)), (b, h, np.isnan(got) ^ np.isnan(w))
        lim = mass_bound(w, before, big, hd, (rs[b + 1] - rs[b]) * nq)
        ok = np.isnan(w) | (np.abs(got - before - w) <= lim)
        assert ok.all(), (b, h, slot[~ok][:8], got[~ok][:8], w[~ok][:8])
    return ref


NAN_ROWS = [
    # nq, hd, [(ctx, rows)], row with a NaN query, width of the table (0: what is needed)
    (2, 128, [(10, 8), (61, 6), (3, 1)], 3, 0),           # few columns, scores kept
    (1, 96, [(62, 12), (0, 5)], 4, 0),
    (2, 96, [(10, 8), (0, 3)], 5, 70000),                 # few columns, scores formed again
    (2, 128, [(0, 40), (0, 1)], 20, 0),                   # chunks
    (1, 96, [(100, 300), (5, 70)], 150, 0),
    (3, 128, [(30, 100), (7, 2), (300, 1), (64, 1)], 33, 0),  # both
]


@pytest.mark.parametrize("nq,hd,seqs,bad,width", NAN_ROWS)
@pytest.mark.parametrize("what", ["nan", "inf", "key"])
def test_mass_beside_rows_that_are_not_finite(nq, hd, seqs, bad, width, what):
    """A row of NaN (by its query, or a key that it sees) makes the masses of the tokens
    that it sees NaN, and no other's."""
    rng = np.random.default_rng([64, nq, hd, bad])
    H = 2
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    qx = rng.normal(size=(H, rs[-1], nq, hd))
    if what == "key":  # of the last row: the rows before do not see it
        t = ctx[0] + seqs[0][1] - 1
        pool["k"][table[0, t // 64], 1, t % 64] = 0x7F
    elif what == "nan":
        qx[1, bad, nq - 1, 5] = np.nan
    else:
        qx[0, bad, 0, :] = -np.inf
    dev, q = to_dev(pool), bf16(qx)
    wide = table
    if width:
        wide = np.full((len(seqs), width), -1, dtype=np.int32)
        wide[:, :table.shape[1]] = table
    mass = torch.full_like(dev["mass"], -7.0)
    say("mass beside rows that are not finite", nq, hd, seqs, bad, width, what)
    o = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(wide), ints(ctx),
                            ints(rs), max(n for _, n in seqs), mass_in=dev["mass"],
                            mass_out=mass)
    torch.cuda.synchronize()
    ref = check_mass(pool, table, ctx, rs, q, mass)
    assert np.array_equal(np.isnan(host(o)), np.isnan(ref[0]))


# ---- scores near the ends of fp32 ----------------------------------------------------

FAR = [(1, [(0, 1), (300, 1), (700, 1), (64, 1)]),          # few columns
       (2, [(90, 8), (5, 3)]),
       (2, [(0, 70), (300, 200)]),                          # chunks
       (1, [(1500, 100), (200, 1), (0, 1), (129, 1), (0, 16)])]  # both


@pytest.mark.parametrize("hd", [96, 128])
@pytest.mark.parametrize("nq,seqs", FAR)
@pytest.mark.parametrize("sign,level", [(1, 2), (-1, 2), (1, 32), (-1, 32), (-1, 60), (1, 100),
                                        (-1, 100), (1, 112), (-1, 112)])
def test_attention_scores_far_from_zero(hd, nq, seqs, sign, level):
    """Scores of some 2^level of either sign: the tokens whose score is the largest share
    the weight alike (their scores are equal and exact), the others, a quarter of it below,
    get none."""
    rng = np.random.default_rng([65, hd, nq, level])
    H = 2
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    # keys of ones and of 1.25, in units of 2^(level - 60): pages and tokens of both
    big = (rng.random((pages, H, 64)) < 0.3) | (rng.random((pages, 1, 1)) < 0.3)
    pool["k"][...] = co.encode(np.where(big, 1.25, 1.0))[..., None]
    s = level - 60
    pool["kv_scale"][..., 0] = 2.0 ** s
    qx = np.full((H, rs[-1], nq, hd), sign * 2.0 ** 60)
    dev, q = to_dev(pool), bf16(qx)
    mass = torch.full_like(dev["mass"], -7.0)
    say("far scores", hd, nq, seqs, sign, level)
    o = foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                            ints(rs), max(n for _, n in seqs), mass_in=dev["mass"],
                            mass_out=mass)
    torch.cuda.synchronize()
    ref = check_mass(pool, table, ctx, rs, q, mass, far=level > 2)
    err, lim = np.abs(host(o) - ref[0]), attention_bound(ref[0], ref[1])
    assert (err <= lim).all(), (np.argwhere(err > lim)[:8], err.max())


@pytest.mark.parametrize("rows", [1, 6, 90])
@pytest.mark.parametrize("what", ["query", "overflow", "mixed"])
def test_attention_scores_of_minus_infinity(rows, what):
    """A row whose scores are all -inf (an infinite query, or products past fp32) is NaN, as
    its softmax is; one that sees no token gives zeros."""
    rng = np.random.default_rng([66, rows])
    H, nq, hd = 1, 2, 96
    seqs = [(300, rows), (0, 2), (700, 1)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    pool["k"][...] = co.encode(1.0)
    pool["kv_scale"][..., 0] = 2.0 ** 60
    table[2] = -1
    qx = rng.normal(size=(H, rs[-1], nq, hd))
    bad = np.zeros((rs[-1], H, nq), dtype=bool)
    bad[rows // 2, 0, 1] = bad[rs[1], 0, 0] = bad[rs[2], 0, 1] = True
    qx[np.swapaxes(bad, 0, 1)] = {"query": -np.inf, "overflow": -2.0 ** 100,
                                  "mixed": -2.0 ** 100}[what]
    if what == "mixed":  # one page in reach: the others lose nothing by it
        pool["kv_scale"][table[0, 0], :, 0] = 2.0 ** 10
    dev, q = to_dev(pool), bf16(qx)
    mass = torch.full_like(dev["mass"], -7.0)
    say("scores of -inf", rows, what)
    o = host(foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                                 ints(rs), rows, mass_in=dev["mass"], mass_out=mass))
    want = bad.copy()
    want[rs[2]] = False                       # sees no token
    if what == "mixed":
        want[rows // 2] = False               # the scores of one page are finite
        ref = co.attend(pool, host(q), table, ctx, rs)
        assert (np.abs(o - ref[0]) <= attention_bound(ref[0], ref[1]))[rows // 2].all()
    assert np.array_equal(np.isnan(o).all(-1), want)
    assert np.isfinite(o[~want]).all() and (o[rs[2]] == 0).all()
    # tokens that a NaN row sees, and no others, get a mass of NaN
    m = host(mass)
    seen = 0 if what == "mixed" else ctx[0] + rows // 2 + 1
    for t in range(ctx[0] + rows):
        assert np.isnan(m[table[0, t // 64], 0, t % 64]) == (t < seen), t


# ---- magnitudes that no code holds -----------------------------------------------------

@pytest.mark.parametrize("hd", [96, 128])
def test_append_magnitudes_past_the_codes(hd):
    """From 1.9375 * 2^127 on a value rounds to 2^128, past fp32, and a rotated key may
    pass it by itself: such tokens are stored as non-finite ones, the largest below are
    held."""
    rng = np.random.default_rng([67, hd])
    H, nq, most = 2, 1, 1.875 * 2.0 ** 127
    ctx, rs, table, pages = batch(rng, [(5, 12), (0, 3)])
    pool = random_pool(rng, pages, H, hd)
    dev = to_dev(pool)
    x = rng.normal(size=(H, rs[-1], nq + 2, hd))
    x[0, 2, 2, 7] = 3.3895e38                   # a value: 1.9921875 * 2^127
    x[1, 4, 2, 0] = -1.9375 * 2.0 ** 127        # the border itself
    x[1, 1, 2, 1] = most                        # held
    x[1, 12, 1, 3] = x[1, 12, 1, 3 + hd // 2] = most   # position 0: held as it is
    x[1, 12:, 0, 3] = x[1, 12:, 0, 3 + hd // 2] = 0.0  # (a query that it leaves finite)
    x[0, 8, 1, 0], x[0, 8, 1, hd // 2] = most, -most   # a key whose rotation passes it
    qkv = bf16(x)
    bad = np.zeros((rs[-1], H), dtype=bool)
    bad[2, 0] = bad[4, 1] = bad[8, 0] = True
    say("append magnitudes", hd)
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                         ints(rs), THETA, SCALE)
    torch.cuda.synchronize()
    got = check_append(pool, dev, host(qkv), table, ctx, rs, q)
    for b, h, i in ((0, 0, 2), (0, 1, 4), (0, 0, 8)):
        t = ctx[b] + i
        assert (got["k"][table[b, 0], h, t] == 0x7F).all()
        assert (got["v"][table[b, 0], h, t // 16, :, t % 16] == 0).all()
    # the queries that see such a token give NaN, the values of the others are finite
    o = host(foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                                 ints(rs), 12))
    want = np.zeros((rs[-1], H), dtype=bool)
    want[2:12, 0] = want[4:12, 1] = True
    assert np.array_equal(np.isnan(o).all((2, 3)), want)
    assert np.isfinite(o[~want]).all()
