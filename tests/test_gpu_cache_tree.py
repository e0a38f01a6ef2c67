"""Trees of drafted tokens over the 8-bit cache (foe_cache_append_tree, foe_cache_attention_ex,
foe_cache_accept) and attention scores of other shapes, against the fp64 oracle."""

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2605_06206_amd import foe
from test_gpu_cache import (DEV, SCALE, THETA, batch, bf16, check_append, check_attention, host,
                            ints, random_pool, same, say, to_dev, to_host)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    foe.lib()


def random_tree(rng, n, back=6):
    """Depths [n] and the rows that each row sees [n, n] (its ancestors and itself)."""
    depth, sees = np.zeros(n, dtype=int), np.eye(n, dtype=bool)
    for i in range(1, n):
        p = max(0, i - int(rng.integers(1, back)))
        depth[i] = depth[p] + 1
        sees[i] |= sees[p]
    return depth, sees


def trees(rng, seqs, **kw):
    """(depth [N], what each of the N rows sees) of a batch."""
    made = [random_tree(rng, n, **kw) for _, n in seqs]
    return (np.concatenate([d for d, _ in made] + [np.zeros(0, dtype=int)]),
            [row for _, s in made for row in s])


def pack(rows, words):
    """int32 [N, words] of the rows' bits."""
    out = np.zeros((len(rows), words * 32), dtype=np.uint8)
    for i, r in enumerate(rows):
        out[i, :len(r)] = r
    bits = np.packbits(out, axis=1, bitorder="little").view(np.int32)
    return torch.from_numpy(bits.copy()).to(DEV)


# ---- append -----------------------------------------------------------------------

class _Depth:
    """The oracle's append with the rows' depths, as check_append calls it."""

    def __init__(self, depth):
        self.depth = depth

    def __enter__(self):
        self.was = co.append
        depth, was = self.depth, co.append
        co.append = lambda *a, **k: was(*a, **k, depth=depth)

    def __exit__(self, *a):
        co.append = self.was


@pytest.mark.parametrize("H,nq,hd,seqs", [
    (1, 1, 96, [(0, 1)]),
    (2, 2, 128, [(0, 5), (63, 1), (64, 2), (60, 9), (127, 1)]),
    (3, 2, 96, [(10, 130), (0, 0), (5, 3), (60, 8)]),
    (1, 4, 128, [(1000, 64), (17, 33)]),
    (1, 64, 128, [(3, 2)]),
])
def test_append_tree_parity(H, nq, hd, seqs):
    say("append tree", H, nq, hd, seqs)
    rng = np.random.default_rng([3, H, nq, hd, len(seqs)])
    ctx, rs, table, pages = batch(rng, seqs)
    depth, _ = trees(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    dev = to_dev(pool)
    qkv = bf16(rng.normal(size=(H, rs[-1], nq + 2, hd)))
    q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                         ints(rs), THETA, SCALE, depth=ints(depth))
    torch.cuda.synchronize()
    with _Depth(depth):
        check_append(pool, dev, host(qkv), table, ctx, rs, q)


def test_append_tree_far_apart_and_cut_depths():
    """Depths in any order, further apart than a page's two sets of sines reach, negative
    and past the largest; positions of the caller's own."""
    rng = np.random.default_rng(4)
    seqs = [(10, 70), (0, 3), (100, 4)]
    depth = np.concatenate([rng.permutation(70) * 3, [-5, 1 << 25, 7], [63, 0, 64, 31]])
    ctx, rs, table, pages = batch(rng, seqs)
    for pos in (None, [130000, 0, 1 << 20]):
        pool = random_pool(rng, pages, 2, 128)
        dev = to_dev(pool)
        qkv = bf16(rng.normal(size=(2, rs[-1], 3, 128)))
        say("append tree, far depths", pos)
        q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                             ints(rs), THETA, SCALE, pos=None if pos is None else ints(pos),
                             depth=ints(depth))
        torch.cuda.synchronize()
        with _Depth(depth):
            check_append(pool, dev, host(qkv), table, ctx, rs, q, pos)


def test_append_tree_of_a_chain_is_append():
    """Depths that count up are the rows' own order, bit for bit."""
    rng = np.random.default_rng(5)
    seqs = [(70, 90), (3, 1), (64, 20)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, 2, 96)
    qkv = bf16(rng.normal(size=(2, rs[-1], 4, 96)))
    depth = np.concatenate([np.arange(n) for _, n in seqs])
    got = []
    say("append chain")
    for d in (None, ints(depth)):
        dev = to_dev(pool)
        q = foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx),
                             ints(rs), THETA, SCALE, depth=d)
        got.append((q, dev))
    assert torch.equal(got[0][0], got[1][0])
    same(to_host(got[1][1]), to_host(got[0][1]))


# ---- attention --------------------------------------------------------------------

def score_error(big, bias, hd):
    """Relative error of a probability.  A score: a sum of hd products (2^-24 each, of `big`),
    its scaling, the cap (a polynomial of relative error 2^-23 with 6 roundings, or an
    exponential and a reciprocal: 16 * 2^-24 of at most `big` cover either), and the bias (its
    slope's rounding, the sum's, and theirs in units of log2 e: 4 * 2^-24); once for the
    probability and once for the maximum and the sum; 1.45 = log2 e, 2^-20 the exponentials."""
    return 2 * 1.45 * 2.0 ** -24 * ((hd + 24) * big + 4 * bias) + 2.0 ** -20


def run_shaped(pool, table, ctx, rs, q, max_rows, mass=False, cap=0.0, slope=None, prefix=None,
               sees=None, depth=None, words=None):
    dev = to_dev(pool)
    mass_out = torch.full_like(dev["mass"], -7.0) if mass else None
    out = torch.full((q.shape[1], q.shape[0], *q.shape[2:]), -3.0, dtype=torch.bfloat16, device=DEV)
    words = words or -(-max_rows // 32)
    foe.cache_attention(
        q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx), ints(rs), max_rows,
        out=out, mass_in=dev["mass"] if mass else None, mass_out=mass_out, cap=cap,
        slope=None if slope is None else torch.tensor(slope, dtype=torch.float32, device=DEV),
        prefix=None if prefix is None else ints(prefix),
        tree=None if sees is None else pack(sees, words),
        depth=None if depth is None else ints(depth))
    torch.cuda.synchronize()
    return out, mass_out


def check_shaped(pool, table, ctx, rs, q, out, mass_out, rows=None, cap=0.0, slope=None,
                 prefix=None, sees=None, depth=None):
    hd = q.shape[3]
    slope32 = None if slope is None else np.asarray(slope, dtype=np.float32)
    o, spread, big, got = co.attend(pool, host(q), table, ctx, rs, rows=rows, mass=True, cap=cap,
                                    slope=slope32, prefix=prefix, tree=sees, depth=depth)
    far = max(c + int(rs[b + 1] - rs[b]) for b, c in enumerate(ctx))
    if depth is not None:
        far += int(np.clip(depth, 0, co.MAX_DEPTH).max())
    rel = score_error(big, 0.0 if slope is None else float(np.abs(slope32).max()) * far, hd)
    g = host(out)
    mine = ~np.isnan(spread)
    err = np.abs(g - o)[mine]
    # a probability and the output are rounded to bf16 once each; a probability below fp32's
    # normal numbers, 2^-126, may be lost, and values are up to 2 (random_pool): 2^-125 a token,
    # twice that for outputs that are not normal themselves
    lim = ((2.0 ** -8 + 2.0 ** -12 + rel) * spread + 2.0 ** -8 * np.abs(o))[mine]
    lim += 2.0 ** -124 * max(c + int(rs[b + 1] - rs[b]) for b, c in enumerate(ctx))
    say(f"error {float((err / np.maximum(lim, 1e-30)).max(initial=0)):.3f} of the bound")
    assert (err <= lim).all()
    if mass_out is None:
        return
    m, touched = host(mass_out), np.zeros(mass_out.shape, dtype=bool)
    for (b, h), w in got.items():
        cols = int(rs[b + 1] - rs[b]) * q.shape[2]
        for t, x in enumerate(w):
            p = table[b, t // 64]
            if not 0 <= p < len(m):
                continue
            touched[p, h, t % 64] = True
            before = float(pool["mass"][p, h, t % 64]) if t < ctx[b] else 0.0
            lim = (rel + cols * 2.0 ** -24) * x + 2.0 ** -23 * abs(before + x) + 1e-37
            assert abs(m[p, h, t % 64] - before - x) <= lim, (b, h, t)
    assert (m[~touched] == -7.0).all()


def slopes(rng, H, nq):
    return 2.0 ** -rng.uniform(0.5, 8, (H, nq))


# columns of the longest: up to 16, 32, 64, 128 and beyond, not all of them full
TREES = [
    # H, nq, hd, [(ctx, rows)]
    (1, 1, 96, [(0, 1)]),
    (2, 2, 128, [(0, 1), (62, 3), (63, 8), (64, 1), (65, 2)]),
    (1, 1, 128, [(1500, 16), (0, 0), (3, 5)]),
    (2, 3, 96, [(50, 10), (0, 7), (255, 1), (256, 9)]),
    (1, 2, 128, [(700, 16), (60, 15), (0, 9)]),
    (1, 1, 96, [(100, 33), (31, 64), (0, 40)]),
    (2, 2, 128, [(130, 32), (64, 17), (1, 1)]),
    (1, 2, 96, [(200, 64), (0, 50), (63, 33)]),
    (1, 4, 128, [(1000, 32), (90, 31)]),
    (1, 17, 128, [(100, 3), (77, 1)]),
    (1, 64, 96, [(130, 2)]),
    (1, 2, 128, [(300, 100), (5, 66), (64, 1)]),
    (1, 3, 96, [(61, 200), (0, 130), (10, 3)]),
    (1, 1, 128, [(100, 300)]),
]


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("H,nq,hd,seqs", TREES)
def test_tree_attention_parity(H, nq, hd, seqs, mass):
    say("tree", H, nq, hd, seqs, mass)
    rng = np.random.default_rng([21, H, nq, hd, len(seqs), seqs[0][0]])
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    depth, sees = trees(rng, seqs)
    q = bf16(1.5 * rng.normal(size=(H, rs[-1], nq, hd)))
    top = max(n for _, n in seqs)
    a = dict(sees=sees, depth=depth)
    out, m = run_shaped(pool, table, ctx, rs, q, top, mass, **a)
    check_shaped(pool, table, ctx, rs, q, out, m, **a)


SHAPES = [
    # H, nq, hd, [(ctx, rows)], what
    (2, 2, 128, [(0, 1), (62, 1), (63, 1), (64, 1), (700, 1)], "cap bias"),
    (1, 2, 128, [(1500, 1)], "cap"),
    (2, 8, 128, [(300, 1), (10, 2)], "bias"),
    (1, 1, 96, [(90, 16), (0, 6), (1000, 2)], "cap bias prefix"),
    (1, 2, 96, [(300, 10), (64, 16), (0, 3)], "cap bias tree"),
    (1, 2, 128, [(300, 32), (100, 20)], "bias tree"),
    (1, 2, 128, [(100, 64), (63, 40), (0, 64)], "cap bias tree prefix"),
    (1, 2, 128, [(100, 40)], "prefix"),
    (1, 2, 96, [(100, 128), (40, 1), (0, 129), (333, 7)], "cap"),
    (1, 3, 128, [(61, 200), (500, 3)], "bias"),
    (2, 1, 128, [(0, 300), (70, 180), (200, 10)], "prefix"),
    (1, 2, 128, [(1000, 257)], "cap bias prefix"),
    (1, 2, 96, [(120, 150), (0, 100)], "cap bias tree"),
    (1, 2, 128, [(120, 150), (0, 100)], "bias depth"),
    (1, 5, 96, [(64, 100), (0, 64), (63, 65)], "cap bias prefix tree"),
    (1, 1, 128, [(30, 9), (130, 12)], "bias depth"),
]


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("H,nq,hd,seqs,what", SHAPES)
def test_shaped_attention_parity(H, nq, hd, seqs, what, mass):
    say("shaped", H, nq, hd, seqs, what, mass)
    rng = np.random.default_rng([22, H, nq, hd, len(seqs), seqs[0][0], len(what)])
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    depth, sees = trees(rng, seqs)
    a = {}
    if "cap" in what:
        a["cap"] = float(rng.choice([2.0, 7.5, 30.0]))
    if "bias" in what:
        a["slope"] = slopes(rng, H, nq)
    if "prefix" in what:
        a["prefix"] = [int(rng.integers(0, c + n + 30)) for c, n in seqs]
        a["prefix"][-1] = int(rng.choice([-4, 0, 1 << 30]))
    if "tree" in what:
        a.update(sees=sees, depth=depth)
    if "depth" in what:
        a["depth"] = depth
    q = bf16(4.0 * rng.normal(size=(H, rs[-1], nq, hd)))
    top = max(n for _, n in seqs)
    out, m = run_shaped(pool, table, ctx, rs, q, top, mass, **a)
    check_shaped(pool, table, ctx, rs, q, out, m, **a)


@pytest.mark.parametrize("i", range(12))
def test_shaped_random_batches(i):
    rng = np.random.default_rng([23, i])
    H, nq = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 4, 7]))
    hd, top = int(rng.choice([96, 128])), int(rng.choice([1, 4, 20, 40, 150]))
    B = int(rng.integers(1, 6 if top > 4 else 20))
    seqs = [(int(2 ** rng.uniform(0, 10)) - 1, int(rng.integers(0, top + 1))) for _ in range(B)]
    seqs[int(rng.integers(B))] = (int(rng.integers(0, 300)), top)
    say("random shaped batch", i, H, nq, hd, seqs)
    ctx, rs, table, pages = batch(rng, seqs, extra=int(rng.integers(0, 3)))
    pool = random_pool(rng, pages, H, hd)
    table[rng.random(table.shape) < 0.05] = -1
    depth, sees = trees(rng, seqs)
    a = {"cap": float(rng.choice([0.0, 3.0, 50.0]))}
    if rng.random() < 0.5:
        a["slope"] = slopes(rng, H, nq)
    if rng.random() < 0.4:
        a["prefix"] = rng.integers(0, 400, B)
    if rng.random() < 0.6:
        a["sees"] = sees
    if rng.random() < 0.6:
        a["depth"] = depth
    if len(a) == 1 and not a["cap"]:
        a["cap"] = 10.0
    q = bf16(2.0 * rng.normal(size=(H, rs[-1], nq, hd)))
    mass = bool(i % 2)
    out, m = run_shaped(pool, table, ctx, rs, q, top, mass, **a)
    check_shaped(pool, table, ctx, rs, q, out, m, **a)


@pytest.mark.parametrize("nq,rows", [(1, 9), (2, 16), (2, 30), (2, 60), (2, 100)])
def test_rows_that_see_nothing_and_masks_of_any_form(nq, rows):
    """Without a context a row may see no token (zeros, no mass), or only later ones; bits
    behind the sequence's rows say nothing; words that a row has too few of are zeros."""
    rng = np.random.default_rng([24, nq, rows])
    H, hd, seqs = 2, 128, [(0, rows), (0, 3), (70, rows - 2)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    sees = [rng.random(160) < 0.3 for _ in range(rs[-1])]
    sees[1][:] = False                # nothing
    sees[2][:] = False
    sees[2][rows:] = True             # bits of rows that are not there
    sees[4][:] = False
    sees[4][rows - 1] = True          # one later row
    q = bf16(1.5 * rng.normal(size=(H, rs[-1], nq, hd)))
    say("rows that see nothing", nq, rows)
    for words in (5, -(-rows // 32)):
        cut = [s[:32 * words] for s in sees]
        out, m = run_shaped(pool, table, ctx, rs, q, rows, True, sees=sees if words == 5 else cut,
                            words=words)
        check_shaped(pool, table, ctx, rs, q, out, m, sees=cut)
        assert (host(out)[1:3] == 0).all()


@pytest.mark.parametrize("nq,rows", [(1, 1), (2, 20), (2, 64), (2, 120)])
def test_capped_scores_of_any_magnitude(nq, rows):
    """Scores from the polynomial's range to past fp32 (capped like any other), caps from the
    smallest to the largest."""
    rng = np.random.default_rng([25, nq, rows])
    H, hd, ctx = 1, 128, 150
    ctx_l, rs, table, pages = batch(rng, [(ctx, rows)])
    pool = random_pool(rng, pages, H, hd)
    for sigma, cap, scale in ((1.0, 2.0 ** -64, 1.0), (1.0, 2.0 ** -9, 1.0), (4.0, 1.0, 1.0),
                              (30.0, 20.0, 1.0), (1.0, 2.0 ** 64, 1.0), (3.0, 2.0 ** 11, 1.0),
                              (1e30, 5.0, 2.0 ** 20), (3e37, 30.0, 2.0 ** 100)):
        p = dict(pool, kv_scale=pool["kv_scale"].copy())
        p["kv_scale"][..., 0] *= scale
        q = bf16(np.abs(sigma * rng.normal(size=(H, rs[-1], nq, hd))))
        if scale > 1:  # (all products of one sign: no sum of infinities of both)
            p["k"] = p["k"] & 0x7F
        say("capped", nq, rows, sigma, cap)
        out, m = run_shaped(p, table, [ctx], rs, q, rows, True, cap=cap)
        g = host(out)
        assert np.isfinite(g).all()
        if sigma <= 30:
            check_shaped(p, table, [ctx], rs, q, out, m, cap=cap)
        else:
            # every score is the cap: the mean of the values that a row sees
            for r in (0, rows - 1):
                k, v, _ = co.tokens(p, table, 0, 0, ctx + r + 1)
                zero = ~(k > 0).any(1)  # (a key of zero codes has a score of zero)
                want = v[~zero].mean(0)
                lim = (2.0 ** -8 + 2.0 ** -12) * np.abs(v).mean(0) + 2.0 ** -8 * np.abs(want)
                assert (np.abs(g[r, 0] - want) <= lim).all()


def test_bias_over_far_places():
    """A slope of zero, a steep one and a negative one; places behind the context that pass
    what the table holds."""
    rng = np.random.default_rng(26)
    H, nq, hd, seqs = 1, 3, 96, [(900, 5), (0, 30), (64, 64)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    depth = rng.integers(0, 3000, rs[-1])
    depth[7] = -9
    q = bf16(1.5 * rng.normal(size=(H, rs[-1], nq, hd)))
    say("bias over far places")
    for a in (dict(depth=depth), {}, dict(depth=depth, sees=trees(rng, seqs)[1])):
        a["slope"] = np.array([[0.0, 3.0, -2.0 ** -6]])
        out, m = run_shaped(pool, table, ctx, rs, q, 64, True, **a)
        check_shaped(pool, table, ctx, rs, q, out, m, **a)


@pytest.mark.parametrize("rows", [1, 12, 30, 60, 110])
def test_absent_pages_and_garbage(rows):
    """Pages that are not there are not seen; slots behind the end and rows that a row's bits
    leave out may hold NaN codes."""
    rng = np.random.default_rng([27, rows])
    H, nq, hd = 2, 2, 96
    seqs = [(200, rows), (0, 1), (130, 1)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    _, sees = trees(rng, seqs)
    bad = rows // 2  # a row that no other sees, with a NaN key
    for r in range(rows):
        if r != bad:
            sees[r][bad] = False
    for b, (c, n) in enumerate(seqs):
        for t in range(c + n, table.shape[1] * 64):
            p = table[b, t // 64]
            pool["k"][p, :, t % 64] = 0x7F
            pool["v"][p, :, (t % 64) // 16, :, t % 16] = 0xFF
    if rows > 1:
        t = 200 + bad
        p = table[0, t // 64]
        pool["k"][p, :, t % 64] = 0x7F
        pool["v"][p, :, (t % 64) // 16, :, t % 16] = 0
    table[0, 1] = pages + 5
    table[2, :] = -3
    q = bf16(rng.normal(size=(H, rs[-1], nq, hd)))
    say("absent pages", rows)
    out, m = run_shaped(pool, table, ctx, rs, q, rows, True, sees=sees, cap=9.0)
    g, m = host(out), host(m)
    assert (g[rs[2]:] == 0).all()
    good = [r for r in range(rs[2]) if rows == 1 or r != bad]
    assert np.isfinite(g[good]).all()
    if rows > 1:  # NaN for the row that sees it, and in the masses of what that row sees
        assert np.isnan(g[bad]).all()
        for t in range(200 + rows):
            p, seen = table[0, t // 64], t < 200 or sees[bad][t - 200]
            if 0 <= p < pages:
                assert np.isnan(m[p, :, t % 64]).all() == seen, t
        sees[bad][:] = False
        clean = dict(pool, k=pool["k"].copy())
        clean["k"][table[0, (200 + bad) // 64], :, (200 + bad) % 64] = 0
        check_shaped(clean, table, ctx, rs, q, out, None, rows=good, sees=sees, cap=9.0)


def test_rows_past_max_rows_and_the_tables_end():
    rng = np.random.default_rng(28)
    H, nq, hd = 1, 2, 128
    pool = random_pool(rng, 6, H, hd)
    table = np.array([[2, 0], [1, 5]], dtype=np.int32)
    ctx, rs = [120, 30], np.array([0, 20, 30])
    depth, sees = trees(rng, [(0, 20), (0, 10)])
    q = bf16(rng.normal(size=(H, 30, nq, hd)))
    say("past the table's end")
    out, m = run_shaped(pool, table, ctx, rs, q, 20, True, sees=sees, depth=depth)
    check_shaped(pool, table, ctx, rs, q, out, m, sees=sees, depth=depth)
    say("past max_rows")
    out, _ = run_shaped(pool, table, ctx, rs, q, 8, False, sees=sees, depth=depth)
    assert (host(out)[8:20] == -3.0).all() and (host(out)[28:] == -3.0).all()
    assert (host(out)[:8] != -3.0).any((1, 2, 3)).all()


@pytest.mark.parametrize("H,nq,hd,ctx,rows,picked", [
    (1, 2, 128, 131071, 1, [0]),
    (1, 2, 128, 131071, 16, [0, 7, 15]),
    (1, 2, 96, 131000, 64, [0, 31, 63]),
])
def test_long_contexts(H, nq, hd, ctx, rows, picked):
    rng = np.random.default_rng(29)
    say("long", ctx, rows)
    ctx_l, rs, table, pages = batch(rng, [(ctx, rows)])
    pool = random_pool(rng, pages, H, hd)
    depth, sees = trees(rng, [(ctx, rows)])
    q = bf16(1.5 * rng.normal(size=(H, rows, nq, hd)))
    for a in (dict(sees=sees, depth=depth), dict(cap=20.0, slope=slopes(rng, H, nq))):
        out, _ = run_shaped(pool, table, [ctx], rs, q, rows, False, **a)
        check_shaped(pool, table, [ctx], rs, q, out, None, rows=picked, **a)


# ---- keeping a path ---------------------------------------------------------------

def random_path(rng, n, m):
    return np.sort(rng.permutation(n)[:m])


def check_accept(pool, table, ctx, rs, path, mass=True):
    want = {n: a.copy() for n, a in pool.items()}
    if not mass:
        want["mass"] = None
    dev = to_dev(pool)
    ref = co.accept(want, table, ctx, rs, path)
    n = foe.cache_accept(dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx), ints(rs),
                         ints(path), mass=dev["mass"] if mass else None)
    torch.cuda.synchronize()
    if not mass:
        want["mass"] = pool["mass"]
    assert np.array_equal(host(n), ref)
    same(to_host(dev), want)
    return ref


@pytest.mark.parametrize("mass", [False, True])
@pytest.mark.parametrize("H,hd,seqs,kept", [
    (1, 96, [(0, 1)], [1]),
    (2, 128, [(0, 8), (60, 9), (63, 2), (64, 5), (127, 1)], [3, 6, 1, 5, 0]),
    (3, 96, [(10, 130), (0, 0), (5, 64), (61, 80)], [100, 0, 64, 70]),
    (1, 128, [(1000, 64), (17, 33)], [12, 33]),
    (8, 96, [(15, 20), (16, 20), (17, 20), (47, 33)], [4, 5, 6, 33]),
])
def test_accept_parity(H, hd, seqs, kept, mass):
    say("accept", H, hd, seqs, kept)
    rng = np.random.default_rng([31, H, hd, len(seqs)])
    ctx, rs, table, pages = batch(rng, seqs)
    path = np.full((len(seqs), max(1, max(kept))), -1)
    for b, m in enumerate(kept):
        path[b, :m] = random_path(rng, seqs[b][1], m)
    check_accept(random_pool(rng, pages, H, hd), table, ctx, rs, path, mass)


def test_accept_paths_that_end_early():
    """Entries that do not ascend, are no rows of the sequence or lie past the table's end
    end the path, whatever follows; contexts and rows are cut to what there is."""
    rng = np.random.default_rng(32)
    seqs = [(10, 12)] * 6
    ctx, rs, table, pages = batch(rng, seqs)
    path = np.array([[0, 3, 3, 5], [0, 5, 2, 7], [-1, 0, 1, 2], [2, 11, 12, 13], [12, 0, 1, 2],
                     [0, 2, 1 << 30, 5]])
    say("accept, paths that end")
    assert list(check_accept(random_pool(rng, pages, 2, 96), table, ctx, rs, path)) == [
        12, 12, 10, 12, 10, 12]
    pool = random_pool(rng, 3, 1, 128)
    assert list(check_accept(pool, np.array([[1, 2]], dtype=np.int32), [120], np.array([0, 20]),
                             np.array([[1, 7, 8, 9]]))) == [122]
    dev = to_dev(pool)
    n = foe.cache_accept(dev["k"], dev["v"], dev["kv_scale"], ints([[1, 2]]), ints([-5]),
                         ints([0, 1 << 30]), ints([[0, 1]]))
    assert int(n) == 2
    n = foe.cache_accept(dev["k"], dev["v"], dev["kv_scale"], ints([[1, 2]]), ints([1 << 30]),
                         ints([0, 4]), ints([[0, 1]]))
    assert int(n) == 128


def test_accept_long_paths():
    """More entries than a workgroup has threads, over many pages."""
    rng = np.random.default_rng(33)
    seqs = [(100, 1500), (0, 700)]
    ctx, rs, table, pages = batch(rng, seqs)
    path = np.full((2, 900), -1)
    path[0, :900] = random_path(rng, 1500, 900)
    path[1, :650] = random_path(rng, 700, 650)
    say("accept, long paths")
    check_accept(random_pool(rng, pages, 1, 96), table, ctx, rs, path)


@pytest.mark.parametrize("hd", [96, 128])
def test_accept_scales_and_special_tokens(hd):
    """Pages whose scales differ by all that fp32 holds, zero tokens, tokens of NaN keys (either
    sign), absent source and destination pages."""
    rng = np.random.default_rng([34, hd])
    H, seqs = 2, [(60, 150), (130, 90), (20, 100), (0, 70)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    pool["kv_scale"] = 2.0 ** rng.choice([-100, -60, 0, 1, 50, 118], pool["kv_scale"].shape)
    for t in (61, 100, 170):   # NaN keys with zero values
        p = table[0, t // 64]
        pool["k"][p, :, t % 64] = 0x7F if t != 100 else 0xFF
        pool["v"][p, :, (t % 64) // 16, :, t % 16] = 0
    for t in range(64):        # zero tokens
        p = table[3, t // 64]
        pool["k"][p, :, t % 64] &= 0x80
        pool["v"][p, :, (t % 64) // 16, :, t % 16] &= 0x80
    table[1, 3] = -1           # a source page
    table[2, 0] = pages + 1    # a destination page
    path = np.full((4, 80), -1)
    path[0, :4] = [1, 40, 110, 149]
    path[1, :80] = random_path(rng, 90, 80)
    path[2, :60] = random_path(rng, 100, 60)
    path[3, :20] = random_path(rng, 60, 20)
    say("accept, scales", hd)
    check_accept(pool, table, ctx, rs, path)


# ---- a run of them together -------------------------------------------------------

@pytest.mark.parametrize("H,nq,hd,stream", [(2, 2, 128, False), (2, 1, 96, True)])
def test_speculative_steps(H, nq, hd, stream):
    """Trees are appended, verified and cut to a path, step after step, and the cache that
    remains holds what the kept tokens alone leave.  A value is rounded to e4m3 once, to the
    same one in units of any scale, but among a scale's subnormals, whose step is 2^-9 of it: there
    two caches may differ by half a step for each of their roundings (one as stored and one as
    rescaled, of either cache), in units of the largest scale that the page had."""
    rng = np.random.default_rng([41, hd])
    B, blocks, steps = 3, 5, 6
    perm = rng.permutation(2 * B * blocks).astype(np.int32)
    t1, t2 = perm[:B * blocks].reshape(B, blocks), perm[B * blocks:].reshape(B, blocks)
    dev = foe.cache_empty(2 * B * blocks, H, hd, DEV)
    kv = (dev["k"], dev["v"], dev["kv_scale"])
    ln = np.array([40, 3, 61])
    st = torch.cuda.Stream() if stream else None
    kw = {"stream": st} if stream else {}
    if stream:
        st.wait_stream(torch.cuda.current_stream())
    qkv = bf16(rng.normal(size=(H, ln.sum(), nq + 2, hd)))
    rs = np.concatenate([[0], np.cumsum(ln)])
    torch.cuda.synchronize()
    for t in (t1, t2):
        foe.cache_append(qkv, *kv, ints(t), ints(np.zeros(B)), ints(rs), THETA, SCALE, **kw)
    largest = np.zeros((2 * B * blocks, H, 2))  # scale that a page had
    for step in range(steps):
        say("speculative step", step, ln)
        n = rng.integers(3, 30, B)
        seqs = list(zip(ln, n))
        rs = np.concatenate([[0], np.cumsum(n)])
        depth, sees = trees(rng, seqs, back=4)
        qkv = bf16(rng.normal(size=(H, rs[-1], nq + 2, hd)))
        top = int(n.max())
        bits = pack(sees, -(-top // 32))
        torch.cuda.synchronize()
        q = foe.cache_append(qkv, *kv, ints(t1), ints(ln), ints(rs), THETA, SCALE,
                             depth=ints(depth), **kw)
        mass = dev["mass"].clone()
        torch.cuda.synchronize()
        out = foe.cache_attention(q, *kv, ints(t1), ints(ln), ints(rs), top, mass_in=mass,
                                  mass_out=dev["mass"], tree=bits, depth=ints(depth), **kw)
        torch.cuda.synchronize()
        pool = to_host(dict(dev, mass=mass))
        largest = np.maximum(largest, pool["kv_scale"])
        check_shaped(pool, t1, ln, rs, q, out, None, sees=sees, depth=depth)
        # a path from the root to some row, and its tokens appended alone
        path = np.full((B, 32), -1)
        keep = []
        for b in range(B):
            leaf = int(rng.integers(n[b]))
            row = np.nonzero(sees[rs[b] + leaf][:n[b]])[0]
            path[b, :len(row)] = row
            keep.append(row)
        new = foe.cache_accept(*kv, ints(t1), ints(ln), ints(rs), ints(path), mass=dev["mass"],
                               **kw)
        torch.cuda.synchronize()
        rows = torch.from_numpy(np.concatenate([rs[b] + keep[b] for b in range(B)])).to(DEV)
        rs2 = np.concatenate([[0], np.cumsum([len(r) for r in keep])])
        q2 = foe.cache_append(qkv[:, rows].contiguous(), *kv, ints(t2), ints(ln), ints(rs2),
                              THETA, SCALE, **kw)
        torch.cuda.synchronize()
        # a path's depths count up: the same positions, and queries
        assert torch.equal(q[:, rows], q2)
        ln = host(new).astype(int)
        assert (ln == [c + len(r) for c, r in zip([s[0] for s in seqs], keep)]).all()
        pool = to_host(dev)
        for b in range(B):
            for h in range(H):
                a, z = (co.tokens(pool, t, b, h, ln[b])[:2] for t in (t1, t2))
                page = np.arange(ln[b]) // 64
                for x in range(2):
                    s = np.maximum(largest[t1[b]], pool["kv_scale"][t2[b]])[page, h, x]
                    off = np.abs(a[x] - z[x])
                    assert (off <= 2 * 2.0 ** -9 * s[:, None]).all(), (b, h, x)
                    # (normal in either cache: the same)
                    assert (off[np.abs(a[x]) >= 2.0 ** -5 * s[:, None]] == 0).all(), (b, h, x)
    # a decode step over both
    qkv = bf16(rng.normal(size=(H, B, nq + 2, hd)))
    torch.cuda.synchronize()
    rs = np.arange(B + 1)
    for t in (t1, t2):
        q = foe.cache_append(qkv, *kv, ints(t), ints(ln), ints(rs), THETA, SCALE, **kw)
        out = foe.cache_attention(q, *kv, ints(t), ints(ln), ints(rs), 1, **kw)
        torch.cuda.synchronize()
        check_attention(to_host(dev), t, ln, rs, q, out, None)


@pytest.mark.parametrize("nq,rows", [(2, 8), (1, 25), (2, 25), (2, 60), (2, 120)])
def test_chain_of_drafts_is_causal(nq, rows):
    """A tree that is a chain: the causal attention's results, within the bounds of both."""
    rng = np.random.default_rng([42, nq, rows])
    H, hd, seqs = 2, 128, [(100, rows), (0, rows), (63, 2)]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    q = bf16(1.5 * rng.normal(size=(H, rs[-1], nq, hd)))
    depth = np.concatenate([np.arange(n) for _, n in seqs])
    sees = [r for _, n in seqs for r in np.tril(np.ones((n, n), dtype=bool))]
    say("chain", nq, rows)
    out, m = run_shaped(pool, table, ctx, rs, q, rows, True, sees=sees, depth=depth)
    check_shaped(pool, table, ctx, rs, q, out, m)


@pytest.mark.parametrize("rows", [1, 14, 30, 60, 150])
def test_graph_replay(rows):
    """A step captured with its append, attention with mass and accept, and replayed with the
    caller's own work between: the eager calls' results each time.  Two graphs share one
    workspace, and replays are ordered on one stream."""
    rng = np.random.default_rng([43, rows])
    H, nq, hd, seqs = 2, 2, 128, [(90, rows), (3, 1), (64, max(1, rows // 2))]
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    depth, sees = trees(rng, seqs)
    path = np.full((3, 8), -1)
    for b, (_, n) in enumerate(seqs):
        m = int(rng.integers(1, min(n, 8) + 1))
        path[b, :m] = random_path(rng, n, m)
    fixed = dict(table=ints(table), ctx=ints(ctx), rs=ints(rs), depth=ints(depth), path=ints(path),
                 tree=pack(sees, -(-rows // 32)),
                 slope=torch.tensor(slopes(rng, H, nq), dtype=torch.float32, device=DEV))
    dev = to_dev(pool)
    start = {n: t.clone() for n, t in dev.items()}
    qkv = torch.zeros((H, int(rs[-1]), nq + 2, hd), dtype=torch.bfloat16, device=DEV)
    mass = torch.zeros_like(dev["mass"])
    q = torch.empty((H, int(rs[-1]), nq, hd), dtype=torch.bfloat16, device=DEV)
    out = torch.empty((int(rs[-1]), H, nq, hd), dtype=torch.bfloat16, device=DEV)
    new_len = torch.empty(3, dtype=torch.int32, device=DEV)
    ws = torch.empty(foe.cache_attention_workspace_bytes(q, fixed["table"], rows, True, shaped=True),
                     dtype=torch.uint8, device=DEV)

    def step(cap):
        f = fixed
        foe.cache_append(qkv, dev["k"], dev["v"], dev["kv_scale"], f["table"], f["ctx"], f["rs"],
                         THETA, SCALE, q=q, depth=f["depth"])
        foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], f["table"], f["ctx"], f["rs"],
                            rows, mass_in=dev["mass"], mass_out=mass, out=out, ws=ws, cap=cap,
                            slope=f["slope"], tree=f["tree"], depth=f["depth"])
        foe.cache_accept(dev["k"], dev["v"], dev["kv_scale"], f["table"], f["ctx"], f["rs"],
                         f["path"], mass=mass, new_len=new_len)

    def reset():
        for n, t in dev.items():
            t.view(torch.uint8).copy_(start[n].view(torch.uint8))
        mass.zero_()
        for t in (out, q):
            t.zero_()

    def result():
        return [t.view(torch.uint8).clone() for t in (out, q, mass, new_len, *dev.values())]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        reset()
        step(9.0)  # warm up
        side.synchronize()
        graphs = []
        say("graph", rows)
        for cap in (9.0, 0.0):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step(cap)
            graphs.append((g, cap))
        for rep in range(4):
            x = bf16(rng.normal(size=qkv.shape))
            qkv.copy_(x)
            g, cap = graphs[rep % 2]
            reset()
            step(cap)
            want = result()
            reset()
            g.replay()
            got = result()
            side.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b), rep


def test_calls_on_two_streams_at_once_repeat():
    """Two streams at a time, each with its own workspace, give the bits of calls one after
    another."""
    rng = np.random.default_rng(44)
    H, nq, hd = 4, 2, 128
    jobs = []
    for rows, a in ((30, dict(cap=5.0)), (1, {}), (64, {}), (200, dict(cap=5.0))):
        seqs = [(500, rows), (1000, rows), (77, 1)]
        ctx, rs, table, pages = batch(rng, seqs)
        dev = to_dev(random_pool(rng, pages, H, hd))
        depth, sees = trees(rng, seqs)
        q = bf16(rng.normal(size=(H, rs[-1], nq, hd)))
        args = (q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx), ints(rs), rows)
        jobs.append((args, dict(a, mass_in=dev["mass"], tree=pack(sees, -(-rows // 32)),
                                depth=ints(depth)), torch.zeros_like(dev["mass"])))
    say("two streams")
    want = []
    for args, a, m in jobs:
        want.append((foe.cache_attention(*args, mass_out=m, **a), m.clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(3):
        got = []
        for i, (args, a, m) in enumerate(jobs):
            m2 = torch.zeros_like(m)
            torch.cuda.synchronize() if i % 2 == 0 else None
            got.append((foe.cache_attention(*args, mass_out=m2, stream=streams[i % 2], **a), m2))
        torch.cuda.synchronize()
        for (o, m), (o2, m2) in zip(want, got):
            assert torch.equal(o, o2) and torch.equal(m, m2)


def test_pool_past_four_gib():
    """Pages whose offsets in the pool pass 32 bits: the same as in a small pool."""
    H, hd, nq, pages = 8, 128, 2, 70000
    rng = np.random.default_rng(45)
    table = np.array([[69999, 3], [66000, 68000]], dtype=np.int32)
    t2 = np.array([[0, 1], [2, 3]], dtype=np.int32)
    seqs = [(50, 40), (30, 64)]
    rs = np.array([0, 40, 104])
    depth, sees = trees(rng, seqs)
    path = np.full((2, 30), -1)
    path[0, :30] = random_path(rng, 40, 30)
    path[1, :20] = random_path(rng, 64, 20)
    old = bf16(rng.normal(size=(H, 80, nq + 2, hd)))
    qkv = bf16(rng.normal(size=(H, 104, nq + 2, hd)))
    got = []
    for t, n in ((table, pages), (t2, 4)):
        dev = foe.cache_empty(n, H, hd, DEV)
        kv = (dev["k"], dev["v"], dev["kv_scale"])
        say("large pool", n)
        foe.cache_append(old, *kv, ints(t), ints([0, 0]), ints([0, 50, 80]), THETA, SCALE)
        q = foe.cache_append(qkv, *kv, ints(t), ints([50, 30]), ints(rs), THETA, SCALE,
                             depth=ints(depth))
        out = foe.cache_attention(q, *kv, ints(t), ints([50, 30]), ints(rs), 64,
                                  mass_in=dev["mass"], mass_out=dev["mass"], tree=pack(sees, 2),
                                  cap=20.0)
        ln = foe.cache_accept(*kv, ints(t), ints([50, 30]), ints(rs), ints(path), mass=dev["mass"])
        torch.cuda.synchronize()
        p = torch.from_numpy(t.reshape(-1)).long().to(DEV)
        pool = to_host({x: y.view(torch.uint8)[p].view(y.dtype) if x in "kv" else y[p]
                        for x, y in dev.items()})
        held = [[x[i, :, :m] for i, m in ((0, 64), (1, 16), (2, 50))]
                for x in (pool["k"], pool["mass"])]
        got.append((q, out, ln, pool["kv_scale"][:3], held))
        del dev, kv
    assert all(torch.equal(a, b) for a, b in zip(got[0][:3], got[1][:3]))
    assert np.array_equal(got[0][3], got[1][3])
    for a, b in zip(got[0][4], got[1][4]):
        assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_empty_batches():
    dev = foe.cache_empty(2, 1, 96, DEV)
    kv = (dev["k"], dev["v"], dev["kv_scale"])
    e = torch.empty
    q = foe.cache_append(e((1, 0, 3, 96), dtype=torch.bfloat16, device=DEV), *kv, ints([[0]]),
                         ints([0]), ints([0, 0]), THETA, depth=ints([]))
    assert q.shape == (1, 0, 1, 96)
    out = foe.cache_attention(q, *kv, ints([[0]]), ints([0]), ints([0, 0]), 1, cap=1.0,
                              tree=torch.empty((0, 1), dtype=torch.int32, device=DEV))
    assert out.shape == (0, 1, 1, 96)
    n = foe.cache_accept(*kv, torch.empty((0, 1), dtype=torch.int32, device=DEV), ints([]),
                         ints([0]), torch.empty((0, 4), dtype=torch.int32, device=DEV))
    assert n.shape == (0,)
    n = foe.cache_accept(*kv, ints([[0]]), ints([3]), ints([0, 0]), ints([[0, 1]]))
    assert int(n) == 3


@pytest.mark.parametrize("nq,top", [(1, 2), (2, 12), (2, 40)])
def test_batches_of_more_sequences_than_threads(nq, top):
    """600 sequences, many without rows: more than any workgroup has threads to look them up."""
    rng = np.random.default_rng([41, nq, top])
    seqs = [(int(rng.integers(0, 70)), int(rng.integers(0, top + 1)) * int(rng.random() < 0.3))
            for _ in range(600)]
    seqs[577] = (65, top)
    say("many sequences", nq, top)
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, 1, 96)
    depth, sees = trees(rng, seqs)
    a = dict(cap=20.0, sees=sees, depth=depth)
    q = bf16(rng.normal(size=(1, rs[-1], nq, 96)))
    out, m = run_shaped(pool, table, ctx, rs, q, top, True, **a)
    check_shaped(pool, table, ctx, rs, q, out, m, **a)


@pytest.mark.parametrize("rows", [1, 9, 30, 120, 300])
def test_mass_in_place(rows):
    """A mass that is added to in place is the one that is written elsewhere."""
    rng = np.random.default_rng([42, rows])
    seqs = [(1900, rows), (333, max(rows // 2, 1)), (0, 0)]
    say("mass in place", rows)
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, 2, 128)
    depth, sees = trees(rng, seqs)
    q = bf16(rng.normal(size=(2, rs[-1], 2, 128)))
    dev = to_dev(pool)
    kw = dict(cap=15.0, tree=pack(sees, -(-rows // 32)), depth=ints(depth))
    args = (q, dev["k"], dev["v"], dev["kv_scale"], ints(table), ints(ctx), ints(rs), rows)
    apart, mine = dev["mass"].clone(), dev["mass"].clone()
    want = foe.cache_attention(*args, mass_in=dev["mass"], mass_out=apart, **kw)
    got = foe.cache_attention(*args, mass_in=mine, mass_out=mine, **kw)
    assert torch.equal(want, got) and torch.equal(apart, mine)


def test_binding_refuses():
    dev = foe.cache_empty(2, 1, 96, DEV)
    kv = (dev["k"], dev["v"], dev["kv_scale"])
    q = torch.zeros((1, 40, 1, 96), dtype=torch.bfloat16, device=DEV)
    args = (q, *kv, ints([[0, 1]]), ints([0]), ints([0, 40]), 40)
    for kw in (dict(slope=torch.zeros((1, 2), device=DEV)), dict(prefix=ints([0, 0])),
               dict(tree=torch.zeros((39, 2), dtype=torch.int32, device=DEV)),
               dict(tree=torch.zeros((40, 1), dtype=torch.int32, device=DEV)),
               dict(depth=ints([0])), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=1e30)):
        with pytest.raises(foe.FoeError):
            foe.cache_attention(*args, **kw)
    for kw in (dict(slope=torch.zeros((1, 1), dtype=torch.bfloat16, device=DEV)),
               dict(depth=torch.zeros(40, device=DEV))):
        with pytest.raises(TypeError):
            foe.cache_attention(*args, **kw)
    with pytest.raises(foe.FoeError):
        foe.cache_attention(*args, cap=1.0, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        foe.cache_attention(*args, depth=torch.zeros(40, dtype=torch.int32))
    with pytest.raises(ValueError):
        foe.cache_attention(*args, tree=torch.zeros((2, 40), dtype=torch.int32, device=DEV).t())
    with pytest.raises(foe.FoeError):
        foe.cache_accept(*kv, ints([[0, 1]]), ints([0]), ints([0, 40]), ints([[0], [1]]))
    with pytest.raises(foe.FoeError):
        foe.cache_accept(*kv, ints([[0, 1]]), ints([0]), ints([0, 40]), ints([[]]).reshape(1, 0))
    x = ints([3])
    with pytest.raises(foe.FoeError):
        foe.cache_accept(*kv, ints([[0, 1]]), x, ints([0, 40]), ints([[0]]), new_len=x)


@pytest.mark.parametrize("cap", [1e-50, -1e-50, 1e-20])
def test_binding_refuses_caps_below_range(cap):
    """A cap that fp32 would round to 0, no cap, is refused like the others below 2^-64."""
    dev = foe.cache_empty(1, 1, 96, DEV)
    q = torch.zeros((1, 1, 1, 96), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(foe.FoeError):
        foe.cache_attention(q, dev["k"], dev["v"], dev["kv_scale"], ints([[0]]), ints([0]),
                            ints([0, 1]), 1, cap=cap)
