"""Trees and other scores over the 8-bit cache at the borders of their forms: one workspace for
batches of all widths, tables too wide for the scores to be kept for the mass, one wide tree beside
single rows, biases over long contexts by bounds that weigh each token, and the masses of accepted
paths alone."""

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2605_06206_amd import foe
from test_gpu_cache import DEV, SCALE, THETA, batch, bf16, host, ints, random_pool, say, to_dev
from test_gpu_cache_tree import check_shaped, pack, run_shaped, slopes, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    foe.lib()


@pytest.mark.parametrize("shaped", [False, True])
@pytest.mark.parametrize("nq,hd", [(2, 128), (1, 96)])
def test_one_workspace_serves_batches_of_all_widths(nq, hd, shaped):
    """A workspace sized for the largest call serves the smaller ones, whichever form they take,
    and none writes past its own size."""
    rng = np.random.default_rng([51, nq, hd])
    H, B, blocks, top = 2, 4, 20, 300
    pool = random_pool(rng, B * blocks, H, hd)
    dev = to_dev(pool)
    table = rng.permutation(B * blocks).astype(np.int32).reshape(B, blocks)

    def size(b, n, rows, mass):
        q = torch.empty((H, n, nq, hd), dtype=torch.bfloat16, device="meta")
        return foe.cache_attention_workspace_bytes(q, ints(table[:b]), rows, mass, shaped=shaped)

    ws = torch.empty(size(B, B * top, top, True), dtype=torch.uint8, device=DEV)
    for rows in (1, 16 // nq, 16 // nq + 1, 32 // nq, 33 // nq, 64, 65, 128, 129, top):
        for b, mass in ((B, True), (2, False), (1, True)):
            seqs = [(int(rng.integers(0, 800)), int(rng.integers(0, rows + 1))) for _ in range(b)]
            seqs[0] = (700, rows)
            say("one workspace", nq, hd, shaped, rows, b, mass)
            ctx, rs = [c for c, _ in seqs], np.concatenate([[0], np.cumsum([n for _, n in seqs])])
            q = bf16(rng.normal(size=(H, rs[-1], nq, hd)))
            depth, sees = trees(rng, seqs)
            a = dict(sees=sees, depth=depth) if shaped else {}
            kw = dict(tree=pack(sees, -(-rows // 32)), depth=ints(depth)) if shaped else {}
            ws.fill_(0xA5)
            m = torch.full_like(dev["mass"], -7.0) if mass else None
            out = foe.cache_attention(
                q, dev["k"], dev["v"], dev["kv_scale"], ints(table[:b]), ints(ctx), ints(rs), rows,
                mass_in=dev["mass"] if mass else None, mass_out=m, ws=ws, **kw)
            torch.cuda.synchronize()
            assert (ws[size(b, int(rs[-1]), rows, mass):] == 0xA5).all()
            check_shaped(pool, table[:b], ctx, rs, q, out, m, **a)


def wide(table):
    """The same pages in a table of the most entries: the scores of 16 columns of two groups, or of
    one of 64 sequences' groups, pass 1 GiB."""
    out = np.full((len(table), 1 << 18), -1, dtype=np.int32)
    out[:, :table.shape[1]] = table
    return out


@pytest.mark.parametrize("H,nq,hd,seqs,what", [
    (2, 2, 128, [(700, 8), (64, 5), (0, 8), (63, 1)], "tree"),
    (2, 1, 96, [(300, 16)], "tree"),
    (3, 4, 96, [(1000, 4), (127, 3), (0, 0), (5, 1)], "tree cap bias"),
    (2, 2, 128, [(90, 8), (1500, 3)], "cap"),
    (2, 16, 96, [(130, 1), (64, 1), (0, 1)], "cap bias"),
    (2, 1, 128, [(200, 16), (10, 9)], "bias prefix"),
    (8, 1, 128, [(40 * b, 1) for b in range(16)], "cap"),
    (4, 1, 96, [(50 * b, 1 + b % 2) for b in range(16)], "tree"),
    # sequences of few columns beside those of more than any few-column form holds
    (2, 2, 128, [(100, 150), (300, 2), (64, 8), (0, 1), (500, 1)], "tree"),
    (2, 1, 96, [(0, 200), (700, 16), (63, 3), (1, 1), (90, 2), (400, 1)], "tree cap bias"),
    (2, 2, 96, [(65, 140), (128, 1), (30, 2), (250, 5)], "cap prefix"),
])
def test_mass_where_scores_are_formed_again(H, nq, hd, seqs, what):
    say("formed again", H, nq, hd, seqs, what)
    rng = np.random.default_rng([52, H, nq, hd, len(seqs), len(what)])
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    depth, sees = trees(rng, seqs)
    a = {}
    if "cap" in what:
        a["cap"] = 8.0
    if "bias" in what:
        a["slope"] = slopes(rng, H, nq)
    if "prefix" in what:
        a["prefix"] = [int(rng.integers(0, c + n + 30)) for c, n in seqs]
    if "tree" in what:
        a.update(sees=sees, depth=depth)
    q = bf16(2.0 * rng.normal(size=(H, rs[-1], nq, hd)))
    top = max(n for _, n in seqs)
    # (what the call takes without the mass, the statistics, and all that scores may take: they
    # are past it, and not kept)
    assert len(seqs) * H * (1 << 18) * min(16, top * nq) * 64 * 4 > 1 << 30
    out, m = run_shaped(pool, wide(table), ctx, rs, q, top, True, **a)
    check_shaped(pool, table, ctx, rs, q, out, m, **a)


@pytest.mark.parametrize("rows,more", [(16, 0), (10, 0), (3, 150)])
def test_nan_rows_where_scores_are_formed_again(rows, more):
    """A row of a NaN key counts, as NaN, for the tokens that it sees alone."""
    rng = np.random.default_rng([53, rows, more])
    H, nq, hd, seqs = 2, 1, 128, [(100, rows), (130, 2)] + ([(20, more)] if more else [])
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    _, sees = trees(rng, seqs)
    bad = rows // 2  # a row that no other sees
    for r in range(rows):
        if r != bad:
            sees[r][bad] = False
    t = 100 + bad
    p = table[0, t // 64]
    pool["k"][p, :, t % 64] = 0x7F
    pool["v"][p, :, (t % 64) // 16, :, t % 16] = 0
    q = bf16(rng.normal(size=(H, rs[-1], nq, hd)))
    say("NaN rows, formed again", rows, more)
    out, m = run_shaped(pool, wide(table), ctx, rs, q, max(rows, more), True, sees=sees, cap=9.0)
    g, m = host(out), host(m)
    good = [r for r in range(rs[-1]) if r != bad]
    assert np.isfinite(g[good]).all() and np.isnan(g[bad]).all()
    for t in range(100 + rows):
        seen = t < 100 or sees[bad][t - 100]
        assert np.isnan(m[table[0, t // 64], :, t % 64]).all() == seen, t
    for t in range(132):
        assert np.isfinite(m[table[1, t // 64], :, t % 64]).all(), t
    sees[bad][:] = False
    pool["k"][p, :, (100 + bad) % 64] = 0
    check_shaped(pool, table, ctx, rs, q, out, None, rows=good, sees=sees, cap=9.0)


@pytest.mark.parametrize("blocks", [1 << 13, 1 << 18])
@pytest.mark.parametrize("H,nq,hd,seqs,what", [
    (2, 2, 128, [(300, 1), (100, 64), (64, 1), (0, 8), (500, 1)], "tree"),
    (2, 1, 96, [(0, 100), (700, 16), (63, 17), (1, 1), (90, 2), (400, 1)], "tree cap bias"),
    (2, 2, 96, [(65, 33), (128, 1), (30, 2), (250, 5)], "cap prefix"),
    (1, 9, 128, [(10, 1), (0, 0), (200, 14), (1500, 2)], "bias"),
    (1, 64, 128, [(10, 2), (200, 0), (99, 0), (1500, 0), (3, 0)], "tree"),
])
def test_a_wide_tree_beside_few_columns(H, nq, hd, seqs, what, blocks):
    """Calls of 65 to 128 columns whose other sequences have few, in tables that hold the pages
    from which both forms are taken."""
    say("wide beside few", H, nq, hd, seqs, what, blocks)
    rng = np.random.default_rng([56, H, nq, hd, len(seqs), len(what)])
    ctx, rs, table, pages = batch(rng, seqs)
    pool = random_pool(rng, pages, H, hd)
    depth, sees = trees(rng, seqs)
    a = {}
    if "cap" in what:
        a["cap"] = 8.0
    if "bias" in what:
        a["slope"] = slopes(rng, H, nq)
    if "prefix" in what:
        a["prefix"] = [int(rng.integers(0, c + n + 30)) for c, n in seqs]
    if "tree" in what:
        a.update(sees=sees, depth=depth)
    q = bf16(1.5 * rng.normal(size=(H, rs[-1], nq, hd)))
    top = max(n for _, n in seqs)
    assert 64 < top * nq <= 128 and (rs[-1] - top) * nq <= 16 * (len(seqs) - 1)
    assert len(seqs) * H * blocks >= 16384
    for mass in (False, True):
        out, m = run_shaped(pool, wide(table)[:, :blocks].copy(), ctx, rs, q, top, mass, **a)
        check_shaped(pool, table, ctx, rs, q, out, m, **a)


def weighed(pool, table, ctx, q, slope, cap=0.0, depth=None, sees=None):
    """One sequence's outputs and masses in fp64, and bounds of their errors that weigh each token
    by its probability.  A score may be off by e_t: its sum of hd products of magnitude a_t in all,
    scaling and cap (hd + 24 roundings of a_t), and the bias: the slope in units of log2 e (two),
    its product with the distance from the page's first token, up to 63 more than the token's own,
    that with the rest, the sum with the score and what is left of the maximum (6 roundings).  A
    probability is then off by e_t and, through the sum, by the mean of all e_t, relatively; by
    2^-16 for the exponential and the sum's additions (a lane's chain has at most 16 for each of
    15 pages).  One below 2^-126 may be lost."""
    H, n, nq, hd = q.shape
    L = ctx + n
    q = host(q)
    slope = np.asarray(slope, dtype=np.float32).astype(np.float64)
    step = np.arange(n) if depth is None else np.clip(depth, 0, co.MAX_DEPTH)
    place, spot = ctx + step, np.concatenate([np.arange(ctx), ctx + step])
    seen = np.arange(L) <= ctx + np.arange(n)[:, None]
    if sees is not None:
        seen = np.ones((n, L), dtype=bool)
        seen[:, ctx:] = np.array([r[:n] for r in sees])
    o, o_lim = np.zeros((n, H, nq, hd)), np.zeros((n, H, nq, hd))
    mass, m_lim = np.zeros((H, L)), np.zeros((H, L))
    far = np.abs(place[:, None] - spot).astype(np.float64)
    for h in range(H):
        k, v, _ = co.tokens(pool, table, 0, h, L)
        for j in range(nq):
            s = q[h, :, j] @ k.T / np.sqrt(hd)
            if cap:
                s = cap * np.tanh(s / cap)
            s = np.where(seen, s - slope[h, j] * far, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            e = np.abs(q[h, :, j]) @ np.abs(k).T / np.sqrt(hd) * (hd + 24)
            e = 1.45 * 2.0 ** -24 * (e + 6 * abs(slope[h, j]) * (far + 63))
            pe = p * (e + (p * e).sum(1, keepdims=True) + 2.0 ** -16)
            o[:, h, j] = p @ v
            # (bf16 for the product with the values and for the output, 2^-12 for its fp32 sums)
            o_lim[:, h, j] = (pe + (2.0 ** -8 + 2.0 ** -12) * p) @ np.abs(v) + \
                2.0 ** -8 * np.abs(o[:, h, j]) + 2.0 ** -124 * L
            mass[h] += p.sum(0)
            m_lim[h] += (pe + n * nq * 2.0 ** -24 * p + 2.0 ** -126).sum(0)
    return o, o_lim, mass, m_lim


@pytest.mark.parametrize("H,nq,hd,ctx,rows,what", [
    (1, 2, 128, 131071, 1, "cap"),
    (1, 4, 96, 130990, 1, ""),
    (1, 2, 128, 131071, 16, "tree"),
    (1, 1, 96, 65000, 64, "tree cap"),
    (2, 2, 128, 20000, 30, "tree"),
    (1, 3, 128, 9001, 90, "cap"),
    (1, 2, 128, 3000, 40, "tree far"),
    (2, 1, 96, 777, 12, "far"),
    (1, 2, 96, 500, 200, "tree far"),
])
def test_bias_by_the_weight_of_each_token(H, nq, hd, ctx, rows, what):
    """Biases over contexts up to the longest, from those that reach a few tokens to those that
    reach all of them, outputs and masses (`far`: some rows stand 2^18 to 2^20 places behind)."""
    rng = np.random.default_rng([54, H, nq, hd, ctx, rows])
    _, rs, table, pages = batch(rng, [(ctx, rows)])
    pool = random_pool(rng, pages, H, hd)
    pool["mass"][:] = 0.0  # (the sum with what was there would hide more)
    depth, sees = trees(rng, [(ctx, rows)])
    q = bf16(1.5 * rng.normal(size=(H, rows, nq, hd)))
    a = {"cap": 20.0 if "cap" in what else 0.0}
    if "tree" in what:
        a.update(sees=sees, depth=depth)
    if "far" in what:
        depth[rows // 2:] += rng.integers(1 << 18, 1 << 20, rows - rows // 2)
        a["depth"] = depth
    for near, end in ((0.9, 0.1), (2.0 ** -5, 2.0 ** -9), (2.0 ** -14, 2.0 ** -18)):
        slope = np.exp(rng.uniform(np.log(end), np.log(near), (H, nq)))
        say("weighed bias", H, nq, hd, ctx, rows, what, near)
        out, m = run_shaped(pool, table, [ctx], rs, q, rows, True, slope=slope, **a)
        o, o_lim, mass, m_lim = weighed(pool, table, ctx, q, slope, **a)
        err = np.abs(host(out) - o)
        say(f"outputs {float((err / o_lim).max()):.3f} of the bound")
        got = host(m).transpose(1, 0, 2)[:, table[0]].reshape(H, -1)[:, :ctx + rows]
        off = np.abs(got - mass)
        say(f"masses {float((off / m_lim).max()):.3f} of the bound")
        assert (err <= o_lim).all() and (off <= m_lim).all()


@pytest.mark.parametrize("nq,hd,back", [(2, 128, 4), (1, 96, 2)])
def test_masses_of_accepted_paths_alone(nq, hd, back):
    """Trees verified without the mass, and the weights of the kept rows added once a path is
    accepted, by a causal call of those rows: bit for bit the masses, and what is then evicted, of a
    cache that never held a rejected draft.  (Every token's largest key and value are the same, so
    that neither cache's pages ever have another scale, and no tree crosses a page, so that both
    form the same sines.)"""
    rng = np.random.default_rng([55, nq, hd])
    H, B, blocks = 2, 3, 6
    perm = rng.permutation(3 * B * blocks).astype(np.int32)
    t1, t2, fresh = (perm[i * B * blocks:(i + 1) * B * blocks].reshape(B, blocks) for i in range(3))
    dev = foe.cache_empty(3 * B * blocks, H, hd, DEV)
    kv, mass = (dev["k"], dev["v"], dev["kv_scale"]), dev["mass"]

    def rows_of(n):
        x = np.clip(rng.normal(size=(H, n, nq + 2, hd)), -4, 4)
        x[..., hd // 2 - 1] = 6.0   # (of the pair that hardly turns)
        return bf16(x)

    ln = np.array([3, 65, 130])
    rs = np.concatenate([[0], np.cumsum(ln)])
    qkv = rows_of(rs[-1])
    for t in (t1, t2):
        q = foe.cache_append(qkv, *kv, ints(t), ints(np.zeros(B)), ints(rs), THETA, SCALE)
        foe.cache_attention(q, *kv, ints(t), ints(np.zeros(B)), ints(rs), 130, mass_in=mass,
                            mass_out=mass)
    for step in range(5):
        n = rng.integers(2, 13, B)
        rs = np.concatenate([[0], np.cumsum(n)])
        depth, sees = trees(rng, list(zip(ln, n)), back=back)
        qkv, top = rows_of(rs[-1]), int(n.max())
        say("masses of paths", step, ln, n)
        q = foe.cache_append(qkv, *kv, ints(t1), ints(ln), ints(rs), THETA, SCALE,
                             depth=ints(depth))
        foe.cache_attention(q, *kv, ints(t1), ints(ln), ints(rs), top, depth=ints(depth),
                            tree=pack(sees, 1))
        path, keep = np.full((B, 25), -1), []
        for b in range(B):
            keep.append(np.nonzero(sees[rs[b] + int(rng.integers(n[b]))][:n[b]])[0])
            if b == step % 4:       # (nothing is accepted)
                keep[b] = keep[b][:0]
            path[b, :len(keep[b])] = keep[b]
        new = foe.cache_accept(*kv, ints(t1), ints(ln), ints(rs), ints(path))
        m = [len(x) for x in keep]
        rs2 = np.concatenate([[0], np.cumsum(m)])
        rows = torch.from_numpy(np.concatenate([rs[b] + keep[b] for b in range(B)])).to(DEV)
        foe.cache_attention(q[:, rows].contiguous(), *kv, ints(t1), ints(ln), ints(rs2), max(m),
                            mass_in=mass, mass_out=mass)
        q2 = foe.cache_append(qkv[:, rows].contiguous(), *kv, ints(t2), ints(ln), ints(rs2), THETA,
                              SCALE)
        foe.cache_attention(q2, *kv, ints(t2), ints(ln), ints(rs2), max(m), mass_in=mass,
                            mass_out=mass)
        torch.cuda.synchronize()
        ln = host(new).astype(int)
        both = [mass.cpu().numpy()[t].transpose(0, 2, 1, 3).reshape(B, H, -1) for t in (t1, t2)]
        for b in range(B):
            assert np.array_equal(both[0][b, :, :ln[b]], both[1][b, :, :ln[b]]), (step, b)
            assert (both[0][b, :, :ln[b]] > 0).all()
    kept = []
    for t in (t1, t2):
        got, _ = foe.cache_evict(*kv, mass.clone(), ints(t), ints(ln), 40, 8, dst_table=ints(fresh))
        kept.append(got)
    torch.cuda.synchronize()
    assert torch.equal(kept[0], kept[1])
