"""Trees over the cache without a GPU: argument checks of the C entry points (no call here
reaches a launch, the addresses are never dereferenced) and pins of the oracle."""

import ctypes
import os
import re

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2605_06206_amd import build as build_mod
from paper_2605_06206_amd import foe

P, P2 = 0x10000, 0x20000
SIZE_MAX = ctypes.c_size_t(-1).value
BF16, F32, INV, UNS, WS = (foe.BF16, foe.F32, foe.FOE_ERR_INVALID, foe.FOE_ERR_UNSUPPORTED,
                           foe.FOE_ERR_WORKSPACE)


@pytest.fixture(scope="module")
def L():
    return foe.lib()


def changed(ok, at, value):
    return [value if i == at else a for i, a in enumerate(ok)]


APPEND = [BF16, 8, 4, 6, 2, 128, 100, 16, 5e5, 16.0, P, P, P, None, P, P, P2, P, P, P, None]


@pytest.mark.parametrize("at,value,rc,msg", [
    (0, 7, INV, "dt"), (0, F32, UNS, "bf16"), (1, 0, INV, "H must"), (2, 65536, INV, "B must"),
    (3, 1 << 26, INV, "N*nq"), (4, 65, INV, "nq must"), (5, 64, UNS, "hd = 96"),
    (6, 0, INV, "n_pages"), (7, 0, INV, "max_blocks"), (8, 0.0, INV, "theta"),
    (10, None, INV, "qkv is NULL"), (10, P2, INV, "q_out must not"), (11, None, INV, "row_start"),
    (12, P + 2, INV, "ctx_len"), (13, P + 1, INV, "pos"), (14, None, INV, "depth is NULL"),
    (14, P + 1, INV, "depth"), (15, None, INV, "block_table"), (16, None, INV, "q_out"),
    (17, P + 4, INV, "k_cache"), (18, None, INV, "v_cache"), (19, None, INV, "kv_scale"),
])
def test_append_tree_rejects(L, at, value, rc, msg):
    assert L.foe_cache_append_tree(*changed(APPEND, at, value)) == rc
    assert "foe_cache_append_tree" in foe.last_error() and msg in foe.last_error()


#         0     1  2  3   4  5    6    7   8   9    10 11 12 13 14 15 16 17 18 19 20 21 22 23 24 25 26
ATTEND = [BF16, 8, 4, 60, 2, 128, 100, 16, 33, 0.0, P, P, P, 2, P, P, P, P, P, P, P, P, P, P, P, P2,
          1 << 40, None]


@pytest.mark.parametrize("at,value,rc,msg", [
    (0, 9, INV, "dt"), (0, F32, UNS, "bf16"), (1, 65, INV, "H must"), (5, 100, UNS, "hd = 96"),
    (8, 0, INV, "max_rows"), (9, -1.0, INV, "cap must"), (9, float("nan"), INV, "cap must"),
    (9, float("inf"), INV, "cap must"), (9, 1e-30, INV, "cap must"), (9, 1e30, INV, "cap must"),
    (10, P + 2, INV, "slope"), (11, P + 1, INV, "prefix"), (12, P + 1, INV, "tree"),
    (13, 1, INV, "tree_words"), (13, 0, INV, "tree_words"), (13, -5, INV, "tree_words"),
    (14, P + 3, INV, "depth"), (15, None, INV, "q is NULL"), (16, None, INV, "row_start"),
    (17, None, INV, "ctx_len"), (18, None, INV, "block_table"), (19, None, INV, "k_cache"),
    (20, P + 8, INV, "v_cache"), (21, None, INV, "kv_scale"), (22, None, INV, "go together"),
    (23, None, INV, "go together"), (22, P + 4, INV, "mass_in"), (24, None, INV, "out is NULL"),
    (25, None, INV, "ws is NULL"), (25, P + 8, INV, "ws is"), (26, 0, WS, "workspace needs"),
])
def test_attention_ex_rejects(L, at, value, rc, msg):
    assert L.foe_cache_attention_ex(*changed(ATTEND, at, value)) == rc
    assert "foe_cache_attention_ex" in foe.last_error() and msg in foe.last_error()


def test_attention_ex_workspace(L):
    f = L.foe_cache_attention_ex_workspace_bytes
    assert f(8, 4, 0, 2, 128, 16, 3, 0) == 0 and f(8, 0, 4, 2, 128, 16, 3, 1) == 0
    assert f(8, 4, 60, 2, 64, 16, 3, 0) == SIZE_MAX and f(8, 4, 60, 2, 128, 16, 0, 0) == SIZE_MAX
    for rows in (1, 8, 16, 17, 32, 33, 60, 1000):
        need = f(8, 4, 60, 2, 128, 16, rows, 1)
        assert 0 < f(8, 4, 60, 2, 128, 16, rows, 0) < need < SIZE_MAX
        call = changed(changed(ATTEND, 8, rows), 26, need - 1)
        assert L.foe_cache_attention_ex(*call) == WS


@pytest.mark.parametrize("name", ["", "_ex"])
@pytest.mark.parametrize("hd", [96, 128])
def test_workspace_of_the_largest_call_serves_smaller_ones(L, name, hd):
    """A server's one workspace, sized for its largest batch: no smaller number of rows, of
    sequences, of pages, of heads or of groups takes more, with and without the mass, whatever
    form and width it takes."""
    f = getattr(L, f"foe_cache_attention{name}_workspace_bytes")
    rng = np.random.default_rng([11, hd])
    assert f(8, 64, 64 * 64, 2, hd, 128, 8, 1) <= f(8, 64, 64 * 64, 2, hd, 128, 64, 1)
    assert f(8, 64, 64 * 64, 1, hd, 128, 32, 0) <= f(8, 64, 64 * 64, 1, hd, 128, 33, 0)
    assert f(1, 1, 2, 2, hd, 1 << 17, 1, 1) <= f(1, 1, 2, 2, hd, 1 << 18, 1, 1)
    for _ in range(300):
        H, nq, B = int(rng.integers(1, 9)), int(rng.integers(1, 9)), int(rng.integers(1, 100))
        blocks = int(2 ** rng.uniform(0, 12))
        N = B * int(2 ** rng.uniform(0, 8))
        top = int(2 ** rng.uniform(0, 8))
        mass = int(rng.integers(2))
        most = f(H, B, N, nq, hd, blocks, top, mass)
        assert 0 < most < SIZE_MAX
        for rows in {1, 2, 3, 16 // nq, 17 // nq, 32 // nq, 64 // nq, 128 // nq, top - 1}:
            if 0 < rows <= top:
                less = [H, B, N, nq, hd, blocks, rows, mass]
                assert f(*less) <= most, (less, top)
                for at, value in ((0, 1), (1, max(1, B // 2)), (2, max(1, N // 3)), (3, 1),
                                  (5, max(1, blocks // 2)), (7, 0)):
                    assert f(*changed(less, at, value)) <= most, (less, at, top)


ACCEPT = [8, 4, 128, 100, 16, 6, P, P, P, P, P, P, P, P, P2, None]


@pytest.mark.parametrize("at,value,rc,msg", [
    (0, 0, INV, "H must"), (1, 65536, INV, "B must"), (2, 64, UNS, "hd = 96"),
    (3, 0, INV, "n_pages"), (4, 0, INV, "max_blocks"), (5, 0, INV, "max_path"),
    (5, (1 << 22) + 1, INV, "max_path"), (6, None, INV, "row_start"), (7, None, INV, "ctx_len"),
    (8, None, INV, "path"), (8, P + 2, INV, "path"), (9, None, INV, "block_table"),
    (10, None, INV, "k_cache"), (11, P + 4, INV, "v_cache"), (12, None, INV, "kv_scale"),
    (13, P + 4, INV, "mass"), (14, None, INV, "new_len"), (14, P, INV, "new_len must not"),
    (8, P2, INV, "path or row_start"), (6, P2, INV, "path or row_start"),
])
def test_accept_rejects(L, at, value, rc, msg):
    assert L.foe_cache_accept(*changed(ACCEPT, at, value)) == rc
    assert "foe_cache_accept" in foe.last_error() and msg in foe.last_error()


# ---- the oracle -------------------------------------------------------------------

def pool_of(rng, pages, H, hd):
    return {"k": np.zeros((pages, H, 64, hd), dtype=np.uint8),
            "v": np.zeros((pages, H, 4, hd, 16), dtype=np.uint8),
            "kv_scale": np.full((pages, H, 2), 2.0 ** -100),
            "mass": rng.random((pages, H, 64)).astype(np.float32)}


def test_oracle_tree_is_each_path_alone():
    """A row of a tree gives what it gives as the last of its own path, appended alone."""
    rng = np.random.default_rng(1)
    H, nq, hd, ctx, n = 1, 2, 16, 70, 12
    parent = [-1, 0, 0, 1, 1, 2, 3, 3, 5, 6, 8, 8]
    depth, sees = np.zeros(n, dtype=int), np.eye(n, dtype=bool)
    for i in range(1, n):
        depth[i] = depth[parent[i]] + 1
        sees[i] |= sees[parent[i]]
    table = np.array([[2, 0]])
    old, qkv = rng.normal(size=(H, ctx, nq + 2, hd)), rng.normal(size=(H, n, nq + 2, hd))
    qkv[:, 0] = 3.0 * np.sign(qkv[:, 0])  # (every path has the largest values: the same scales)
    base = pool_of(rng, 3, H, hd)
    co.append(base, old, table, [0], [0, ctx], 1e4, 1.0)
    pool = {k: v.copy() for k, v in base.items()}
    q, _ = co.append(pool, qkv, table, [ctx], [0, n], 1e4, 1.0, depth=depth)
    for a in ({}, dict(cap=2.0), dict(slope=np.array([[0.3, 0.01]]))):
        o = co.attend(pool, q, table, [ctx], [0, n], tree=sees, depth=depth, **a)[0]
        for r in range(n):
            path = np.nonzero(sees[r])[0]
            alone = {k: v.copy() for k, v in base.items()}
            q1, _ = co.append(alone, qkv[:, path], table, [ctx], [0, len(path)], 1e4, 1.0)
            o1 = co.attend(alone, q1, table, [ctx], [0, len(path)], **a)[0]
            np.testing.assert_allclose(o[r], o1[-1], rtol=1e-12, atol=1e-12)
            # and keeping the path leaves that cache
            kept = {k: v.copy() for k, v in pool.items()}
            ln = co.accept(kept, table, [ctx], [0, n], np.array([list(path) + [-1]]))
            assert ln[0] == ctx + len(path)
            np.testing.assert_array_equal(kept["kv_scale"], alone["kv_scale"])
            for name, rows in (("k", lambda x: x), ("v", co._v_rows)):
                np.testing.assert_array_equal(rows(kept[name][0, 0])[:ln[0] - 64],
                                              rows(alone[name][0, 0])[:ln[0] - 64])


def test_oracle_scores_by_hand():
    """Two keys of known scores: the cap, the bias and the masks are the formulas'."""
    hd = 16
    pool = pool_of(np.random.default_rng(0), 1, 1, hd)
    pool["kv_scale"][:] = 1.0
    pool["k"][0, 0, :3] = co.encode(np.array([[4.0], [8.0], [2.0]]) * np.eye(hd)[0])
    for t, x in enumerate((1.0, 2.0, 4.0)):
        pool["v"][0, 0, 0, :, t] = co.encode(np.full(hd, x))
    q = np.zeros((1, 1, 1, hd))
    q[..., 0] = 1.0                    # scores 1, 2 and 0.5
    table, v = np.array([[0]]), np.array([1.0, 2.0, 4.0])

    def want(s):
        p = np.exp(s)
        return (p / p.sum()) @ v[:len(s)]

    def got(**a):
        return co.attend(pool, q, table, [2], [0, 1], **a)[0][0, 0, 0, 0]

    s = np.array([1.0, 2.0, 0.5])
    assert np.isclose(got(), want(s))
    assert np.isclose(got(cap=1.5), want(1.5 * np.tanh(s / 1.5)))
    assert np.isclose(got(slope=np.array([[0.25]])), want(s - 0.25 * np.array([2, 1, 0])))
    assert np.isclose(got(slope=np.array([[0.25]]), depth=[3]), want(s - 0.25 * np.array([5, 4, 0])))
    assert np.isclose(got(tree=[[False]]), want(s[:2]))
    assert np.isclose(got(tree=[[True]]), want(s))
    assert np.isclose(got(tree=[[False]], prefix=[3]), want(s))
    q2 = np.concatenate([q, q], 1)
    o = co.attend(pool, q2, table, [1], [0, 2], prefix=[3])[0][:, 0, 0, 0]
    assert np.allclose(o, want(s))     # the prefix reaches the later row
    o = co.attend(pool, q2, table, [1], [0, 2], prefix=[2])[0][:, 0, 0, 0]
    assert np.allclose(o, [want(s[:2]), want(s)])


def test_oracle_accept_by_hand():
    """Tokens 2, 3, 4, 5 behind a context of 2; rows 1 and 3 stay, as tokens 2 and 3."""
    rng = np.random.default_rng(2)
    pool = pool_of(rng, 1, 1, 16)
    pool["kv_scale"][:] = 4.0
    x = np.array([1.0, 2.0, 256.0, 8.0, 448.0, 32.0])
    pool["k"][0, 0, :6] = co.encode(x[:, None] * np.ones(16))
    for t in range(6):
        pool["v"][0, 0, 0, :, t] = co.encode(np.full(16, -x[t]))
    mass = pool["mass"].copy()
    ln = co.accept(pool, np.array([[0]]), [2], [0, 4], np.array([[1, 3, 3]]))
    assert ln[0] == 4
    want = 4.0 * np.array([1.0, 2.0, 8.0, 32.0])
    assert (pool["kv_scale"] == 2.0 ** -1).all()   # 128 / 448 < 1/2 <= 256 / 448
    np.testing.assert_array_equal(co.decode(pool["k"][0, 0, :4, 0]) * 0.5, want)
    np.testing.assert_array_equal(co.decode(pool["v"][0, 0, 0, 0, :4]) * -0.5, want)
    np.testing.assert_array_equal(pool["mass"][0, 0, :4], mass[0, 0, [0, 1, 3, 5]])
    np.testing.assert_array_equal(pool["k"][0, 0, 4:6], co.encode(x[4:, None] * np.ones(16)))


def test_tanh_polynomials_are_as_exact_as_they_say():
    """The cap's polynomials (csrc/kv_attention.hip): the relative errors that stand at their
    coefficients, as written and in fp32, up to the last digit that is given."""
    with open(os.path.join(build_mod.CSRC, "kv_attention.hip")) as f:
        src = f.read()
    for poly, bound, exact, single in (("kTanhPoly", "kTanhBound", 8.2e-8, 8.9e-8),
                                       ("kTanhLow", "kTanhNear", 7.4e-8, 8.4e-8)):
        end = float(re.search(rf"float {bound} = ([0-9.]+)f;", src)[1])
        said = src[:src.index(f"double {poly}[")].rsplit(f"|x| <= {bound}", 1)[1]
        assert all(f"{e:.1e}".replace("e-0", "e-") in said for e in (exact, single))
        c = np.array([float(x) for x in
                      re.search(rf"double {poly}\[\d\] = {{([^}}]+)}}", src)[1].split(",")])
        x = np.linspace(1e-4, end, 400001)
        for k, want in ((c, exact), (c.astype(np.float32).astype(float), single)):
            y = np.polynomial.polynomial.polyval(x * x, k)
            worst = np.abs(y * x / np.tanh(x) - 1).max()
            assert want - 1e-9 < worst < want + 1e-9, (poly, worst)
