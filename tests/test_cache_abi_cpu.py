"""Argument checks of the cache's C entry points (host only: no call here reaches a
launch, the addresses are never dereferenced)."""

import ctypes

import pytest

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


APPEND = [BF16, 8, 4, 6, 2, 128, 100, 16, 5e5, 16.0, P, P, P, None, P, P2, P, P, P, None]


@pytest.mark.parametrize("at,value,rc,msg", [
    (0, 7, INV, "dt"), (0, F32, UNS, "bf16"), (1, 0, INV, "H must"), (1, 65, INV, "H must"),
    (2, -1, INV, "B must"), (2, 65536, INV, "B must"), (3, -1, INV, "N*nq"),
    (3, 1 << 26, INV, "N*nq"), (4, 0, INV, "nq must"), (4, 65, INV, "nq must"),
    (5, 64, UNS, "hd = 96"), (6, 0, INV, "n_pages"), (7, 0, INV, "max_blocks"),
    (7, (1 << 18) + 1, INV, "max_blocks"), (8, 0.0, INV, "theta"), (8, float("nan"), INV, "theta"),
    (9, -1.0, INV, "scale"), (10, None, INV, "qkv is NULL"), (10, P + 8, INV, "qkv is not"),
    (10, P2, INV, "q_out must not"), (11, None, INV, "row_start"), (12, P + 2, INV, "ctx_len"),
    (13, P + 1, INV, "pos"), (14, None, INV, "block_table"), (15, None, INV, "q_out"),
    (16, P + 4, INV, "k_cache"), (17, None, INV, "v_cache"), (18, None, INV, "kv_scale"),
])
def test_append_rejects(L, at, value, rc, msg):
    assert L.foe_cache_append(*changed(APPEND, at, value)) == rc
    assert msg in foe.last_error()


ATTEND = [BF16, 8, 4, 6, 2, 128, 100, 16, 3, P, P, P, P, P, P, P, P, P, P, P2, 1 << 40, None]


@pytest.mark.parametrize("at,value,rc,msg", [
    (0, 9, INV, "dt"), (0, F32, UNS, "bf16"), (1, 65, INV, "H must"), (5, 100, UNS, "hd = 96"),
    (8, 0, INV, "max_rows"), (8, -3, INV, "max_rows"), (9, None, INV, "q is NULL"),
    (10, None, INV, "row_start"), (11, None, INV, "ctx_len"), (12, None, INV, "block_table"),
    (13, None, INV, "k_cache"), (14, P + 8, INV, "v_cache"), (15, None, INV, "kv_scale"),
    (16, None, INV, "go together"), (17, None, INV, "go together"), (16, P + 4, INV, "mass_in"),
    (18, None, INV, "out is NULL"), (19, None, INV, "ws is NULL"), (19, P + 8, INV, "ws is"),
    (20, 0, WS, "workspace needs"),
])
def test_attention_rejects(L, at, value, rc, msg):
    assert L.foe_cache_attention(*changed(ATTEND, at, value)) == rc
    assert msg in foe.last_error()


EVICT = [8, 4, 128, 100, 16, 128, 16, P, P, P, 2, P, P, P, P, P, P, None, 0, None]


LONG = 513  # pages: more tokens than a workgroup of the selection holds


def test_evict_workspace(L):
    assert L.foe_cache_evict_workspace_bytes(8, 4, 512) == 0
    need = L.foe_cache_evict_workspace_bytes(8, 4, LONG)
    assert 0 < need < SIZE_MAX
    assert L.foe_cache_evict_workspace_bytes(8, -1, LONG) == SIZE_MAX
    long = changed(EVICT, 4, LONG)
    assert L.foe_cache_evict(*long) == INV and "ws is NULL" in foe.last_error()
    long[17:19] = P2, need - 1
    assert L.foe_cache_evict(*long) == WS and "workspace needs" in foe.last_error()


@pytest.mark.parametrize("at,value,rc,msg", [
    (0, 0, INV, "H must"), (1, -1, INV, "B must"), (2, 64, UNS, "hd = 96"), (3, 0, INV, "n_pages"),
    (4, 0, INV, "max_blocks"), (5, 0, INV, "keep"), (5, 129, INV, "dst_blocks"),
    (6, -1, INV, "recent"), (6, 129, INV, "recent"), (7, None, INV, "length"),
    (8, None, INV, "block_table"), (9, None, INV, "dst_table"), (10, 1, INV, "dst_blocks"),
    (11, None, INV, "k_cache"), (12, None, INV, "v_cache"), (13, None, INV, "kv_scale"),
    (14, None, INV, "mass is NULL"), (15, P + 2, INV, "kept"), (16, None, INV, "new_len"),
])
def test_evict_rejects(L, at, value, rc, msg):
    assert L.foe_cache_evict(*changed(EVICT, at, value)) == rc
    assert msg in foe.last_error()


def test_tables_past_the_limit(L):
    for call, ok, at_b, at_blocks in ((L.foe_cache_append, APPEND, 2, 7),
                                      (L.foe_cache_attention, ATTEND, 2, 7),
                                      (L.foe_cache_evict, EVICT, 1, 4)):
        args = changed(changed(ok, at_b, (1 << 13) + 1), at_blocks, 1 << 18)
        assert call(*args) == INV and "B*max_blocks" in foe.last_error()
    assert L.foe_cache_attention_workspace_bytes(8, (1 << 13) + 1, 4, 2, 128, 1 << 18, 1,
                                                 0) == SIZE_MAX


def test_empty_calls_are_noops(L):
    empty = [None] * 20
    assert L.foe_cache_append(BF16, 8, 4, 0, 2, 128, 1, 1, 5e5, 1.0, *empty[:10]) == foe.FOE_OK
    assert L.foe_cache_attention(BF16, 8, 4, 0, 2, 128, 1, 1, 1, *empty[:11], 0,
                                 None) == foe.FOE_OK
    assert L.foe_cache_evict(8, 0, 128, 1, 1, 1, 0, None, None, None, 1,
                             *empty[:7], 0, None) == foe.FOE_OK


def test_workspace_bytes(L):
    f = L.foe_cache_attention_workspace_bytes
    assert f(8, 4, 0, 2, 128, 16, 1, 0) == 0
    plain, mass = f(8, 64, 64, 2, 128, 128, 1, 0), f(8, 64, 64, 2, 128, 128, 1, 1)
    assert plain <= mass < SIZE_MAX
    assert f(8, 4, 6, 2, 128, 16, 6, 1) == f(8, 4, 6, 2, 128, 16, 100, 1)
    for bad in ((0, 4, 6, 2, 128, 16, 1, 0), (8, 4, 6, 2, 64, 16, 1, 0), (8, 4, 6, 2, 128, 0, 1, 0),
                (8, 4, 6, 2, 128, 16, 0, 0)):
        assert f(*bad) == SIZE_MAX
        assert foe.last_error()
