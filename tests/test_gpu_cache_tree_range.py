"""Trees and other scores over the 8-bit cache at the borders of their forms: one workspace for
batches of all widths."""

import numpy as np
import pytest
import torch

from paper_2605_06206_amd import foe
from test_gpu_cache import DEV, batch, bf16, ints, random_pool, say, to_dev
from test_gpu_cache_tree import check_shaped, pack, trees

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
