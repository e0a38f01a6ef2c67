"""The prompt's attention with scores far from zero, against the fp64 oracle."""

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from paper_2605_06206_amd import foe
from test_gpu_attention import attn_part_err, rel_err, say, to_dev

pytestmark = pytest.mark.gpu
TOL = 2e-2  # as test_gpu_attention: bf16 storage of v, p, o and the output


@pytest.mark.parametrize("S,nq,hd", [(1, 2, 128), (65, 1, 96), (200, 2, 128), (330, 3, 96),
                                     (129, 1, 128), (700, 2, 96)])
@pytest.mark.parametrize("sign,level", [(1, 2), (-1, 2), (1, 20), (-1, 20), (1, 24), (-1, 24)])
def test_scores_far_from_zero(S, nq, hd, sign, level):
    """Scores up to the documented 2^29 (2^28.1 at most here).
    Queries and keys of equal elements in every dim, in units of 2^(level / 2), a third of
    them 1.25 times the others: the tokens whose score is the largest share the weight
    alike (their scores are equal and exact).  Positions are scaled down until nothing turns."""
    rng = np.random.default_rng([71, S, nq, hd])
    H, d = 2, 64
    x = rng.normal(size=(H, S, d)).astype(np.float32)
    x = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    x[:, :, 0] = np.where(rng.random((H, S)) < 0.3, 1.25, 1.0)
    groups = []
    for _ in range(H):
        w = np.zeros(((nq + 2) * hd, d))
        w[:nq * hd, 0] = sign * 2.0 ** (level // 2)   # queries and keys: of the first element
        w[nq * hd:(nq + 1) * hd, 0] = 2.0 ** (level // 2)
        w[(nq + 1) * hd:, 1:] = 0.2 * rng.normal(size=(hd, d - 1))
        wo = 0.2 * rng.normal(size=(d, nq * hd))
        groups.append({n: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16).double()
                       .numpy() for n, a in (("w_qkv", w), ("w_o", wo))})
    say("far scores", S, nq, hd, sign, level)
    got = foe.group_attention(to_dev(x), to_dev(np.stack([g["w_qkv"] for g in groups])),
                              to_dev(np.concatenate([g["w_o"] for g in groups], axis=1)), nq,
                              500000.0, 1e30)
    torch.cuda.synchronize()
    got = got.float().cpu().numpy()
    ref, _ = ao.attention_block(x, groups, nq, hd, 500000.0, 1e30)
    e_full, e_attn = rel_err(got, ref), attn_part_err(got, ref, x.mean(axis=0))
    say(f"rel err r_full {e_full:.2e}, attention part {e_attn:.2e}")
    assert np.isfinite(got).all()
    assert e_full <= TOL and e_attn <= TOL
