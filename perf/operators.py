"""The operators of the 8-bit key/value cache, as cases that can be timed and checked.

A cache is a pool of pages of 64 tokens for H groups of one key/value head each:

- ``k``  [pages, H, 64, hd] e4m3 codes, one row per token;
- ``v``  [pages, H, 4, hd, 16] e4m3 codes, dims by tokens within 16 tokens;
- ``kv_scale`` [pages, H, 2] fp32, powers of two (keys, values): value = code * scale;
- ``mass`` [pages, H, 64] fp32, the attention weight that each token has received.

``block_table`` [B, blocks] names the pages of each sequence in order, ``ctx_len`` [B] the
tokens that it holds, ``row_start`` [B + 1] the new rows of each sequence in the packed batch.

Three kinds of case:

- ``append``: new rows [q | k | v] are rotated, q is returned, k and v go into the cache;
- ``attend``: the rows' queries over the cache (row i of a sequence sees its first ctx + i + 1
  tokens), with or without the mass that the tokens receive;
- ``evict``: each group keeps its last ``recent`` tokens and those with the largest mass before
  them, ``keep`` in all, moved into other pages.

The plain forms are the definitions in 32 bits (rotary angles in 64); ``exact`` has them in 64.
"""

from __future__ import annotations

import math

import torch

own = False

# Rotary base and position scaling of both attention models.
THETA, ROPE_SCALE = 500000.0, 16.0
PAGE = 64
E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -100


def listed():
    big = dict(H=8, nq=2, hd=128)    # the 7B model: eight groups, two query heads each
    small = dict(H=8, nq=1, hd=96)   # the 1B model: one query head per group
    step, small_step = (dict(c, chunks=0, rows=1) for c in (big, small))  # one token each
    return [
        # A decode step of 128 requests: one new token each, at ragged lengths.
        dict(step, kind="append", name="append_step", B=128, ctx_lo=200, ctx_hi=8000),
        # A 4096-token chunk of a prompt, behind 1000 tokens that end inside a page.
        dict(big, kind="append", name="append_prompt", B=1, chunks=1, rows=4096, ctx_lo=1000,
             ctx_hi=1000),
        # One request decoding: the latency of the smallest call.
        dict(step, kind="attend", name="attend_one", B=1, ctx_lo=1500, ctx_hi=1500,
             mass=False),
        # A decode step of 64 requests with ragged contexts.
        dict(step, kind="attend", name="attend_step", B=64, ctx_lo=256, ctx_hi=8192,
             mass=False),
        # The same for the small model, with the mass that eviction goes by.
        dict(small_step, kind="attend", name="attend_step_mass", B=48, ctx_lo=100, ctx_hi=4096,
             mass=True),
        # Four long-document requests decoding.
        dict(step, kind="attend", name="attend_step_long", B=4, ctx_lo=131071, ctx_hi=131071,
             mass=False),
        # A prefill chunk over what earlier chunks of the prompt left.
        dict(big, kind="attend", name="attend_chunk", B=1, chunks=1, rows=2048, ctx_lo=6144,
             ctx_hi=6144, mass=False),
        # The last chunk of a 32768-token prompt: the largest product.
        dict(big, kind="attend", name="attend_chunk_long", B=1, chunks=1, rows=4096,
             ctx_lo=28672, ctx_hi=28672, mass=False),
        # A chunk of one prompt that rides along with sixteen decoding requests, with the mass.
        dict(big, kind="attend", name="attend_mixed_mass", B=17, chunks=1, rows=512, ctx_lo=300,
             ctx_hi=4000, mass=True),
        # One request's cache cut to half.
        dict(big, kind="evict", name="evict_one", B=1, ctx_lo=4096, ctx_hi=4096, keep=2048,
             recent=256),
        # A batch of ragged lengths cut to one budget (some sequences are within it).
        dict(big, kind="evict", name="evict_batch", B=24, ctx_lo=2000, ctx_hi=16000, keep=4000,
             recent=512),
        # Two long documents cut to half.
        dict(big, kind="evict", name="evict_long", B=2, ctx_lo=131000, ctx_hi=131072, keep=65536,
             recent=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    nq, hd = rng.choice([(2, 128), (1, 96), (1, 128), (2, 96), (4, 128), (3, 96)])
    c = dict(H=rng.choice([1, 2, 4, 8, 8]), nq=nq, hd=hd)
    kind = rng.choice(["append", "attend", "attend", "attend", "evict"])
    if kind == "evict":
        B = _log_int(rng, 1, 32)
        hi = _log_int(rng, 64, 262144 // B)
        keep = rng.randint(1, hi)
        return dict(c, kind=kind, B=B, ctx_lo=rng.randint(0, hi), ctx_hi=hi, keep=keep,
                    recent=rng.randint(0, keep))
    what = rng.choice(["step", "step", "chunk", "mixed"])
    B = 1 if what == "chunk" else _log_int(rng, 1, 128) if what == "step" else rng.randint(2, 24)
    most = {"step": 1, "chunk": 4096 if nq <= 2 else 2000, "mixed": 600}[what]
    c.update(kind=kind, B=B, chunks=0 if what == "step" else rng.randint(1, min(B, 3)),
             rows=1 if what == "step" else _log_int(rng, 2, most))
    hi = _log_int(rng, 16, {"step": 400000 // B, "chunk": 28000, "mixed": 4096}[what])
    c.update(ctx_lo=rng.randint(0, hi), ctx_hi=hi)
    return c if kind == "append" else dict(c, mass=rng.random() < 0.5)


def _batch(case):
    """New rows and context of each sequence: the last `chunks` sequences have chunks of about
    `rows` rows, the others one row; contexts spread over [ctx_lo, ctx_hi]."""
    B = case["B"]
    rows = [1] * B
    for i in range(case.get("chunks", 0)):
        rows[B - 1 - i] = max(1, case["rows"] - 37 * i)
    lo, hi = case["ctx_lo"], case["ctx_hi"]
    ctx = [lo + int((hi - lo) * (((b + 1) * 0.6180339887498949) % 1.0)) for b in range(B)]
    return ([0] * B if case["kind"] == "evict" else rows), ctx


def _scale_for(amax):
    """The smallest power of two s, at least 2^-100, with amax <= 448 s."""
    m, e = torch.frexp(amax)          # amax = m 2^e, 448 = 0.875 * 2^9
    s = torch.ldexp(torch.ones_like(m), torch.where(m <= 0.875, e - 9, e - 8))
    return torch.where(amax > 0, s, torch.zeros_like(s)).clamp_min(MIN_SCALE)


def _codes(x):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _bytes(codes):
    return codes.view(torch.uint8)


def _floats(codes):
    return codes.view(torch.float8_e4m3fn).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    B, H, nq, hd = case["B"], case["H"], case["nq"], case["hd"]
    rows, ctx = _batch(case)
    N = sum(rows)
    blocks = max(1, max((c + r + PAGE - 1) // PAGE for c, r in zip(ctx, rows)))
    dst_blocks = (case["keep"] + PAGE - 1) // PAGE if case["kind"] == "evict" else 0
    pages = B * (blocks + dst_blocks)
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    st = {"case": case, "ws": None, "ctx_len": ints(ctx),
          "block_table": order[:B * blocks].reshape(B, blocks).contiguous()}
    # what earlier steps left: keys and values of unit scale whose blocks differ in magnitude
    st["kv_scale"] = torch.empty((pages, H, 2), dtype=torch.float32, device="cuda")
    for i, (name, shape) in enumerate((("k", (PAGE, hd)), ("v", (PAGE // 16, hd, 16)))):
        x = normal(pages, H, *shape)
        one = (pages, H) + (1,) * len(shape)
        x *= (0.3 * normal(*one)).exp()
        s = _scale_for(x.flatten(2).abs().amax(-1))
        st["kv_scale"][:, :, i] = s
        st[name] = _codes(x / s.reshape(one))
        del x
    if case["kind"] == "evict":
        # heavy-tailed masses, some of them equal (tokens that no query looked at)
        mass = (2.0 * normal(pages, H, PAGE)).exp() / (blocks * PAGE)
        st["mass"] = mass * (torch.rand(mass.shape, generator=gen, device="cuda") > 0.05)
        st["dst_table"] = order[B * blocks:].reshape(B, dst_blocks).contiguous()
        return st
    st["row_start"] = ints([sum(rows[:b]) for b in range(B + 1)])
    st["max_rows"] = max(rows)
    if case["kind"] == "append":
        st["qkv"] = normal(H, N, nq + 2, hd).to(torch.bfloat16)
        return st
    st["q"] = (1.5 * normal(H, N, nq, hd)).to(torch.bfloat16)
    st["mass_in"] = st["mass_out"] = None
    if case["mass"]:
        st["mass_in"] = (2.0 * normal(pages, H, PAGE)).exp() / (blocks * PAGE)
        st["mass_out"] = torch.zeros_like(st["mass_in"])
    return st


# ---- one pass ------------------------------------------------------------------


def run(st):
    kind = st["case"]["kind"]
    if kind == "append":
        q = _append_own(st) if own else _append(st)
        return {"q": q, "k": st["k"], "v": st["v"], "kv_scale": st["kv_scale"]}
    if kind == "attend":
        o = _attend_own(st) if own else _attend(st)
        return {"o": o} if st["mass_out"] is None else {"o": o, "mass": st["mass_out"]}
    kept, new_len = _evict_own(st) if own else _evict(st)
    return {"kept": kept, "new_len": new_len, "k": st["k"], "v": st["v"],
            "kv_scale": st["kv_scale"], "mass": st["mass"]}


def _append_own(st):
    from paper_2605_06206_amd import foe

    return foe.cache_append(st["qkv"], st["k"], st["v"], st["kv_scale"], st["block_table"],
                            st["ctx_len"], st["row_start"], THETA, ROPE_SCALE)


def _attend_own(st):
    from paper_2605_06206_amd import foe

    if st["ws"] is None:
        n = foe.cache_attention_workspace_bytes(st["q"], st["block_table"], st["max_rows"],
                                                st["mass_out"] is not None)
        st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return foe.cache_attention(st["q"], st["k"], st["v"], st["kv_scale"], st["block_table"],
                               st["ctx_len"], st["row_start"], st["max_rows"],
                               mass_in=st["mass_in"], mass_out=st["mass_out"], ws=st["ws"])


def _evict_own(st):
    from paper_2605_06206_amd import foe

    return foe.cache_evict(st["k"], st["v"], st["kv_scale"], st["mass"], st["block_table"],
                           st["ctx_len"], st["case"]["keep"], st["case"]["recent"],
                           st["dst_table"])


def _rows_of(st, N):
    """Sequence and index within it of each packed row."""
    row = torch.arange(N, device="cuda")
    seq = torch.searchsorted(st["row_start"][1:].contiguous(), row, right=True)
    return seq, row - st["row_start"][seq]


def _append(st):
    case, qkv = st["case"], st["qkv"]
    H, N, _, hd = qkv.shape
    nq, half = case["nq"], hd // 2
    seq, i = _rows_of(st, N)
    slot = st["ctx_len"][seq].long() + i
    # rotation by the position (the token's place in its sequence)
    inv = THETA ** (-2.0 * torch.arange(half, dtype=torch.float64, device="cuda") / hd)
    ang = (slot.double() / ROPE_SCALE)[:, None] * inv
    cos, sin = ang.cos().float()[None, :, None], ang.sin().float()[None, :, None]
    x = qkv[:, :, :nq + 1].float()
    a, b = x[..., :half], x[..., half:]
    x = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    q = x[:, :, :nq].to(torch.bfloat16)
    kv = torch.stack([x[:, :, nq], qkv[:, :, nq + 1].float()])        # [2, H, N, hd]
    # each block's scale: what its new tokens need, and no less than it had if it held tokens
    page = st["block_table"].long()[seq, slot // PAGE]                 # [N]
    amax = kv.abs().amax(-1).permute(2, 1, 0).contiguous()            # [N, H, 2]
    pages = st["kv_scale"].shape[0]
    need = torch.zeros((pages, H, 2), device="cuda").index_reduce_(0, page, amax, "amax")
    new = torch.zeros(pages, dtype=torch.bool, device="cuda").index_fill_(0, page, True)
    first = (st["ctx_len"].long() // PAGE).clamp_max(st["block_table"].shape[1] - 1)
    part = st["block_table"].long().gather(1, first[:, None])[:, 0]   # the block at the end
    held = torch.zeros(pages, dtype=torch.bool, device="cuda")
    held[part] = st["ctx_len"] % PAGE > 0
    old = st["kv_scale"]
    scale = _scale_for(need)
    scale = torch.where(held[:, None, None], torch.maximum(scale, old), scale)
    scale = torch.where(new[:, None, None], scale, old)
    ratio = (old / scale)[part]                                        # [B, H, 2]
    kb, vb = _bytes(st["k"]), _bytes(st["v"])
    kb[part] = _bytes(_codes(_floats(kb[part]) * ratio[:, :, 0, None, None]))
    vb[part] = _bytes(_codes(_floats(vb[part]) * ratio[:, :, 1, None, None, None]))
    st["kv_scale"].copy_(scale)
    codes = _codes(kv.permute(0, 2, 1, 3) / scale[page].permute(2, 0, 1)[..., None])  # [2,N,H,hd]
    t = slot % PAGE
    heads = torch.arange(H, device="cuda")[None]
    kb[page[:, None], heads, t[:, None]] = _bytes(codes[0])
    vb = vb.transpose(-1, -2)
    vb[page[:, None], heads, (t // 16)[:, None], (t % 16)[:, None]] = _bytes(codes[1])
    return q


def _values(st, table):
    """Keys and values [B, H, blocks * 64, hd] of the pages of a table."""
    p = table.long()
    B, n = p.shape
    s = st["kv_scale"][p]                                              # [B, n, H, 2]
    k = _floats(_bytes(st["k"])[p]) * s[..., 0, None, None]            # [B, n, H, 64, hd]
    v = _floats(_bytes(st["v"])[p]) * s[..., 1, None, None, None]      # [B, n, H, 4, hd, 16]
    H, hd = k.shape[2], k.shape[-1]
    k = k.transpose(1, 2).reshape(B, H, n * PAGE, hd)
    v = v.transpose(-1, -2).transpose(1, 2).reshape(B, H, n * PAGE, hd)
    return k, v


def _attend(st):
    q = st["q"]
    H, N, nq, hd = q.shape
    B, blocks = st["block_table"].shape
    R, L = st["max_rows"], blocks * PAGE
    seq, i = _rows_of(st, N)
    k, v = _values(st, st["block_table"])
    qp = torch.zeros((B, H, R, nq, hd), device="cuda")
    qp[seq, :, i] = q.transpose(0, 1).float()
    s = qp.reshape(B, H, R * nq, hd) @ k.transpose(2, 3).contiguous()
    s = s.reshape(B, H, R, nq, L).mul_(1.0 / math.sqrt(hd))
    seen = (st["ctx_len"].long()[:, None] + torch.arange(R, device="cuda")[None] + 1)  # [B, R]
    key = torch.arange(L, device="cuda")
    s.masked_fill_(key >= seen[:, None, :, None, None], -math.inf)
    s -= s.amax(-1, keepdim=True)
    p = s.exp_()
    p /= p.sum(-1, keepdim=True)
    o = (p.reshape(B, H, R * nq, L) @ v).reshape(B, H, R, nq, hd)
    if st["mass_out"] is not None:
        there = torch.zeros((B, R), dtype=torch.bool, device="cuda")
        there[seq, i] = True
        got = torch.where(there[:, None, :, None, None], p, torch.zeros_like(p)).sum((2, 3))
        n = st["row_start"][1:] - st["row_start"][:-1]
        pg = st["block_table"].long()
        ctx = st["ctx_len"].long()[:, None, None]
        before = st["mass_in"][pg].transpose(1, 2).reshape(B, H, L)
        got = got + torch.where(key < ctx, before, torch.zeros_like(before))
        valid = key < ctx + n.long()[:, None, None]
        keep = st["mass_out"][pg].transpose(1, 2).reshape(B, H, L)
        got = torch.where(valid, got, keep)
        st["mass_out"][pg] = got.reshape(B, H, blocks, PAGE).transpose(1, 2)
    return o[seq, :, i].to(torch.bfloat16)                             # [N, H, nq, hd]


def _evict(st):
    case = st["case"]
    keep, recent, H = case["keep"], case["recent"], case["H"]
    B, blocks = st["block_table"].shape
    L = blocks * PAGE
    n = st["ctx_len"].long()
    mass = st["mass"][st["block_table"].long()].transpose(1, 2).reshape(B, H, L)
    slot = torch.arange(L, device="cuda")
    key = torch.where(slot >= (n - recent)[:, None, None], math.inf, mass)
    key = torch.where(slot < n[:, None, None], key, -math.inf)
    m = n.clamp_max(keep)                                              # kept tokens
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    width = order.shape[-1]
    j = torch.arange(keep, device="cuda")
    kept = torch.full((B, H, keep), L, dtype=torch.long, device="cuda")
    kept[..., :width] = torch.where(j[:width] < m[:, None, None], order, L)
    kept = kept.sort(-1).values
    there = j < m[:, None, None]                                       # [B, 1, keep]
    D = st["dst_table"].shape[1]
    pad = D * PAGE - keep
    src = torch.nn.functional.pad(torch.where(kept < L, kept, 0), (0, pad))
    there = torch.nn.functional.pad(there.expand(B, H, keep), (0, pad))
    sp = st["block_table"].long()[torch.arange(B, device="cuda")[:, None, None], src // PAGE]
    t, heads = src % PAGE, torch.arange(H, device="cuda")[None, :, None]
    sc = st["kv_scale"][sp, heads]                                     # [B, H, D * 64, 2]
    kb, vb = _bytes(st["k"]), _bytes(st["v"]).transpose(-1, -2)
    kv = torch.stack([_floats(kb[sp, heads, t].contiguous()),
                      _floats(vb[sp, heads, t // 16, t % 16].contiguous())])
    kv *= sc.permute(3, 0, 1, 2)[..., None]                            # [2, B, H, D * 64, hd]
    amax = torch.where(there, kv.abs().amax(-1), 0.0).reshape(2, B, H, D, PAGE).amax(-1)
    s = _scale_for(amax)                                               # [2, B, H, D]
    kv /= s.repeat_interleave(PAGE, -1)[..., None]
    at = there.nonzero(as_tuple=True)
    dp, dt = st["dst_table"].long()[at[0], at[2] // PAGE], at[2] % PAGE
    kb[dp, at[1], dt] = _bytes(_codes(kv[0][at]))
    vb[dp, at[1], dt // 16, dt % 16] = _bytes(_codes(kv[1][at]))
    st["mass"][dp, at[1], dt] = st["mass"][sp[at], at[1], t[at]]
    used = (torch.arange(D, device="cuda") * PAGE < m[:, None]).nonzero(as_tuple=True)
    st["kv_scale"][st["dst_table"].long()[used]] = s.permute(1, 3, 2, 0)[used]
    return torch.where(kept < L, kept, -1).int(), m.int()


# ---- what a pass cannot do without ------------------------------------------------


def work(case):
    H, nq, hd = case["H"], case["nq"], case["hd"]
    rows, ctx = _batch(case)
    N = sum(rows)
    if case["kind"] == "append":
        return {"bytes": H * N * hd * (2 * (nq + 2) + 2 * nq + 2),
                "flops": 6 * H * N * (nq + 1) * hd}
    if case["kind"] == "evict":
        m = sum(min(c, case["keep"]) for c in ctx)
        return {"bytes": H * (4 * sum(ctx) + m * (4 * hd + 8)), "flops": 0}
    tokens = sum(c + r for c, r in zip(ctx, rows))
    pairs = sum(r * c + r * (r + 1) // 2 for c, r in zip(ctx, rows))
    per_token = 2 * hd + (8 if case["mass"] else 0)
    return {"bytes": H * (per_token * tokens + 4 * N * nq * hd), "flops": 4 * H * nq * hd * pairs}


# ---- the same in 64 bits ------------------------------------------------------------


def _exact_scale(amax):
    up = torch.ceil(torch.log2(amax.clamp_min(1e-300) / E4M3_MAX))
    return (2.0 ** up).clamp_min(MIN_SCALE)


def _exact_pages(st, table, b, h):
    """Keys and values [blocks * 64, hd] of sequence b's group h."""
    p = table[b].long()
    s = st["kv_scale"][p, h].double()
    k = _floats(_bytes(st["k"])[p, h]).double() * s[:, 0, None, None]
    v = _floats(_bytes(st["v"])[p, h]).double() * s[:, 1, None, None, None]
    return k.flatten(0, 1), v.transpose(2, 3).reshape(-1, k.shape[-1])


def _exact_rotated(x, pos):
    half = x.shape[-1] // 2
    inv = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                    pos.double()[:, None] / ROPE_SCALE * inv)
    y = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * z
    return torch.cat([y.real, y.imag], -1)


def _exact_append(st, rows, ctx):
    """Codes before their rounding: the values in units of their block's scale."""
    case, H = st["case"], st["case"]["H"]
    nq = case["nq"]
    k, v, scale = st["k"].double(), st["v"].double(), st["kv_scale"].double()
    qs, r0 = [], 0
    for b, (n, c) in enumerate(zip(rows, ctx)):
        x = st["qkv"][:, r0:r0 + n].double()
        pos = torch.arange(c, c + n, device="cuda")
        rot = _exact_rotated(x[:, :, :nq + 1].transpose(1, 2), pos)    # [H, nq + 1, n, hd]
        qs.append(rot[:, :nq].transpose(1, 2))
        r0 += n
        new = torch.stack([rot[:, nq], x[:, :, nq + 1]])               # [2, H, n, hd]
        for blk in range(c // PAGE, (c + n - 1) // PAGE + 1):
            p = st["block_table"][b, blk].long()
            lo, hi = max(c, blk * PAGE), min(c + n, blk * PAGE + PAGE)
            mine = new[:, :, lo - c:hi - c]
            s = _exact_scale(mine.abs().amax((2, 3)))                  # [2, H]
            if lo > blk * PAGE:
                s = torch.maximum(s, scale[p].t())
                k[p] *= (scale[p, :, 0] / s[0])[:, None, None]
                v[p] *= (scale[p, :, 1] / s[1])[:, None, None, None]
            scale[p] = s.t()
            mine = mine / s[:, :, None, None]
            k[p, :, lo % PAGE:lo % PAGE + hi - lo] = mine[0]
            vt = v[p].transpose(1, 2).reshape(H, -1, PAGE)             # [H, hd, 64]
            vt[:, :, lo % PAGE:lo % PAGE + hi - lo] = mine[1].transpose(1, 2)
            v[p] = vt.reshape(H, -1, PAGE // 16, 16).transpose(1, 2)
    return {"q": torch.cat(qs, 1), "k": k, "v": v, "kv_scale": scale}


def _exact_attend(st, rows, ctx):
    H, N, nq, hd = st["q"].shape
    o = torch.empty((N, H, nq, hd), dtype=torch.float64, device="cuda")
    mass = None if st["mass_out"] is None else st["mass_out"].double()
    r0 = 0
    for b, (n, c) in enumerate(zip(rows, ctx)):
        p = st["block_table"][b, :(c + n + PAGE - 1) // PAGE].long()
        for h in range(H):
            k, v = _exact_pages(st, st["block_table"], b, h)
            k, v = k[:c + n], v[:c + n]
            got = torch.zeros(c + n, dtype=torch.float64, device="cuda")
            for a in range(0, n, 1024):
                e = min(a + 1024, n)
                q = st["q"][h, r0 + a:r0 + e].double().flatten(0, 1) / math.sqrt(hd)
                s = (q @ k.t()).reshape(e - a, nq, c + n)
                late = torch.arange(c + n, device="cuda") > torch.arange(c + a, c + e,
                                                                         device="cuda")[:, None]
                w = s.masked_fill(late[:, None], -math.inf).softmax(-1)
                o[r0 + a:r0 + e, h] = (w.flatten(0, 1) @ v).reshape(e - a, nq, hd)
                got += w.sum((0, 1))
            if mass is not None:
                m = mass[p, h].flatten()
                m[:c + n] = got
                m[:c] += st["mass_in"][p, h].flatten()[:c].double()
                mass[p, h] = m.reshape(-1, PAGE)
        r0 += n
    return {"o": o} if mass is None else {"o": o, "mass": mass}


def _exact_evict(st, ctx):
    case = st["case"]
    H, keep, recent = case["H"], case["keep"], case["recent"]
    k, v, scale = st["k"].double(), st["v"].double(), st["kv_scale"].double()
    mass = st["mass"].double()
    kept = torch.full((case["B"], H, keep), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(ctx):
        m = min(n, keep)
        for h in range(H):
            w = mass[st["block_table"][b].long(), h].flatten()[:n]
            old = max(0, n - recent)
            ids = torch.arange(n, device="cuda")
            if n > keep:
                # stable: of equal masses the earlier token comes first
                top = torch.sort(-w[:old], stable=True).indices[:keep - (n - old)]
                ids = torch.cat([top.sort().values, ids[old:]])
            kept[b, h, :m] = ids.int()
            kk, vv = _exact_pages(st, st["block_table"], b, h)
            for blk in range((m + PAGE - 1) // PAGE):
                t = ids[blk * PAGE:(blk + 1) * PAGE]
                p, c = st["dst_table"][b, blk].long(), len(t)
                a, z = kk[t], vv[t]
                s = _exact_scale(torch.stack([a.abs().amax(), z.abs().amax()]))
                scale[p, h] = s
                k[p, h, :c] = a / s[0]
                zt = v[p, h].transpose(0, 1).reshape(-1, PAGE)
                zt[:, :c] = (z / s[1]).t()
                v[p, h] = zt.reshape(-1, PAGE // 16, 16).transpose(0, 1)
                mass[p, h, :c] = w[t]
    new_len = torch.tensor([min(n, keep) for n in ctx], dtype=torch.int32, device="cuda")
    return {"kept": kept, "new_len": new_len, "k": k, "v": v, "kv_scale": scale, "mass": mass}


def exact(case, seed):
    rows, ctx = _batch(case)
    if case["kind"] == "evict" and sum(min(c, case["keep"]) for c in ctx) * case["H"] > 500_000:
        return None  # block by block, over twenty seconds
    st = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(st, rows, ctx)
    if case["kind"] == "attend":
        return _exact_attend(st, rows, ctx)
    return _exact_evict(st, ctx)
