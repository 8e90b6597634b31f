"""A cache held in 4 bits, and what a serving step does with it: the append that rotates on the way (with the rows read back), the
attention over the whole cache, the choice of the pages that a query attends, and the attention over chosen pages.  Each as
elementary torch operations (`own` false) or as the library's calls (`own` true)."""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16                      # tokens of a block, features that share a scale
TDTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
FLT_MAX = float(np.finfo(np.float32).max)


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _append(B, new_lo, new_hi, ctx_hi, n_q, n_kv, d, page, rot, axes, interleaved, dtype, theta, mix):
    return dict(op="append", B=B, new_lo=new_lo, new_hi=new_hi, ctx_lo=0, ctx_hi=ctx_hi, n_q=n_q, n_kv=n_kv, d=d, page=page, rot=rot,
                axes=axes, interleaved=interleaved, dtype=dtype, theta=theta, mix=mix)


def _attn(B, new_lo, new_hi, ctx_lo, ctx_hi, n_q, n_kv, d, page, dtype, cap, alibi, prefix, mix):
    return dict(op="attn", B=B, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, n_q=n_q, n_kv=n_kv, d=d, page=page,
                dtype=dtype, cap=cap, alibi=alibi, prefix=prefix, mix=mix)


def _select(B, new_lo, new_hi, ctx_lo, ctx_hi, n_q, n_kv, d, page, dtype, n_select, first, recent, mix):
    return dict(op="select", B=B, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, n_q=n_q, n_kv=n_kv, d=d, page=page,
                dtype=dtype, n_select=n_select, first=first, recent=recent, mix=mix)


def _sparse(B, new_lo, new_hi, ctx_lo, ctx_hi, n_q, n_kv, d, page, dtype, n_select, cap, mix):
    return dict(op="sparse", B=B, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, n_q=n_q, n_kv=n_kv, d=d, page=page,
                dtype=dtype, n_select=n_select, cap=cap, mix=mix)


def listed():
    return [
        # a decode step of the 8B backbone: one token for each of 128 requests, small pages
        dict(name="append_decode", **_append(128, 1, 1, 32768, 32, 8, 128, 16, 128, 1, False, "bf16", 500000.0, 1)),
        # prompts of ragged lengths, 33 thousand tokens
        dict(name="append_prompts", **_append(48, 1, 1400, 1024, 32, 8, 128, 64, 128, 1, False, "bf16", 500000.0, 2)),
        # prompts with images in them in fp32, time, height and width, half of each small head rotated
        dict(name="append_images_fp32", **_append(5, 1, 900, 777, 8, 8, 64, 32, 32, 3, True, "fp32", 10000.0, 3)),
        # one request, a short cache: latency
        dict(name="attn_one_request", **_attn(1, 1, 1, 777, 777, 32, 8, 128, 16, "bf16", 0.0, False, False, 4)),
        # a long-context batch of the 8B backbone: 0.5 G values each for K and V
        dict(name="attn_long_batch", **_attn(16, 1, 1, 32768, 32768, 32, 8, 128, 64, "bf16", 0.0, False, False, 5)),
        # the 7B backbone's heads, ragged lengths, capped scores, small pages in any order
        dict(name="attn_ragged_capped", **_attn(32, 1, 1, 16, 8192, 32, 32, 128, 16, "bf16", 30.0, False, False, 6)),
        # a chunk of a long prompt for each of two requests, a bidirectional prefix (an image)
        dict(name="attn_chunk", **_attn(2, 1024, 1024, 8192, 8192, 32, 8, 128, 64, "bf16", 0.0, False, True, 7)),
        # a mixed step in fp32: short drafts to verify, a bias by distance, heads of 64
        dict(name="attn_drafts_fp32", **_attn(8, 1, 9, 64, 2048, 8, 8, 64, 32, "fp32", 0.0, True, False, 8)),
        # a decode step over very long caches: which 64 of 1024 pages each head reads
        dict(name="select_decode", **_select(16, 1, 1, 65536, 65536, 32, 8, 128, 64, "bf16", 64, 1, 2, 9)),
        # drafts to verify, small pages, ragged caches
        dict(name="select_drafts", **_select(8, 1, 9, 500, 30000, 32, 8, 128, 16, "bf16", 128, 1, 4, 10)),
        # the decode step's attention over those pages
        dict(name="sparse_decode", **_sparse(16, 1, 1, 65536, 65536, 32, 8, 128, 64, "bf16", 64, 0.0, 11)),
        # a few tokens of each request in fp32, small pages, capped scores
        dict(name="sparse_drafts_fp32", **_sparse(6, 1, 9, 100, 9000, 8, 8, 64, 16, "fp32", 48, 20.0, 12)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "select", "sparse"])
    mix = rng.randrange(1 << 30)
    n_kv, g = rng.choice([(8, 4), (8, 1), (32, 1), (4, 8), (8, 2)])
    d, page, dtype = rng.choice([64, 128]), rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "bf16", "fp32"])
    if op == "append":
        B = _log(rng, 1, 128)
        new_hi = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, 16384 // B))
        rot = rng.choice([d, d, d // 2, 48])
        return _append(B, 1, new_hi, _log(rng, 16, 8192), n_kv * g, n_kv, d, page, rot, rng.choice([1, 2, 3]), rng.random() < 0.5, dtype,
                       rng.choice([10000.0, 500000.0]), mix)
    if op == "attn":
        cap, alibi, prefix = rng.choice([0.0, 20.0, 50.0]), rng.random() < 0.3, rng.random() < 0.3
        kind = rng.choice(["decode", "decode", "drafts", "chunk"])
        if kind == "decode":
            ctx = _log(rng, 1, 32768)
            B = _log(rng, 1, max(1, min(64, (1 << 19) // (ctx * max(1, n_kv // 8)))))
            return _attn(B, 1, 1, max(1, ctx // 8), ctx, n_kv * g, n_kv, d, page, dtype, cap, alibi, False, mix)
        if kind == "drafts":
            ctx = _log(rng, 16, 8192)
            return _attn(_log(rng, 1, 16), 1, rng.randint(2, 9), 16, ctx, n_kv * g, n_kv, d, page, dtype, cap, alibi, prefix, mix)
        ctx = _log(rng, 64, 8192)
        nq = min(ctx, _log(rng, 16, 700))
        if dtype == "fp32":
            nq, ctx = min(nq, 128), min(ctx, 2048)
        return _attn(rng.randint(1, 2), max(1, nq // 2), nq, max(nq, ctx // 2), ctx, n_kv * g, n_kv, d, page, dtype, cap, alibi, prefix, mix)
    new_hi = rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 128)])
    ctx = max(new_hi, _log(rng, 16, 65536))
    B = _log(rng, 1, max(1, min(32, (1 << 20) // ctx, 256 // new_hi)))
    n_select = _log(rng, 4, 128)
    if op == "select":
        return _select(B, 1, new_hi, max(1, ctx // 8), ctx, n_kv * g, n_kv, d, page, dtype, n_select, rng.randint(0, 2), rng.randint(1, 2), mix)
    n_select = max(1, min(n_select, (1 << 22) // (B * new_hi * n_kv * page)))
    return _sparse(B, 1, new_hi, max(1, ctx // 8), ctx, n_kv * g, n_kv, d, page, dtype, n_select, rng.choice([0.0, 20.0]), mix)


def _lengths(case):
    """(cached tokens before the step, new tokens) of every request: part of the case, the same for every seed."""
    rng = random.Random(case["mix"])
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["B"])]
    if case["op"] == "append":
        return [rng.randint(0, case["ctx_hi"]) for _ in new], new
    after = [max(n, rng.randint(case["ctx_lo"], case["ctx_hi"])) for n in new]
    return [a - n for a, n in zip(after, new)], new


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _table(case, before, new, gen):
    """Pages handed out in any order, block table rows in any order, as in a pool that has been in use."""
    P, B = case["page"], case["B"]
    pages = [-(-(b + n) // P) for b, n in zip(before, new)]
    width, n_pages = max(pages), sum(pages) + 8
    perm = torch.randperm(n_pages, generator=gen, device="cuda", dtype=torch.int32)
    first = _ints(np.concatenate([[0], np.cumsum(pages)[:-1]]).tolist(), torch.int64)
    col = torch.arange(width, device="cuda")
    at = (first[:, None] + col[None]).clamp(max=n_pages - 1)
    rows = torch.where(col[None] < _ints(pages, torch.int64)[:, None], perm[at], torch.zeros_like(perm[at]))
    slots = torch.randperm(B, generator=gen, device="cuda", dtype=torch.int32)
    table = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    table[slots.long()] = rows
    return table, slots, n_pages, width


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


# ---------------------------------------------------------------------------------------------------------------
# the format: e2m1 codes, an e4m3 scale for each 16 features of a token, blocks of 16 tokens
#   [K codes 16 x d/2 | V codes, by token pairs | K scales 16 x d/16 | V scales d/16 x 16]
# ---------------------------------------------------------------------------------------------------------------
def _quantise(x, unit):
    """x [..., d] fp32 -> (codes uint8 [..., d], scales e4m3 [..., d/16]), in fp32 steps."""
    y = x.unflatten(-1, (-1, BLOCK))
    a = y.abs().amax(-1)
    s8 = (a * float(np.float32(1.0 / (6.0 * unit)))).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = s8.float()
    r = torch.where(s > 0, float(np.float32(1.0 / unit)) / s, torch.zeros_like(s))
    y = y * r[..., None]
    m = y.abs()
    m = torch.where(m < 2, (m * 2).round() / 2, torch.where(m < 4, m.round(), (m / 2).round() * 2)).clamp(max=6.0)
    code = torch.where(m <= 2, m * 2, torch.where(m < 4, m + 2, 4 + m / 2))        # 0 .5 1 1.5 2 3 4 6 -> 0 .. 7
    code = code.to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    return code.flatten(-2), s8


def _pack(kc, ks, vc, vs):
    """codes [..., 16, d], scales [..., 16, d/16] of blocks -> bytes [..., 18 d]."""
    d = kc.shape[-1]
    lead = kc.shape[:-2]
    kb = (kc[..., 0::2] | kc[..., 1::2] << 4).flatten(-2)
    vb = (vc[..., 0::2] | vc[..., 1::2] << 4).view(*lead, 2, 4, 2, 8, d // 16)
    n = len(lead)
    vb = vb.permute(*range(n), n, n + 3, n + 1, n + 2, n + 4).flatten(-5)
    return torch.cat([kb, vb, ks.view(torch.uint8).flatten(-2), vs.view(torch.uint8).transpose(-1, -2).flatten(-2)], -1)


def _unpack(blocks, which):
    """bytes [..., 18 d] -> values [..., 16, d] in fp32 (of unit 1)."""
    d = blocks.shape[-1] // 18
    lead = blocks.shape[:-1]
    n = len(lead)
    if which == 0:
        codes = blocks[..., : 8 * d].unflatten(-1, (16, d // 2))
        scales = blocks[..., 16 * d: 17 * d].unflatten(-1, (16, d // 16))
    else:
        codes = blocks[..., 8 * d: 16 * d].unflatten(-1, (2, 8, 4, 2, d // 16))
        codes = codes.permute(*range(n), n, n + 2, n + 3, n + 1, n + 4).reshape(*lead, 16, d // 2)
        scales = blocks[..., 17 * d:].unflatten(-1, (d // 16, 16)).transpose(-1, -2)
    lut = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=blocks.device)
    pair = torch.stack([lut[torch.arange(256, device=blocks.device) % 16], lut[torch.arange(256, device=blocks.device) // 16]], -1)
    v = pair[codes.int()].view(*lead, 16, d // 16, 16)
    return (v * scales.contiguous().view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _bounds(values, valid):
    """values [..., tokens, d], valid [..., tokens] -> (int8 [..., 2, d] largest and smallest value of every feature, scale)."""
    inf = float("inf")
    top = torch.where(valid[..., None], values, torch.full_like(values, -inf)).amax(-2)
    low = torch.where(valid[..., None], values, torch.full_like(values, inf)).amin(-2)
    both = torch.stack([top, low], -2)
    a = both.abs().amax((-1, -2))
    s = (a * float(np.float32(1.0 / 127.0))).clamp(min=2.0 ** -60)
    codes = (both * (1.0 / s)[..., None, None]).round().clamp(-127, 127)
    return torch.where(torch.isfinite(codes), codes, torch.zeros_like(codes)).to(torch.int8), s


# ---------------------------------------------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, n_q, n_kv, d, P, dt = case["op"], case["n_q"], case["n_kv"], case["d"], case["page"], TDTYPE[case["dtype"]]
    before, new = _lengths(case)
    table, slots, n_pages, width = _table(case, before, new, gen)
    T, B = sum(new), case["B"]
    cu = _ints([0] + np.cumsum(new).tolist())
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), _ints(new, torch.int64))
    pos = torch.arange(T, device="cuda") - cu[:-1].long()[seq] + _ints(before, torch.int64)[seq]
    s = dict(case=case, table=table, slots=slots, n_pages=n_pages, width=width, n_tokens=T, max_new=max(new), cu=cu, seq=seq.int(),
             pos=pos.int(), lens=_ints([b + n for b, n in zip(before, new)]),
             k_unit=2.0 ** -2 if op == "append" else 1.0, v_unit=2.0 ** -4 if op == "append" else 1.0)
    if op == "select":
        centre = _normal(gen, n_pages, n_kv, 1, d)
        line = centre + _normal(gen, n_pages, n_kv, 2, d).abs() * torch.tensor([1.0, -1.0], device="cuda")[:, None]
        s["bounds"], s["bound_scales"] = _bounds(line, torch.ones(n_pages, n_kv, 2, dtype=torch.bool, device="cuda"))
    else:
        shape = (n_pages, n_kv, P // BLOCK, BLOCK, d)
        centre = _normal(gen, n_pages, n_kv, 1, 1, d) * 0.5
        kq = _quantise(centre + _normal(gen, *shape), s["k_unit"])
        vq = _quantise(_normal(gen, *shape), s["v_unit"])
        s["blocks"] = _pack(*kq, *vq)
        s["bounds"] = torch.zeros(n_pages, n_kv, 2, d, dtype=torch.int8, device="cuda")
        s["bound_scales"] = torch.zeros(n_pages, n_kv, device="cuda")
    if op == "append":
        # the fused projection's output: q | k | v of every token in one row
        qkv = _normal(gen, T, (n_q + 2 * n_kv) * d).to(dt)
        s |= dict(q=qkv[:, : n_q * d].view(T, n_q, d), k=qkv[:, n_q * d: (n_q + n_kv) * d].view(T, n_kv, d),
                  v=qkv[:, (n_q + n_kv) * d:].view(T, n_kv, d), rows=table.long()[slots.long()[seq], pos // P] * P + pos % P)
        # (images: height and width beside the time)
        axes = [pos] + [torch.randint(0, 64, (T,), generator=gen, device="cuda") for _ in range(case["axes"] - 1)]
        s["axes_pos"] = torch.stack(axes).int()
        # pages that the step touches: page of (request, j-th page from its first new token on)
        first = [b // P for b in before]
        touched = [(b, f + j) for b, (f, bb, n) in enumerate(zip(first, before, new)) for j in range((bb + n - 1) // P - f + 1)]
        s["touched"] = torch.tensor(touched, device="cuda")
        return s
    s["q"] = (_normal(gen, T, n_q, d) * 2.5).to(dt)
    if op == "attn":
        s |= dict(slopes=None, prefix=None)
        if case["alibi"]:
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, n_q + 1, device="cuda", dtype=torch.float32) / n_q)
        if case["prefix"]:
            s["prefix"] = (torch.rand(B, generator=gen, device="cuda") * s["lens"]).int()
    if op == "sparse":
        # chosen pages: the query's own one, the first one, others at random
        S, own_page = case["n_select"], pos // P
        key = torch.rand(T, n_kv, width, generator=gen, device="cuda")
        col = torch.arange(width, device="cuda")
        key = torch.where(col == own_page[:, None, None], 2.0, torch.where(col == 0, 1.5, key))
        key = torch.where(col <= own_page[:, None, None], key, -1.0)
        top, idx = key.topk(min(S, width), dim=-1)
        idx = torch.where(top >= 0, idx, torch.full_like(idx, width)).sort(-1).values
        idx = torch.nn.functional.pad(torch.where(idx < width, idx, torch.full_like(idx, -1)), (0, S - idx.shape[-1]), value=-1)
        s["pages"] = idx.int().contiguous()
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _sections(half, axes):
    return (half,) if axes == 1 else (half // 2, half - half // 2) if axes == 2 else (
        half // 4, (half - half // 4) // 2, half - half // 4 - (half - half // 4) // 2)


def _axis_of(case):
    """Axis that each frequency index follows: runs of the sections' lengths, or taken in turn while a section lasts."""
    half, axes = case["rot"] // 2, case["axes"]
    sec = _sections(half, axes)
    if not case["interleaved"]:
        return np.repeat(np.arange(axes), sec)
    j = np.arange(half)
    a = j % axes
    return np.where(j // axes < np.asarray(sec)[a], a, 0)


def _plain_append(s):
    c = s["case"]
    P, rot, d = c["page"], c["rot"], c["d"]
    half = rot // 2
    freq = c["theta"] ** (-2.0 * torch.arange(half, device="cuda", dtype=torch.float64) / rot)
    ang = s["axes_pos"].double()[torch.as_tensor(_axis_of(c), device="cuda")].T * freq          # [T][half]
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def turn(x):
        x = x.float()
        x1, x2 = x[..., :half], x[..., half:rot]
        return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin, x[..., rot:]], -1)
    q, k, v = turn(s["q"]), turn(s["k"]), s["v"].float()
    (kc, ks), (vc, vs) = _quantise(k, s["k_unit"]), _quantise(v, s["v_unit"])
    # into the blocks: bytes of the tokens' rows
    page, tok = s["rows"] // P, s["rows"] % P
    blk, r = tok // BLOCK, tok % BLOCK
    raw, T, H = s["blocks"], s["n_tokens"], c["n_kv"]
    parts = [x.squeeze(-1) for x in raw.unsqueeze(-1).split([8 * d, 8 * d, d, d], dim=3)]
    parts[0].unflatten(-1, (16, d // 2))[page, :, blk, r] = kc[..., 0::2] | kc[..., 1::2] << 4
    parts[1].unflatten(-1, (2, 8, 4, 2, d // 16)).permute(0, 1, 2, 3, 5, 6, 4, 7)[page, :, blk, r // 8, r // 2 % 4, r % 2] = (
        vc[..., 0::2] | vc[..., 1::2] << 4).view(T, H, 8, d // 16)
    parts[2].unflatten(-1, (16, d // 16))[page, :, blk, r] = ks.view(torch.uint8)
    parts[3].unflatten(-1, (d // 16, 16)).transpose(-1, -2)[page, :, blk, r] = vs.view(torch.uint8)
    # the touched pages' bounds
    b, j = s["touched"].T
    pid = s["table"].long()[s["slots"].long()[b], j]
    line = _unpack(raw[pid], 0).flatten(2, 3)                                                   # [pages][H][P][d]
    valid = (j[:, None] * P + torch.arange(P, device="cuda") < s["lens"].long()[b][:, None])[:, None].expand(-1, H, -1)
    s["bounds"][pid], s["bound_scales"][pid] = _bounds(line, valid)
    # the rows that the new tokens now have
    kv = [_unpack(raw[page, :, blk], w)[torch.arange(T, device="cuda"), :, r] * u for w, u in ((0, s["k_unit"]), (1, s["v_unit"]))]
    dt = s["q"].dtype
    return dict(q=q.to(dt), k=kv[0].to(dt), v=kv[1].to(dt), bounds=s["bounds"], bound_scales=s["bound_scales"])


def _queries(s):
    """(queries [B][H][g N][d] fp32, padded to the longest, positions [B][N]; tokens' places in that)."""
    c = s["case"]
    n_q, n_kv, d, B, N = c["n_q"], c["n_kv"], c["d"], c["B"], s["max_new"]
    cu, lens = s["cu"].long(), s["lens"].long()
    i = torch.arange(N, device="cuda")
    q = s["q"][(cu[:-1, None] + i).clamp(max=s["n_tokens"] - 1)].float()
    q = q.view(B, N, n_kv, n_q // n_kv, d).permute(0, 2, 3, 1, 4).reshape(B, n_kv, -1, d)
    return q, (lens - (cu[1:] - cu[:-1]))[:, None] + i


def _plain_attn(s):
    c = s["case"]
    n_q, n_kv, d, P, B = c["n_q"], c["n_kv"], c["d"], c["page"], c["B"]
    g, N, L = n_q // n_kv, s["max_new"], s["width"] * c["page"]
    raw = s["blocks"][s["table"].long()[s["slots"].long()]]                 # [B][pages][H][P / 16][18 d]
    k, v = [_unpack(raw, w).permute(0, 2, 1, 3, 4, 5).reshape(B, n_kv, L, d) for w in (0, 1)]
    q, pos = _queries(s)
    x = (q @ k.transpose(-1, -2)).view(B, n_kv, g, N, L) * (1.0 / math.sqrt(d))
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    t = torch.arange(L, device="cuda")
    if c["alibi"]:
        x = x - s["slopes"].view(n_kv, g)[None, :, :, None, None] * (pos[:, :, None] - t).abs()[:, None, None].float()
    seen = t <= pos[..., None]
    if c["prefix"]:
        seen = seen | (t < s["prefix"].long()[:, None, None])
    seen = seen & (t < s["lens"].long()[:, None, None])
    x = x.masked_fill(~seen[:, None, None], float("-inf"))
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = (p.view(B, n_kv, g * N, L) @ v).view(B, n_kv, g, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, n_q, d)
    seq = s["seq"].long()
    return dict(out=o[seq, torch.arange(s["n_tokens"], device="cuda") - s["cu"].long()[seq]].to(s["q"].dtype))


def _plain_select(s):
    c = s["case"]
    n_q, n_kv, P, B, S, N, W = c["n_q"], c["n_kv"], c["page"], c["B"], c["n_select"], s["max_new"], s["width"]
    q, pos = _queries(s)
    top = q.abs().amax(-1)
    s_q = (top * float(np.float32(1.0 / 127.0))).clamp(2.0 ** -60, 2.0 ** 100)
    codes = (q * (1.0 / s_q)[..., None]).round().clamp(-127, 127)
    pid = s["table"].long()[s["slots"].long()]                              # [B][W]
    both = s["bounds"][pid].float().permute(0, 2, 3, 1, 4)                  # [B][H][2][W][d]
    s_p = s["bound_scales"][pid].permute(0, 2, 1)                           # [B][H][W]
    # whole numbers below 2^24: exact in fp32 in any order
    whole = codes.clamp(min=0) @ both[:, :, 0].transpose(-1, -2) + codes.clamp(max=0) @ both[:, :, 1].transpose(-1, -2)
    score = (s_q[..., None] * s_p[:, :, None]) * whole
    score = torch.where(torch.isnan(score), torch.full_like(score, FLT_MAX), score)
    score = score.view(B, n_kv, n_q // n_kv, N, W).amax(2)                  # [B][H][N][W]
    own_page, j = (pos // P)[:, None, :, None], torch.arange(W, device="cuda")
    inf = float("inf")
    score = torch.where((j < c["first"]) | (j > own_page - c["recent"]), inf, score)
    score = torch.where(j <= own_page, score, -inf)
    key, idx = score.sort(dim=-1, descending=True, stable=True)
    idx = torch.where(key > -inf, idx, W)[..., :S].sort(-1).values
    idx = torch.nn.functional.pad(torch.where(idx < W, idx, -1), (0, max(0, S - W)), value=-1)
    seq = s["seq"].long()
    return dict(pages=idx.permute(0, 2, 1, 3)[seq, torch.arange(s["n_tokens"], device="cuda") - s["cu"].long()[seq]].int())


def _plain_sparse(s):
    c = s["case"]
    n_q, n_kv, d, P, T = c["n_q"], c["n_kv"], c["d"], c["page"], s["n_tokens"]
    g, S = n_q // n_kv, c["n_select"]
    rows = s["table"].long()[s["slots"].long()[s["seq"].long()]]            # [T][W]
    chosen = s["pages"].long()                                              # [T][H][S]
    pid = rows[:, None].expand(-1, n_kv, -1).gather(-1, chosen.clamp(min=0))
    raw = s["blocks"][pid, torch.arange(n_kv, device="cuda")[:, None]]       # [T][H][S][P / 16][18 d]
    k, v = [_unpack(raw, w).reshape(T, n_kv, S * P, d) for w in (0, 1)]
    t = (chosen[..., None] * P + torch.arange(P, device="cuda")).view(T, n_kv, S * P)
    seen = ((chosen >= 0)[..., None].expand(-1, -1, -1, P).reshape(T, n_kv, S * P)) & (t <= s["pos"].long()[:, None, None])
    x = (s["q"].float().view(T, n_kv, g, d) @ k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    x = x.masked_fill(~seen[:, :, None], float("-inf"))
    p = torch.exp(x - x.amax(-1, keepdim=True))
    return dict(out=((p / p.sum(-1, keepdim=True)) @ v).view(T, n_q, d).to(s["q"].dtype))


# ---------------------------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2603_22910_b200 import binding
    c = s["case"]
    op = c["op"]
    if "cache" not in s:                       # made once, as a program does
        cfg = binding.make_config(n_layers=1, n_q_heads=c["n_q"], n_kv_heads=c["n_kv"], head_dim=c["d"], group_size=1, n_retained_heads=0,
                                  page_tokens=c["page"], max_batch=c["B"], max_pages_per_seq=s["width"], n_pages=s["n_pages"],
                                  dtype=binding.ECHOKV_BF16 if c["dtype"] == "bf16" else binding.ECHOKV_FP32)
        s["cache"] = binding.Fp4Cache(cfg, k_unit=s["k_unit"], v_unit=s["v_unit"], blocks=s.get("blocks"), bounds=s["bounds"],
                                      bound_scales=s["bound_scales"])
        if op == "append":
            s["rotation"] = binding.Rotation(cfg, c["theta"], n_axes=c["axes"], sections=_sections(c["rot"] // 2, c["axes"]), rot_dim=c["rot"],
                                             interleaved=c["interleaved"])
    cache = s["cache"]
    if op == "append":
        q = cache.append(s["k"], s["v"], s["rows"], q=s["q"], rotation=s["rotation"], positions=s["axes_pos"])
        k, v = cache.read(s["rows"])
        return dict(q=q, k=k, v=v, bounds=s["bounds"], bound_scales=s["bound_scales"])
    if op == "attn":
        return dict(out=cache.attention(s["q"], s["table"], s["lens"], cu_tokens=s["cu"], max_new=s["max_new"], seq_slots=s["slots"],
                                        softcap=c["cap"], alibi_slopes=s["slopes"], prefix_lens=s["prefix"]))
    if op == "select":
        return dict(pages=cache.select_pages(s["q"], s["table"], s["seq"], s["pos"], c["n_select"], n_first=c["first"], n_recent=c["recent"],
                                             seq_slots=s["slots"]))
    return dict(out=cache.sparse_attention(s["q"], s["table"], s["seq"], s["pos"], s["pages"], seq_slots=s["slots"], softcap=c["cap"]))


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attn": _plain_attn, "select": _plain_select, "sparse": _plain_sparse}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------
# what cannot be done without, and the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    before, new = _lengths(case)
    T, P, n_q, n_kv, d = sum(new), case["page"], case["n_q"], case["n_kv"], case["d"]
    e = 2 if case["dtype"] == "bf16" else 4
    pair = 2 * n_kv * (d // 2 + d // 16)                       # a token's K and V in the cache
    if case["op"] == "append":
        # q in and out, k and v in and read back, the cache written once and read once; bounds of the touched pages (keys of a
        # page that were there before, too)
        touched = sum((b + n - 1) // P - b // P + 1 for b, n in zip(before, new))
        old = sum(b % P for b in before)
        return {"bytes": T * ((2 * n_q + 4 * n_kv) * d * e + 2 * pair + 8 + 4 * case["axes"]) + old * pair // 2 + touched * n_kv * (2 * d + 4),
                "flops": T * (3 * n_q + 12 * n_kv) * d}
    after = [b + n for b, n in zip(before, new)]
    if case["op"] == "attn":
        pairs = sum(n * a - n * (n - 1) // 2 for a, n in zip(after, new))
        return {"bytes": sum(after) * pair + T * n_q * d * 2 * e, "flops": 4 * pairs * n_q * d}
    pos = [b + i for b, n in zip(before, new) for i in range(n)]
    if case["op"] == "select":
        pages = sum(-(-a // P) for a in after)
        seen = sum(p // P + 1 for p in pos)
        return {"bytes": pages * (n_kv * (2 * d + 4) + 4) + T * (n_q * d * e + n_kv * case["n_select"] * 4), "flops": 2 * seen * n_q * 2 * d}
    tokens = sum(min(p + 1, (min(case["n_select"], p // P + 1) - 1) * P + p % P + 1) for p in pos)
    return {"bytes": tokens * pair + T * (n_q * d * 2 * e + n_kv * case["n_select"] * 4), "flops": 4 * tokens * n_q * d}


def _row64(raw, which, d):
    """[n][18 d] bytes of blocks -> [16 n][d] values in 64 bits, from the bits of the codes and scales."""
    n = len(raw)
    tok, f = torch.meshgrid(torch.arange(16, device="cuda"), torch.arange(d, device="cuda"), indexing="ij")
    if which == 0:
        at, sc = tok * (d // 2) + f // 2, 16 * d + tok * (d // 16) + f // 16
    else:
        w = d // 16                                          # bytes of a lane's share of a token
        at = 8 * d + (((tok // 8 * 8 + f // (d // 8)) * 4 + tok % 8 // 2) * 2 + tok % 2) * w + f % (d // 8) // 2
        sc = 17 * d + f // 16 * 16 + tok
    code = raw[:, at.flatten()].long() >> (f.flatten() % 2 * 4) & 15
    ex, man = code >> 1 & 3, (code & 1).double()
    mag = torch.where(ex == 0, man / 2, (1 + man / 2) * 2.0 ** (ex - 1).double())
    byte = raw[:, sc.flatten()].long()
    ex, man = byte >> 3 & 15, (byte & 7).double()
    scale = torch.where(ex == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * 2.0 ** (ex - 7).double())
    return (mag * torch.where(code >= 8, -1.0, 1.0) * scale).view(n * 16, d)


def _softmax64(q, k, v, hidden, cap, bias):
    x = q @ k.T / math.sqrt(q.shape[-1])
    if cap:
        x = torch.tanh(x / cap) * cap
    if bias is not None:
        x = x - bias
    return torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v


def exact(case, seed):
    if case["op"] == "select":
        return None                                          # whole numbers
    s = prepare(case, seed)
    n_q, n_kv, d, P = case["n_q"], case["n_kv"], case["d"], case["page"]
    if case["op"] == "append":
        half, rot = case["rot"] // 2, case["rot"]
        pos = s["axes_pos"].cpu().numpy().astype(np.float64)
        z = np.exp(1j * pos[_axis_of(case)].T * case["theta"] ** (-np.arange(half) / half))[:, None, :]
        x = s["q"].double().cpu().numpy()
        y = (x[..., :half] + 1j * x[..., half:rot]) * z
        # (what is held in 4 and 8 bits has no value in more bits than it is held in)
        return dict(q=np.concatenate([y.real, y.imag, x[..., rot:]], -1), k=None, v=None, bounds=None, bound_scales=None)
    table, cu, slots, lens = (s[n].cpu().tolist() for n in ("table", "cu", "slots", "lens"))
    out = torch.empty(s["n_tokens"], n_q, d, dtype=torch.float64, device="cuda")
    if case["op"] == "attn":
        prefix = s["prefix"].cpu().tolist() if case["prefix"] else [0] * case["B"]
        for b in range(case["B"]):
            n = lens[b]
            pages = torch.tensor(table[slots[b]][: -(-n // P)], device="cuda")
            at = torch.arange(n - (cu[b + 1] - cu[b]), n, device="cuda", dtype=torch.float64)[:, None]
            t = torch.arange(n, device="cuda", dtype=torch.float64)
            hidden = (t > at) & (t >= prefix[b])
            for h in range(n_kv):
                k, v = [_row64(s["blocks"][pages, h].flatten(0, 1), w, d)[:n] for w in (0, 1)]
                for j in range(h * n_q // n_kv, (h + 1) * n_q // n_kv):
                    bias = float(s["slopes"][j]) * (at - t).abs() if case["alibi"] else None
                    out[cu[b]:cu[b + 1], j] = _softmax64(s["q"][cu[b]:cu[b + 1], j].double(), k, v, hidden, case["cap"], bias)
        return dict(out=out.cpu().numpy())
    if s["n_tokens"] * n_kv > 3000:
        return None
    seq, pos, chosen = (s[n].cpu().tolist() for n in ("seq", "pos", "pages"))
    g = n_q // n_kv
    for i in range(s["n_tokens"]):
        for h in range(n_kv):
            mine = [p for p in chosen[i][h] if p >= 0]
            raw = s["blocks"][torch.tensor([table[slots[seq[i]]][p] for p in mine], device="cuda"), h].flatten(0, 1)
            t = (torch.tensor(mine, device="cuda")[:, None] * P + torch.arange(P, device="cuda")).flatten()
            out[i, h * g:(h + 1) * g] = _softmax64(s["q"][i, h * g:(h + 1) * g].double(), _row64(raw, 0, d), _row64(raw, 1, d),
                                                   (t > pos[i])[None], case["cap"], None)
    return dict(out=out.cpu().numpy())
