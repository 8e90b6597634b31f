"""What one serving step needs around the attention over a cache held in 8 bits: the plan of the step (block table and
slot map from request lengths), the rotary positions of the new queries and keys, the append that quantises, and the
attention.  Each as elementary torch operations (`own` false) or as the library's calls (`own` true)."""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16                      # tokens that share a scale
QMAX = {"int8": 127.0, "e4m3": 448.0}
TDTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _plan(B, new_lo, new_hi, ctx_lo, ctx_hi, page, mix):
    return dict(op="plan", B=B, new_lo=new_lo, new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, page=page, mix=mix)


def _rotate(T, n_q, n_kv, d, rot, axes, interleaved, dtype, inverse, pos_hi, theta, mix):
    return dict(op="rotate", T=T, n_q=n_q, n_kv=n_kv, d=d, rot=rot, axes=axes, interleaved=interleaved, dtype=dtype,
                inverse=inverse, pos_hi=pos_hi, theta=theta, mix=mix)


def _append(B, new_lo, new_hi, ctx_hi, n_kv, d, page, fmt, dtype, mix):
    return dict(op="append", B=B, new_lo=new_lo, new_hi=new_hi, ctx_hi=ctx_hi, n_kv=n_kv, d=d, page=page, fmt=fmt,
                dtype=dtype, mix=mix)


def _attn(B, nq_lo, nq_hi, ctx_lo, ctx_hi, n_q, n_kv, d, page, fmt, dtype, cap, alibi, prefix, mix):
    return dict(op="attn", B=B, nq_lo=nq_lo, nq_hi=nq_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, n_q=n_q, n_kv=n_kv, d=d,
                page=page, fmt=fmt, dtype=dtype, cap=cap, alibi=alibi, prefix=prefix, mix=mix)


def listed():
    return [
        # a decode step of a full batch: one token per request, every sixteenth request needs a page
        dict(name="plan_decode", **_plan(256, 1, 1, 1, 8192, 16, 1)),
        # a step that also takes in prompts: ragged chunks, 33 thousand tokens
        dict(name="plan_prompts", **_plan(64, 1, 1024, 0, 16384, 16, 2)),
        # decode: 64 tokens, the 8B backbone's heads, plain text positions
        dict(name="rotate_decode", **_rotate(64, 32, 8, 128, 128, 1, False, "bf16", False, 131072, 500000.0, 3)),
        # a prompt with images and video in it: time, height and width
        dict(name="rotate_video", **_rotate(16385, 32, 8, 128, 128, 3, False, "bf16", False, 32768, 1000000.0, 4)),
        # the gradient's pass of the same on the 7B backbone's heads in fp32, half of each head rotated
        dict(name="rotate_inverse", **_rotate(2049, 32, 32, 128, 64, 3, True, "fp32", True, 8192, 10000.0, 5)),
        # decode: one token per request joins its block; one in sixteen completes it
        dict(name="append_decode", **_append(128, 1, 1, 32768, 8, 128, 16, "int8", "bf16", 6)),
        # prompts: ragged lengths, 33 thousand tokens
        dict(name="append_prompts", **_append(48, 1, 1400, 1024, 8, 128, 64, "e4m3", "bf16", 7)),
        # one request, a short cache: latency
        dict(name="attn_one_request", **_attn(1, 1, 1, 777, 777, 32, 8, 128, 16, "int8", "bf16", 0.0, False, False, 8)),
        # a long-context batch of the 8B backbone: 0.5 G codes each for K and V
        dict(name="attn_long_batch", **_attn(16, 1, 1, 32768, 32768, 32, 8, 128, 64, "int8", "bf16", 0.0, False, False, 9)),
        # the 7B backbone's heads, ragged lengths, capped scores, e4m3 codes, small pages in any order
        dict(name="attn_ragged_capped", **_attn(32, 1, 1, 16, 8192, 32, 32, 128, 16, "e4m3", "bf16", 30.0, False, False, 10)),
        # a chunk of a long prompt per request, a bidirectional prefix (an image), capped scores
        dict(name="attn_chunk", **_attn(2, 1024, 1024, 8192, 8192, 32, 8, 128, 64, "e4m3", "bf16", 50.0, False, True, 11)),
        # a mixed step in fp32: short drafts to verify, a bias by distance, heads of 64
        dict(name="attn_drafts_fp32", **_attn(8, 1, 9, 64, 2048, 8, 8, 64, 32, "int8", "fp32", 0.0, True, False, 12)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "rotate", "append", "attn", "attn"])
    mix = rng.randrange(1 << 30)
    n_kv, g = rng.choice([(8, 4), (8, 1), (32, 1), (4, 8), (8, 2)])
    d, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    if op == "plan":
        B = _log(rng, 1, 512)
        new_hi = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, 32768 // B))
        return _plan(B, rng.choice([0, 1]), new_hi, 0, _log(rng, 16, 32768), page, mix)
    if op == "rotate":
        rot = rng.choice([d, d, d // 2])
        return _rotate(_log(rng, 1, 8192), n_kv * g, n_kv, d, rot, rng.choice([1, 2, 3]), rng.random() < 0.5,
                       rng.choice(["bf16", "fp32"]), rng.random() < 0.5, _log(rng, 64, 1000000),
                       rng.choice([10000.0, 500000.0]), mix)
    fmt, dtype = rng.choice(["int8", "e4m3"]), rng.choice(["bf16", "bf16", "fp32"])
    if op == "append":
        B = _log(rng, 1, 128)
        new_hi = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, 16384 // B))
        return _append(B, 1, new_hi, _log(rng, 16, 8192), n_kv, d, page, fmt, dtype, mix)
    cap, alibi, prefix = rng.choice([0.0, 20.0, 50.0]), rng.random() < 0.3, rng.random() < 0.3
    kind = rng.choice(["decode", "decode", "drafts", "chunk"])
    if kind == "decode":
        ctx = _log(rng, 1, 32768)
        B = _log(rng, 1, max(1, min(64, (1 << 19) // (ctx * max(1, n_kv // 8)))))
        return _attn(B, 1, 1, max(1, ctx // 8), ctx, n_kv * g, n_kv, d, page, fmt, dtype, cap, alibi, False, mix)
    if kind == "drafts":
        ctx = _log(rng, 16, 8192)
        return _attn(_log(rng, 1, 16), 1, rng.randint(2, 9), 16, ctx, n_kv * g, n_kv, d, page, fmt, dtype, cap, alibi, prefix, mix)
    ctx = _log(rng, 64, 8192)
    nq = min(ctx, _log(rng, 16, 700))
    if dtype == "fp32":
        nq, ctx = min(nq, 128), min(ctx, 2048)
    return _attn(rng.randint(1, 2), max(1, nq // 2), nq, max(nq, ctx // 2), ctx, n_kv * g, n_kv, d, page, fmt, dtype, cap, alibi, prefix, mix)


def _lengths(case):
    """(cached tokens before the step, new tokens) of every request: part of the case, the same for every seed."""
    rng = random.Random(case["mix"])
    op, B = case["op"], case["B"]
    if op == "attn":
        new = [rng.randint(case["nq_lo"], case["nq_hi"]) for _ in range(B)]
        after = [max(n, rng.randint(case["ctx_lo"], case["ctx_hi"])) for n in new]
        return [a - n for a, n in zip(after, new)], new
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(B)]
    if op == "plan":
        return [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(B)], new
    # append: prompts are cut at block borders, decode steps stand anywhere
    before = [rng.randint(0, case["ctx_hi"]) for _ in range(B)]
    if case["new_hi"] > 1:
        before = [b // BLOCK * BLOCK for b in before]
    return before, new


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _pages(before, new, page):
    return [-(-(b + n) // page) for b, n in zip(before, new)]


def _table(case, before, new, gen):
    """Pages handed out in any order, block table rows in any order, as in a pool that has been in use."""
    pages = _pages(before, new, case["page"])
    width, n_pages, B = max(max(pages), 1), sum(pages) + 8, case["B"]
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


def _codes(gen, fmt, n_pages, n_kv, page, d):
    x = torch.randn(n_pages, n_kv, page, d, generator=gen, device="cuda", dtype=torch.bfloat16)
    if fmt == "int8":
        codes = (x * 40).round_().clamp_(-127, 127).to(torch.int8)
    else:
        codes = (x * 140).clamp_(-448, 448).to(torch.float8_e4m3fn)
    spread = torch.rand(n_pages, n_kv, page // BLOCK, generator=gen, device="cuda") + 0.5
    return codes, spread * ((1 / 40) if fmt == "int8" else (1 / 140))


# ---------------------------------------------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "plan":
        before, new = _lengths(case)
        B, P = case["B"], case["page"]
        pages = _pages(before, new, P)
        width, n_pages = max(max(pages), 1), sum(pages) + 8
        used = sum(_pages(before, [0] * B, P))
        perm = torch.randperm(n_pages, generator=gen, device="cuda", dtype=torch.int32)
        table = torch.zeros(B, width, dtype=torch.int32, device="cuda")
        slots = torch.randperm(B, generator=gen, device="cuda", dtype=torch.int32)
        old = _ints(_pages(before, [0] * B, P), torch.int64)
        col = torch.arange(width, device="cuda")
        at = ((old.cumsum(0) - old)[:, None] + col[None]).clamp(max=n_pages - 1)
        table[slots.long()] = torch.where(col[None] < old[:, None], perm[at], torch.zeros_like(perm[at]))
        free = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        free[: n_pages - used] = perm[used:]
        s |= dict(table=table, slots=slots, seq_lens=_ints(before), new_lens=_ints(new), free_pages=free,
                  free_count=_ints([n_pages - used]), n_tokens=sum(new), n_pages=n_pages, width=width)
        return s
    if case["op"] == "rotate":
        T, n_q, n_kv, d = case["T"], case["n_q"], case["n_kv"], case["d"]
        # the fused projection's output: q | k | v of every token in one row
        qkv = _normal(gen, T, (n_q + 2 * n_kv) * d).to(TDTYPE[case["dtype"]])
        pos = torch.randint(0, case["pos_hi"], (case["axes"], T), generator=gen, device="cuda", dtype=torch.int32)
        s |= dict(q=qkv[:, : n_q * d].view(T, n_q, d), k=qkv[:, n_q * d:(n_q + n_kv) * d].view(T, n_kv, d), pos=pos)
        return s
    before, new = _lengths(case)
    n_kv, d, P, dt = case["n_kv"], case["d"], case["page"], TDTYPE[case["dtype"]]
    table, slots, n_pages, width = _table(case, before, new, gen)
    T, B = sum(new), case["B"]
    kc, ks = _codes(gen, case["fmt"], n_pages, n_kv, P, d)
    vc, vs = _codes(gen, case["fmt"], n_pages, n_kv, P, d)
    s |= dict(table=table, slots=slots, n_pages=n_pages, width=width, n_tokens=T, max_new=max(new), kc=kc, ks=ks, vc=vc, vs=vs,
              kt=_normal(gen, B, n_kv, BLOCK, d).to(dt), vt=_normal(gen, B, n_kv, BLOCK, d).to(dt),
              cu=_ints([0] + np.cumsum(new).tolist()), lens=_ints([b + n for b, n in zip(before, new)]))
    if case["op"] == "append":
        seq = torch.repeat_interleave(torch.arange(B, device="cuda"), _ints(new, torch.int64))
        pos = torch.arange(T, device="cuda") - s["cu"][:-1].long()[seq] + _ints(before, torch.int64)[seq]
        s |= dict(k=_normal(gen, T, n_kv, d).to(dt), v=_normal(gen, T, n_kv, d).to(dt), seq=seq.int(),
                  rows=table.long()[slots.long()[seq], pos // P] * P + pos % P, max_blocks=(max(new) + 2 * BLOCK - 2) // BLOCK,
                  n_full=sum((b % BLOCK + n) // BLOCK for b, n in zip(before, new)))
        return s
    n_q = case["n_q"]
    s |= dict(q=(_normal(gen, T, n_q, d) * 2.5).to(dt), max_len=max(b + n for b, n in zip(before, new)), slopes=None, prefix=None)
    if case["alibi"]:
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, n_q + 1, device="cuda", dtype=torch.float32) / n_q)
    if case["prefix"]:
        s["prefix"] = (torch.rand(B, generator=gen, device="cuda") * s["lens"]).int()
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _plain_plan(s):
    P, n = s["case"]["page"], s["n_tokens"]
    lens, new, count = s["seq_lens"].long(), s["new_lens"].long(), s["free_count"].long()
    old = (lens + P - 1) // P
    need = (lens + new + P - 1) // P - old
    upto = need.cumsum(0)
    served = ((need == 0) | (upto <= count)) & (new.cumsum(0) <= n)
    take = torch.where(served, new, torch.zeros_like(new))
    cu = torch.nn.functional.pad(take.cumsum(0), (1, 0))
    after = lens + take
    slots = s["slots"].long()
    col = torch.arange(s["width"], device="cuda")[None]
    fresh = (col >= old[:, None]) & (col < (old + need)[:, None]) & served[:, None]
    at = (count - 1 - ((upto - need)[:, None] + col - old[:, None])).clamp(0, s["n_pages"] - 1)
    rows = torch.where(fresh, s["free_pages"][at], s["table"][slots])
    s["table"][slots] = rows
    tok = torch.arange(n, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
    live = seq < len(lens)
    q = seq.clamp(max=len(lens) - 1)
    pos = tok - cu[q] + lens[q]
    slot = rows[q, (pos // P).clamp(0, s["width"] - 1)].long() * P + pos % P
    none = torch.full_like(tok, -1)
    return dict(table=s["table"], cu=cu.int(), positions=torch.where(live, pos, none).int(), seqs=torch.where(live, seq, none).int(),
                rows=torch.where(live, slot, none), lens=after.int(), count=(count - torch.where(served, need, torch.zeros_like(need)).sum()).int())


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


def _plain_rotate(s):
    c = s["case"]
    rot = c["rot"]
    half = rot // 2
    freq = c["theta"] ** (-2.0 * torch.arange(half, device="cuda", dtype=torch.float64) / rot)
    ang = s["pos"].double()[torch.as_tensor(_axis_of(c), device="cuda")].T * freq          # [T][half]
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    sin = -sin if c["inverse"] else sin

    def turn(x):
        x1, x2, rest = x[..., :half].float(), x[..., half:rot].float(), x[..., rot:]
        return torch.cat([(x1 * cos - x2 * sin).to(x.dtype), (x2 * cos + x1 * sin).to(x.dtype), rest], -1)
    return dict(q=turn(s["q"]), k=turn(s["k"]))


def _plain_append(s):
    c = s["case"]
    P, n_kv, d, B, fmt = c["page"], c["n_kv"], c["d"], c["B"], c["fmt"]
    rows, cu, slots = s["rows"], s["cu"].long(), s["slots"].long()
    new = cu[1:] - cu[:-1]
    off = rows[cu[:-1].clamp(max=len(rows) - 1)] % BLOCK                    # rows of the first block that wait in the tail
    r = torch.arange(BLOCK, device="cuda")
    at = torch.arange(s["max_blocks"], device="cuda")[None, :, None] * BLOCK + r - off[:, None, None]   # token of the step
    fresh = (at >= 0) & (at < new[:, None, None])
    tok = (cu[:-1, None, None] + at).clamp(0, len(rows) - 1)
    full = fresh[..., BLOCK - 1]                                            # blocks that the step completes
    last = tok[..., BLOCK - 1]
    b_at, j_at = torch.nonzero_static(full, size=s["n_full"]).T
    row0 = rows[last[b_at, j_at]] - (BLOCK - 1)
    page, inside = row0 // P, row0 % P
    part = (off + new) // BLOCK                                             # the block that stays open, if any
    has = fresh[torch.arange(B, device="cuda"), part.clamp(max=s["max_blocks"] - 1)] & (part < s["max_blocks"])[:, None]
    tok_open = tok[torch.arange(B, device="cuda"), part.clamp(max=s["max_blocks"] - 1)]
    out = {}
    inv_q = np.float32(1.0) / np.float32(QMAX[fmt])
    floor = 2.0 ** -100
    for x, tail, codes, scales, name in ((s["k"], s["kt"], s["kc"], s["ks"], "k"), (s["v"], s["vt"], s["vc"], s["vs"], "v")):
        old = tail[slots[b_at]].permute(0, 2, 1, 3)                         # [blocks][16][heads][d]
        blk = torch.where(fresh[b_at, j_at][..., None, None], x[tok[b_at, j_at]], old).float()
        amax = blk.abs().amax(dim=(1, 3))
        ok = torch.isfinite(amax)
        scale = torch.where(ok, (amax * float(inv_q)).clamp(min=floor), torch.full_like(amax, float("nan")))
        y = torch.where(ok[:, None, :, None], blk * torch.reciprocal(scale)[:, None, :, None], torch.zeros_like(blk))
        y = (y.round() if fmt == "int8" else y).clamp(-QMAX[fmt], QMAX[fmt]).to(CODE[fmt])
        raw = codes.view(torch.uint8)
        raw[page[:, None], :, inside[:, None] + r] = y.view(torch.uint8)
        scales[page, :, inside // BLOCK] = scale
        mine = tail[slots]
        tail[slots] = torch.where(has[:, None, :, None], x[tok_open].permute(0, 2, 1, 3), mine)
        out |= {name + "_codes": codes, name + "_scales": scales, name + "_tail": tail}
    return out


def _plain_attn(s):
    c = s["case"]
    n_q, n_kv, d, P, B = c["n_q"], c["n_kv"], c["d"], c["page"], c["B"]
    g, L, N = n_q // n_kv, s["max_len"], s["max_new"]
    lens, cu, slots = s["lens"].long(), s["cu"].long(), s["slots"].long()
    t = torch.arange(L, device="cuda")
    page = s["table"].long()[slots][:, t // P]                              # [B][L]
    open_ = t[None] >= (lens // BLOCK * BLOCK)[:, None]

    def rows(codes, scales, tail):
        x = codes.view(torch.uint8)[page, :, t % P].view(codes.dtype)                      # [B][L][heads][d]
        x = x.float() * scales[page, :, t % P // BLOCK][..., None]
        w = tail[slots].permute(0, 2, 1, 3)[:, t % BLOCK].float()
        return torch.where(open_[..., None, None], w, x).permute(0, 2, 1, 3)
    k, v = rows(s["kc"], s["ks"], s["kt"]), rows(s["vc"], s["vs"], s["vt"])
    new = cu[1:] - cu[:-1]
    i = torch.arange(N, device="cuda")
    q = s["q"][(cu[:-1, None] + i).clamp(max=s["n_tokens"] - 1)].float()    # [B][N][n_q][d]
    q = q.view(B, N, n_kv, g, d).permute(0, 2, 3, 1, 4).reshape(B, n_kv, g * N, d)
    x = (q @ k.transpose(-1, -2)).view(B, n_kv, g, N, L) * (1.0 / math.sqrt(d))
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    pos = (lens - new)[:, None] + i                                         # [B][N]
    if c["alibi"]:
        x = x - s["slopes"].view(n_kv, g)[None, :, :, None, None] * (pos[:, :, None] - t).abs()[:, None, None].float()
    seen = t <= pos[..., None]
    if c["prefix"]:
        seen = seen | (t < s["prefix"].long()[:, None, None])
    seen = seen & (t < lens[:, None, None])
    x = x.masked_fill(~seen[:, None, None], float("-inf"))
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = (p.view(B, n_kv, g * N, L) @ v).view(B, n_kv, g, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, n_q, d)
    tok = torch.arange(s["n_tokens"], device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), tok, right=True)
    return dict(out=o[seq, tok - cu[seq]].to(s["q"].dtype))


# ---------------------------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------------------------
def _config(s):
    from paper_2603_22910_b200 import binding
    c = s["case"]
    bf16 = c.get("dtype", "bf16") == "bf16"
    return binding.make_config(n_layers=1, n_q_heads=c.get("n_q", c.get("n_kv", 8)), n_kv_heads=c.get("n_kv", 8), head_dim=c.get("d", 128),
                               group_size=1, n_retained_heads=0, page_tokens=c.get("page", 16), max_batch=c.get("B", 1),
                               max_pages_per_seq=s.get("width", 1), n_pages=s.get("n_pages", 1),
                               dtype=binding.ECHOKV_BF16 if bf16 else binding.ECHOKV_FP32)


def _own(s):
    from paper_2603_22910_b200 import binding
    c = s["case"]
    if "cfg" not in s:                       # made once, as a program does
        s["cfg"] = _config(s)
        if c["op"] in ("append", "attn"):
            s["cache"] = binding.QuantCache(s["cfg"], c["fmt"], k_codes=s["kc"], v_codes=s["vc"], k_scales=s["ks"], v_scales=s["vs"],
                                            k_tail=s["kt"], v_tail=s["vt"])
        if c["op"] == "rotate":
            s["sections"] = _sections(c["rot"] // 2, c["axes"])
    if c["op"] == "plan":
        p = binding.plan_tokens(s["cfg"], s["table"], s["seq_lens"], s["new_lens"], s["free_pages"], s["free_count"],
                                s["n_tokens"], seq_slots=s["slots"])
        return dict(table=s["table"], cu=p.cu_tokens, positions=p.positions, seqs=p.token_seqs, rows=p.slot_map, lens=p.seq_lens,
                    count=p.free_count)
    if c["op"] == "rotate":
        q, k = binding.rotate(s["cfg"], s["q"], s["k"], s["pos"], c["theta"], sections=s["sections"], rot_dim=c["rot"],
                              interleaved=c["interleaved"], inverse=c["inverse"])
        return dict(q=q, k=k)
    cache = s["cache"]
    if c["op"] == "append":
        cache.append(s["k"], s["v"], s["rows"], s["seq"], s["cu"], seq_slots=s["slots"])
        return dict(k_codes=s["kc"], k_scales=s["ks"], k_tail=s["kt"], v_codes=s["vc"], v_scales=s["vs"], v_tail=s["vt"])
    out = cache.attention(s["q"], s["table"], s["lens"], cu_tokens=s["cu"], max_new=s["max_new"], seq_slots=s["slots"],
                          softcap=c["cap"], alibi_slopes=s["slopes"], prefix_lens=s["prefix"])
    return dict(out=out)


def run(state):
    if own:
        return _own(state)
    return {"plan": _plain_plan, "rotate": _plain_rotate, "append": _plain_append, "attn": _plain_attn}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------
# what cannot be done without, and the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "rotate":
        n = case["T"] * (case["n_q"] + case["n_kv"]) * case["d"]
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * n * e + 4 * case["T"] * case["axes"], "flops": 3 * n}
    before, new = _lengths(case)
    T, B, P = sum(new), case["B"], case["page"]
    if op == "plan":
        need = sum(-(-(b + n) // P) - -(-b // P) for b, n in zip(before, new))
        return {"bytes": 4 * (5 * B + 2) + 8 * need + 16 * T, "flops": 8 * (B + T)}
    e = 2 if case["dtype"] == "bf16" else 4
    D = case["n_kv"] * case["d"]
    if op == "append":
        full = sum((b % BLOCK + n) // BLOCK for b, n in zip(before, new))
        waited = sum(b % BLOCK for b, n in zip(before, new) if b % BLOCK + n >= BLOCK)
        left = sum(min(n, (b + n) % BLOCK) for b, n in zip(before, new))
        return {"bytes": 2 * (T * D * e + waited * D * e + full * (BLOCK * D + 4 * case["n_kv"]) + left * D * e) + 12 * T,
                "flops": 2 * 3 * full * BLOCK * D}
    after = [b + n for b, n in zip(before, new)]
    codes = sum(a // BLOCK * BLOCK * D + a % BLOCK * D * e + a // BLOCK * 4 * case["n_kv"] for a in after)
    pairs = sum(n * a - n * (n - 1) // 2 for a, n in zip(after, new))
    return {"bytes": 2 * codes + T * case["n_q"] * case["d"] * 2 * e, "flops": 4 * pairs * case["n_q"] * case["d"]}


def _exact_scales(case, s):
    before, new = _lengths(case)
    rows, cu, slots = s["rows"].cpu().numpy(), s["cu"].cpu().numpy(), s["slots"].cpu().numpy()
    out = dict(k_codes=None, k_scales=None, k_tail=None, v_codes=None, v_scales=None, v_tail=None)
    for n in "kv":
        x, tail = s[n].abs().double(), s[n + "t"].abs().double()
        scales = s[n + "s"].double().cpu().numpy().copy()
        for b in range(case["B"]):
            o = before[b] % BLOCK
            line = torch.cat([tail[slots[b], :, :o].transpose(0, 1), x[cu[b]:cu[b + 1]]])
            m = len(line) // BLOCK
            if m:
                top = line[: m * BLOCK].view(m, BLOCK, case["n_kv"], case["d"]).amax(dim=(1, 3)).cpu().numpy() / QMAX[case["fmt"]]
                row = rows[cu[b] + np.arange(1, m + 1) * BLOCK - 1 - o]
                scales[row // case["page"], :, row % case["page"] // BLOCK] = np.maximum(top, 2.0 ** -100)
        out[n + "_scales"] = scales
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "plan":
        return None                                      # whole numbers
    if op == "append":
        return _exact_scales(case, s)                    # codes and copies have no value in more bits than they are held in
    if op == "rotate":
        half, rot = case["rot"] // 2, case["rot"]
        axis = _axis_of(case)
        pos = s["pos"].cpu().numpy().astype(np.float64)
        z = np.exp((-1j if case["inverse"] else 1j) * pos[axis].T * case["theta"] ** (-np.arange(half) / half))[:, None, :]

        def turned(x):
            x = x.double().cpu().numpy()
            y = (x[..., :half] + 1j * x[..., half:rot]) * z
            return np.concatenate([y.real, y.imag, x[..., rot:]], -1)
        return dict(q=turned(s["q"]), k=turned(s["k"]))
    n_q, n_kv, d, P = case["n_q"], case["n_kv"], case["d"], case["page"]
    table, cu, slots, lens = (s[n].cpu().tolist() for n in ("table", "cu", "slots", "lens"))
    prefix = s["prefix"].cpu().tolist() if case["prefix"] else [0] * case["B"]
    out = torch.empty(s["n_tokens"], n_q, d, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        n, m = lens[b], lens[b] // BLOCK * BLOCK
        pages = torch.tensor(table[slots[b]][: -(-n // P)], device="cuda")
        at = torch.arange(cu[b + 1] - cu[b], device="cuda", dtype=torch.float64)[:, None] + (n - (cu[b + 1] - cu[b]))
        t = torch.arange(n, device="cuda", dtype=torch.float64)
        hidden = (t > at) & (t >= prefix[b])
        for h in range(n_kv):
            kv = []
            for codes, scales, tail in ((s["kc"], s["ks"], s["kt"]), (s["vc"], s["vs"], s["vt"])):
                x = codes.view(torch.uint8)[pages, h].view(codes.dtype).float().double().view(-1, BLOCK, d) * scales[pages, h].double().view(-1, 1, 1)
                kv.append(torch.cat([x.view(-1, d)[:m], tail[slots[b], h].double()[: n - m]]))
            for j in range(h * n_q // n_kv, (h + 1) * n_q // n_kv):
                x = s["q"][cu[b]:cu[b + 1], j].double() @ kv[0].T / math.sqrt(d)
                if case["cap"]:
                    x = torch.tanh(x / case["cap"]) * case["cap"]
                if case["alibi"]:
                    x -= float(s["slopes"][j]) * (at - t).abs()
                out[cu[b]:cu[b + 1], j] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ kv[1]
    return dict(out=out.cpu().numpy())
