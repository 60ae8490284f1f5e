"""Cases of the chunked-prefill operators: block tables built on the GPU, rotary positions fused with the append into
the paged pool, and attention of a chunk of new tokens over that pool, with the score caps, biases and masks it takes.

`run` makes the calls a program makes of these operators (`own` true), or computes the same in elementary torch
operations (`own` false).  Pools and tables are laid out as everywhere in this package: kv_pool[slab][block][K|V]
[kv head][slot][dim] in bf16, blocks of 16 tokens, request r's blocks in kv_indices[kv_indptr[r]:kv_indptr[r + 1]].
"""
import math
import random

import torch

own = False

BS = 16                      # tokens per pool block
DEV = "cuda:0"
SCORES = 1 << 30             # scores the plain forms hold at a time
VALUES = 1 << 28             # and values of K (or V) in 32 bits

# --------------------------------------------------------------------------- cases
_LENS = dict(chunks=0, chunk_lo=1, chunk_hi=1)
_ATTN = dict(kind="attn", heads=32, kv_heads=8, dim=128, layers=1, q_scale=1.0, softcap=0.0, window=0, alibi=False, docs=0,
             prefix=False, **_LENS)
_ROPE = dict(kind="rope", heads=32, kv_heads=8, dim=128, rot=128, axes=1, adjacent=False, cycled=False, dtype="bf16", pad=0, far=4096)
_STEP = {**_ATTN, **_ROPE, "kind": "step"}


def listed():
    return [
        # one decode step of the 64-request batch: a new token each, hardly a block to hand out
        dict(name="tables_decode_64", kind="tables", batch=64, ctx_lo=512, ctx_hi=2048, new_lo=1, new_hi=1, lens=1, **_LENS),
        # the 512-request batch: most requests verify a few drafted tokens, sixteen bring a piece of their prompt
        dict(name="tables_mixed_512", kind="tables", batch=512, ctx_lo=128, ctx_hi=4096, new_lo=1, new_hi=5, lens=2,
             chunks=16, chunk_lo=100, chunk_hi=1000),
        # the rows of one verification round (64 requests, five rows each), written to the pool one by one
        dict(_ROPE, name="rope_round_320", rows=320, lens=3),
        # a prompt with images and video: three position axes, and the captured launch is wider than the batch
        dict(_ROPE, name="rope_axes_8192", rows=8192, axes=3, pad=192, far=100000, lens=4),
        # small heads, part of each head rotated, neighbouring pairs, axes in turn, 32-bit projections
        dict(_ROPE, name="rope_partial_d64", rows=1777, heads=8, kv_heads=2, dim=64, rot=48, axes=3, adjacent=True, cycled=True,
             dtype="fp32", far=1000000, lens=5),
        # single tokens: the decode step of 64 requests, four layers under one plan
        dict(_ATTN, name="attn_token_64", batch=64, ctx_lo=512, ctx_hi=2048, new_lo=1, new_hi=1, layers=4, lens=6),
        # single tokens over few long contexts: every request has to be split over many SMs
        dict(_ATTN, name="attn_token_long", batch=5, ctx_lo=30000, ctx_hi=120000, new_lo=1, new_hi=1, layers=2, lens=7),
        # a whole prompt at once, nothing cached
        dict(_ATTN, name="attn_prompt_8192", batch=1, ctx_lo=0, ctx_hi=0, new_lo=8192, new_hi=8192, lens=8),
        # a chunk of a long prompt over what is cached already, odd sizes
        dict(_ATTN, name="attn_chunk_long", batch=1, ctx_lo=62221, ctx_hi=62221, new_lo=2047, new_hi=2047, lens=9),
        # scores capped by a tanh, keys within a window: four prompts of odd length
        dict(_ATTN, name="attn_cap_window", batch=4, ctx_lo=300, ctx_hi=3000, new_lo=1500, new_hi=2500, q_scale=6.0, softcap=30.0,
             window=1024, lens=10),
        # packed documents with a bias on distance, a prefix that sees itself both ways, small heads
        dict(_ATTN, name="attn_docs_bias_d64", heads=12, kv_heads=4, dim=64, batch=3, ctx_lo=100, ctx_hi=1000, new_lo=1000,
             new_hi=4000, alibi=True, docs=700, prefix=True, lens=11),
        # a serving step that mixes decoding requests with pieces of prompts: tables, plan, then append and attention per layer
        dict(_STEP, name="step_mixed_128", batch=128, ctx_lo=1024, ctx_hi=8192, new_lo=1, new_hi=1, chunks=6,
             chunk_lo=150, chunk_hi=700, layers=4, pad=128, lens=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tables", "rope", "rope", "attn", "attn", "attn", "attn", "step"])
    lens = rng.randrange(1, 1 << 20)
    if kind == "tables":
        hi = _log_int(rng, 16, 32768)
        return dict(kind=kind, batch=_log_int(rng, 1, 512), ctx_lo=0, ctx_hi=hi, new_lo=0, new_hi=rng.randint(1, 9),
                    chunks=rng.randint(0, 3), chunk_lo=10, chunk_hi=_log_int(rng, 11, 2000), lens=lens)
    heads, kv_heads = rng.choice([(32, 8), (8, 2), (8, 8), (40, 8), (28, 4), (12, 4), (24, 1), (5, 5)])
    dim = rng.choice([64, 128])
    if kind == "rope":
        rot = 2 * rng.randint(3, dim // 2)
        axes = rng.randint(1, 4)
        return dict(_ROPE, heads=heads, kv_heads=kv_heads, dim=dim, rows=_log_int(rng, 1, 8192), rot=rot, axes=axes,
                    adjacent=rng.random() < 0.5, cycled=rng.random() < 0.5, dtype=rng.choice(["bf16", "fp32"]),
                    pad=rng.choice([0, 0, 7]), far=_log_int(rng, 10, 1000000), lens=lens)
    c = dict(_ATTN, heads=heads, kv_heads=kv_heads, dim=dim, lens=lens, layers=rng.randint(1, 2))
    if kind == "step":
        return dict(_STEP, heads=heads, kv_heads=kv_heads, dim=dim, rot=2 * rng.randint(8, dim // 2), lens=lens, axes=1,
                    pad=rng.randint(0, 50), batch=_log_int(rng, 2, 64), ctx_lo=0, ctx_hi=_log_int(rng, 100, 8000), new_lo=0,
                    new_hi=rng.randint(1, 3), chunks=rng.randint(1, 2), chunk_lo=5, chunk_hi=_log_int(rng, 50, 1000), layers=2)
    shape = rng.choice(["token", "few", "chunk", "prompts"])
    if shape == "token":
        c.update(batch=_log_int(rng, 1, 128), ctx_lo=0, ctx_hi=_log_int(rng, 100, 16000), new_lo=1, new_hi=1)
    elif shape == "few":
        c.update(batch=_log_int(rng, 1, 64), ctx_lo=10, ctx_hi=_log_int(rng, 100, 8000), new_lo=0, new_hi=rng.randint(2, 40),
                 chunks=1, chunk_lo=1, chunk_hi=9)
    elif shape == "chunk":
        ctx, new = _log_int(rng, 1000, 40000), _log_int(rng, 100, 2000)
        c.update(batch=1, ctx_lo=ctx, ctx_hi=ctx, new_lo=new, new_hi=new)
    else:
        c.update(batch=rng.randint(1, 4), ctx_lo=0, ctx_hi=rng.choice([0, 500]), new_lo=10, new_hi=_log_int(rng, 100, 4000))
    extra = rng.choice(["none", "none", "cap", "window", "bias", "docs", "prefix", "all"])
    if extra in ("cap", "all"):
        c.update(softcap=rng.choice([15.0, 30.0, 50.0]), q_scale=rng.choice([1.0, 6.0]))
    if extra in ("window", "all"):
        c.update(window=_log_int(rng, 1, 2000))
    if extra in ("bias", "all"):
        c.update(alibi=True)
    if extra in ("docs", "all"):
        c.update(docs=_log_int(rng, 5, 1000))
    if extra in ("prefix", "all"):
        c.update(prefix=True)
    return c


# --------------------------------------------------------------------------- lengths
def _lengths(case):
    """Committed and new tokens of each request, from the case alone."""
    rng = random.Random(case["lens"])
    ctx = [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["batch"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    for r in rng.sample(range(case["batch"]), min(case["chunks"], case["batch"])):
        new[r] = rng.randint(case["chunk_lo"], case["chunk_hi"])
    return ctx, new


def _offsets(sizes):
    out = [0]
    for s in sizes:
        out.append(out[-1] + s)
    return out


def _blocks(tokens):
    return (tokens + BS - 1) // BS


def _doc_starts(case, ctx, new):
    """Position at which each new row's document starts (packed documents), as one list over the requests."""
    rng = random.Random(case["lens"] + 1)
    out = []
    for c, n in zip(ctx, new):
        start, left = max(0, c - rng.randint(0, case["docs"])), rng.randint(1, 2 * case["docs"])
        for i in range(n):
            if left == 0:
                start, left = c + i, rng.randint(1, 2 * case["docs"])
            left -= 1
            out.append(start)
    return out


def _prefixes(case, ctx, new):
    rng = random.Random(case["lens"] + 2)
    return [rng.randint(0, c + n) for c, n in zip(ctx, new)]


def _sections(case):
    """Rotated pairs of each position axis: equal shares, the first axis takes the rest."""
    pairs = case["rot"] // 2
    share = [pairs // case["axes"]] * case["axes"]
    share[0] += pairs - sum(share)
    return share


def _axis_of_pair(case):
    sections = _sections(case)
    if not case["cycled"]:
        return [a for a, s in enumerate(sections) for _ in range(s)]
    n = case["axes"]
    return [j % n if j % n > 0 and j // n < sections[j % n] else 0 for j in range(case["rot"] // 2)]


# --------------------------------------------------------------------------- inputs
def _normal(gen, *shape, scale=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, scale, generator=gen).to(dtype)


def _on_gpu(values, dtype):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _prepare_tables(case, gen):
    """Blocks the requests hold, one row each, and the list of free blocks."""
    ctx, new = _lengths(case)
    rng = random.Random(case["lens"] + 3)
    need = [_blocks(c + n) for c, n in zip(ctx, new)]
    held_n = [_blocks(c) + (rng.randint(0, 2) if rng.random() < 0.25 else 0) for c in ctx]    # some kept blocks of rejected drafts
    width = max(max(need), max(held_n)) + 4
    took = sum(max(0, a - b) for a, b in zip(need, held_n))
    total = sum(held_n) + took + 64
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    held = torch.full((len(ctx), width), -1, dtype=torch.int32, device=DEV)
    col = torch.arange(width, device=DEV)[None, :]
    start = _on_gpu(_offsets(held_n), torch.int64)
    n_held = _on_gpu(held_n, torch.int32)
    mine = col < n_held[:, None]
    held[mine] = ids[(start[:-1, None] + col)[mine]]
    rows, pad = sum(new), case.get("pad", 0)
    s = dict(ctx_len=_on_gpu(ctx, torch.int32), new_len=_on_gpu(new, torch.int32), held=held, n_held=n_held,
             free_blocks=ids[sum(held_n):].contiguous(), free_begin=_on_gpu([3], torch.int64), num_blocks=total,
             max_rows=max(1, rows + pad), max_entries=max(1, sum(need)))
    i32 = dict(dtype=torch.int32, device=DEV)
    i64 = dict(dtype=torch.int64, device=DEV)
    s.update(kv_indptr=torch.zeros(len(ctx) + 1, **i64), kv_indices=torch.full((s["max_entries"] + 5,), -7, **i32),
             q_indptr=torch.zeros(len(ctx) + 1, **i64), slot_map=torch.zeros(s["max_rows"], **i64),
             positions=torch.zeros(s["max_rows"], **i32), row_req=torch.zeros(s["max_rows"], **i32),
             n_held_new=torch.zeros(len(ctx), **i32), free_end=torch.zeros(1, **i64))
    return s


def _prepare_rope(case, gen):
    rows, h, hkv, d = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    total = rows + case["pad"]
    dtype = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    blocks = _blocks(rows + 5) + 9
    ids = torch.randperm(blocks, generator=gen, device=DEV)
    at = torch.arange(rows, device=DEV) + 5                               # the rows begin inside a block
    slots = torch.full((total,), -1, dtype=torch.int64, device=DEV)
    slots[:rows] = ids[at // BS] * BS + at % BS
    qkv = _normal(gen, total, (h + 2 * hkv) * d, dtype=dtype)            # as one projection leaves them
    positions = torch.randint(0, case["far"], (case["axes"], total), generator=gen, device=DEV, dtype=torch.int32)
    return dict(qkv=qkv, positions=positions, slot_map=slots, num_blocks=blocks, inv_freq=_inv_freq(case),
                pool=_normal(gen, 1, blocks, 2, hkv, BS, d), q_out=_normal(gen, total, h, d), pair_axis=_on_gpu(_axis_of_pair(case), torch.int64))


def _inv_freq(case):
    j = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
    return (1e6 ** (-2.0 * j / case["rot"])).float()


def _groups(ctx, new, heads, width):
    """Requests of like length together, with the largest row slice whose scores the plain form may hold."""
    order = sorted((r for r in range(len(ctx)) if new[r]), key=lambda r: (new[r], ctx[r]))
    out = []
    for r in order:
        cells = (len(out[-1]["reqs"]) + 1) * max(out[-1]["keys"], ctx[r] + new[r]) if out else 0
        if not out or cells * heads * new[r] > SCORES or cells * width > VALUES or new[r] > 2 * out[-1]["low"] + 8:
            out.append(dict(reqs=[], keys=0, rows=0, low=new[r]))
        g = out[-1]
        g["reqs"].append(r)
        g["keys"] = max(g["keys"], ctx[r] + new[r])
        g["rows"] = max(g["rows"], new[r])
    for g in out:
        g["slice"] = max(1, min(g["rows"], SCORES // (heads * g["keys"] * len(g["reqs"]))))
        g["reqs"] = _on_gpu(g["reqs"], torch.int64)
    return out


def _prepare_attn(case, gen):
    ctx, new = _lengths(case)
    h, hkv, d, layers = case["heads"], case["kv_heads"], case["dim"], case["layers"]
    need = [_blocks(c + n) for c, n in zip(ctx, new)]
    live, rows = max(1, sum(need)), max(1, sum(new))
    num_blocks = live + max(4, live // 8)
    s = dict(num_blocks=num_blocks, max_rows=rows,
             kv_indices=torch.randperm(num_blocks, generator=gen, device=DEV)[:live].to(torch.int32),
             kv_indptr=_on_gpu(_offsets(need), torch.int64), q_indptr=_on_gpu(_offsets(new), torch.int64),
             ctx_len=_on_gpu(ctx, torch.int32), pool=torch.empty(layers, num_blocks, 2, hkv, BS, d, dtype=torch.bfloat16, device=DEV),
             q=_normal(gen, layers, rows, h, d, scale=case["q_scale"]))
    for layer in range(layers):
        s["pool"][layer] = _normal(gen, num_blocks, 2, hkv, BS, d)
    s.update(_score_options(case, ctx, new))
    s.update(o=torch.zeros(layers, rows, h, d, dtype=torch.bfloat16, device=DEV),
             lse=torch.zeros(layers, rows, h, dtype=torch.float32, device=DEV), groups=_groups(ctx, new, h, hkv * d))
    return s


def _score_options(case, ctx, new):
    s = dict(prefix_len=None, row_first=None, slopes=None)
    if case["prefix"]:
        s["prefix_len"] = _on_gpu(_prefixes(case, ctx, new), torch.int32)
    if case["docs"]:
        s["row_first"] = _on_gpu(_doc_starts(case, ctx, new) or [0], torch.int32)
    if case["alibi"]:
        s["slopes"] = torch.pow(2.0, -8.0 * torch.arange(1, case["heads"] + 1, dtype=torch.float64, device=DEV) / case["heads"]).float()
    return s


def _prepare_step(case, gen):
    ctx, new = _lengths(case)
    h, hkv, d, layers = case["heads"], case["kv_heads"], case["dim"], case["layers"]
    s = _prepare_tables(case, gen)
    s["pool"] = torch.empty(layers, s["num_blocks"], 2, hkv, BS, d, dtype=torch.bfloat16, device=DEV)
    for layer in range(layers):
        s["pool"][layer] = _normal(gen, s["num_blocks"], 2, hkv, BS, d)
    s.update(qkv=_normal(gen, layers, s["max_rows"], (h + 2 * hkv) * d), inv_freq=_inv_freq(case), pair_axis=_on_gpu(_axis_of_pair(case), torch.int64),
             q_out=torch.zeros(layers, s["max_rows"], h, d, dtype=torch.bfloat16, device=DEV),
             o=torch.zeros(layers, s["max_rows"], h, d, dtype=torch.bfloat16, device=DEV),
             lse=torch.zeros(layers, s["max_rows"], h, dtype=torch.float32, device=DEV), groups=_groups(ctx, new, h, hkv * d))
    s.update(_score_options(case, ctx, new))
    return s


_handles = {}


def _handle(case, s, layers):
    """The worker's context and plan buffer: made once for its sizes, kept as long as the worker lives."""
    batch = case.get("batch", 1)
    h, hkv, d = case.get("heads", 32), case.get("kv_heads", 8), case.get("dim", 128)
    key = (h, hkv, d, layers, s["num_blocks"], batch)
    if key not in _handles:
        import paper_2609_29364_b200 as nsd

        _handles.clear()
        _handles[key] = nsd.VerifyContext(num_layers=layers, num_q_heads=h, num_kv_heads=hkv, head_dim=d, block_size=BS,
                                          num_blocks=s["num_blocks"], region_b_begin=0, max_batch=batch, max_gamma=1, vocab_size=2,
                                          max_table_entries=1)
    return _handles[key]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"tables": _prepare_tables, "rope": _prepare_rope, "attn": _prepare_attn, "step": _prepare_step}[case["kind"]](case, gen)
    s["case"] = case
    if own:
        s["nsd"] = _handle(case, s, case.get("layers", 1))
        if case["kind"] in ("attn", "step"):
            s["plan"] = torch.empty(s["nsd"].nsd_chunk_plan_bytes(s["max_rows"]), dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------- one pass
def run(s):
    return {"tables": _run_tables, "rope": _run_rope, "attn": _run_attn, "step": _run_step}[s["case"]["kind"]](s)


def _tables(s):
    if own:
        s["nsd"].nsd_block_tables(s["ctx_len"], s["new_len"], s["held"], s["n_held"], s["free_blocks"], s["free_begin"], s["kv_indptr"],
                                  s["kv_indices"], s["q_indptr"], s["slot_map"], s["positions"], s["row_req"], s["n_held_new"], s["free_end"])
    else:
        _plain_tables(s)


def _run_tables(s):
    _tables(s)
    return {k: s[k] for k in ("kv_indptr", "kv_indices", "q_indptr", "slot_map", "positions", "row_req", "held", "n_held_new", "free_end")}


def _rope(s, layer, qkv, q_out, positions):
    c = s["case"]
    nq, nk = c["heads"] * c["dim"], c["kv_heads"] * c["dim"]
    q, k, v = qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:]
    if own:
        s["nsd"].nsd_rope_append(s["pool"], layer, q, k, v, q_out, positions, _sections(c), s["inv_freq"], s["slot_map"],
                                 adjacent=c["adjacent"], cycled=c["cycled"])
    else:
        _plain_rope(s, layer, q, k, v, q_out, positions)


def _run_rope(s):
    _rope(s, 0, s["qkv"], s["q_out"], s["positions"])
    return {"q_out": s["q_out"], "pool": s["pool"]}


def _plan(s):
    s["nsd"].nsd_chunk_plan(s["plan"], s["max_rows"], s["q_indptr"], s["ctx_len"], s["kv_indptr"], window=s["case"]["window"],
                            prefix_len=s["prefix_len"], row_first=s["row_first"])


def _attn(s, layer, q, o, lse):
    if own:
        s["nsd"].nsd_chunk_attn(s["plan"], s["max_rows"], s["pool"], q, o, lse, s["kv_indices"], layer=layer,
                                softcap=s["case"]["softcap"], alibi_slopes=s["slopes"])
    else:
        for g in s["groups"]:
            for first in range(0, g["rows"], g["slice"]):
                _plain_attn(s, layer, q, o, lse, g, first)


def _run_attn(s):
    if own:
        _plan(s)
    for layer in range(s["case"]["layers"]):
        _attn(s, layer, s["q"][layer], s["o"][layer], s["lse"][layer])
    return {"o": s["o"], "lse": s["lse"]}


def _run_step(s):
    _tables(s)
    if own:
        _plan(s)
    for layer in range(s["case"]["layers"]):
        _rope(s, layer, s["qkv"][layer], s["q_out"][layer], s["positions"][None])
        _attn(s, layer, s["q_out"][layer], s["o"][layer], s["lse"][layer])
    return {k: s[k] for k in ("kv_indptr", "kv_indices", "slot_map", "q_out", "pool", "o", "lse")}


# --------------------------------------------------------------------------- plain forms
def _plain_tables(s):
    """Prefix sums and searches; entries and rows past the last request keep what they hold, padding rows get -1."""
    ctx, new, n_held = s["ctx_len"].long(), s["new_len"].long(), s["n_held"].long()
    need = (ctx + new + BS - 1) // BS
    take = (need - n_held).clamp(min=0)
    zero = torch.zeros(1, dtype=torch.int64, device=ctx.device)
    kv_indptr = torch.cat([zero, need.cumsum(0)])
    q_indptr = torch.cat([zero, new.cumsum(0)])
    take_at = take.cumsum(0) - take
    # blocks from the free list behind those a request holds
    col = torch.arange(s["held"].shape[1], device=ctx.device)[None, :]
    fresh = (col >= n_held[:, None]) & (col < need[:, None])
    at = s["free_begin"] + take_at[:, None] + (col - n_held[:, None])
    held = torch.where(fresh, s["free_blocks"][at.clamp(0, s["free_blocks"].numel() - 1)], s["held"])
    s["held"].copy_(held)
    s["n_held_new"].copy_(n_held + take)
    s["free_end"].copy_(s["free_begin"] + take.sum())
    # the tables, end to end
    e = torch.arange(s["kv_indices"].numel(), device=ctx.device)
    r = torch.searchsorted(kv_indptr, e, right=True) - 1
    inside = e < kv_indptr[-1]
    r = r.clamp(0, ctx.numel() - 1)
    s["kv_indices"].copy_(torch.where(inside, held[r, (e - kv_indptr[r]).clamp(0, held.shape[1] - 1)], s["kv_indices"]))
    s["kv_indptr"].copy_(kv_indptr)
    s["q_indptr"].copy_(q_indptr)
    # the rows
    i = torch.arange(s["max_rows"], device=ctx.device)
    inside = i < q_indptr[-1]
    r = (torch.searchsorted(q_indptr, i, right=True) - 1).clamp(0, ctx.numel() - 1)
    pos = ctx[r] + i - q_indptr[r]
    slot = held[r, (pos // BS).clamp(0, held.shape[1] - 1)].long() * BS + pos % BS
    s["slot_map"].copy_(torch.where(inside, slot, -1))
    s["positions"].copy_(torch.where(inside, pos, 0))
    s["row_req"].copy_(torch.where(inside, r, -1))


def _plain_rope(s, layer, q, k, v, q_out, positions):
    """Angles in 64 bits, the rotation in 32; padding rows (slot -1) are left alone."""
    c = s["case"]
    d, half = c["dim"], c["rot"] // 2
    angle = positions[s["pair_axis"]].t().double() * s["inv_freq"].double()               # [rows][pairs]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def rotate(x):
        x = x.reshape(x.shape[0], -1, d).float()
        if c["adjacent"]:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        return torch.cat([turned, x[..., 2 * half:]], dim=-1).to(torch.bfloat16)

    real = (s["slot_map"] >= 0)
    q_out.copy_(torch.where(real[:, None, None], rotate(q), q_out))
    pool = s["pool"][layer]
    slot = s["slot_map"].clamp(min=0)
    block, at = slot // BS, slot % BS
    # a padding row stores what its place holds already: the last real row's, at the last real row's place
    last = torch.where(real, torch.arange(real.numel(), device=real.device), 0).cummax(0).values
    block, at = block[last], at[last]
    pool[block, 0, :, at] = rotate(k)[last]
    pool[block, 1, :, at] = v.reshape(v.shape[0], -1, d).to(torch.bfloat16)[last]


def _plain_attn(s, layer, q, o, lse, g, first):
    """Scores, weights and sums of one slice of the rows of a group of requests, in 32 bits."""
    c, reqs = s["case"], g["reqs"]
    h, hkv, d = c["heads"], c["kv_heads"], c["dim"]
    n, keys = min(g["slice"], g["rows"] - first), g["keys"]
    start, ctx = s["q_indptr"][reqs], s["ctx_len"][reqs].long()
    count = s["q_indptr"][reqs + 1] - start
    i = first + torch.arange(n, device=q.device)[None, :]
    real = i < count[:, None]                                                             # [requests][rows]
    row = torch.where(real, start[:, None] + i, start[:, None])
    j = torch.arange(keys, device=q.device)
    at = torch.arange(_blocks(keys), device=q.device)[None, :]
    inside = at < (s["kv_indptr"][reqs + 1] - s["kv_indptr"][reqs])[:, None]
    block = s["kv_indices"][torch.where(inside, s["kv_indptr"][reqs][:, None] + at, s["kv_indptr"][reqs][:, None])].long()
    kv = s["pool"][layer][block].float()                                                  # [requests][blocks][2][hkv][16][d]
    kv = kv.permute(2, 0, 3, 1, 4, 5).reshape(2, reqs.numel(), hkv, -1, d)[..., :keys, :]
    qq = q[row].float().reshape(reqs.numel(), n, hkv, h // hkv, d).permute(0, 2, 3, 1, 4).reshape(reqs.numel(), hkv, -1, d)
    score = (qq @ kv[0].transpose(-1, -2)).reshape(reqs.numel(), hkv, h // hkv, n, keys) * (1.0 / math.sqrt(d))
    pos = ctx[:, None] + i
    if c["softcap"]:
        score = torch.tanh(score / c["softcap"]) * c["softcap"]
    if s["slopes"] is not None:
        score = score + s["slopes"].reshape(1, hkv, h // hkv, 1, 1) * (j - pos[..., None]).float()[:, None, None]
    stop, begin = pos + 1, torch.zeros_like(pos)
    if s["prefix_len"] is not None:
        stop = torch.maximum(stop, torch.minimum(s["prefix_len"][reqs].long(), ctx + count)[:, None])
    if c["window"]:
        begin = (pos + 1 - c["window"]).clamp(min=0)
    if s["row_first"] is not None:
        begin = torch.maximum(begin, s["row_first"][row].long())
    seen = ((j >= begin[..., None]) & (j < stop[..., None]))[:, None, None]
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = weight.sum(-1, keepdim=True)
    value = torch.where((j < (ctx + count)[:, None])[:, None, :, None], kv[1], 0.0)
    out = (weight.reshape(reqs.numel(), hkv, -1, keys) @ value).reshape(weight.shape[:-1] + (d,)) / torch.where(total > 0, total, 1.0)
    out = out.permute(0, 3, 1, 2, 4).reshape(reqs.numel(), n, h, d)
    log_sum = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(reqs.numel(), n, h)
    o[row[real]] = out[real].to(torch.bfloat16)
    lse[row[real]] = log_sum[real]


# --------------------------------------------------------------------------- work
def _row_bytes(case):
    size = 4 if case["dtype"] == "fp32" else 2
    h, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    return (h + 2 * hkv) * d * (size + 2) + 8 + 4 * case["axes"]


def _visible(case, ctx, new):
    """(row, key) pairs that take part, and the keys of each request that some row sees."""
    first = _doc_starts(case, ctx, new) if case["docs"] else None
    prefix = _prefixes(case, ctx, new) if case["prefix"] else [0] * len(ctx)
    pairs, keys, row = 0, 0, 0
    for c, n, p in zip(ctx, new, prefix):
        low, high, p = c + n, 0, min(p, c + n)
        if not (first or case["window"] or case["prefix"]):
            pairs += n * c + n * (n + 1) // 2
            low, high = 0, c + n if n else 0
        else:
            for i in range(n):
                begin = max(0, c + i + 1 - case["window"]) if case["window"] else 0
                begin = max(begin, first[row + i]) if first else begin
                stop = max(c + i + 1, p)
                if stop > begin:
                    pairs += stop - begin
                    low, high = min(low, begin), max(high, stop)
        keys += max(0, high - low)
        row += n
    return pairs, keys


def work(case):
    if case["kind"] == "rope":
        rows = case["rows"]
        return {"bytes": rows * _row_bytes(case) + 8 * case["pad"], "flops": 3 * rows * case["rot"] * (case["heads"] + case["kv_heads"])}
    ctx, new = _lengths(case)
    rows, blocks = sum(new), sum(_blocks(c + n) for c, n in zip(ctx, new))
    # lengths, held blocks and free list in; offsets, tables, slots, positions and owners out
    table_bytes = len(ctx) * (4 * 3 + 8 * 2 + 4) + 8 * blocks + 16 * rows
    if case["kind"] == "tables":
        return {"bytes": table_bytes, "flops": rows + blocks}
    pairs, keys = _visible(case, ctx, new)
    h, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    layer_bytes = keys * 2 * hkv * d * 2 + rows * h * (2 * d * 2 + 4) + 4 * blocks
    flops = 4 * d * h * pairs
    if case["kind"] == "step":
        layer_bytes += rows * _row_bytes(case)
        flops += 3 * rows * case["rot"] * (h + hkv)
    else:
        table_bytes = 0
    return {"bytes": case["layers"] * layer_bytes + table_bytes, "flops": case["layers"] * flops}


# --------------------------------------------------------------------------- 64 bits, from the definitions
def _exact_tables(case, s):
    """Request by request, on the host."""
    ctx, new = _lengths(case)
    held, n_held, free = s["held"].tolist(), s["n_held"].tolist(), s["free_blocks"].tolist()
    nxt = int(s["free_begin"])
    indices, slots, where, owner = [], [], [], []
    for r, (c, n) in enumerate(zip(ctx, new)):
        need = -(-(c + n) // BS)
        while n_held[r] < need:
            held[r][n_held[r]] = free[nxt]
            nxt, n_held[r] = nxt + 1, n_held[r] + 1
        indices += held[r][:need]
        for t in range(c, c + n):
            slots.append(held[r][t // BS] * BS + t % BS)
            where.append(t)
            owner.append(r)
    spare = s["kv_indices"].numel() - len(indices)
    pad = s["max_rows"] - len(slots)
    t = lambda v, dt: torch.tensor(v, dtype=dt, device=DEV)  # noqa: E731
    return {"kv_indptr": t(_offsets([-(-(c + n) // BS) for c, n in zip(ctx, new)]), torch.int64), "kv_indices": t(indices + [-7] * spare, torch.int32),
            "q_indptr": t(_offsets(new), torch.int64), "slot_map": t(slots + [-1] * pad, torch.int64), "positions": t(where + [0] * pad, torch.int32),
            "row_req": t(owner + [-1] * pad, torch.int32), "held": t(held, torch.int32), "n_held_new": t(n_held, torch.int32), "free_end": t([nxt], torch.int64)}


def _exact_rope(case, qkv, positions, slots, inv_freq, pool, q_out):
    """Each pair as a complex number turned by its angle."""
    h, hkv, d, rot = case["heads"], case["kv_heads"], case["dim"], case["rot"]
    keep = slots >= 0
    x = qkv[keep].double().reshape(-1, h + 2 * hkv, d)
    axis = _axis_of_pair(case)
    theta = torch.stack([positions[axis[p]][keep].double() * float(inv_freq[p]) for p in range(rot // 2)], -1)
    first = torch.arange(0, rot, 2, device=DEV) if case["adjacent"] else torch.arange(rot // 2, device=DEV)
    second = first + (1 if case["adjacent"] else rot // 2)
    z = torch.complex(x[:, :h + hkv, first], x[:, :h + hkv, second]) * torch.polar(torch.ones_like(theta), theta)[:, None]
    x[:, :h + hkv, first], x[:, :h + hkv, second] = z.real, z.imag
    q_out, pool = q_out.double(), pool.double()
    q_out[keep] = x[:, :h]
    b, t = slots[keep] // BS, slots[keep] % BS
    pool[b, 0, :, t] = x[:, h:h + hkv]
    pool[b, 1, :, t] = x[:, h + hkv:]
    return q_out, pool


def _exact_attn(case, s, q, pool, indptr, indices):
    """Head by head and request by request, weights from exp(score - log-sum)."""
    ctx, new = _lengths(case)
    h, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    rows = q.shape[0]
    o = torch.zeros(rows, h, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(rows, h, dtype=torch.float64, device=DEV)
    docs = torch.tensor(_doc_starts(case, ctx, new), device=DEV) if case["docs"] else None
    prefix = _prefixes(case, ctx, new) if case["prefix"] else None
    at = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        total = c + n
        if not n:
            continue
        mine = indices[indptr[r]:indptr[r] + -(-total // BS)].long()
        kv = pool[mine].permute(1, 2, 0, 3, 4).reshape(2, hkv, -1, d)[:, :, :total].double()
        key = torch.arange(total, device=DEV)
        step = max(1, (1 << 28) // total)
        for a in range(0, n, step):
            m = min(step, n - a)
            p = c + a + torch.arange(m, device=DEV)
            far = p if prefix is None else p.clamp(min=prefix[r] - 1)
            hide = key[None] > far[:, None]
            if case["window"]:
                hide |= key[None] <= p[:, None] - case["window"]
            if docs is not None:
                hide |= key[None] < docs[at + a:at + a + m, None]
            for head in range(h):
                z = q[at + a:at + a + m, head].double() @ kv[0, head // (h // hkv)].t() / math.sqrt(d)
                if case["softcap"]:
                    z = case["softcap"] * torch.tanh(z / case["softcap"])
                if case["alibi"]:
                    z -= float(s["slopes"][head]) * (p[:, None] - key[None])
                z.masked_fill_(hide, float("-inf"))
                log_sum = torch.logsumexp(z, -1)
                lse[at + a:at + a + m, head] = log_sum
                z = torch.exp(z - log_sum[:, None])
                z.masked_fill_(hide, 0.0)
                o[at + a:at + a + m, head] = z @ kv[1, head // (h // hkv)]
        at += n
    return o, lse


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "tables":
        return _exact_tables(case, s)
    if kind == "rope":
        q_out, pool = _exact_rope(case, s["qkv"], s["positions"], s["slot_map"], s["inv_freq"], s["pool"][0], s["q_out"])
        return {"q_out": q_out, "pool": pool[None]}
    if kind == "attn":
        ctx, new = _lengths(case)
        indptr = _offsets([-(-(c + n) // BS) for c, n in zip(ctx, new)])
        both = [_exact_attn(case, s, s["q"][k], s["pool"][k], indptr, s["kv_indices"]) for k in range(case["layers"])]
        return {"o": torch.stack([b[0] for b in both]), "lse": torch.stack([b[1] for b in both])}
    t = _exact_tables(case, s)
    out = {k: t[k] for k in ("kv_indptr", "kv_indices", "slot_map")}
    made = []
    for k in range(case["layers"]):
        q, pool = _exact_rope(case, s["qkv"][k], t["positions"][None], t["slot_map"], s["inv_freq"], s["pool"][k], s["q_out"][k])
        # attention reads what the cache and the query buffer hold: values of 16 bits
        made.append((q, pool) + _exact_attn(case, s, q.to(torch.bfloat16), pool.to(torch.bfloat16), t["kv_indptr"].tolist(), t["kv_indices"]))
    out.update({k: torch.stack([m[i] for m in made]) for i, k in enumerate(("q_out", "pool", "o", "lse"))})
    return out
