"""Cases of two families of operators over the paged pool.

The 8-bit cache: K and V quantised as they are written (`append`), whole blocks parked in 8 bits and fetched back (`pack`,
`unpack`), and attention that reads the 8-bit blocks (`attn8`).  A row of one token and kv head is held as e4m3 codes and one
power of two, 2^e: e is the least integer from -126 on with max|x| <= 448 2^e, the codes are x 2^-e rounded to nearest even.
kv8[slab][block][K|V][kv head][slot][dim], scales[slab][block][kv head][K|V][slot] (the exponent plus 127).

Attention for a batch whose requests share long prefixes, each read once for the whole group (`prefix`).

`run` makes the calls a program makes of these operators (`own` true), or computes the same in elementary torch
operations (`own` false).  The 16-bit pool is kv_pool[slab][block][K|V][kv head][slot][dim] in bf16, blocks of 16 tokens,
request r's blocks in kv_indices[kv_indptr[r]:kv_indptr[r + 1]].
"""
import math
import random

import torch

own = False

BS = 16                      # tokens per pool block
DEV = "cuda:0"
SCORES = 1 << 29             # scores the plain forms hold at a time
VALUES = 1 << 28             # and values of K (or V) in 32 bits
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu

# --------------------------------------------------------------------------- cases
_SHAPE = dict(heads=32, kv_heads=8, dim=128, layers=1)
_APPEND = dict(_SHAPE, kind="append", rot=0, pad=0, dtype="bf16", far=4096)
_STORE = dict(_SHAPE, dtype="bf16")
_ATTN = dict(_SHAPE, kind="attn8", window=0)
_PREFIX = dict(_SHAPE, kind="prefix")


def listed():
    return [
        # the rows of one verification round (64 requests, five rows each): k and v come rotated, q is not touched
        dict(_APPEND, name="append_round_320", rows=320, lens=1),
        # a prompt: q and k turn, k and v are quantised; the captured launch is wider than the batch
        dict(_APPEND, name="append_prompt_8192", rows=8192, rot=128, pad=192, far=100000, lens=2),
        # one request leaves the worker: its blocks, scattered over the pool, are parked in 8 bits
        dict(_STORE, name="pack_request_67", kind="pack", blocks=67, layers=4, lens=3),
        # a bank is emptied: the blocks of some thirty requests of a thousand tokens
        dict(_STORE, name="pack_bank_2048", kind="pack", blocks=2048, layers=4, lens=4),
        # one request comes back
        dict(_STORE, name="unpack_request_67", kind="unpack", blocks=67, layers=4, lens=5),
        # a bank is filled
        dict(_STORE, name="unpack_bank_2048", kind="unpack", blocks=2048, layers=4, lens=6),
        # the decode step of 64 requests, four layers under one plan
        dict(_ATTN, name="attn8_token_64", batch=64, ctx_lo=512, ctx_hi=2048, new_lo=1, new_hi=1, layers=4, lens=7),
        # a verification round of 512 requests: an anchor and up to four drafted tokens each
        dict(_ATTN, name="attn8_verify_512", batch=512, ctx_lo=128, ctx_hi=4096, new_lo=3, new_hi=5, lens=8),
        # few long contexts: every request is split over many SMs
        dict(_ATTN, name="attn8_token_long", batch=5, ctx_lo=30000, ctx_hi=120000, new_lo=1, new_hi=1, layers=2, lens=9),
        # 64 requests decode behind one system prompt
        dict(_PREFIX, name="prefix_token_64", groups=1, members_lo=64, members_hi=64, shared_lo=4000, shared_hi=4000, own_lo=30,
             own_hi=700, new_lo=1, new_hi=1, layers=4, lens=10),
        # 256 requests verify drafted tokens behind a long document
        dict(_PREFIX, name="prefix_verify_256", groups=1, members_lo=256, members_hi=256, shared_lo=32777, shared_hi=32777, own_lo=100,
             own_hi=2000, new_lo=3, new_hi=5, lens=11),
        # samples of several prompts: groups of odd sizes, some of one request, small heads
        dict(_PREFIX, name="prefix_groups_d64", heads=16, kv_heads=4, dim=64, groups=12, members_lo=1, members_hi=24, shared_lo=50,
             shared_hi=6000, own_lo=0, own_hi=1500, new_lo=1, new_hi=4, lens=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "pack", "unpack", "attn8", "attn8", "attn8", "prefix", "prefix", "prefix"])
    lens = rng.randrange(1, 1 << 20)
    heads, kv_heads = rng.choice([(32, 8), (8, 2), (8, 8), (40, 8), (28, 4), (12, 4), (24, 1), (5, 5)])
    shape = dict(heads=heads, kv_heads=kv_heads, dim=rng.choice([64, 128]), lens=lens)
    if kind == "append":
        return {**_APPEND, **shape, "rows": _log_int(rng, 1, 8192), "rot": rng.choice([0, 2 * rng.randint(3, shape["dim"] // 2)]),
                "pad": rng.choice([0, 0, 7]), "dtype": rng.choice(["bf16", "fp32"]), "far": _log_int(rng, 10, 1000000)}
    if kind in ("pack", "unpack"):
        return {**_STORE, **shape, "kind": kind, "blocks": _log_int(rng, 1, 2000), "layers": rng.randint(1, 4)}
    shape["layers"] = rng.randint(1, 2)
    if kind == "attn8":
        c = {**_ATTN, **shape, "window": rng.choice([0, 0, 0, _log_int(rng, 1, 2000)])}
        how = rng.choice(["token", "verify", "verify", "few"])
        if how == "token":
            c.update(batch=_log_int(rng, 1, 128), ctx_lo=0, ctx_hi=_log_int(rng, 100, 16000), new_lo=1, new_hi=1)
        elif how == "verify":
            c.update(batch=_log_int(rng, 1, 256), ctx_lo=10, ctx_hi=_log_int(rng, 100, 6000), new_lo=0, new_hi=rng.randint(2, 9))
        else:
            c.update(batch=rng.randint(1, 4), ctx_lo=0, ctx_hi=_log_int(rng, 1000, 60000), new_lo=1, new_hi=_log_int(rng, 2, 40))
        return c
    many = rng.random() < 0.5
    return {**_PREFIX, **shape, "groups": 1 if many else rng.randint(2, 9), "members_lo": 1, "members_hi": _log_int(rng, 2, 200 if many else 24),
            "shared_lo": 0, "shared_hi": _log_int(rng, 30, 24000 if many else 6000), "own_lo": 0, "own_hi": _log_int(rng, 20, 1500),
            "new_lo": rng.randint(0, 1), "new_hi": rng.randint(1, 6)}


# --------------------------------------------------------------------------- lengths
def _offsets(sizes):
    out = [0]
    for s in sizes:
        out.append(out[-1] + s)
    return out


def _blocks(tokens):
    return (tokens + BS - 1) // BS


def _lengths(case):
    """Committed and new tokens of each request, from the case alone; for groups also their requests and shared lengths."""
    rng = random.Random(case["lens"])
    if case["kind"] == "attn8":
        ctx = [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["batch"])]
        new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
        return ctx, new, None, None
    members = [rng.randint(case["members_lo"], case["members_hi"]) for _ in range(case["groups"])]
    shared = [rng.randint(case["shared_lo"], case["shared_hi"]) for _ in range(case["groups"])]
    ctx = [p + rng.randint(case["own_lo"], case["own_hi"]) for m, p in zip(members, shared) for _ in range(m)]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in ctx]
    return ctx, new, members, shared


# --------------------------------------------------------------------------- inputs
def _normal(gen, *shape, scale=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, scale, generator=gen).to(dtype)


def _on_gpu(values, dtype):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _kv(gen, *shape, dtype=torch.bfloat16):
    """Rows of K and V as a model leaves them: tokens of unlike size, a few channels that stand out."""
    x = torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=gen)
    x *= torch.exp2(0.7 * torch.empty(shape[:-1] + (1,), dtype=torch.float32, device=DEV).normal_(generator=gen))
    x[..., ::29] *= 4.0
    return x.to(dtype)


def _exponent(top):
    """The least e >= -126 with top <= 448 2^e: 448 = 0.875 2^9, and frexp gives top = m 2^x with 0.5 <= m < 1."""
    m, x = torch.frexp(top)
    return torch.where(top > 0, x - 9 + (m > 0.875).to(x.dtype), -126).clamp(min=-126)


def _quantise(x):
    """Codes and exponents of rows of 32-bit values."""
    e = _exponent(x.abs().amax(-1))
    inverse = ((127 - e) << 23).view(torch.float32)                       # 2^-e, exactly
    return (x * inverse[..., None]).to(E4M3), e


def _values(codes, scales):
    """What 8-bit blocks [..][K|V][kv head][slot][dim] with scales [..][kv head][K|V][slot] stand for, in 32 bits."""
    return codes.float() * scales.float().transpose(-3, -2)[..., None]


def _prepare_append(case, gen):
    rows, h, hkv, d = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    total = rows + case["pad"]
    dtype = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    blocks = _blocks(rows + 5) + 9
    ids = torch.randperm(blocks, generator=gen, device=DEV)
    at = torch.arange(rows, device=DEV) + 5                               # the rows begin inside a block
    slots = torch.full((total,), -1, dtype=torch.int64, device=DEV)
    slots[:rows] = ids[at // BS] * BS + at % BS
    codes, e = _quantise(_kv(gen, 1, blocks, 2, hkv, BS, d).float())
    s = dict(kv=_kv(gen, total, 2 * hkv, d, dtype=dtype).reshape(total, -1), slot_map=slots, num_blocks=blocks, kv8=codes,
             scales=(e + 127).to(torch.uint8).transpose(-3, -2).contiguous().view(E8M0), q=None, q_out=None, positions=None, inv_freq=None)
    if case["rot"]:
        j = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
        s.update(q=_normal(gen, total, h * d, dtype=dtype), q_out=_normal(gen, total, h, d), inv_freq=(1e6 ** (-2.0 * j / case["rot"])).float(),
                 positions=torch.randint(0, case["far"], (1, total), generator=gen, device=DEV, dtype=torch.int32))
    return s


def _prepare_store(case, gen):
    """A pool of 16-bit blocks and one of 8-bit blocks, and pairs of a block here and one there."""
    n, hkv, d, layers = case["blocks"], case["kv_heads"], case["dim"], case["layers"]
    num_blocks = n + 5
    s = dict(num_blocks=num_blocks, src=torch.randperm(num_blocks, generator=gen, device=DEV)[:n].to(torch.int32),
             dst=torch.randperm(num_blocks, generator=gen, device=DEV)[:n].to(torch.int32),
             pool=torch.empty(layers, num_blocks, 2, hkv, BS, d, dtype=torch.bfloat16, device=DEV))
    s.update(_cache8(gen, layers, num_blocks, hkv, d))
    for layer in range(layers):
        s["pool"][layer] = _kv(gen, num_blocks, 2, hkv, BS, d)
    return s


def _cache8(gen, layers, num_blocks, hkv, d):
    kv8 = torch.empty(layers, num_blocks, 2, hkv, BS, d, dtype=E4M3, device=DEV)
    scales = torch.empty(layers, num_blocks, hkv, 2, BS, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 28) // (2 * hkv * BS * d))
    for layer in range(layers):
        for b in range(0, num_blocks, step):
            codes, e = _quantise(_kv(gen, min(step, num_blocks - b), 2, hkv, BS, d).float())
            kv8[layer, b:b + step] = codes
            scales[layer, b:b + step] = (e + 127).to(torch.uint8).transpose(-3, -2)
    return dict(kv8=kv8, scales=scales.view(E8M0))


def _prepare_attn(case, gen):
    ctx, new, members, shared = _lengths(case)
    h, hkv, d, layers = case["heads"], case["kv_heads"], case["dim"], case["layers"]
    need = [_blocks(c + n) for c, n in zip(ctx, new)]
    # the full blocks of a group's prefix are the same for its members; the rest of a table is the request's own
    common = [0] * len(ctx) if members is None else [p // BS for m, p in zip(members, shared) for _ in range(m)]
    group = list(range(len(ctx))) if members is None else [g for g, m in enumerate(members) for _ in range(m)]
    first = {}
    for r, g in enumerate(group):
        first.setdefault(g, r)
    live = sum(need) - sum(c for r, c in enumerate(common) if first[group[r]] != r)
    num_blocks = max(1, live) + max(4, live // 8)
    ids = torch.randperm(num_blocks, generator=gen, device=DEV).to(torch.int32)
    tables, at = [], 0
    for r, n in enumerate(need):
        if first[group[r]] == r:
            tables.append(ids[at:at + n])
            at += n
        else:
            tables.append(torch.cat([tables[first[group[r]]][:common[r]], ids[at:at + n - common[r]]]))
            at += n - common[r]
    rows = max(1, sum(new))
    s = dict(num_blocks=num_blocks, max_rows=rows, kv_indices=torch.cat(tables + [ids[:1]]), kv_indptr=_on_gpu(_offsets(need), torch.int64),
             q_indptr=_on_gpu(_offsets(new), torch.int64), ctx_len=_on_gpu(ctx, torch.int32), q=_normal(gen, layers, rows, h, d),
             o=torch.zeros(layers, rows, h, d, dtype=torch.bfloat16, device=DEV),
             lse=torch.zeros(layers, rows, h, dtype=torch.float32, device=DEV))
    if members is None:
        s.update(_cache8(gen, layers, num_blocks, hkv, d))
        s["slices"] = _slices(range(len(ctx)), ctx, new, [0] * len(ctx), h, hkv * d)
        return s
    s["pool"] = torch.empty(layers, num_blocks, 2, hkv, BS, d, dtype=torch.bfloat16, device=DEV)
    for layer in range(layers):
        s["pool"][layer] = _kv(gen, num_blocks, 2, hkv, BS, d)
    # a prefix that does not end with its block: every member keeps its own copy of that block's shared tokens
    for r, g in enumerate(group):
        if first[g] != r and shared[g] % BS:
            s["pool"][:, tables[r][common[r]].long(), :, :, :shared[g] % BS] = s["pool"][:, tables[first[g]][common[r]].long(), :, :, :shared[g] % BS]
    begin = _offsets(members)
    s.update(group_indptr=_on_gpu(begin, torch.int64), prefix_len=_on_gpu(shared, torch.int32),
             groups=[dict(rows=(sum(new[:a]), sum(new[:b])), shared=p, table=tables[a][:_blocks(p)].long(), slices=_slices(range(a, b), ctx, new, [p] * len(ctx), h, hkv * d))
                     for a, b, p in zip(begin, begin[1:], shared)])
    return s


def _slices(reqs, ctx, new, skip, heads, width):
    """Requests of like length together, as many as the plain form may hold scores and values of."""
    out = []
    for r in sorted((r for r in reqs if new[r]), key=lambda r: (new[r], ctx[r])):
        keys = ctx[r] + new[r] - skip[r]
        cells = (len(out[-1]["reqs"]) + 1) * max(out[-1]["keys"], keys) if out else 0
        if not out or cells * heads * new[r] > SCORES or cells * width > VALUES or new[r] > 2 * out[-1]["rows"] + 8:
            out.append(dict(reqs=[], keys=0, rows=0, skip=skip[r]))
        g = out[-1]
        g["reqs"].append(r)
        g["keys"], g["rows"] = max(g["keys"], keys), max(g["rows"], new[r])
    for g in out:
        g["reqs"] = _on_gpu(g["reqs"], torch.int64)
    return out


_handles = {}


def _handle(case, s):
    """The worker's context: made once for its sizes, kept as long as the worker lives."""
    batch = max(1, s["ctx_len"].numel()) if "ctx_len" in s else 1
    key = (case["heads"], case["kv_heads"], case["dim"], case["layers"], s["num_blocks"], batch)
    if key not in _handles:
        import paper_2609_29364_b200 as nsd

        _handles.clear()
        _handles[key] = nsd.VerifyContext(num_layers=case["layers"], num_q_heads=case["heads"], num_kv_heads=case["kv_heads"], head_dim=case["dim"],
                                          block_size=BS, num_blocks=s["num_blocks"], region_b_begin=0, max_batch=batch, max_gamma=1, vocab_size=2,
                                          max_table_entries=1)
    return _handles[key]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind = case["kind"]
    s = {"append": _prepare_append, "pack": _prepare_store, "unpack": _prepare_store, "attn8": _prepare_attn, "prefix": _prepare_attn}[kind](case, gen)
    s["case"] = case
    if own:
        s["nsd"] = _handle(case, s)
        if kind == "attn8":
            s["plan"] = torch.empty(s["nsd"].nsd_kv8_plan_bytes(s["max_rows"]), dtype=torch.uint8, device=DEV)
        if kind == "prefix":
            s["plan"] = torch.empty(s["nsd"].nsd_prefix_plan_bytes(s["max_rows"]), dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------- one pass
def run(s):
    return {"append": _run_append, "pack": _run_pack, "unpack": _run_unpack, "attn8": _run_attn8, "prefix": _run_prefix}[s["case"]["kind"]](s)


def _run_append(s):
    c = s["case"]
    wk = c["kv_heads"] * c["dim"]
    k, v = s["kv"][:, :wk], s["kv"][:, wk:]
    if own:
        s["nsd"].nsd_kv8_append(s["kv8"], s["scales"], 0, s["q"], k, v, s["q_out"], s["slot_map"], s["positions"], [c["rot"] // 2] if c["rot"] else [],
                                s["inv_freq"])
    else:
        _plain_append(s, k, v)
    out = {"kv8": s["kv8"], "scales": s["scales"]}
    return out if s["q"] is None else {**out, "q_out": s["q_out"]}


def _run_pack(s):
    if own:
        s["nsd"].nsd_kv8_pack(s["pool"], s["kv8"], s["scales"], s["src"], s["dst"])
    else:
        codes, e = _quantise(s["pool"][:, s["src"].long()].float())
        s["kv8"].view(torch.uint8)[:, s["dst"].long()] = codes.view(torch.uint8)
        s["scales"].view(torch.uint8)[:, s["dst"].long()] = (e + 127).to(torch.uint8).transpose(-3, -2)
    return {"kv8": s["kv8"], "scales": s["scales"]}


def _run_unpack(s):
    if own:
        s["nsd"].nsd_kv8_unpack(s["kv8"], s["scales"], s["pool"], s["src"], s["dst"])
    else:
        src = s["src"].long()
        s["pool"][:, s["dst"].long()] = _values(s["kv8"].view(torch.uint8)[:, src].view(E4M3), s["scales"].view(torch.uint8)[:, src].view(E8M0)).to(torch.bfloat16)
    return {"pool": s["pool"]}


def _run_attn8(s):
    c = s["case"]
    if own:
        s["nsd"].nsd_kv8_plan(s["plan"], s["max_rows"], s["q_indptr"], s["ctx_len"], s["kv_indptr"], window=c["window"])
        for layer in range(c["layers"]):
            s["nsd"].nsd_kv8_attn(s["plan"], s["max_rows"], s["kv8"], s["scales"], s["q"][layer], s["o"][layer], s["lse"][layer], s["kv_indices"], layer=layer)
    else:
        for layer in range(c["layers"]):
            for g in s["slices"]:
                _finish(s, layer, g, *_plain_part(s, layer, g))
    return {"o": s["o"], "lse": s["lse"]}


def _run_prefix(s):
    c = s["case"]
    if own:
        s["nsd"].nsd_prefix_plan(s["plan"], s["max_rows"], s["group_indptr"], s["prefix_len"], s["q_indptr"], s["ctx_len"], s["kv_indptr"])
        for layer in range(c["layers"]):
            s["nsd"].nsd_prefix_attn(s["plan"], s["max_rows"], s["pool"], s["q"][layer], s["o"][layer], s["lse"][layer], s["kv_indices"], layer=layer)
    else:
        for layer in range(c["layers"]):
            for g in s["groups"]:
                _plain_group(s, layer, g)
    return {"o": s["o"], "lse": s["lse"]}


# --------------------------------------------------------------------------- plain forms
def _plain_append(s, k, v):
    """Angles in 64 bits, the rotation in 32, then codes; padding rows (slot -1) are left alone."""
    c = s["case"]
    d, half = c["dim"], c["rot"] // 2

    def rotate(x):
        x = x.reshape(x.shape[0], -1, d).float()
        if not half:
            return x
        angle = s["positions"][0].double()[:, None] * s["inv_freq"].double()
        cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], dim=-1)

    real = s["slot_map"] >= 0
    if s["q"] is not None:
        s["q_out"].copy_(torch.where(real[:, None, None], rotate(s["q"]).to(torch.bfloat16), s["q_out"]))
    # a padding row stores what its place holds already: the last real row's, at the last real row's place
    last = torch.where(real, torch.arange(real.numel(), device=real.device), 0).cummax(0).values
    slot = s["slot_map"].clamp(min=0)[last]
    codes, e = _quantise(torch.stack([rotate(k), v.reshape(v.shape[0], -1, d).float()], 1)[last])               # [rows][K|V][kv head]
    s["kv8"].view(torch.uint8)[0, slot // BS, :, :, slot % BS] = codes.view(torch.uint8)
    s["scales"].view(torch.uint8)[0, slot // BS, :, :, slot % BS] = (e + 127).to(torch.uint8).transpose(1, 2)


def _plain_part(s, layer, g):
    """Largest score, sum of weights and weighted values of the requests of a slice over the keys from `skip` on, in 32 bits."""
    c, reqs = s["case"], g["reqs"]
    h, hkv, d = c["heads"], c["kv_heads"], c["dim"]
    n, keys, skip = g["rows"], g["keys"], g["skip"]
    q = s["q"][layer]
    start, ctx = s["q_indptr"][reqs], s["ctx_len"][reqs].long()
    count = s["q_indptr"][reqs + 1] - start
    i = torch.arange(n, device=q.device)[None, :]
    row = torch.where(i < count[:, None], start[:, None] + i, start[:, None])
    at = skip // BS + torch.arange(_blocks(skip % BS + keys), device=q.device)[None, :]
    inside = at < (s["kv_indptr"][reqs + 1] - s["kv_indptr"][reqs])[:, None]
    block = s["kv_indices"][torch.where(inside, s["kv_indptr"][reqs][:, None] + at, s["kv_indptr"][reqs][:, None])].long()
    if "pool" in s:
        kv = s["pool"][layer][block].float()
    else:
        kv = _values(s["kv8"][layer].view(torch.uint8)[block].view(E4M3), s["scales"][layer].view(torch.uint8)[block].view(E8M0))
    kv = kv.permute(2, 0, 3, 1, 4, 5).reshape(2, reqs.numel(), hkv, -1, d)[..., skip % BS:skip % BS + keys, :]
    qq = q[row].float().reshape(reqs.numel(), n, hkv, h // hkv, d).permute(0, 2, 3, 1, 4).reshape(reqs.numel(), hkv, -1, d)
    score = (qq @ kv[0].transpose(-1, -2)).reshape(reqs.numel(), hkv, h // hkv, n, keys) * (1.0 / math.sqrt(d))
    j, pos = skip + torch.arange(kv.shape[3], device=q.device), ctx[:, None] + i
    seen = j <= pos[..., None]
    if c.get("window"):
        seen &= j > pos[..., None] - c["window"]
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    value = torch.where((j < (ctx + count)[:, None])[:, None, :, None], kv[1], 0.0)
    out = (weight.reshape(reqs.numel(), hkv, -1, kv.shape[3]) @ value).reshape(weight.shape[:-1] + (d,))
    return tuple(x.permute(0, 3, 1, 2, 4).reshape(reqs.numel(), n, h, -1) for x in (top, weight.sum(-1, keepdim=True), out))


def _finish(s, layer, g, top, total, out):
    reqs = g["reqs"]
    start = s["q_indptr"][reqs]
    i = torch.arange(g["rows"], device=start.device)[None, :]
    real = i < (s["q_indptr"][reqs + 1] - start)[:, None]
    row = (start[:, None] + i)[real]
    s["o"][layer][row] = (out / torch.where(total > 0, total, 1.0))[real].to(torch.bfloat16)
    s["lse"][layer][row] = (top + total.log()).squeeze(-1)[real]


def _plain_group(s, layer, g):
    """The shared keys in one product for all rows of the group, each request's own keys, and the two joined."""
    c, (a, b), p = s["case"], g["rows"], g["shared"]
    h, hkv, d = c["heads"], c["kv_heads"], c["dim"]
    tops, totals, outs = [], [], []
    step = max(1, SCORES // (h * max(1, p)))
    if p and b > a:
        kv = s["pool"][layer][g["table"]].permute(1, 2, 0, 3, 4).reshape(2, hkv, -1, d)[:, :, :p].float()
        for r in range(a, b, step):
            q = s["q"][layer][r:min(b, r + step)].float().reshape(-1, hkv, h // hkv, d).permute(1, 0, 2, 3).reshape(hkv, -1, d)
            score = (q @ kv[0].transpose(-1, -2)) * (1.0 / math.sqrt(d))
            top = score.amax(-1, keepdim=True)
            weight = torch.exp(score - top)
            for to, x in ((tops, top), (totals, weight.sum(-1, keepdim=True)), (outs, weight @ kv[1])):
                to.append(x.reshape(hkv, -1, h // hkv, x.shape[-1]).permute(1, 0, 2, 3).reshape(-1, h, x.shape[-1]))
    for sl in g["slices"]:
        top, total, out = _plain_part(s, layer, sl)
        if p:
            start = s["q_indptr"][sl["reqs"]]
            i = torch.arange(sl["rows"], device=start.device)[None, :]
            row = (torch.where(i < (s["q_indptr"][sl["reqs"] + 1] - start)[:, None], start[:, None] + i, start[:, None]) - a)
            top0 = torch.cat(tops)[row]
            m = torch.maximum(top, top0)
            w0, w1 = torch.exp(top0 - m), torch.exp(top - m)
            top, total, out = m, total * w1 + torch.cat(totals)[row] * w0, out * w1 + torch.cat(outs)[row] * w0
        _finish(s, layer, sl, top, total, out)


# --------------------------------------------------------------------------- work
def _pairs(case, ctx, new):
    """(row, key) pairs that take part, and the keys of each request that some row sees."""
    pairs, keys, w = 0, [], case.get("window", 0)
    for c, n in zip(ctx, new):
        if not n:
            keys.append(0)
            continue
        pairs += sum(min(c + i + 1, w) for i in range(n)) if w else n * c + n * (n + 1) // 2
        keys.append(min(c + n, w + n - 1) if w else c + n)
    return pairs, keys


def work(case):
    h, hkv, d, layers = case["heads"], case["kv_heads"], case["dim"], case["layers"]
    row8 = 2 * hkv * (d + 1)                                              # a token in the 8-bit cache
    if case["kind"] == "append":
        size, rows = 4 if case["dtype"] == "fp32" else 2, case["rows"]
        got = rows * (2 * hkv * d * size + row8 + 8) + 8 * case["pad"]
        if case["rot"]:
            got += rows * (h * d * (size + 2) + 4)
        return {"bytes": got, "flops": rows * (4 * hkv * d + (3 * case["rot"] * (h + hkv) if case["rot"] else 0))}
    if case["kind"] in ("pack", "unpack"):
        cells = case["blocks"] * layers * BS
        return {"bytes": cells * (2 * hkv * d * 2 + row8) + 8 * case["blocks"], "flops": cells * 4 * hkv * d}
    ctx, new, members, shared = _lengths(case)
    rows, blocks = sum(new), sum(_blocks(c + n) for c, n in zip(ctx, new))
    pairs, keys = _pairs(case, ctx, new)
    tokens, each = sum(keys), row8
    if members:
        at, each = _offsets(members), 2 * hkv * d * 2
        live = [sum(1 for n in new[a:b] if n) for a, b in zip(at, at[1:])]
        tokens -= sum(p * (m - 1) for p, m in zip(shared, live) if m)
    return {"bytes": layers * (tokens * each + rows * h * (2 * d * 2 + 4)) + 4 * blocks, "flops": layers * 4 * d * h * pairs}


# --------------------------------------------------------------------------- 64 bits, from the definitions
def _exact_codes(x):
    """The value each element is held as, and the power of two of its row, from the grid of e4m3: steps of 2^(E - 3) for
    2^E <= |y| < 2^(E + 1), and of 2^-9 below 2^-6."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.full_like(top, 2.0 ** -126)
    big = top > 448 * scale
    scale[big] = torch.exp2(torch.ceil(torch.log2(top[big] / 448)))
    scale = torch.where(big & (scale * 224 >= top), scale / 2, scale)    # the logarithm may have come out a little high
    scale = torch.where(big & (scale * 448 < top), scale * 2, scale)     # or low
    y = x / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, scale[..., 0]


def _exact_append(case, s):
    h, hkv, d, rot = case["heads"], case["kv_heads"], case["dim"], case["rot"]
    keep = s["slot_map"] >= 0
    kv = s["kv"][keep].double().reshape(-1, 2, hkv, d)
    out = {}
    if rot:
        theta = s["positions"][0][keep].double()[:, None] * s["inv_freq"].double()
        turn = torch.polar(torch.ones_like(theta), theta)[:, None]

        def turned(x):
            z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
            return torch.cat([z.real, z.imag, x[..., rot:]], -1)

        kv[:, 0] = turned(kv[:, 0])
        out["q_out"] = s["q_out"].double()
        out["q_out"][keep] = turned(s["q"][keep].double().reshape(-1, h, d))
    codes, scale = _exact_codes(kv)
    out["kv8"], out["scales"] = s["kv8"].double(), s["scales"].double()
    b, t = s["slot_map"][keep] // BS, s["slot_map"][keep] % BS
    out["kv8"][0, b, :, :, t] = codes
    out["scales"][0, b, :, :, t] = scale.transpose(1, 2)
    return out


def _exact_attn(case, s, layer):
    """Request by request and head by head over its own whole table, weights from exp(score - log-sum)."""
    ctx, new, _, _ = _lengths(case)
    h, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    o = torch.zeros(s["max_rows"], h, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["max_rows"], h, dtype=torch.float64, device=DEV)
    at, entry = 0, 0
    for c, n in zip(ctx, new):
        mine = s["kv_indices"][entry:entry + -(-(c + n) // BS)].long()
        entry += mine.numel()
        if not n:
            continue
        if case["kind"] == "attn8":
            kv = s["kv8"][layer].view(torch.uint8)[mine].view(E4M3).double() * s["scales"][layer].view(torch.uint8)[mine].view(E8M0).double().transpose(1, 2)[..., None]
        else:
            kv = s["pool"][layer][mine].double()
        kv = kv.permute(1, 2, 0, 3, 4).reshape(2, hkv, -1, d)[:, :, :c + n]
        z = torch.einsum("nkgd,kjd->kgnj", s["q"][layer][at:at + n].double().reshape(n, hkv, -1, d), kv[0]) / math.sqrt(d)
        far = (c + torch.arange(n, device=DEV))[:, None] - torch.arange(c + n, device=DEV)[None]
        z.masked_fill_((far < 0) | (far >= (case.get("window") or c + n + 1)), float("-inf"))
        log_sum = torch.logsumexp(z, -1)
        lse[at:at + n] = log_sum.permute(2, 0, 1).reshape(n, h)
        o[at:at + n] = torch.einsum("kgnj,kjd->nkgd", torch.exp(z - log_sum[..., None]), kv[1]).reshape(n, h, d)
        at += n
    return o, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(case, s)
    if case["kind"] == "pack":
        kv8, scales = s["kv8"].double(), s["scales"].double()
        for layer in range(case["layers"]):
            codes, scale = _exact_codes(s["pool"][layer][s["src"].long()].double())
            kv8[layer][s["dst"].long()] = codes
            scales[layer][s["dst"].long()] = scale.transpose(1, 2)
        return {"kv8": kv8, "scales": scales}
    if case["kind"] == "unpack":
        pool = s["pool"].double()
        for layer in range(case["layers"]):
            codes, scale = s["kv8"][layer].double()[s["src"].long()], s["scales"][layer].double()[s["src"].long()]
            pool[layer][s["dst"].long()] = codes * scale.transpose(1, 2)[..., None]
        return {"pool": pool}
    both = [_exact_attn(case, s, k) for k in range(case["layers"])]
    return {"o": torch.stack([b[0] for b in both]), "lse": torch.stack([b[1] for b in both])}
