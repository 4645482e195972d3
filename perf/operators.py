"""What the ragged-batch operators over the paged cache are measured on.

Three families: attention of ragged chunks over the cache (``extend``), rotary positions with the cache write
(``rope_append``), and the upkeep of the pages (``pages_copy``, ``pages_branch``, ``pages_compact``).  ``run`` makes one
pass, in elementary torch operations where ``own`` is false and through the library where it is true.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a serving tick that mixes one prompt chunk with running sequences (the 16/2/4-head, 4K-token configuration)
        dict(name="extend mixed 16 seqs", op="extend", batch=16, n_q=16, n_k=2, n_v=4, d_qk=128, d_v=128, dtype="bf16",
             page=16, past_lo=500, past_hi=4095, chunk_lo=512, chunk_hi=512, ones=15, pad=7, lens=1),
        # verification of a few guessed tokens over long contexts (the 32/4/8-head configuration, 16-token pages)
        dict(name="extend verify 5 tokens 32k", op="extend", batch=16, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128,
             dtype="bf16", page=16, past_lo=4096, past_hi=32700, chunk_lo=2, chunk_hi=5, ones=3, pad=0, lens=2),
        # chunked prefill of several prompts, some with a cached prefix (compute-bound)
        dict(name="extend prefill chunks", op="extend", batch=4, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16",
             page=128, past_lo=0, past_hi=6144, chunk_lo=1500, chunk_hi=2048, ones=0, pad=0, lens=3),
        # the 64-channel head layout of the 1.5B model, a decode tick with short contexts: latency
        dict(name="extend ticks d64", op="extend", batch=8, n_q=32, n_k=4, n_v=16, d_qk=64, d_v=64, dtype="bf16",
             page=64, past_lo=1, past_hi=2047, chunk_lo=1, chunk_hi=3, ones=5, pad=0, lens=4),
        # the fp32 mode (16/2/4 heads of 64 channels), small chunks
        dict(name="extend f32 chunks", op="extend", batch=4, n_q=16, n_k=2, n_v=4, d_qk=64, d_v=64, dtype="f32",
             page=16, past_lo=0, past_hi=1024, chunk_lo=17, chunk_hi=100, ones=0, pad=3, lens=5),
        # a decode tick's rotation and append: latency
        dict(name="rope tick 16 rows", op="rope", batch=16, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16",
             page=16, past_lo=100, past_hi=30000, chunk_lo=1, chunk_hi=1, ones=0, pad=0, lens=6, rot=128,
             interleaved=False, mscale=1.0),
        # prompt chunks with interleaved pairs over half of the head and stretched positions
        dict(name="rope chunks interleaved", op="rope", batch=8, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16",
             page=16, past_lo=0, past_hi=120000, chunk_lo=900, chunk_hi=2048, ones=0, pad=5, lens=7, rot=64,
             interleaved=True, mscale=1.2079),
        # a few pages, as a host-side allocator copies them before a shared page is written
        dict(name="copy 24 pages", op="pages_copy", n_k=2, n_v=4, d_qk=128, d_v=128, dtype="bf16", page=16, pool=512,
             count=24),
        # a long sequence brought into pages of its own
        dict(name="copy 4096 pages", op="pages_copy", n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16", page=16,
             pool=16384, count=4096),
        # sampling several continuations of running prompts: the old ones leave, the new ones branch, all get their next token
        dict(name="branch 64 slots 32k", op="pages_branch", slots=64, kids=24, n_k=4, n_v=8, d_qk=128, d_v=128,
             dtype="bf16", page=16, pool=98304, max_len=32768, past_lo=1000, past_hi=32000, new=1, lens=8),
        dict(name="compact 700 pages", op="pages_compact", slots=12, n_k=4, n_v=16, d_qk=64, d_v=64, dtype="bf16",
             page=64, pool=700, live=400, row=64),
        # a pool of a few GB at six tenths of its pages after many sequences have left
        dict(name="compact 48k pages", op="pages_compact", slots=64, n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16",
             page=16, pool=49152, live=29491, row=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


_HEADS = [(16, 2, 4, 128, 128), (32, 4, 8, 128, 128), (32, 4, 16, 64, 64), (32, 4, 16, 64, 128), (32, 8, 8, 128, 128),
          (16, 4, 2, 128, 128), (12, 2, 4, 128, 128)]


def draw(rng):
    op = rng.choice(["extend", "extend", "rope", "pages_copy", "pages_branch", "pages_compact"])
    n_q, n_k, n_v, d_qk, d_v = rng.choice(_HEADS)
    heads = dict(n_k=n_k, n_v=n_v, d_qk=d_qk, d_v=d_v)
    page = rng.choice([16, 16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    lens = rng.randrange(1 << 20)
    if op == "extend":
        hi = _log(rng, 1, 2048 if dtype == "bf16" else 160)
        batch = _log(rng, 1, max(1, min(24, 4000 // hi)))
        past = _log(rng, 8, 30000 if hi <= 64 and dtype == "bf16" else 4000 if dtype == "bf16" else 1200)
        past = min(past, 190000 // batch, 16000000 // (batch * hi))
        return dict(op=op, batch=batch, n_q=n_q, **heads, dtype=dtype, page=page, past_lo=past // rng.randint(1, 9),
                    past_hi=past, chunk_lo=max(1, hi // 2), chunk_hi=hi, ones=rng.randint(0, batch // 2),
                    pad=rng.randint(0, 9), lens=lens)
    if op == "rope":
        hi = _log(rng, 1, 2048)
        return dict(op=op, batch=_log(rng, 1, max(1, min(16, 5500 // hi))), n_q=n_q, **heads, dtype=dtype, page=page,
                    past_lo=0, past_hi=_log(rng, 10, 120000), chunk_lo=max(1, hi // 2), chunk_hi=hi, ones=0,
                    pad=rng.randint(0, 9), lens=lens, rot=d_qk // rng.choice([1, 1, 2, 4]),
                    interleaved=rng.random() < 0.5, mscale=rng.choice([1.0, 1.1386]))
    if op == "pages_copy":
        count = _log(rng, 4, (1 << 14) // page)
        return dict(op=op, **heads, dtype=dtype, page=page, pool=count * 2 + rng.randint(1, 900), count=count)
    if op == "pages_branch":
        slots = rng.randint(4, 64)
        max_len = _log(rng, 1024, min(32768, 600000 // slots))
        return dict(op=op, slots=slots, kids=rng.randint(1, slots // 2), **heads, dtype="bf16", page=page,
                    pool=slots * (-(-max_len // page) + 2) // 2 * 3, max_len=max_len, past_lo=max_len // 9,
                    past_hi=max_len * 9 // 10, new=rng.choice([1, 1, 5, 60]), lens=lens)
    pool = _log(rng, 400, (1 << 19) // page)
    live = int(pool * rng.uniform(0.2, 0.95))
    return dict(op=op, slots=rng.randint(2, 64), **heads, dtype="bf16", page=page, pool=pool, live=live,
                row=-(-live // 2) + rng.randint(0, 9))


# ---------------------------------------------------------------------------------------------------------- inputs

def _lengths(case):
    """(past, new) of every sequence, from the case alone."""
    r = random.Random(case["lens"])
    past = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["batch"])]
    new = [r.randint(case["chunk_lo"], case["chunk_hi"]) for _ in range(case["batch"])]
    for b in r.sample(range(case["batch"]), case["ones"]):
        new[b] = 1
    return past, new


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32 if dtype == torch.float32 else torch.bfloat16)


def _pools(gen, case, pages):
    dtype = DTYPES[case["dtype"]]
    return (_normal(gen, (pages, case["n_k"], case["page"], case["d_qk"]), dtype),
            _normal(gen, (pages, case["n_v"], case["page"], case["d_v"]), dtype))


def _ragged(case, gen, written_only):
    """Pools, tables and lengths of a ragged batch.  `written_only`: pages for the rows a call writes alone (positions
    below them belong to a page that is not read, page 0)."""
    past, new = _lengths(case)
    page = case["page"]
    first = [p // page if written_only else 0 for p in past]
    last = [-(-(p + n) // page) for p, n in zip(past, new)]
    pages = sum(e - f for f, e in zip(first, last)) + 3
    order = torch.randperm(pages - 1, generator=gen, device=DEV).to(torch.int32) + 1
    table = torch.zeros((len(past), max(last)), dtype=torch.int32, device=DEV)
    at = 0
    for b, (f, e) in enumerate(zip(first, last)):
        table[b, f:e] = order[at:at + e - f]
        at += e - f
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    k, v = _pools(gen, case, pages)
    return dict(past=_int(past), cu=_int(cu), rows=cu[-1], total=cu[-1] + case["pad"], longest=max(new),
                reach=max(last) * page, table=table, k=k, v=v, past_host=past, new_host=new)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case=case)
    op = case["op"]
    dtype = DTYPES[case["dtype"]]
    if op == "extend":
        s.update(_ragged(case, gen, False))
        s["q"] = _normal(gen, (s["total"], case["n_q"], case["d_qk"]), dtype)
        s["scale"] = case["d_qk"] ** -0.5
        s["out"] = torch.full((s["total"], case["n_q"], case["d_v"]), 0.125, dtype=dtype, device=DEV)
        s["lse"] = torch.full((s["total"], case["n_q"]), 0.125, dtype=torch.float32, device=DEV)
    elif op == "rope":
        s.update(_ragged(case, gen, True))
        s["q"] = _normal(gen, (s["total"], case["n_q"], case["d_qk"]), dtype)
        s["k_new"] = _normal(gen, (s["total"], case["n_k"], case["d_qk"]), dtype)
        s["v_new"] = _normal(gen, (s["total"], case["n_v"], case["d_v"]), dtype)
        s["out"] = torch.full((s["total"], case["n_q"], case["d_qk"]), 0.125, dtype=dtype, device=DEV)
        half = case["rot"] // 2
        s["inv_freq"] = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    elif op == "pages_copy":
        s["k"], s["v"] = _pools(gen, case, case["pool"])
        ids = torch.randperm(case["pool"], generator=gen, device=DEV)[:2 * case["count"]].to(torch.int32)
        s["src"], s["dst"] = ids[:case["count"]].contiguous(), ids[case["count"]:].contiguous()
        s["seqlens"], s["table"] = _int([0]), torch.full((1, 1), -1, dtype=torch.int32, device=DEV)
    elif op == "pages_branch":
        slots, page, kids = case["slots"], case["page"], case["kids"]
        r = random.Random(case["lens"])
        lens = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(slots)]
        row = -(-case["max_len"] // page) + 4
        order = torch.randperm(case["pool"], generator=gen, device=DEV).to(torch.int32)
        table = torch.full((slots, row), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(lens):
            held = -(-n // page)
            table[b, :held] = order[at:at + held]
            at += held
        refs = torch.zeros(case["pool"], dtype=torch.int32, device=DEV)
        refs[order[:at].long()] = 1
        ids = torch.randperm(slots, generator=gen, device=DEV).to(torch.int32)
        s["children"] = ids[:kids].contiguous()
        parents = ids[kids:][torch.randint(0, slots - kids, (kids,), generator=gen, device=DEV)]
        s["parents"] = parents.contiguous()
        s["cu"] = torch.arange(slots + 1, dtype=torch.int32, device=DEV) * case["new"]
        s["seqlens"], s["table"], s["refs"] = _int(lens), table, refs
        s["granted"] = torch.zeros(slots, dtype=torch.int32, device=DEV)
        s["k"], s["v"] = _pools(gen, case, case["pool"])
    else:
        # `live` pages at random places, dealt to the slots; every slot past the first also shares one page of the first
        slots, live, row = case["slots"], case["live"], case["row"]
        order = torch.randperm(case["pool"], generator=gen, device=DEV)[:live].to(torch.int32)
        per = min(row - 1, live // slots)
        table = torch.full((slots, row), -1, dtype=torch.int32, device=DEV)
        refs = torch.zeros(case["pool"], dtype=torch.int32, device=DEV)
        table[:, 1:1 + per] = order[:slots * per].view(slots, per)
        table[:, 0] = order[0]
        refs[order.long()] = 1  # what no slot names is held by somebody else (a pinned prefix)
        refs[order[0].long()] = slots + 1
        s["seqlens"] = torch.full((slots,), (1 + per) * case["page"], dtype=torch.int32, device=DEV)
        s["table"], s["refs"] = table, refs
        s["table_out"], s["refs_out"] = torch.empty_like(table), torch.empty_like(refs)
        s["live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        s["k"], s["v"] = _pools(gen, case, case["pool"])
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

def _row_places(s):
    """Sequence and place within it of every row."""
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=s["rows"])
    return seq, torch.arange(s["rows"], device=DEV) - s["cu"].long()[seq]


def _plain_extend(s):
    c = s["case"]
    B, Q, L = c["batch"], s["longest"], s["reach"]
    seq, place = _row_places(s)
    rows = (s["cu"][:-1, None].long() + torch.arange(Q, device=DEV)).clamp(max=s["total"] - 1)
    q = s["q"][rows].float().permute(0, 2, 1, 3).reshape(B, c["n_k"], -1, c["d_qk"])  # [B, n_k, heads * Q, d]
    pages = s["table"].long()
    k = s["k"][pages].permute(0, 2, 1, 3, 4).reshape(B, c["n_k"], L, c["d_qk"]).float()
    v = s["v"][pages].permute(0, 2, 1, 3, 4).reshape(B, c["n_v"], L, c["d_v"]).float()
    x = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).view(B, c["n_q"], Q, L)
    sees = torch.arange(L, device=DEV) <= (s["past"][:, None].long() + torch.arange(Q, device=DEV))[:, :, None]
    x.masked_fill_(~sees[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, c["n_v"], -1, L), v).view(B, c["n_q"], Q, c["d_v"]) / total
    lse = (top + total.log())[..., 0]
    s["out"][:s["rows"]] = o[seq, :, place].to(s["out"].dtype)
    s["lse"][:s["rows"]] = lse[seq, :, place]
    return {"out": s["out"], "lse": s["lse"]}


def _rotated(x, cos, sin, rot, interleaved):
    y = x.float().clone()
    if interleaved:
        a, b = x[..., 0:rot:2].float(), x[..., 1:rot:2].float()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :rot // 2].float(), x[..., rot // 2:rot].float()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return y.to(x.dtype)


def _plain_rope(s):
    c = s["case"]
    seq, place = _row_places(s)
    pos = s["past"].long()[seq] + place
    angle = pos.double()[:, None] * s["inv_freq"]
    cos, sin = (angle.cos() * c["mscale"]).float()[:, None], (angle.sin() * c["mscale"]).float()[:, None]
    n = s["rows"]
    s["out"][:n] = _rotated(s["q"][:n], cos, sin, c["rot"], c["interleaved"])
    page = s["table"].long()[seq, pos // c["page"]]
    s["k"][page, :, pos % c["page"]] = _rotated(s["k_new"][:n], cos, sin, c["rot"], c["interleaved"])
    s["v"][page, :, pos % c["page"]] = s["v_new"][:n]
    return {"q": s["out"], "k": s["k"], "v": s["v"]}


def _plain_copy(s):
    for pool in (s["k"], s["v"]):
        pool[s["dst"].long()] = pool[s["src"].long()]
    return {"k": s["k"], "v": s["v"]}


def _count_refs(refs, ids, sign):
    refs.index_add_(0, ids.clamp(min=0).flatten().long(), ((ids >= 0).to(refs.dtype) * sign).flatten())


def _plain_branch(s):
    page, table, refs, lens = s["case"]["page"], s["table"], s["refs"], s["seqlens"]
    at = torch.arange(table.shape[1], device=DEV)
    kids, parents = s["children"].long(), s["parents"].long()
    # the children's old pages go back
    _count_refs(refs, table[kids], -1)
    table[kids] = -1
    lens[kids] = 0
    # the children share what their parents have filled
    shared = torch.where(at < ((lens[parents] + page - 1) // page)[:, None], table[parents], -1)
    _count_refs(refs, shared, 1)
    table[kids] = shared
    lens[kids] = lens[parents]
    # every slot gets pages of its own for its next tokens
    new = s["cu"][1:] - s["cu"][:-1]
    first, end = lens // page, torch.where(new > 0, (lens + new + page - 1) // page, 0)
    spread = (refs[table.clamp(min=0).long()] > 1) & (table >= 0)
    need = (at >= first[:, None]) & (at < end[:, None]) & ((table < 0) | spread)
    demand = need.sum(1)
    s["granted"].copy_((demand == 0) | (demand.cumsum(0) <= (refs == 0).sum()))
    need &= s["granted"][:, None] > 0
    free = torch.sort((refs > 0).to(torch.int8), stable=True).indices
    fresh = free[(need.flatten().cumsum(0) - 1).clamp(min=0).view_as(need)].to(table.dtype)
    slot = (need.gather(1, first[:, None].long())[:, 0] & (table.gather(1, first[:, None].long())[:, 0] >= 0)
            & (lens % page > 0)).nonzero()[:, 0]  # slots whose half-filled page has other holders
    src, dst = table[slot, first[slot].long()].long(), fresh[slot, first[slot].long()].long()
    for pool in (s["k"], s["v"]):
        pool[dst] = pool[src]
    _count_refs(refs, torch.where(need, table, -1), -1)
    _count_refs(refs, torch.where(need, fresh, -1), 1)
    table.copy_(torch.where(need, fresh, table))
    return {"table": table, "refs": refs, "seqlens": lens, "granted": s["granted"], "k": s["k"], "v": s["v"]}


def _plain_compact(s):
    refs, table = s["refs"], s["table"]
    held = refs > 0
    count = held.sum()
    ids = torch.arange(refs.numel(), device=DEV)
    src = (held & (ids >= count)).nonzero()[:, 0]
    dst = (~held & (ids < count)).nonzero()[:, 0]
    to = ids.to(table.dtype)
    to[src] = dst.to(table.dtype)
    for pool in (s["k"], s["v"]):
        pool[dst] = pool[src]
    s["table_out"].copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    s["refs_out"].copy_(refs)
    s["refs_out"][dst] = refs[src]
    s["refs_out"][src] = 0
    s["live"].copy_(count)
    return {"table": s["table_out"], "refs": s["refs_out"], "live": s["live"], "k": s["k"], "v": s["v"]}


_PLAIN = {"extend": _plain_extend, "rope": _plain_rope, "pages_copy": _plain_copy, "pages_branch": _plain_branch,
          "pages_compact": _plain_compact}


# ------------------------------------------------------------------------------------------------- the library's calls

def _own_cache(api, s, seqlens):
    c = s["case"]
    return api.KVCache(s["k"], s["v"], seqlens, s["table"].shape[1] * c["page"], page_table=s["table"],
                       page_size=c["page"])


def _own_extend(api, s):
    c = s["case"]
    api.diffqkv_extend(s["q"], s["cu"], _own_cache(api, s, s["past"]), c["n_k"], c["n_v"], s["scale"], out=s["out"],
                       lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_rope(api, s):
    c = s["case"]
    api.diffqkv_rope_append(s["q"], s["k_new"], s["v_new"], s["cu"], _own_cache(api, s, s["past"]), s["inv_freq"],
                            interleaved=c["interleaved"], magnitude=c["mscale"], q_out=s["out"])
    return {"q": s["out"], "k": s["k"], "v": s["v"]}


def _own_copy(api, s):
    c = s["case"]
    api.diffqkv_pages_copy(s["src"], s["dst"], _own_cache(api, s, s["seqlens"]), c["n_k"], c["n_v"])
    return {"k": s["k"], "v": s["v"]}


def _own_branch(api, s):
    c = s["case"]
    cache = _own_cache(api, s, s["seqlens"])
    api.diffqkv_pages_free(s["children"], cache, s["refs"])
    api.diffqkv_pages_fork(s["parents"], s["children"], cache, s["refs"])
    api.diffqkv_pages_reserve(s["cu"], cache, s["refs"], c["n_k"], c["n_v"], granted=s["granted"])
    return {"table": s["table"], "refs": s["refs"], "seqlens": s["seqlens"], "granted": s["granted"], "k": s["k"],
            "v": s["v"]}


def _own_compact(api, s):
    c = s["case"]
    api.diffqkv_pages_compact(_own_cache(api, s, s["seqlens"]), s["refs"], c["n_k"], c["n_v"], table_out=s["table_out"],
                              refs_out=s["refs_out"], live=s["live"])
    return {"table": s["table_out"], "refs": s["refs_out"], "live": s["live"], "k": s["k"], "v": s["v"]}


_OWN = {"extend": _own_extend, "rope": _own_rope, "pages_copy": _own_copy, "pages_branch": _own_branch,
        "pages_compact": _own_compact}


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2501_13629_b200 import api
        return _OWN[op](api, state)
    return _PLAIN[op](state)


# ------------------------------------------------------------------------------------------------------------- work

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    page_bytes = case["page"] * (case["n_k"] * case["d_qk"] + case["n_v"] * case["d_v"]) * size
    token_bytes = page_bytes // case["page"]
    if case["op"] == "extend":
        past, new = _lengths(case)
        rows, tokens = sum(new), sum(past) + sum(new)
        seen = sum(n * p + n * (n + 1) // 2 for p, n in zip(past, new))
        pages = sum(-(-(p + n) // case["page"]) for p, n in zip(past, new))
        return {"bytes": rows * case["n_q"] * ((case["d_qk"] + case["d_v"]) * size + 4) + tokens * token_bytes + 4 * pages,
                "flops": 2 * seen * case["n_q"] * (case["d_qk"] + case["d_v"])}
    if case["op"] == "rope":
        rows = sum(_lengths(case)[1])
        return {"bytes": 2 * rows * (case["n_q"] * case["d_qk"] * size + token_bytes),
                "flops": 3 * rows * (case["n_q"] + case["n_k"]) * case["rot"]}
    if case["op"] == "pages_copy":
        return {"bytes": case["count"] * (2 * page_bytes + 8), "flops": 0}
    if case["op"] == "pages_branch":
        r = random.Random(case["lens"])
        lens = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["slots"])]
        kid_pages = case["kids"] * sum(-(-n // case["page"]) for n in lens) / case["slots"]  # on average
        # rows freed, read and written; their counts down and up; counts searched for free pages; half-filled pages copied
        copied = min(2 * case["kids"], case["slots"]) * page_bytes
        return {"bytes": 4 * kid_pages * 7 + 4 * case["pool"] + 2 * copied, "flops": 0}
    moved = case["live"] * (case["pool"] - case["live"]) / case["pool"]  # on average
    return {"bytes": moved * 2 * page_bytes + 8 * case["pool"] + 8 * case["slots"] * case["row"], "flops": 0}


# ------------------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_extend(s):
    c = s["case"]
    out, lse = s["out"].double(), s["lse"].double()
    at = 0
    for b in range(c["batch"]):
        past, n = s["past_host"][b], s["new_host"][b]
        t = past + n
        held = s["table"][b, :-(-t // c["page"])].long()
        k = s["k"][held].transpose(0, 1).flatten(1, 2)[:, :t]
        v = s["v"][held].transpose(0, 1).flatten(1, 2)[:, :t]
        hidden = torch.ones((n, t), dtype=torch.bool, device=DEV).triu(past + 1)
        for h in range(c["n_q"]):
            x = s["q"][at:at + n, h].double() @ k[h * c["n_k"] // c["n_q"]].double().T * s["scale"]
            x = x.masked_fill(hidden, -math.inf)
            z = torch.logsumexp(x, 1)
            out[at:at + n, h] = torch.exp(x - z[:, None]) @ v[h * c["n_v"] // c["n_q"]].double()
            lse[at:at + n, h] = z
        at += n
    return {"out": out, "lse": lse}


def _exact_rope(s):
    c = s["case"]
    half = c["rot"] // 2
    q_out, k_pool, v_pool = s["out"].double(), s["k"].double(), s["v"].double()
    pair = torch.arange(half, device=DEV)
    one, two = (2 * pair, 2 * pair + 1) if c["interleaved"] else (pair, pair + half)
    at = 0
    for b in range(c["batch"]):
        past, n = s["past_host"][b], s["new_host"][b]
        pos = torch.arange(past, past + n, device=DEV)
        turn = torch.polar(torch.full((n, 1, half), float(c["mscale"]), dtype=torch.float64, device=DEV),
                           torch.outer(pos.double(), s["inv_freq"])[:, None])
        page, slot = s["table"][b].long()[pos // c["page"]], pos % c["page"]
        turned = []
        for x in (s["q"], s["k_new"]):
            x = x[at:at + n].double()
            z = torch.complex(x[..., one], x[..., two]) * turn
            x[..., one], x[..., two] = z.real, z.imag
            turned.append(x)
        q_out[at:at + n] = turned[0]
        k_pool[page, :, slot] = turned[1]
        v_pool[page, :, slot] = s["v_new"][at:at + n].double()
        at += n
    return {"q": q_out, "k": k_pool, "v": v_pool}


def exact(case, seed):
    if case["op"] == "extend":
        return _exact_extend(prepare(case, seed))
    if case["op"] == "rope":
        return _exact_rope(prepare(case, seed))
    return None  # whole numbers and bytes moved as they are
