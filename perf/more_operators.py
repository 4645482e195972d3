"""What the windowed, shared-prefix and normalising operators over the paged cache are measured on.

Three families: attention of ragged chunks within a sliding window and to the first tokens (``window``), attention of
sequences that share a prefix (``shared``), and norms of query and key heads with rotary positions and the cache write
(``norm``).  ``run`` makes one pass, in elementary torch operations where ``own`` is false and through the library where
it is true.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a decode tick of a windowed layer (the 16/2/4-head, 4K-token configuration): latency
        dict(name="window tick 16 seqs", op="window", batch=16, n_q=16, n_k=2, n_v=4, d_qk=128, d_v=128, dtype="bf16",
             page=16, past_lo=500, past_hi=4095, chunk_lo=1, chunk_hi=1, ones=0, pad=0, lens=1, window=1024, sinks=4),
        # verification of a few guessed tokens, long contexts behind a 4K window (the 32/4/8-head configuration)
        dict(name="window verify 5 tokens 4k", op="window", batch=32, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128,
             dtype="bf16", page=16, past_lo=4096, past_hi=32700, chunk_lo=2, chunk_hi=5, ones=6, pad=0, lens=2,
             window=4096, sinks=4),
        # chunked prefill of several prompts through a windowed layer (compute-bound)
        dict(name="window prefill chunks", op="window", batch=4, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16",
             page=128, past_lo=0, past_hi=6144, chunk_lo=1500, chunk_hi=2048, ones=0, pad=0, lens=3, window=2048,
             sinks=0),
        # one prompt chunk among running sequences, 64-channel heads, an odd window and a first block that stays visible
        dict(name="window mixed d64", op="window", batch=12, n_q=32, n_k=4, n_v=16, d_qk=64, d_v=64, dtype="bf16",
             page=64, past_lo=200, past_hi=8000, chunk_lo=700, chunk_hi=700, ones=11, pad=5, lens=4, window=1500,
             sinks=130),
        # the fp32 mode (16/2/4 heads of 64 channels), small chunks
        dict(name="window f32 chunks", op="window", batch=4, n_q=16, n_k=2, n_v=4, d_qk=64, d_v=64, dtype="f32", page=16,
             past_lo=100, past_hi=2000, chunk_lo=17, chunk_hi=100, ones=0, pad=3, lens=5, window=300, sinks=4),
        # a few samples of each of a few prompts, one token each (the 16/2/4-head, 4K-token configuration): latency
        dict(name="shared 4 x 4 samples", op="shared", groups=4, batch=16, n_q=16, n_k=2, n_v=4, d_qk=128, d_v=128,
             dtype="bf16", page=16, prefix_lo=1000, prefix_hi=3500, past_lo=1, past_hi=500, chunk_lo=1, chunk_hi=1, pad=0,
             lens=6),
        # many users behind one long instruction, one token each (the 32/4/8-head configuration)
        dict(name="shared 16k by 64 seqs", op="shared", groups=1, batch=64, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128,
             dtype="bf16", page=16, prefix_lo=16384, prefix_hi=16384, past_lo=50, past_hi=1500, chunk_lo=1, chunk_hi=1,
             pad=0, lens=7),
        # prompts behind two common instructions, in chunks, 64-channel keys and 128-channel values
        dict(name="shared chunks", op="shared", groups=2, batch=8, n_q=32, n_k=4, n_v=16, d_qk=64, d_v=128, dtype="bf16",
             page=64, prefix_lo=3000, prefix_hi=5000, past_lo=0, past_hi=700, chunk_lo=150, chunk_hi=600, pad=9, lens=8),
        # a decode tick's norms, rotation and append: latency
        dict(name="norm tick 16 rows", op="norm", batch=16, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16",
             page=16, past_lo=100, past_hi=30000, chunk_lo=1, chunk_hi=1, ones=0, pad=0, lens=9, rot=128,
             interleaved=False, per_head=False),
        # prompt chunks, the whole head turned
        dict(name="norm chunks", op="norm", batch=8, n_q=32, n_k=4, n_v=8, d_qk=128, d_v=128, dtype="bf16", page=16,
             past_lo=0, past_hi=120000, chunk_lo=900, chunk_hi=2048, ones=0, pad=5, lens=10, rot=128, interleaved=False,
             per_head=False),
        # the fp32 mode, half of a 64-channel head turned as neighbouring pairs, a weight for each head
        dict(name="norm f32 interleaved", op="norm", batch=6, n_q=32, n_k=4, n_v=16, d_qk=64, d_v=64, dtype="f32",
             page=64, past_lo=0, past_hi=9000, chunk_lo=200, chunk_hi=700, ones=1, pad=2, lens=11, rot=32,
             interleaved=True, per_head=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


_HEADS = [(16, 2, 4, 128, 128), (32, 4, 8, 128, 128), (32, 4, 16, 64, 64), (32, 4, 16, 64, 128), (32, 8, 8, 128, 128),
          (16, 4, 2, 128, 128), (12, 2, 4, 128, 128)]


def draw(rng):
    op = rng.choice(["window", "window", "shared", "shared", "norm"])
    n_q, n_k, n_v, d_qk, d_v = rng.choice(_HEADS)
    case = dict(op=op, n_q=n_q, n_k=n_k, n_v=n_v, d_qk=d_qk, d_v=d_v, page=rng.choice([16, 16, 32, 64, 128]),
                dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), lens=rng.randrange(1 << 20), pad=rng.randint(0, 9))
    small = case["dtype"] == "f32"
    if op == "window":
        hi = _log(rng, 1, 160 if small else 2048)
        batch = _log(rng, 1, max(1, min(32, 3000 // hi)))
        past = min(_log(rng, 8, 1200 if small else 30000 if hi <= 64 else 4000), 600000 // batch, 16000000 // (batch * hi))
        case.update(batch=batch, past_lo=past // rng.randint(1, 9), past_hi=past, chunk_lo=max(1, hi // 2), chunk_hi=hi,
                    ones=rng.randint(0, batch // 2), window=_log(rng, 1, 4096), sinks=rng.choice([0, 1, 4, 64, 200]))
    elif op == "shared":
        hi = _log(rng, 1, 60 if small else 600)
        batch = _log(rng, 2, max(2, min(64, 2400 // hi)))
        groups = rng.randint(1, max(1, batch // 2))
        prefix = min(_log(rng, 16, 1200 if small else 16384), 1000000 // batch, 9000000 // (batch * hi), 60000 // groups)
        tail = min(_log(rng, 1, 300 if small else 1500), 50000 // batch)
        case.update(batch=batch, groups=groups, prefix_lo=max(1, prefix // rng.randint(1, 4)), prefix_hi=prefix, past_lo=0,
                    past_hi=tail, chunk_lo=max(1, hi // 2), chunk_hi=hi)
    else:
        hi = _log(rng, 1, 2048)
        case.update(batch=_log(rng, 1, max(1, min(16, 5500 // hi))), past_lo=0, past_hi=_log(rng, 10, 120000),
                    chunk_lo=max(1, hi // 2), chunk_hi=hi, ones=0, rot=d_qk // rng.choice([1, 1, 2, 4]),
                    interleaved=rng.random() < 0.5, per_head=rng.random() < 0.3)
    return case


# ---------------------------------------------------------------------------------------------------------- inputs

def _lengths(case):
    """(tokens cached before, new rows) of every sequence, from the case alone."""
    r = random.Random(case["lens"])
    past = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["batch"])]
    new = [r.randint(case["chunk_lo"], case["chunk_hi"]) for _ in range(case["batch"])]
    for b in r.sample(range(case["batch"]), case.get("ones", 0)):
        new[b] = 1
    if case["op"] == "shared":
        first, prefix = _groups(case)
        for g, p in enumerate(prefix):
            for b in range(first[g], first[g + 1]):
                past[b] += p
    return past, new


def _groups(case):
    """First sequence of every group (and the end), tokens that each shares."""
    r = random.Random(case["lens"] + 1)
    first = [0] + sorted(r.sample(range(1, case["batch"]), case["groups"] - 1)) + [case["batch"]]
    return first, [r.randint(case["prefix_lo"], case["prefix_hi"]) for _ in range(case["groups"])]


def _kept(case, past, new):
    """Pages of a sequence that hold a token which the call reads or writes."""
    page = case["page"]
    end = -(-(past + new) // page)
    if case["op"] == "norm":
        return list(range(past // page, end))
    if case["op"] == "window":
        low = max(0, past - case["window"] + 1) // page
        front = min(-(-case["sinks"] // page), low)
        return list(range(front)) + list(range(low, end))
    return list(range(end))


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32 if dtype == torch.float32 else torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype, page = DTYPES[case["dtype"]], case["page"]
    past, new = _lengths(case)
    s = dict(case=case, past_host=past, new_host=new)
    # pages at random places; a windowed layer's pages that no row can see have been given back, entries without a page are -1
    last = max(-(-(p + n) // page) for p, n in zip(past, new))
    rows = torch.full((len(past), last), -1, dtype=torch.int32)
    at, half_filled = 0, []
    if case["op"] == "shared":
        first, prefix = _groups(case)
        s.update(cu_groups=_int(first), prefix_lens=_int(prefix), first_host=first, prefix_host=prefix)
        for g, p in enumerate(prefix):
            for b in range(first[g], first[g + 1]):
                whole, end = p // page, -(-(past[b] + new[b]) // page)
                lead = b == first[g]
                if not lead:
                    rows[b, :whole] = rows[first[g], :whole]
                    if p % page:
                        half_filled.append((first[g], b, whole, p % page))
                begin = 0 if lead else whole
                rows[b, begin:end] = torch.arange(at, at + end - begin, dtype=torch.int32)
                at += end - begin
    else:
        for b, (p, n) in enumerate(zip(past, new)):
            held = _kept(case, p, n)
            rows[b, held] = torch.arange(at, at + len(held), dtype=torch.int32)
            at += len(held)
    pages = at + 3
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    rows = rows.to(DEV)
    s["table"] = torch.where(rows >= 0, order[rows.clamp(min=0).long()], -1).contiguous()
    s["k"] = _normal(gen, (pages, case["n_k"], page, case["d_qk"]), dtype)
    s["v"] = _normal(gen, (pages, case["n_v"], page, case["d_v"]), dtype)
    for a, b, x, n in half_filled:  # the shared part of a page that a sequence has gone on to write
        for pool in (s["k"], s["v"]):
            pool[s["table"][b, x].long(), :, :n] = pool[s["table"][a, x].long(), :, :n]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    total = cu[-1] + case["pad"]
    s.update(past=_int(past), cu=_int(cu), rows=cu[-1], total=total, longest=max(new), reach=last * page)
    s["q"] = _normal(gen, (total, case["n_q"], case["d_qk"]), dtype)
    if case["op"] == "norm":
        half = case["rot"] // 2
        s["k_new"] = _normal(gen, (total, case["n_k"], case["d_qk"]), dtype) * 3
        s["v_new"] = _normal(gen, (total, case["n_v"], case["d_v"]), dtype)
        shape = lambda h: (h, case["d_qk"]) if case["per_head"] else (case["d_qk"],)  # noqa: E731
        s["q_weight"] = 1 + 0.2 * _normal(gen, shape(case["n_q"]), dtype)
        s["k_weight"] = 1 + 0.2 * _normal(gen, shape(case["n_k"]), dtype)
        s["eps"] = 1e-6
        s["inv_freq"] = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        s["out"] = torch.full((total, case["n_q"], case["d_qk"]), 0.125, dtype=dtype, device=DEV)
    else:
        s["scale"] = case["d_qk"] ** -0.5
        s["out"] = torch.full((total, case["n_q"], case["d_v"]), 0.125, dtype=dtype, device=DEV)
        s["lse"] = torch.full((total, case["n_q"]), 0.125, dtype=torch.float32, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

def _row_places(s):
    """Sequence and place within it of every row."""
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=s["rows"])
    return seq, torch.arange(s["rows"], device=DEV) - s["cu"].long()[seq]


def _plain_attention(s):
    c = s["case"]
    B, Q, L = c["batch"], s["longest"], s["reach"]
    seq, place = _row_places(s)
    rows = (s["cu"][:-1, None].long() + torch.arange(Q, device=DEV)).clamp(max=s["total"] - 1)
    q = s["q"][rows].float().permute(0, 2, 1, 3).reshape(B, c["n_k"], -1, c["d_qk"])  # [B, n_k, heads * Q, d]
    pages = s["table"].long().clamp(min=0)
    k = s["k"][pages].permute(0, 2, 1, 3, 4).reshape(B, c["n_k"], L, c["d_qk"]).float()
    x = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).view(B, c["n_q"], Q, L)
    del k
    v = s["v"][pages].permute(0, 2, 1, 3, 4).reshape(B, c["n_v"], L, c["d_v"]).float()
    at = (s["past"][:, None].long() + torch.arange(Q, device=DEV))[:, :, None]
    token = torch.arange(L, device=DEV)
    sees = token <= at
    if c["op"] == "window":
        sees = sees & ((token < c["sinks"]) | (token > at - c["window"]))
    x.masked_fill_(~sees[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, c["n_v"], -1, L), v).view(B, c["n_q"], Q, c["d_v"]) / total
    lse = (top + total.log())[..., 0]
    s["out"][:s["rows"]] = o[seq, :, place].to(s["out"].dtype)
    s["lse"][:s["rows"]] = lse[seq, :, place]
    return {"out": s["out"], "lse": s["lse"]}


def _plain_turned(x, weight, eps, cos, sin, rot, interleaved):
    y = x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * weight.float()
    z = y.clone()
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        z[..., 0:rot:2], z[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        z[..., :rot // 2], z[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return z.to(x.dtype)


def _plain_norm(s):
    c = s["case"]
    seq, place = _row_places(s)
    pos = s["past"].long()[seq] + place
    angle = pos.double()[:, None] * s["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    n = s["rows"]
    turn = (s["eps"], cos, sin, c["rot"], c["interleaved"])
    s["out"][:n] = _plain_turned(s["q"][:n], s["q_weight"], *turn)
    page = s["table"].long()[seq, pos // c["page"]]
    s["k"][page, :, pos % c["page"]] = _plain_turned(s["k_new"][:n], s["k_weight"], *turn)
    s["v"][page, :, pos % c["page"]] = s["v_new"][:n]
    return {"q": s["out"], "k": s["k"], "v": s["v"]}


# ------------------------------------------------------------------------------------------------- the library's calls

def _own_cache(api, s):
    c = s["case"]
    return api.KVCache(s["k"], s["v"], s["past"], s["table"].shape[1] * c["page"], page_table=s["table"],
                       page_size=c["page"])


def _own_window(api, s):
    c = s["case"]
    api.diffqkv_extend_window(s["q"], s["cu"], _own_cache(api, s), c["n_k"], c["n_v"], s["scale"], c["window"],
                              sinks=c["sinks"], out=s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_shared(api, s):
    c = s["case"]
    api.diffqkv_extend_shared(s["q"], s["cu"], _own_cache(api, s), s["cu_groups"], s["prefix_lens"], c["n_k"], c["n_v"],
                              s["scale"], out=s["out"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_norm(api, s):
    api.diffqkv_norm_rope_append(s["q"], s["k_new"], s["v_new"], s["cu"], _own_cache(api, s), s["inv_freq"],
                                 s["q_weight"], s["k_weight"], s["eps"], interleaved=s["case"]["interleaved"],
                                 q_out=s["out"])
    return {"q": s["out"], "k": s["k"], "v": s["v"]}


_OWN = {"window": _own_window, "shared": _own_shared, "norm": _own_norm}


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2501_13629_b200 import api
        return _OWN[op](api, state)
    return _plain_norm(state) if op == "norm" else _plain_attention(state)


# ------------------------------------------------------------------------------------------------------------- work

def _pairs(case, past, n):
    """(row, token) pairs that are visible, and tokens that some row sees."""
    whole = n * past + n * (n + 1) // 2
    if case["op"] != "window":
        return whole, past + n
    w, first = case["window"], case["sinks"]
    # row at p sees min(p + 1, w) tokens of the window and min(first, max(0, p + 1 - w)) in front of it
    pairs = sum(min(p + 1, w) + min(first, max(0, p + 1 - w)) for p in range(past, past + n))
    low = max(0, past + 1 - w)
    return pairs, past + n - low + min(first, low)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    token_bytes = (case["n_k"] * case["d_qk"] + case["n_v"] * case["d_v"]) * size
    past, new = _lengths(case)
    rows = sum(new)
    if case["op"] == "norm":
        return {"bytes": 2 * rows * (case["n_q"] * case["d_qk"] * size + token_bytes),
                "flops": rows * (case["n_q"] + case["n_k"]) * (4 * case["d_qk"] + 3 * case["rot"])}
    pairs = tokens = 0
    for p, n in zip(past, new):
        x, y = _pairs(case, p, n)
        pairs, tokens = pairs + x, tokens + y
    if case["op"] == "shared":  # a prefix is read once
        first, prefix = _groups(case)
        tokens -= sum((first[g + 1] - first[g] - 1) * p for g, p in enumerate(prefix))
    return {"bytes": rows * case["n_q"] * ((case["d_qk"] + case["d_v"]) * size + 4) + tokens * token_bytes
            + 4 * (tokens // case["page"]), "flops": 2 * pairs * case["n_q"] * (case["d_qk"] + case["d_v"])}


# ------------------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_attention(s):
    c = s["case"]
    out, lse = s["out"].double(), s["lse"].double()
    at = 0
    for b in range(c["batch"]):
        past, n = s["past_host"][b], s["new_host"][b]
        t = past + n
        held = s["table"][b, :-(-t // c["page"])].long().clamp(min=0)
        k = s["k"][held].transpose(0, 1).flatten(1, 2)[:, :t]
        v = s["v"][held].transpose(0, 1).flatten(1, 2)[:, :t]
        i, j = torch.arange(past, t, device=DEV)[:, None], torch.arange(t, device=DEV)[None]
        hidden = j > i
        if c["op"] == "window":
            hidden |= (i - j >= c["window"]) & (j >= c["sinks"])
        for h in range(c["n_q"]):
            x = s["q"][at:at + n, h].double() @ k[h * c["n_k"] // c["n_q"]].double().T * s["scale"]
            x = x.masked_fill(hidden, -math.inf)
            z = torch.logsumexp(x, 1)
            out[at:at + n, h] = torch.exp(x - z[:, None]) @ v[h * c["n_v"] // c["n_q"]].double()
            lse[at:at + n, h] = z
        at += n
    return {"out": out, "lse": lse}


def _exact_norm(s):
    c = s["case"]
    half = c["rot"] // 2
    q_out, k_pool, v_pool = s["out"].double(), s["k"].double(), s["v"].double()
    pair = torch.arange(half, device=DEV)
    one, two = (2 * pair, 2 * pair + 1) if c["interleaved"] else (pair, pair + half)
    at = 0
    for b in range(c["batch"]):
        past, n = s["past_host"][b], s["new_host"][b]
        pos = torch.arange(past, past + n, device=DEV)
        turn = torch.polar(torch.ones((n, 1, half), dtype=torch.float64, device=DEV),
                           torch.outer(pos.double(), s["inv_freq"])[:, None])
        page, slot = s["table"][b].long()[pos // c["page"]], pos % c["page"]
        turned = []
        for x, w in ((s["q"], s["q_weight"]), (s["k_new"], s["k_weight"])):
            x = x[at:at + n].double()
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["d_qk"] + s["eps"]) * w.double()
            z = torch.complex(x[..., one], x[..., two]) * turn
            x[..., one], x[..., two] = z.real, z.imag
            turned.append(x)
        q_out[at:at + n] = turned[0]
        k_pool[page, :, slot] = turned[1]
        v_pool[page, :, slot] = s["v_new"][at:at + n].double()
        at += n
    return {"q": q_out, "k": k_pool, "v": v_pool}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_norm(s) if case["op"] == "norm" else _exact_attention(s)
