"""The operators of a cache's life in a decode loop, through the public entry points and in plain torch: a row is rotated and
written, read for a batch that shares its first rows, weighed, and in the end dropped.

  op "append"  sfi_rope_append: rotary positions for the new rows' queries and keys, keys and values into the cache
  op "shared"  sfi_shared_attn: dense attention of a batch whose sequences hold the same first rows, which are read once
  op "weigh"   sfi_weight_attn: dense attention that adds every row's share of the softmax to the row's running weight
  op "evict"   sfi_evict: sink rows, the heaviest rows between and the recent rows, in their order, into a smaller cache

A case is one call.  The caches are flat tensors or pools of blocks with a block table, as a context of the library takes them.
Sequences' lengths run from `lo` to `hi` in even steps over the batch (the seed decides which sequence has which), so a
case's work does not depend on the seed.
"""
import math

import torch

own = False

D = 128
N_SINK = 4
BASE = 500000.0


def _case(op, batch, hq, hkv, lo, hi, **more):
    c = dict(op=op, batch=batch, hq=hq, hkv=hkv, lo=lo, hi=hi, page=0, layout="htd", out_bf16=False)
    c.update({"append": dict(new=1, rot=128, pairs="half", scaling="none", factor=1.0, far=0),
              "shared": dict(own_lo=1, own_hi=1, support=0.01),
              "weigh": dict(decay=1.0, support=0.01),
              "evict": dict(budget=0, recent=128, spare=64)}[op])
    assert set(more) <= set(c) | {"name"}
    c.update(more)
    return c


def listed():
    return [
        # every step of a few users on an 8B-class model: one row each, hardly any work
        _case("append", 4, 32, 8, 1000, 2000, name="append token"),
        # a prompt written into an empty cache in one go; queries, keys and values come out of one projection
        _case("append", 1, 32, 8, 8192, 8192, new=8192, scaling="turns", factor=8.0, name="append prompt"),
        # prompts of several requests at their own lengths, paged, half of each head rotated in the interleaved layout, at far positions
        _case("append", 16, 40, 8, 700, 2011, new=2011, rot=64, pairs="interleaved", scaling="dims", factor=4.0, far=900001, page=16,
              name="append prompts far paged"),
        # two dozen query columns per head over a short shared instruction: where latency counts
        _case("shared", 6, 8, 2, 2048, 2048, own_lo=16, own_hi=64, name="shared small"),
        # ordinary serving: a long system prompt, every user a conversation behind it, paged, outputs in the model's bf16
        _case("shared", 32, 32, 8, 16384, 16384, own_lo=100, own_hi=1201, page=16, out_bf16=True, name="shared system prompt"),
        # a document that many users ask about, a few hundred query columns per head
        _case("shared", 64, 64, 8, 32768, 32768, own_lo=33, own_hi=512, name="shared document"),
        # one stream with a short cache
        _case("weigh", 1, 8, 2, 2048, 2048, name="weigh tiny"),
        # the bounded caches of a batch, near the length at which they are cut again
        _case("weigh", 16, 32, 8, 4200, 6000, decay=0.98, name="weigh batch"),
        # long chain-of-thought generation on a paged cache
        _case("weigh", 8, 40, 8, 20011, 24571, page=16, support=0.0, out_bf16=True, name="weigh cot paged"),
        # one short cache cut to a quarter
        _case("evict", 1, 8, 2, 4096, 4096, budget=960, recent=64, name="evict tiny"),
        # the bounded caches of a batch, cut once they have grown by half
        _case("evict", 16, 32, 8, 5800, 6200, budget=3960, recent=128, name="evict batch"),
        # after long prompts: what is kept of each goes into a small paged cache
        _case("evict", 4, 32, 8, 30011, 60000, budget=4001, recent=256, page=16, name="evict prompts paged"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: batches of 1 to 64, caches of 1 to 60000 rows, groups of 1 to 16 heads."""
    while True:
        op = rng.choice(["append", "shared", "weigh", "evict"])
        hkv = rng.choice([1, 2, 4, 8, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
        batch = _log_int(rng, 1, 64)
        more = dict(page=rng.choice([0, 0, 16, 64]), layout=rng.choice(["htd", "thd"]), out_bf16=rng.random() < 0.3)
        if op == "append":
            hi = _log_int(rng, 1, 8192)
            new = rng.choice([1, min(hi, _log_int(rng, 1, 64)), hi])
            scaling = rng.choice(["none", "linear", "turns", "dims"])
            more.update(new=new, rot=rng.choice([16, 32, 64, 96, 128, 128, 128]), pairs=rng.choice(["half", "interleaved"]), scaling=scaling,
                        factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]), far=rng.choice([0, rng.randint(1, 1000000)]),
                        out_bf16=False)
        elif op == "shared":
            hi = _log_int(rng, 64, 40000)
            own_hi = _log_int(rng, 1, 2000)
            more.update(own_hi=own_hi, own_lo=rng.choice([0, 1, own_hi, max(1, own_hi // 3)]), support=rng.choice([0.0, 0.01]))
        elif op == "weigh":
            hi = _log_int(rng, 1, 40000)
            more.update(decay=rng.choice([1.0, 0.9, 0.99]), support=rng.choice([0.0, 0.01]))
        else:
            hi = _log_int(rng, 200, 60000)
            more.update(budget=_log_int(rng, 1, min(6000, hi)), recent=rng.choice([1, 64, 128, rng.randint(1, 300)]), spare=rng.randint(0, 100))
        lo = max(1, int(hi * rng.choice([1.0, rng.uniform(0.25, 1.0)])))
        c = _case(op, batch, hq, hkv, lo, hi, **more)
        rows = c["hi"] + c.get("own_hi", 0)
        w = work(c)
        # no more work than the largest listed cases, and no cache of more than 3 GB
        if 4 * batch * hkv * rows * D <= 3e9 and w["bytes"] <= 9e8 and w["flops"] <= 7e10:
            return c


def _lengths(c):
    """Length of the sequence of each rank, shortest first: rows of the cache, for "shared" the rows it shares with the first sequence."""
    n, lo, hi = c["batch"], c["lo"], c["hi"]
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _own_lengths(c):
    n, lo, hi = c["batch"], c["own_lo"], c["own_hi"]
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _new_rows(c, length):
    return min(c["new"], length)


def _kept(c, length):
    """(rows between sink and recent rows that are kept, rows of the cache afterwards)."""
    n_j = max(0, length - c["recent"] - N_SINK)
    k = min(c["budget"], n_j)
    return k, length - n_j + k


def _cache(c, gen, rows, zero):
    """K and V of `rows` rows for every sequence (flat [B, Hkv, rows, D], or pools of blocks), and the block table."""
    b, hkv, page = c["batch"], c["hkv"], c["page"]
    if page:
        per = (rows + page - 1) // page
        shape = (b * per, hkv, page, D) if c["layout"] == "htd" else (b * per, page, hkv, D)
        table = torch.randperm(b * per, generator=gen, device="cuda").to(torch.int32).view(b, per)
    else:
        shape, table = (b, hkv, rows, D), None
    K = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    if not zero:
        K.normal_(generator=gen)
        V.normal_(generator=gen)
        if c.get("support"):
            x4 = torch.rand(shape[:-1], generator=gen, device="cuda") < c["support"]
            K.mul_((1 + 3 * x4).to(torch.bfloat16).unsqueeze(-1))
    return K, V, table


def _context(c, cache, rows, budget, recent):
    from paper_2603_12038_amd.binding import SfiContext, sfi_set_block_table
    ctx = SfiContext(c["batch"], c["hq"], c["hkv"], rows, budget, N_SINK, recent, cache["K"], cache["V"], page_size=c["page"],
                     page_layout=c["layout"], out_bf16=c["out_bf16"])
    if cache["table"] is not None:
        sfi_set_block_table(ctx.handle, cache["table"], cache["table"].numel())
    return ctx


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    b, hq, hkv = c["batch"], c["hq"], c["hkv"]
    order = torch.randperm(b, generator=gen, device="cuda").tolist()
    ranked = _lengths(c)
    lens = [ranked[r] for r in order]
    s = {"case": c, "lens": lens}
    if c["op"] == "append":
        rows, new = c["hi"], c["new"]
        s["qkv"] = torch.empty((b, new, hq + 2 * hkv, D), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        s["q"], s["k"], s["v"] = s["qkv"].split([hq, hkv, hkv], dim=2)
        n_new = [_new_rows(c, n) for n in lens]
        s["n_new"] = _i32(n_new)
        first = [n - m for n, m in zip(lens, n_new)]
        s["pos"] = _i32([r + c["far"] for r in first]) if c["far"] else None
        s["q_out"] = torch.zeros((b, new, hq, D), dtype=torch.bfloat16, device="cuda")
        # the tokens that are no padding, as (sequence, place in the batch of new rows, cache row, position)
        s["token"] = torch.tensor([(i, t, first[i] + t, first[i] + t + c["far"]) for i in range(b) for t in range(n_new[i])], device="cuda").T.contiguous()
    elif c["op"] == "shared":
        ranked_own = _own_lengths(c)
        shared = [c["hi"] if i == 0 else n for i, n in enumerate(lens)]  # the first sequence holds all of the shared rows
        lens = [n + ranked_own[r] for n, r in zip(shared, order)]
        rows = c["hi"] + c["own_hi"]
        s["shared_len"] = _i32(shared)
        s["lens"], s["shared"] = lens, shared
    else:
        rows = c["hi"]
    s["ctx_len"] = _i32(s["lens"])
    s["K"], s["V"], s["table"] = _cache(c, gen, rows, c["op"] == "append")
    s["rows"] = rows
    if c["op"] in ("shared", "weigh"):
        s["q"] = torch.empty((b, hq, D), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        s["out"] = torch.zeros((b, hq, D), dtype=torch.bfloat16 if c["out_bf16"] else torch.float32, device="cuda")
    if c["op"] in ("weigh", "evict"):
        # what earlier steps have left: a few heavy rows, many light ones, some that have never been looked at
        w = torch.empty((b, hkv, rows), device="cuda").normal_(generator=gen).mul_(3.0).exp_().mul_(0.1 / rows)
        w.mul_(torch.rand((b, hkv, rows), generator=gen, device="cuda") > 0.05)
        s["weights"] = w
    if c["op"] == "weigh":
        s["weights_out"] = torch.zeros_like(s["weights"])
    budget, recent = c.get("budget", 0), c.get("recent", 128)
    if c["op"] == "evict":
        rows_out = max(_kept(c, n)[1] for n in s["lens"]) + c["spare"]
        small = {}
        small["K"], small["V"], small["table"] = _cache(c, gen, rows_out, True)
        small["rows"] = rows_out
        small["weights"] = torch.zeros((b, hkv, rows_out), device="cuda")
        small["row_pos"] = torch.zeros((b, hkv, rows_out), dtype=torch.int32, device="cuda")
        small["ctx_len"] = torch.zeros(b, dtype=torch.int32, device="cuda")
        s["small"] = small
        s["row_pos"] = torch.arange(rows, dtype=torch.int32, device="cuda").expand(b, hkv, rows).contiguous()
        s["kept"] = torch.zeros((b, hkv, budget), dtype=torch.int32, device="cuda")
        s["n_kept"] = torch.zeros((b, hkv), dtype=torch.int32, device="cuda")
    if own:
        s["ctx"] = _context(c, s, rows, budget, recent)
        s["h"] = s["ctx"].handle
        if c["op"] == "append":
            from paper_2603_12038_amd import sfi_set_rope
            scaling = {"none": None, "linear": dict(kind="linear", factor=c["factor"]),
                       "turns": dict(kind="turns", factor=c["factor"], low=1.0, high=4.0, orig_ctx=8192),
                       "dims": dict(kind="dims", factor=c["factor"], low=1.0, high=32.0, orig_ctx=8192)}[c["scaling"]]
            sfi_set_rope(s["h"], c["rot"], BASE, interleaved=c["pairs"] == "interleaved", scaling=scaling, magnitude=_magnitude(c))
        if c["op"] == "evict":
            s["small"]["ctx"] = _context(c, s["small"], s["small"]["rows"], budget, recent)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "dims" else 1.0


def _freqs(c):
    """Radians per position of each pair, in 64 bits."""
    n = c["rot"]
    i = torch.arange(n // 2, dtype=torch.float64, device="cuda")
    f = BASE ** (-2.0 * i / n)
    if c["scaling"] == "linear":
        return f / c["factor"]
    if c["scaling"] == "turns":  # pairs that turn often within the trained context are left, those that turn seldom are stretched
        keep = ((8192.0 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / c["factor"])
    if c["scaling"] == "dims":  # the same with a ramp along the pairs' numbers
        lo = max(math.floor(n * math.log(8192 / (2 * math.pi * 32.0)) / (2 * math.log(BASE))), 0)
        hi = min(math.ceil(n * math.log(8192 / (2 * math.pi * 1.0)) / (2 * math.log(BASE))), n - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * ((1.0 - ramp) + ramp / c["factor"])
    return f


def _rotate(c, x, angle):
    """x: [tokens, heads, D] in 32 bits, angle: [tokens, pairs] in 64 bits."""
    rot = c["rot"]
    cos, sin = (angle.cos() * _magnitude(c)).float()[:, None], (angle.sin() * _magnitude(c)).float()[:, None]
    head, rest = x[..., :rot], x[..., rot:]
    if c["pairs"] == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, rest), dim=-1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2), rest), dim=-1)


def _put(c, pool, table, seq, row, values):
    """Rows `row` of sequences `seq` of a cache: values [n, Hkv, D]."""
    if not c["page"]:
        pool[seq, :, row] = values
    elif c["layout"] == "htd":
        pool[table[seq, row // c["page"]].long(), :, row % c["page"]] = values
    else:
        pool[table[seq, row // c["page"]].long(), row % c["page"]] = values


def _rows(c, pool, table, seq, row):
    """Rows row[...] of sequences seq[...] as [..., Hkv, D]."""
    if not c["page"]:
        return pool.transpose(1, 2)[seq, row]
    if c["layout"] == "htd":
        return pool.transpose(1, 2)[table[seq, row // c["page"]].long(), row % c["page"]]
    return pool[table[seq, row // c["page"]].long(), row % c["page"]]


def _append(s):
    c = s["case"]
    seq, place, row, position = s["token"]
    angle = position.double()[:, None] * _freqs(c)
    s["q_out"][seq, place] = _rotate(c, s["q"][seq, place].float(), angle).to(torch.bfloat16)
    _put(c, s["K"], s["table"], seq, row, _rotate(c, s["k"][seq, place].float(), angle).to(torch.bfloat16))
    _put(c, s["V"], s["table"], seq, row, s["v"][seq, place])
    return s["q_out"], s["K"], s["V"]


def _store(s, o):
    s["out"].copy_(o)
    return s["out"]


def _shared(s):
    c = s["case"]
    b, hq, hkv = c["batch"], c["hq"], c["hkv"]
    g, n, m = hq // hkv, c["hi"], c["own_hi"]
    scale = 1.0 / math.sqrt(D)
    q = s["q"].float().view(b, hkv, g, D)
    shared, length = s["shared_len"].long(), s["ctx_len"].long()
    at = torch.arange(n, device="cuda")
    first = torch.zeros_like(at)
    K = _rows(c, s["K"], s["table"], first, at).float().transpose(0, 1)  # [Hkv, n, D] of the first sequence
    V = _rows(c, s["V"], s["table"], first, at).float().transpose(0, 1).contiguous()
    y = torch.matmul(q.permute(1, 0, 2, 3).reshape(hkv, b * g, D), K.transpose(1, 2).contiguous()).view(hkv, b, g, n).permute(1, 0, 2, 3) * scale
    y = y.masked_fill((at >= shared[:, None])[:, None, None], -math.inf)
    seq = torch.arange(b, device="cuda")[:, None]
    row = shared[:, None] + torch.arange(m, device="cuda")
    there = row < length[:, None]
    row = torch.where(there, row, 0)
    k = _rows(c, s["K"], s["table"], seq, row).float().permute(0, 2, 3, 1).contiguous()  # [B, Hkv, D, m]
    v = _rows(c, s["V"], s["table"], seq, row).float().transpose(1, 2).contiguous()
    z = (torch.matmul(q, k) * scale).masked_fill(~there[:, None, None], -math.inf)
    top = torch.maximum(y.amax(-1, keepdim=True), z.amax(-1, keepdim=True))
    y, z = (y - top).exp(), (z - top).exp()
    norm = y.sum(-1, keepdim=True) + z.sum(-1, keepdim=True)
    o = torch.matmul(y.permute(1, 0, 2, 3).reshape(hkv, b * g, n), V).view(hkv, b, g, D).permute(1, 0, 2, 3) + torch.matmul(z, v)
    return _store(s, (o / norm).reshape(b, hq, D))


def _all_rows(s, pool):
    """The whole cache as [B, Hkv, rows, D] in 32 bits."""
    c = s["case"]
    if not c["page"]:
        return pool.float()
    seq = torch.arange(c["batch"], device="cuda")[:, None]
    return _rows(c, pool, s["table"], seq, torch.arange(s["rows"], device="cuda")[None]).transpose(1, 2).float().contiguous()


def _weigh(s):
    c = s["case"]
    b, hq, hkv = c["batch"], c["hq"], c["hkv"]
    q = s["q"].float().view(b, hkv, hq // hkv, D)
    there = torch.arange(s["rows"], device="cuda") < s["ctx_len"][:, None]
    y = torch.matmul(q, _all_rows(s, s["K"]).transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    y = y.masked_fill(~there[:, None, None], -math.inf)
    p = (y - y.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p, _all_rows(s, s["V"]))
    s["weights_out"].copy_(torch.where(there[:, None], c["decay"] * s["weights"] + p.mean(2), s["weights_out"]))
    return _store(s, o.view(b, hq, D)), s["weights_out"]


def _evict(s):
    c, small = s["case"], s["small"]
    b, hkv, n, m, k = c["batch"], c["hkv"], s["rows"], small["rows"], c["budget"]
    length = s["ctx_len"].long()[:, None, None]
    at = torch.arange(n, device="cuda")
    among = (at >= N_SINK) & (at < length - c["recent"])
    w = torch.where(s["weights"] > 0, s["weights"], 0.0)
    best = torch.where(among, w, -1.0).sort(dim=-1, descending=True, stable=True).indices[..., :k]
    n_j = (length - c["recent"] - N_SINK).clamp(min=0)
    n_kept = n_j.clamp(max=k)
    nth = torch.arange(k, device="cuda")
    kept = torch.where(nth < n_kept, best, n).sort(dim=-1).values
    s["kept"].copy_(torch.where(nth < n_kept, kept, -1))
    s["n_kept"].copy_(n_kept[..., 0].expand(b, hkv))
    after = length - n_j + n_kept
    to = torch.arange(m, device="cuda").expand(b, hkv, m)
    sink = length.clamp(max=N_SINK)
    middle = torch.gather(kept, 2, (to - sink).clamp(0, k - 1))
    source = torch.where(to < sink, to, torch.where(to < sink + n_kept, middle, to + (length - after)))
    live = to < after
    source = torch.where(live, source, 0)
    small["weights"].copy_(torch.where(live, torch.gather(s["weights"], 2, source), 0.0))
    small["row_pos"].copy_(torch.where(live, torch.gather(s["row_pos"], 2, source), small["row_pos"]))
    small["ctx_len"].copy_(after[:, 0, 0])
    seq = torch.arange(b, device="cuda")[:, None, None]
    head = torch.arange(hkv, device="cuda")[:, None]
    if not c["page"]:
        src, dst = (seq, head, source), (seq, head, to)
    else:
        page = c["page"]
        sb, db = s["table"][seq, source // page].long(), small["table"][seq, to // page].long()
        src = (sb, head, source % page) if c["layout"] == "htd" else (sb, source % page, head)
        dst = (db, head, to % page) if c["layout"] == "htd" else (db, to % page, head)
    small["K"][dst] = torch.where(live[..., None], s["K"][src], small["K"][dst])
    small["V"][dst] = torch.where(live[..., None], s["V"][src], small["V"][dst])
    return small["K"], small["V"], small["weights"], small["row_pos"], small["ctx_len"], s["kept"], s["n_kept"]


def run(s):
    c = s["case"]
    if not own:
        return {"append": _append, "shared": _shared, "weigh": _weigh, "evict": _evict}[c["op"]](s)
    import paper_2603_12038_amd as sfi
    if c["op"] == "append":
        sfi.sfi_rope_append(s["h"], s["q"], s["k"], s["v"], s["ctx_len"], s["n_new"], s["pos"], s["q_out"], s["K"], s["V"])
        return s["q_out"], s["K"], s["V"]
    if c["op"] == "shared":
        sfi.sfi_shared_attn(s["h"], s["q"], s["K"], s["V"], s["ctx_len"], s["shared_len"], 0, c["hi"], s["rows"], s["out"])
        return s["out"]
    if c["op"] == "weigh":
        sfi.sfi_weight_attn(s["h"], s["q"], s["K"], s["V"], s["ctx_len"], s["rows"], c["decay"], s["weights"], s["weights_out"], s["out"])
        return s["out"], s["weights_out"]
    small = s["small"]
    sfi.sfi_evict(s["h"], s["K"], s["V"], s["ctx_len"], s["rows"], c["budget"], s["weights"], s["row_pos"], small["ctx"].handle,
                  small["K"], small["V"], small["ctx_len"], None, small["weights"], small["row_pos"], s["kept"], s["n_kept"])
    return small["K"], small["V"], small["weights"], small["row_pos"], small["ctx_len"], s["kept"], s["n_kept"]


def work(case):
    """What each operator cannot do without: the new rows read and written; the shared rows once, every other row once, and four
    operations per element of a row and query head; the rows that are kept read and written and the weights looked at."""
    c = case
    g = c["hq"] // c["hkv"]
    heads = c["hq"] + 2 * c["hkv"]
    io = c["batch"] * c["hq"] * D * (2 + (2 if c["out_bf16"] else 4))
    if c["op"] == "append":
        tokens = sum(_new_rows(c, n) for n in _lengths(c))
        return {"bytes": tokens * heads * D * 4, "flops": tokens * (c["hq"] + c["hkv"]) * c["rot"] * 3}
    if c["op"] == "shared":
        own_rows = sum(_own_lengths(c))
        seen = own_rows + sum(_lengths(c))
        return {"bytes": (c["hi"] + own_rows) * c["hkv"] * 4 * D + io, "flops": seen * c["hkv"] * 4 * g * D}
    if c["op"] == "weigh":
        rows = sum(_lengths(c)) * c["hkv"]
        return {"bytes": rows * (4 * D + 8) + io, "flops": rows * 4 * g * D}
    kept = sum(_kept(c, n)[1] for n in _lengths(c)) * c["hkv"]
    looked = sum(_lengths(c)) * c["hkv"]
    return {"bytes": kept * (8 * D + 16) + looked * 4, "flops": looked}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _sequence(s, pool, i, n):
    """Rows [0, n) of sequence i as [Hkv, n, D], in 64 bits."""
    c = s["case"]
    if not c["page"]:
        return pool[i, :, :n].double()
    pages = pool[s["table"][i, :(n + c["page"] - 1) // c["page"]].long()]
    if c["layout"] == "thd":
        pages = pages.transpose(1, 2)
    return pages.transpose(0, 1).reshape(c["hkv"], -1, D)[:, :n].double()


def _attention(q, K, V):
    """q: [Hq, D], K, V: [Hkv, n, D] in 64 bits -> output [Hq, D] and softmax weights [Hq, n]."""
    g = q.shape[0] // K.shape[0]
    K, V = K.repeat_interleave(g, 0), V.repeat_interleave(g, 0)
    p = torch.softmax((K * q[:, None]).sum(-1) / math.sqrt(D), dim=-1)
    return (p[..., None] * V).sum(1), p


def _turning(c, i):
    """Radians per position of pair i."""
    period = 2 * math.pi * math.exp(math.log(BASE) * 2 * i / c["rot"])  # positions per turn, unscaled
    stretched = period * c["factor"]
    if c["scaling"] == "turns":
        keep = min(1.0, max(0.0, (8192 / period - 1.0) / 3.0))
    elif c["scaling"] == "dims":
        def pair_with(turns):  # the pair that makes so many turns in the trained context
            return c["rot"] / 2 * math.log(8192 / turns / (2 * math.pi)) / math.log(BASE)
        lo, hi = max(0, math.floor(pair_with(32.0))), min(c["rot"] - 1, math.ceil(pair_with(1.0)))
        keep = 1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
    else:
        keep = 0.0
    return keep * 2 * math.pi / period + (1.0 - keep) * 2 * math.pi / stretched


def exact(case, seed):
    global own
    kept_own, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept_own
    c = s["case"]
    b = c["batch"]
    if c["op"] == "append":
        rot, half = c["rot"], c["rot"] // 2
        q_out = torch.zeros(s["q_out"].shape, dtype=torch.float64, device="cuda")
        K = torch.zeros(s["K"].shape, dtype=torch.float64, device="cuda")
        V = torch.zeros_like(K)
        f = torch.tensor([_turning(c, i) for i in range(half)], dtype=torch.float64, device="cuda")
        gain = 1.0 if c["scaling"] != "dims" else 1.0 + math.log(c["factor"]) / 10.0
        for i in range(b):
            n = _new_rows(c, s["lens"][i])
            r0 = s["lens"][i] - n
            row = torch.arange(r0, r0 + n, device="cuda")
            turn = torch.polar(torch.full((n, half), gain, dtype=torch.float64, device="cuda"), (row + c["far"])[:, None] * f)[:, None]

            def rotated(x):
                x = x.double().clone()
                even, odd = (slice(0, half), slice(half, rot)) if c["pairs"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
                z = torch.complex(x[..., even], x[..., odd]) * turn
                x[..., even], x[..., odd] = z.real, z.imag
                return x

            q_out[i, :n] = rotated(s["q"][i, :n])
            for dst, val in ((K, rotated(s["k"][i, :n])), (V, s["v"][i, :n].double())):
                if not c["page"]:
                    dst[i, :, r0:r0 + n] = val.transpose(0, 1)
                else:
                    blk = s["table"][i].long()[row // c["page"]]
                    if c["layout"] == "htd":
                        dst[blk, :, row % c["page"]] = val
                    else:
                        dst[blk, row % c["page"]] = val
        return q_out, K, V
    if c["op"] == "shared":
        lead = (_sequence(s, s["K"], 0, c["hi"]), _sequence(s, s["V"], 0, c["hi"]))
        out = []
        for i in range(b):
            n, m = s["shared"][i], s["lens"][i]
            mine = (_sequence(s, s["K"], i, m), _sequence(s, s["V"], i, m))
            K, V = (torch.cat((a[:, :n], x[:, n:]), dim=1) for a, x in zip(lead, mine))
            out.append(_attention(s["q"][i].double(), K, V)[0])
        return torch.stack(out)
    if c["op"] == "weigh":
        g = c["hq"] // c["hkv"]
        out, weights = [], torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda")
        for i in range(b):
            n = s["lens"][i]
            o, p = _attention(s["q"][i].double(), _sequence(s, s["K"], i, n), _sequence(s, s["V"], i, n))
            out.append(o)
            weights[i, :, :n] = c["decay"] * s["weights"][i, :, :n].double() + p.view(c["hkv"], g, n).mean(1)
        return torch.stack(out), weights
    # rows are moved, not computed: only the moved weights are numbers
    small = s["small"]
    w = torch.zeros(small["weights"].shape, dtype=torch.float64)
    weights = s["weights"].double().cpu()
    for i in range(b):
        n = s["lens"][i]
        k, after = _kept(c, n)
        for h in range(c["hkv"]):
            row = weights[i, h, :n]
            sinks, recent = row[:min(N_SINK, n)], row[max(min(N_SINK, n), n - c["recent"]):]
            middle = row[N_SINK:N_SINK + n - c["recent"] - N_SINK] if n > c["recent"] + N_SINK else row[:0]
            best = sorted(range(len(middle)), key=lambda j, m=middle.tolist(): (-m[j], j))[:k]
            w[i, h, :after] = torch.cat((sinks, middle[sorted(best)], recent))
    return None, None, w.cuda(), None, None, None, None
