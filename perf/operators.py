"""Performance cases of the paged cache: what happens to a compressed cache after the prompt, when
new tokens come in one by one.

Four kinds of pass:
  tables   the page tables of every (layer, sequence, KV head), from row counts: `admit` takes the
           selection of new prompts, `extend` a decode step (some sequences idle, some released)
  fill     the retained rows of the prompts gathered into their pages
  rotate   rotary positions of a prompt's queries and keys, or (backward) of their gradients; and
           `append`, the single-token form that writes the new key and value rows into the pages
  attend   attention of one new token per sequence over the pages

Row counts of heads are uneven, as a layer-wide selection leaves them.  They belong to the case;
the seed draws the pages that they lie in and all values.  Rows of a page behind a head's last row
are uninitialised memory in earnest: NaN in the cases that say so.
"""
from __future__ import annotations

import math

import torch

own = False


# ----------------------------------------------------------------------------- cases
def _case(kind, **kw):
    c = dict(kind=kind, layers=1, q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", batch=1, rows=128,
             len_seed=1, page_rows=64)
    if kind == "tables":
        c.update(form="extend", tokens=1, others=0)
    if kind == "fill":
        c.update(tokens=1021, window=32, held=0)
    if kind in ("rotate", "append"):
        c.update(tokens=1, rotary_dim=128, layout="halves", scaling="plain", base=500000.0, start=0)
    if kind == "rotate":
        c.update(backward=False)
    if kind == "attend":
        c.update(softcap=0.0, empty=False, garbage=False)
    c.update(kw)
    return c


def listed():
    return [
        # page tables of a decode step: 32 layers, a serving batch of 8, one token each
        _case("tables", name="tables_token", layers=32, batch=8, rows=600),
        # the prompts of a batch get their pages: 32K contexts at 2048 rows per head, beside running ones
        _case("tables", name="tables_prompts", form="admit", layers=32, batch=4, rows=2048, others=4),
        # the retained rows of a short chat prompt, all layers
        _case("fill", name="fill_1k", layers=32, rows=128),
        # the retained rows of the headline workload
        _case("fill", name="fill_32k", layers=32, tokens=32768, rows=2048),
        # queries and keys of one layer of a 32K prompt, frequencies scaled for long contexts
        _case("rotate", name="rotate_32k", tokens=32768, scaling="bands"),
        # gradients of a training step far into a long context, adjacent pairs, half of the head, fp32
        _case("rotate", name="rotate_grad_f32", tokens=2049, dtype="f32", rotary_dim=64, layout="pairs",
              scaling="ramp", base=10000.0, start=129022, backward=True),
        # one new token of one sequence: latency
        _case("append", name="append_token", start=32768),
        # one new token of each of 256 sequences
        _case("append", name="append_256", batch=256, start=5000),
        # one fp32 layer of a small model with capped logits, one of three sequences empty: latency
        _case("attend", name="attend_tiny_f32", q_heads=4, kv_heads=2, head_dim=64, dtype="f32", batch=3, rows=64,
              page_rows=16, softcap=30.0, empty=True, garbage=True),
        # one layer of a serving batch of ragged prompts at strong compression
        _case("attend", name="attend_batch", batch=8, rows=150, garbage=True),
        # all layers of a 128K context, seven query heads per KV head, capped logits
        _case("attend", name="attend_gqa7", layers=28, q_heads=28, kv_heads=4, rows=1024, page_rows=128, softcap=50.0),
        # one layer of a large serving batch of long contexts: bound by the read of the cache
        _case("attend", name="attend_large", batch=64, rows=2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["tables", "fill", "rotate", "append", "attend"], [3, 2, 3, 2, 6])[0]
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (28, 4), (8, 2), (32, 4), (16, 16), (32, 2)])
    dtype, head_dim = rng.choices([("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)], [6, 2, 1, 1])[0]
    es = 2 if dtype == "bf16" else 4
    c = _case(kind, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype,
              len_seed=rng.randrange(1 << 20), page_rows=rng.choice([16, 32, 64, 64, 128, 256]))
    if kind == "tables":
        c["layers"] = rng.choice([1, 4, 16, 28, 32])
        c["batch"] = _log_int(rng, 1, max(1, 2048 // (c["layers"] * kv_heads)))
        c["rows"] = _log_int(rng, 1, 4096)
        c["form"] = rng.choice(["admit", "extend", "extend"])
        if c["form"] == "admit":
            c["others"] = rng.randrange(0, 5)
        else:
            c["tokens"] = rng.choice([1, 1, 1, 5, 32])
    elif kind == "fill":
        c["layers"] = rng.choice([1, 4, 16, 28, 32])
        c["batch"] = rng.choice([1, 1, 3, 8])
        most = 4.2e9 / (2 * c["layers"] * kv_heads * head_dim * es * c["batch"])
        c["tokens"] = _log_int(rng, 100, min(131072, most))
        c["window"] = rng.choice([16, 32, 64])
        c["rows"] = max(c["window"], min(c["tokens"] // 3, _log_int(rng, 64, 4096)))
        c["held"] = rng.choice([0, 0, 7, 100])
    elif kind in ("rotate", "append"):
        if kind == "rotate":
            most = 32768 * 40 * 128 * 2 / ((q_heads + kv_heads) * head_dim * es)
            c["tokens"] = _log_int(rng, 1, most)
            c["backward"] = rng.random() < 0.4
        else:
            c["batch"] = _log_int(rng, 1, 256)
            c["tokens"] = rng.choice([1, 1, 1, 5])
        c["rotary_dim"] = rng.choice([head_dim, head_dim, head_dim // 2, 16, 48])
        c["layout"] = rng.choice(["halves", "halves", "pairs"])
        c["scaling"] = rng.choice(["plain", "linear", "base", "bands", "ramp"])
        c["base"] = rng.choice([10000.0, 500000.0])
        c["start"] = rng.choice([0, _log_int(rng, 1, 2000000)])
    else:
        c["layers"] = rng.choice([1, 1, 1, 4, 28])
        c["batch"] = _log_int(rng, 1, 64)
        heads = c["layers"] * c["batch"] * kv_heads
        # rows: as many as the largest listed case reads, and room for the plain form's padding
        most = 64 * 8 * 2048 * 128 * 2 / (heads * head_dim * es)
        c["rows"] = _log_int(rng, 1, max(2, min(100000, most, 6e9 / (heads * 4 * (4 * head_dim + q_heads // kv_heads * 4)))))
        c["softcap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        c["empty"] = rng.random() < 0.3
        c["garbage"] = rng.random() < 0.5
    return c


# ----------------------------------------------------------------------------- inputs
def _row_counts(c, batch=None):
    """Rows per (layer, sequence, KV head): uneven by a factor of ten or so, at most four times the mean."""
    g = torch.Generator().manual_seed(c["len_seed"])
    batch = c["batch"] if batch is None else batch
    x = torch.exp(0.8 * torch.randn((c["layers"], batch, c["kv_heads"]), generator=g, dtype=torch.float64))
    n = (c["rows"] * x / x.mean()).round().clamp(1, 4 * c["rows"]).long()
    if c.get("empty") and batch > 1:
        n[:, 1] = 0
    return n


def _added(c):
    """Rows that a decode step adds to each sequence: -1 for one that is released."""
    g = torch.Generator().manual_seed(c["len_seed"] + 1)
    add = torch.randint(1, c["tokens"] + 1, (c["batch"],), generator=g)
    add[4::5] = 0
    if c["batch"] > 2:
        add[2] = -1
    return add


def _ceil(a, b):
    return -(-a // b)


def _pages(c, rows, spare, g):
    """A page table for these rows and the ring of free pages, pages in random order."""
    ps = c["page_rows"]
    held = _ceil(rows, ps)
    used = int(held.sum())
    n_pages = max(1, used + spare)
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    most = int(_ceil(4 * c["rows"] + c.get("tokens", 0) + c.get("held", 0) + 1, ps))
    first = (held.reshape(-1).cumsum(0) - held.reshape(-1)).view(*held.shape, 1)
    col = torch.arange(most).expand(*held.shape, most)
    at = torch.where(col < held.unsqueeze(-1), first + col, -1).cuda()
    table = torch.where(at >= 0, order[at.clamp(min=0)], -1).int()
    taken = int(torch.randint(0, n_pages, (1,), generator=g, device="cuda"))
    free = torch.empty_like(order)
    free[(taken + torch.arange(n_pages, device="cuda")) % n_pages] = order.roll(-used)
    counters = torch.tensor([taken, taken + n_pages - used], dtype=torch.int64, device="cuda")
    return n_pages, most, table, free, counters


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, L, B, H, Hq, d, ps = _dtype(c), c["layers"], c["batch"], c["kv_heads"], c["q_heads"], c["head_dim"], c["page_rows"]

    def randn(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)

    s = dict(c=c)
    if c["kind"] == "tables":
        if c["form"] == "extend":
            rows = _row_counts(c)
            s["add"] = _added(c).int().cuda()
            s["slots"] = torch.empty((L, B, c["tokens"], H), dtype=torch.int32, device="cuda")
            spare = 3 + L * B * H * _ceil(c["tokens"], ps)
        else:
            # sequences [others, others + batch) of the cache are new, the others hold rows
            every = _row_counts(c, c["others"] + B)
            rows, new = every.clone(), every[:, c["others"]:]
            rows[:, c["others"]:] = 0
            hoff = torch.zeros((L, B, H + 1), dtype=torch.int64)
            hoff[:, :, 1:] = new.cumsum(2)
            s["head_offsets"] = hoff.int().cuda()
            s["first_row"] = torch.empty((L, B, H), dtype=torch.int32, device="cuda")
            spare = 3 + int(_ceil(new, ps).sum())
        s["n_pages"], s["max_pages"], s["table"], s["free"], s["counters"] = _pages(c, rows, spare, g)
        s["head_rows"] = rows.int().cuda()
        s["rows_out"], s["counters_out"] = torch.empty_like(s["head_rows"]), torch.empty_like(s["counters"])
    elif c["kind"] == "fill":
        n, w, T = c["tokens"], c["window"], c["tokens"] * B
        P = n - w
        s["k"], s["v"] = randn(L, H, T, d), randn(L, H, T, d)
        k = min(H * (c["rows"] - w), H * P)
        # heads weigh differently, so a layer-wide choice leaves them uneven numbers of rows
        weight = torch.exp(0.5 * torch.randn((L, B, H, 1), generator=g, device="cuda"))
        hoff = torch.zeros((L, B, H + 1), dtype=torch.int64, device="cuda")
        keep = torch.zeros((L, B, H * P), dtype=torch.int32, device="cuda")
        for b in range(B):
            flat = (torch.rand((L, H, P), generator=g, device="cuda") * weight[:, b]).reshape(L, H * P)
            best = flat.topk(k, dim=1, sorted=False).indices.sort(dim=1).values
            count = torch.zeros((L, H), dtype=torch.int64, device="cuda")
            count.scatter_add_(1, best // P, torch.ones_like(best))
            hoff[:, b, 1:] = (count + w).cumsum(1)
            keep[:, b, :k] = (best % P).int()
        s["keep_idx"], s["head_offsets"] = keep.view(L, -1), hoff.int()
        rows = (hoff[:, :, 1:] - hoff[:, :, :-1]).cpu()
        s["most"] = int(rows.max())
        c["rows"] = max(c["rows"], _ceil(s["most"], 4))
        # the pool holds any spread of the rows over the heads: up to a page per head more than they fill
        pool = L * B * (_ceil(H * (w + c["held"]) + k, ps) + H)
        held = rows + c["held"]
        s["n_pages"], s["max_pages"], s["table"], _, _ = _pages(c, held, pool - int(_ceil(held, ps).sum()), g)
        s["first_row"] = torch.full((L, B, H), c["held"], dtype=torch.int32, device="cuda")
        s["k_pages"] = torch.zeros((s["n_pages"], ps, d), dtype=dt, device="cuda")
        s["v_pages"] = torch.zeros_like(s["k_pages"])
        s["cu_seqlens"] = torch.arange(0, T + 1, n, dtype=torch.int32, device="cuda")
    elif c["kind"] in ("rotate", "append"):
        N = c["tokens"] * (B if c["kind"] == "append" else 1)
        # the projections' output: queries, keys and values of a token side by side
        s["qkv"] = randn(N, (Hq + 2 * H) * d)
        s["q"] = s["qkv"][:, : Hq * d].view(N, Hq, d)
        s["k"] = s["qkv"][:, Hq * d: (Hq + H) * d].view(N, H, d)
        s["v"] = s["qkv"][:, (Hq + H) * d:].view(N, H, d)
        freqs, s["scale"] = frequencies(c)
        s["freqs"] = freqs.cuda()
        s["q_out"] = torch.empty((N, Hq, d), dtype=dt, device="cuda")
        if c["kind"] == "rotate":
            s["positions"] = (c["start"] + torch.arange(N, device="cuda")).int()
            # keys in the order that the score step reads, [H_kv, tokens, d]
            s["k_out"] = torch.empty((H, N, d), dtype=dt, device="cuda").permute(1, 0, 2)
        else:
            first = c["start"] + torch.randint(0, 4000, (B, 1), generator=g, device="cuda")
            s["positions"] = (first + torch.arange(c["tokens"], device="cuda")).int().reshape(-1)
            heads = B * H
            s["n_pages"], s["max_pages"] = heads, 1
            page = torch.randperm(heads, generator=g, device="cuda").view(B, 1, H)
            row = torch.randint(0, ps - c["tokens"] + 1, (B, 1, H), generator=g, device="cuda")
            slots = page * ps + row + torch.arange(c["tokens"], device="cuda").view(1, -1, 1)
            slots[6::7] = -1                    # sequences without a new token
            s["slots"] = slots.int().view(1, B, c["tokens"], H)
            s["k_pages"] = torch.zeros((heads, ps, d), dtype=dt, device="cuda")
            s["v_pages"] = torch.zeros_like(s["k_pages"])
    else:
        rows = _row_counts(c)
        s["n_pages"], s["max_pages"], s["table"], _, _ = _pages(c, rows, 2, g)
        s["head_rows"] = rows.int().cuda()
        s["most"] = max(1, int(rows.max()))
        s["k_pages"], s["v_pages"] = randn(s["n_pages"], ps, d), randn(s["n_pages"], ps, d)
        heavy = 1 + 2 * (torch.rand((s["n_pages"], ps, 1), generator=g, device="cuda") < 0.01)
        s["k_pages"] *= heavy.to(dt)
        s["v_pages"] *= torch.exp(0.5 * randn(s["n_pages"], ps, 1, dtype=torch.float32)).to(dt)
        if c["garbage"]:
            col = torch.arange(s["max_pages"] * ps, device="cuda")
            behind = col >= s["head_rows"].unsqueeze(-1)
            page = s["table"].repeat_interleave(ps, dim=-1)
            at = (page.long() * ps + col % ps)[behind & (page >= 0)]
            s["k_pages"].view(-1, d)[at] = float("nan")
            s["v_pages"].view(-1, d)[at] = float("nan")
        s["q"] = 1.5 * randn(L, B, Hq, d)
        s["out"] = torch.empty((L, B, Hq, d), dtype=dt, device="cuda")
        s["lse"] = torch.empty((L, B, Hq), dtype=torch.float32, device="cuda")
    return s


def frequencies(c):
    """Radians per position of each rotated pair (64 bits), and the factor on the rotated vectors.
    plain: base^(-2i/r); linear: positions divided by the factor; base: a larger base, factor^(r/(r-2))
    times; bands: slow frequencies divided, fast ones kept, a line between two wavelengths; ramp: the
    line runs over the pairs' numbers, and the vectors grow with the factor's logarithm."""
    r, base, kind, factor, original = c["rotary_dim"], c["base"], c["scaling"], 8.0, 8192.0
    i = torch.arange(0, r, 2, dtype=torch.float64)
    if kind == "base":
        base = base * factor ** (r / (r - 2))
    f = base ** (-i / r)
    scale = 1.0
    if kind == "linear":
        f = f / factor
    elif kind == "bands":
        low, high = 1.0, 4.0
        keep = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = keep * f + (1 - keep) * f / factor
    elif kind == "ramp":
        fast, slow = 32.0, 1.0
        lo = max(0, math.floor(r * math.log(original / (fast * 2 * math.pi)) / (2 * math.log(base))))
        hi = min(r - 1, math.ceil(r * math.log(original / (slow * 2 * math.pi)) / (2 * math.log(base))))
        slow_share = ((i / 2 - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        f = f / factor * slow_share + f * (1 - slow_share)
        scale = 0.1 * math.log(factor) + 1.0
    return f, scale


# ----------------------------------------------------------------------------- the framework's calls
def _lava(s):
    """The package and the descriptors that a program keeps beside its cache, made at the first pass."""
    import paper_2509_09754_b200 as lava
    c = s["c"]
    if "cache" not in s:
        code = lava.LAVA_BF16 if c["dtype"] == "bf16" else lava.LAVA_F32
        if "n_pages" in s:
            s["cache"] = lava.CacheDesc(
                n_layers=c["layers"], batch=c["batch"] + c.get("others", 0), n_q_heads=c["q_heads"],
                n_kv_heads=c["kv_heads"], head_dim=c["head_dim"], dtype=code, page_rows=c["page_rows"],
                max_pages=s["max_pages"], n_pages=s["n_pages"], softcap=c.get("softcap", 0.0))
        else:
            s["cache"] = None
        if "freqs" in s:
            s["rotary"] = lava.RotaryDesc(
                head_dim=c["head_dim"], rotary_dim=c["rotary_dim"], dtype=code, interleaved=c["layout"] == "pairs",
                backward=c.get("backward", False), scale=s["scale"])
        if c["kind"] == "attend":
            s["ws"] = torch.zeros(lava.lava_cache_workspace_bytes(s["cache"]), dtype=torch.uint8, device="cuda")
        if c["kind"] == "fill":
            T, d = s["k"].shape[2], c["head_dim"]
            s["desc"] = lava.LayerDesc(
                n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=d, window=c["window"], dtype=code,
                batch=c["batch"], max_seqlen=c["tokens"], cu_seqlens=s["cu_seqlens"], total_tokens=T,
                k_stride_head=T * d, k_stride_tok=d, v_stride_head=T * d, v_stride_tok=d)
    return lava


def _run_own(s):
    c = s["c"]
    lava = _lava(s)
    cache = s["cache"]
    if c["kind"] == "tables":
        if c["form"] == "extend":
            lava.lava_page_extend(cache, s["add"], s["head_rows"], s["table"], s["free"], s["counters"], s["slots"],
                                  head_rows_out=s["rows_out"], counters_out=s["counters_out"])
            return {"rows": s["rows_out"], "table": s["table"], "free": s["free"], "counters": s["counters_out"],
                    "slots": s["slots"]}
        lava.lava_page_admit(cache, c["others"], s["head_offsets"], s["head_rows"], s["table"], s["free"],
                             s["counters"], s["first_row"], head_rows_out=s["rows_out"],
                             counters_out=s["counters_out"])
        return {"rows": s["rows_out"], "table": s["table"], "counters": s["counters_out"], "first": s["first_row"]}
    if c["kind"] == "fill":
        lava.lava_compact_kv_pages(s["desc"], cache, 0, s["k"], s["v"], s["k"].stride(0), s["v"].stride(0),
                                   s["keep_idx"], s["head_offsets"], s["first_row"], s["table"], s["k_pages"],
                                   s["v_pages"])
        return {"k": s["k_pages"], "v": s["v_pages"]}
    if c["kind"] == "rotate":
        lava.lava_rotary(s["rotary"], s["freqs"], s["positions"], s["q"], s["k"], s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "append":
        lava.lava_rotary_append(s["rotary"], s["freqs"], cache, 0, s["positions"], s["q"], s["k"], s["v"],
                                s["q_out"], s["slots"], s["k_pages"], s["v_pages"])
        return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}
    lava.lava_decode_attention_pages(cache, 0, s["q"], s["k_pages"], s["v_pages"], s["table"], s["head_rows"],
                                     s["out"], s["lse"], s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


# ----------------------------------------------------------------------------- the plain forms
def _take_pages(s, before, after, released):
    """Pages for heads that grow from `before` to `after` rows ([heads], in order): the next entries of the
    ring go to the heads in order, and the pages of released heads go to the ring's end.  Returns the new
    table, ring and counters."""
    ps, n, most = s["c"]["page_rows"], s["n_pages"], s["max_pages"]
    table = s["table"].view(-1, most)
    old, new = (before + ps - 1) // ps, (after + ps - 1) // ps
    take = torch.where(released, 0, new - old)
    give = torch.where(released, old, 0)
    first = take.cumsum(0) - take
    col = torch.arange(most, device="cuda").view(1, -1)
    at = s["counters"][0] + first.view(-1, 1) + col - old.view(-1, 1)
    grown = (col >= old.view(-1, 1)) & (col < (old + take).view(-1, 1))
    filled = torch.where(grown, s["free"][at % n], table)
    to = s["counters"][1] + (give.cumsum(0) - give).view(-1, 1) + col
    ring = torch.cat([s["free"], s["free"].new_zeros(1)])        # a place more for what is not given back
    ring[torch.where(col < give.view(-1, 1), to % n, n)] = table
    counters = s["counters"] + torch.stack([take.sum(), give.sum()])
    return filled, ring[:n], counters


def _tables_plain(s):
    c = s["c"]
    L, H, ps = c["layers"], c["kv_heads"], c["page_rows"]
    before = s["head_rows"].long().view(-1)
    if c["form"] == "extend":
        B, T = c["batch"], c["tokens"]
        add = s["add"].long().view(1, B, 1).expand(L, B, H).reshape(-1)
        released = add < 0
        after = torch.where(released, 0, before + add)
        table, ring, counters = _take_pages(s, before, after, released)
        j = torch.arange(T, device="cuda").view(1, T)
        row = before.view(-1, 1) + j
        page = table.long().gather(1, (row // ps).clamp(max=s["max_pages"] - 1))
        slot = torch.where(j < add.view(-1, 1), page * ps + row % ps, -1)
        slots = slot.view(L, B, H, T).permute(0, 1, 3, 2).contiguous().int()
        return {"rows": after.int().view(L, B, H), "table": table.view(s["table"].shape), "free": ring,
                "counters": counters, "slots": slots}
    B = c["batch"] + c["others"]
    hoff = s["head_offsets"].long()
    add = torch.zeros((L, B, H), dtype=torch.int64, device="cuda")
    add[:, c["others"]:] = hoff[:, :, 1:] - hoff[:, :, :-1]
    after = before + add.view(-1)
    table, _, counters = _take_pages(s, before, after, torch.zeros_like(before, dtype=torch.bool))
    first = before.view(L, B, H)[:, c["others"]:].int().contiguous()
    return {"rows": after.int().view(L, B, H), "table": table.view(s["table"].shape), "counters": counters,
            "first": first}


def _fill_plain(s):
    c = s["c"]
    L, B, H, ps, n, w, d = c["layers"], c["batch"], c["kv_heads"], c["page_rows"], c["tokens"], c["window"], c["head_dim"]
    hoff = s["head_offsets"].long()
    count = (hoff[:, :, 1:] - hoff[:, :, :-1]).unsqueeze(-1)                  # [L, B, H, 1]
    # row j of every head; past its end the last row once more
    j = torch.arange(s["most"], device="cuda").view(1, 1, 1, -1).minimum(count - 1)
    head = torch.arange(H, device="cuda").view(1, 1, H, 1)
    entry = hoff[:, :, :H].unsqueeze(-1) - head * w + j
    kept = s["keep_idx"].view(L, B, -1).gather(2, entry.clamp(max=H * (n - w) - 1).view(L, B, -1)).view(entry.shape)
    tok = torch.where(j < count - w, kept.long(), n - count + j)
    tok = tok + torch.arange(B, device="cuda").view(1, B, 1, 1) * n
    src = ((torch.arange(L, device="cuda").view(L, 1, 1, 1) * H + head) * (B * n) + tok).view(-1)
    row = s["first_row"].long().unsqueeze(-1) + j
    dst = (s["table"].long().gather(3, row // ps) * ps + row % ps).view(-1)
    s["k_pages"].view(-1, d)[dst] = s["k"].view(-1, d)[src]
    s["v_pages"].view(-1, d)[dst] = s["v"].view(-1, d)[src]
    return {"k": s["k_pages"], "v": s["v_pages"]}


def _turn(s, x):
    """Rotates the leading rotary_dim elements of x [tokens, heads, d], angles in 64 bits."""
    c = s["c"]
    r = c["rotary_dim"]
    angle = s["positions"].double().view(-1, 1, 1) * s["freqs"]
    cos, sin = (angle.cos() * s["scale"]).float(), (angle.sin() * s["scale"]).float()
    if c.get("backward"):
        sin = -sin
    x = x.float()
    if c["layout"] == "pairs":
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2: r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., r:]], dim=-1).to(s["qkv"].dtype)


def _append_plain(s):
    c = s["c"]
    d = c["head_dim"]
    slots = s["slots"].long().view(-1)
    # rows without a place go to one more row behind the pool
    at = torch.where(slots >= 0, slots, s["n_pages"] * c["page_rows"])
    pages = []
    for pool, rows in ((s["k_pages"], _turn(s, s["k"])), (s["v_pages"], s["v"])):
        flat = torch.cat([pool.view(-1, d), pool.new_zeros(1, d)])
        flat[at] = rows.reshape(-1, d)
        pages.append(flat[:-1].view(pool.shape))
    return {"q": _turn(s, s["q"]), "k": pages[0], "v": pages[1]}


def _gathered(s, pool):
    """The rows of every head side by side, [heads, most, d], zeros behind a head's last one; and which are rows."""
    c = s["c"]
    ps = c["page_rows"]
    j = torch.arange(s["most"], device="cuda")
    rows = s["head_rows"].long().view(-1, 1)
    page = s["table"].view(rows.shape[0], -1).long()[:, j // ps].clamp(min=0)
    there = j < rows
    x = pool.view(-1, c["head_dim"])[(page * ps + j % ps).view(-1)].view(rows.shape[0], s["most"], -1)
    return torch.where(there.unsqueeze(-1), x.float(), 0.0), there


def _attend_plain(s):
    c = s["c"]
    L, B, Hq, H, d = c["layers"], c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"]
    k, there = _gathered(s, s["k_pages"])
    q = s["q"].float().view(L * B * H, Hq // H, d)
    x = torch.matmul(q, k.transpose(1, 2)) * d ** -0.5
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    x = torch.where(there.unsqueeze(1), x, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    v, _ = _gathered(s, s["v_pages"])
    out = torch.matmul(e, v) / torch.where(total == 0, 1.0, total)
    lse = torch.log(total) + top
    return {"out": out.view(L, B, Hq, d).to(s["q"].dtype), "lse": lse.view(L, B, Hq)}


def run(s):
    if own:
        return _run_own(s)
    kind = s["c"]["kind"]
    if kind == "tables":
        return _tables_plain(s)
    if kind == "fill":
        return _fill_plain(s)
    if kind == "rotate":
        return {"q": _turn(s, s["q"]), "k": _turn(s, s["k"])}
    if kind == "append":
        return _append_plain(s)
    return _attend_plain(s)


# ----------------------------------------------------------------------------- 64 bits
def _turn_exact(s, x):
    """The rotation as a complex product, in 64 bits."""
    c = s["c"]
    r = c["rotary_dim"]
    z = torch.polar(torch.full_like(s["freqs"], s["scale"]).expand(x.shape[0], -1),
                    s["positions"].double().outer(s["freqs"])).unsqueeze(1)
    z = z.conj() if c.get("backward") else z
    x = x.double()
    lead = x[..., :r]
    pairs = lead.unflatten(-1, (r // 2, 2)) if c["layout"] == "pairs" else lead.unflatten(-1, (2, r // 2)).transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
    turned = turned if c["layout"] == "pairs" else turned.transpose(-1, -2)
    return torch.cat([turned.flatten(-2), x[..., r:]], dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] in ("tables", "fill"):
        return None                              # whole numbers, and rows copied bit for bit
    if c["kind"] == "rotate":
        return {"q": _turn_exact(s, s["q"]), "k": _turn_exact(s, s["k"])}
    d, ps = c["head_dim"], c["page_rows"]
    if c["kind"] == "append":
        pool, keys = s["k_pages"].double().view(-1, d), _turn_exact(s, s["k"]).reshape(-1, d)
        slots = s["slots"].view(-1).long()
        pool[slots[slots >= 0]] = keys[slots >= 0]
        return {"q": _turn_exact(s, s["q"]), "k": pool.view(s["k_pages"].shape), "v": None}
    # head by head, softmax from torch in 64 bits
    L, B, Hq, H = c["layers"], c["batch"], c["q_heads"], c["kv_heads"]
    out = torch.zeros((L * B * H, Hq // H, d), dtype=torch.float64, device="cuda")
    lse = torch.full((L * B * H, Hq // H), -math.inf, dtype=torch.float64, device="cuda")
    q = s["q"].double().view(out.shape)
    table, counts = s["table"].view(L * B * H, -1).long(), s["head_rows"].view(-1).tolist()
    for h, n in enumerate(counts):
        if n == 0:
            continue
        pages = table[h, : _ceil(n, ps)]
        k = s["k_pages"][pages].view(-1, d)[:n].double()
        v = s["v_pages"][pages].view(-1, d)[:n].double()
        x = q[h] @ k.T / math.sqrt(d)
        if c["softcap"]:
            x = c["softcap"] * torch.tanh(x / c["softcap"])
        out[h] = torch.softmax(x, dim=-1) @ v
        lse[h] = torch.logsumexp(x, dim=-1)
    return {"out": out.view(L, B, Hq, d), "lse": lse.view(L, B, Hq)}


# ----------------------------------------------------------------------------- work
def work(case):
    c = dict(case)
    L, B, H, Hq, d, ps = c["layers"], c["batch"], c["kv_heads"], c["q_heads"], c["head_dim"], c["page_rows"]
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "tables":
        if c["form"] == "extend":
            rows, add = _row_counts(c), _added(c).view(1, B, 1)
            moved = torch.where(add < 0, _ceil(rows, ps), _ceil(rows + add, ps) - _ceil(rows, ps))
            # rows and slots of every head; a page number is read in one place and written to another
            return {"bytes": L * B * H * (8 + 4 * c["tokens"]) + 8 * int(moved.sum()) + 4 * B + 32, "flops": 0}
        new = _row_counts(c, c["others"] + B)[:, c["others"]:]
        return {"bytes": L * (B + c["others"]) * H * 8 + L * B * H * 8 + 8 * int(_ceil(new, ps).sum()) + 32, "flops": 0}
    if c["kind"] == "fill":
        rows = L * B * H * c["rows"]
        return {"bytes": rows * (4 * d * es + 4), "flops": 0}
    if c["kind"] in ("rotate", "append"):
        N = c["tokens"] * (B if c["kind"] == "append" else 1)
        written = 2 * N * (Hq + H) * d * es + 4 * N
        if c["kind"] == "append":
            written += 2 * N * H * d * es + 4 * N * H
        return {"bytes": written, "flops": 3 * N * (Hq + H) * c["rotary_dim"]}
    rows = int(_row_counts(c).sum())
    return {"bytes": rows * 2 * d * es + L * B * Hq * (2 * d * es + 4) + 4 * rows // ps + 4 * L * B * H,
            "flops": 4 * rows * (Hq // H) * d}
