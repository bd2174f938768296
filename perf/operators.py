"""The cache operators around the verify step, as they are measured: attention of ragged chunks of new
tokens over the paged cache, rotary positions applied on the way into the cache, and the upkeep of its
pages (forking branches, making room, closing holes).

Every case is a dict of plain values.  `prepare` makes its inputs, `run` is one pass through the operator:
in plain torch operations where `own` is false, through the library's entry points where it is true.
"""
import math
import random

import torch

own = False

PAGE, DIM = 16, 128
ROPE_BASE = 1.0e6          # the usual base of long-context rotary embeddings; any positive number would do


# ------------------------------------------------------------------------------------------------ cases
def listed():
    """The head shapes are those of the repository's workloads: 8 / 2 (tiny), 16 / 2 (3B), 40 / 8 (32B)."""
    return [
        # the smallest call: one new token for each of four short branches; its time is latency
        {"name": "attn_one_token_small", "op": "attn", "hq": 8, "hkv": 2, "prefix": 256, "chunks": 0, "chunk_lo": 1, "chunk_hi": 1,
         "ctx_lo": 0, "ctx_hi": 0, "singles": 4, "single_lo": 200, "single_hi": 256, "lse": False, "layout": 1},
        # plain decoding of 64 branches of different questions: every key is read for one token, so bandwidth counts
        {"name": "attn_one_token_64", "op": "attn", "hq": 40, "hkv": 8, "prefix": 0, "chunks": 0, "chunk_lo": 1, "chunk_hi": 1,
         "ctx_lo": 0, "ctx_hi": 0, "singles": 64, "single_lo": 1024, "single_hi": 8192, "lse": False, "layout": 2},
        # prompts of the length the workloads have (below 800 tokens), ragged, nothing cached yet
        {"name": "attn_prompts_24", "op": "attn", "hq": 16, "hkv": 2, "prefix": 0, "chunks": 24, "chunk_lo": 90, "chunk_hi": 799,
         "ctx_lo": 0, "ctx_hi": 0, "singles": 0, "single_lo": 1, "single_hi": 1, "lse": True, "layout": 3},
        # a serving step: one piece of a long prompt beside 31 branches that decode one token each
        {"name": "attn_mixed_step", "op": "attn", "hq": 40, "hkv": 8, "prefix": 512, "chunks": 1, "chunk_lo": 1021, "chunk_hi": 1021,
         "ctx_lo": 5000, "ctx_hi": 5000, "singles": 31, "single_lo": 1000, "single_hi": 8000, "lse": False, "layout": 4},
        # the largest: 8192 new tokens on top of 24576 cached ones, bound by the tensor cores
        {"name": "attn_long_prompt", "op": "attn", "hq": 40, "hkv": 8, "prefix": 0, "chunks": 1, "chunk_lo": 8192, "chunk_hi": 8192,
         "ctx_lo": 24576, "ctx_hi": 24576, "singles": 0, "single_lo": 1, "single_hi": 1, "lse": True, "layout": 5},
        # the verify step's rows (gamma 3, 16 branches) on their way into the cache: latency
        {"name": "rope_verify_rows", "op": "rope", "hq": 40, "hkv": 8, "prefix": 512, "n": 16, "rows_lo": 4, "rows_hi": 4,
         "ctx_lo": 300, "ctx_hi": 4096, "axes": 1, "pairs": 64, "interleaved": False, "layout": 6},
        # a batch of long prompts, one position axis: bandwidth
        {"name": "rope_prompts", "op": "rope", "hq": 40, "hkv": 8, "prefix": 0, "n": 11, "rows_lo": 700, "rows_hi": 1900,
         "ctx_lo": 0, "ctx_hi": 2000, "axes": 1, "pairs": 64, "interleaved": False, "layout": 7},
        # image and video tokens: time, height and width, positions of tokens far into a sequence
        {"name": "rope_three_axes", "op": "rope", "hq": 16, "hkv": 2, "prefix": 32, "n": 5, "rows_lo": 501, "rows_hi": 2500,
         "ctx_lo": 0, "ctx_hi": 100000, "axes": 3, "pairs": 64, "interleaved": True, "layout": 8},
        # 16 branches of one question resampled, then room for the next step's 4 rows: few pages are copied
        {"name": "fork_16", "op": "fork", "layers": 64, "hq": 40, "hkv": 8, "prefix": 512, "n": 16, "children": 16, "len_lo": 200,
         "len_hi": 700, "rows": 4, "spare": 64, "layout": 9},
        # the smallest fork: four branches from one, few layers
        {"name": "fork_4_from_1", "op": "fork", "layers": 4, "hq": 8, "hkv": 2, "prefix": 256, "n": 1, "children": 4, "len_lo": 37,
         "len_hi": 37, "rows": 6, "spare": 32, "layout": 10},
        # half of 24 branches have finished and left holes behind: about half of the pages that remain move
        {"name": "compact_24", "op": "compact", "layers": 64, "hq": 40, "hkv": 8, "prefix": 512, "n": 24, "kept": 12, "len_lo": 100,
         "len_hi": 900, "spare": 40, "layout": 11},
        # a small model's pool: few layers and two KV heads, many pages
        {"name": "compact_small_pages", "op": "compact", "layers": 6, "hq": 16, "hkv": 2, "prefix": 512, "n": 64, "kept": 41, "len_lo": 1024,
         "len_hi": 4000, "spare": 500, "layout": 12},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "rope", "fork", "compact"])
    layout = rng.randrange(100, 1 << 20)
    hq, hkv = rng.choice([(8, 2), (16, 2), (40, 8), (8, 8), (12, 1), (28, 4), (32, 8)])
    if kind == "attn":
        chunks = rng.choice([0, 1, 1, 2, 5, _spread(rng, 1, 24)])
        hi = _spread(rng, 2, 8192 // max(1, chunks))
        ctx = rng.choice([0, _spread(rng, 1, 16000 // max(1, chunks))])
        singles = rng.choice([0, _spread(rng, 1, 64)]) if chunks else _spread(rng, 1, 64)
        far = _spread(rng, 16, 8192)
        return {"op": "attn", "hq": hq, "hkv": hkv, "prefix": 16 * rng.choice([0, 0, _spread(rng, 1, 64)]), "chunks": chunks,
                "chunk_lo": max(1, hi // rng.choice([1, 2, 8])), "chunk_hi": hi, "ctx_lo": ctx // 2, "ctx_hi": ctx, "singles": singles,
                "single_lo": max(1, far // 8), "single_hi": far, "lse": rng.random() < 0.5, "layout": layout}
    if kind == "rope":
        n = _spread(rng, 1, 64)
        hi = _spread(rng, 1, 14000 // n)
        return {"op": "rope", "hq": hq, "hkv": hkv, "prefix": 16 * rng.choice([0, _spread(rng, 1, 64)]), "n": n, "rows_lo": max(1, hi // 3),
                "rows_hi": hi, "ctx_lo": 0, "ctx_hi": _spread(rng, 1, 60000 // n), "axes": rng.choice([1, 2, 3, 4]),
                "pairs": rng.choice([64, 64, 32, 48, 20]), "interleaved": rng.random() < 0.5, "layout": layout}
    hkv = rng.choice([1, 2, 4, 8])
    case = {"op": kind, "layers": _spread(rng, 1, 64), "hq": 8, "hkv": hkv, "prefix": 16 * rng.choice([0, _spread(rng, 1, 64)]),
            "n": _spread(rng, 1, 32)}
    far = _spread(rng, 20, max(21, min(4000, 200000 // (case["n"] * case["layers"] * hkv // 4 + 1))))
    case |= {"len_lo": max(1, far // 5), "len_hi": far, "spare": 0, "layout": layout}
    if kind == "fork":
        case |= {"children": _spread(rng, 1, 32), "rows": rng.randrange(1, 65)}
        case["spare"] = case["children"] * 6 + rng.randrange(100)
    else:
        case |= {"kept": rng.randrange(0, case["n"] + 1), "spare": rng.randrange(200)}
    return case


# ----------------------------------------------------------------- what a case fixes, whatever the seed is
def _plan(case):
    """Lengths and page tables of a case, on the host: they belong to the case, so that work() knows them."""
    r = random.Random(case["layout"])
    shared = case["prefix"] // PAGE
    if case["op"] in ("attn", "rope"):
        if case["op"] == "attn":
            kinds = ["c"] * case["chunks"] + ["s"] * case["singles"]
            r.shuffle(kinds)
            chunk = [r.randint(case["chunk_lo"], case["chunk_hi"]) if k == "c" else 1 for k in kinds]
            ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) if k == "c" else r.randint(case["single_lo"], case["single_hi"]) - 1 for k in kinds]
        else:
            chunk = [r.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["n"])]
            ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["n"])]
        lens = [c + x for c, x in zip(chunk, ctx)]
        need = [-(-x // PAGE) for x in lens]
        pages = list(range(shared + sum(need) + 3))
        r.shuffle(pages)
        at, rows = shared, []
        for n in need:
            rows.append(pages[:shared] + pages[at:at + n])
            at += n
        return {"chunk": chunk, "lens": lens, "rows": rows, "pages": len(pages)}
    lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["n"])]
    need = [-(-x // PAGE) for x in lens]
    pages = list(range(shared + sum(need) + case["spare"]))
    r.shuffle(pages)
    at, rows = shared, []
    for n in need:
        rows.append(pages[:shared] + pages[at:at + n])
        at += n
    plan = {"lens": lens, "rows": rows, "pages": len(pages)}
    if case["op"] == "fork":
        plan["parents"] = [r.randrange(case["n"]) for _ in range(case["children"])]
    else:
        kept = set(r.sample(range(case["n"]), case["kept"]))
        plan["rows"] = [row if b in kept else [] for b, row in enumerate(rows)]
    return plan


def _axis_of_pair(case):
    """Which position axis turns which pair: alternating for images and video, so that every axis has high and low frequencies."""
    return [i % case["axes"] for i in range(case["pairs"])]


def _inv_freq(case):
    return [ROPE_BASE ** (-i / case["pairs"]) for i in range(case["pairs"])]


def work(case):
    plan = _plan(case)
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "attn":
        keys = sum(plan["lens"]) + case["prefix"]                       # every cached token once, the shared ones once
        rows = sum(plan["chunk"])
        seen = sum(c * (case["prefix"] + n - c) + c * (c + 1) // 2 for c, n in zip(plan["chunk"], plan["lens"]))
        return {"bytes": keys * hkv * DIM * 4 + rows * hq * DIM * 4 + (rows * hq * 4 if case["lse"] else 0), "flops": 4 * DIM * hq * seen}
    if case["op"] == "rope":
        rows = sum(plan["chunk"])
        return {"bytes": rows * (2 * hq * DIM * 2 + 4 * hkv * DIM * 2 + 4 * case["axes"]), "flops": rows * (hq + hkv) * case["pairs"] * 6}
    page = hkv * PAGE * DIM * 2 * 2 * case["layers"]                    # one page of K and V in every layer
    table = max(len(x) for x in plan["rows"]) * len(plan["rows"]) * 4
    if case["op"] == "fork":
        copies, seen = 0, set()
        for p in plan["parents"]:
            copies += p in seen and (case["prefix"] + plan["lens"][p]) % PAGE != 0
            seen.add(p)
        return {"bytes": 2 * copies * page + 2 * table + 2 * plan["pages"] * 4, "flops": 0}
    used = {p for row in plan["rows"] for p in row}
    return {"bytes": 2 * sum(p >= len(used) for p in used) * page + 2 * table + 3 * plan["pages"] * 4, "flops": 0}


# ----------------------------------------------------------------------------------------------- inputs
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(rows, width):
    return _ints([row + [-1] * (width - len(row)) for row in rows])


def prepare(case, seed):
    plan = _plan(case)
    gen = torch.Generator("cuda").manual_seed(seed)
    hq, hkv = case["hq"], case["hkv"]
    layers = case.get("layers", 1)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    width = max(1, max(len(row) for row in plan["rows"]))
    if case["op"] == "fork":
        width += -(-case["rows"] // PAGE) + 1
    s = {"case": case, "prefix": case["prefix"], "hq": hq, "hkv": hkv, "n": len(plan["rows"]), "table": _table(plan["rows"], width),
         "lens": _ints(plan["lens"])}
    s["k"], s["v"] = normal(layers, plan["pages"], hkv, PAGE, DIM), normal(layers, plan["pages"], hkv, PAGE, DIM)
    if case["op"] in ("attn", "rope"):
        starts = [0]
        for c in plan["chunk"]:
            starts.append(starts[-1] + c)
        s |= {"starts": starts, "row_start": _ints(starts), "rows": starts[-1], "chunk": plan["chunk"], "total": [case["prefix"] + x for x in plan["lens"]]}
        qkv = normal(s["rows"], hq + 2 * hkv, DIM)                      # the projection's result: q, k and v side by side
        s["q"], s["k_new"], s["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["out"] = torch.empty(s["rows"], hq, DIM, device="cuda", dtype=torch.bfloat16)
        s["branch"] = torch.repeat_interleave(torch.arange(s["n"], device="cuda"), _ints(plan["chunk"]).long(), output_size=s["rows"])
        if case["op"] == "attn":
            s["lse"] = torch.empty(s["rows"], hq, device="cuda") if case["lse"] else None
            # branches whose plain form runs as one padded batch: equal chunks, scores of at most 2 GB
            s["groups"] = _groups(plan["chunk"], s["total"], hq)
        else:
            at = torch.arange(s["rows"], device="cuda") - s["row_start"].long()[s["branch"]]
            at = at + (s["lens"].long()[s["branch"]] - _ints(plan["chunk"]).long()[s["branch"]]) + case["prefix"]
            s["place"] = at                                             # each row's place in its sequence
            # text moves all axes together; the further axes of images run over a grid
            grid = [at] + [torch.randint(0, 200, (s["rows"],), generator=gen, device="cuda") + at // 4 for _ in range(case["axes"] - 1)]
            s["positions"] = torch.stack(grid).to(torch.int32).contiguous()
            s["axis"], s["inv_freq"] = _axis_of_pair(case), _inv_freq(case)
    else:
        s["refs"] = torch.zeros(plan["pages"], dtype=torch.int32, device="cuda")
        held = s["table"][s["table"] >= 0].long()
        s["refs"].scatter_add_(0, held, torch.ones_like(held, dtype=torch.int32))
        s["new_refs"] = torch.empty_like(s["refs"])
        if case["op"] == "fork":
            s["parents"] = _ints(plan["parents"])
            s["more"] = torch.full((case["children"],), case["rows"], dtype=torch.int32, device="cuda")     # rows to come, for each branch
            s["new_table"] = torch.empty(case["children"], width, dtype=torch.int32, device="cuda")
            s["new_lens"] = torch.empty(case["children"], dtype=torch.int32, device="cuda")
        else:
            s["new_table"] = torch.empty_like(s["table"])
            s["page_map"] = torch.empty(plan["pages"], dtype=torch.int32, device="cuda")
            s["n_used"] = torch.empty(1, dtype=torch.int32, device="cuda")
    if own:
        # the handle that a server keeps: a context for this model and pool, and its lists of pools and frequencies
        import paper_2505_19634_b200 as tts
        s["ctx"] = tts.TtsContext(hq, hkv, max(s["n"], case.get("children", 1)), 1, width, plan["pages"])
        if case["op"] == "attn":
            s["ctx"].tts_chunk_reserve(s["rows"])
        elif case["op"] == "rope":
            s["rope"] = tts.TtsRope(s["axis"], s["inv_freq"], case["interleaved"])
        else:
            s["pools"] = tts.TtsPools(list(s["k"]), list(s["v"]))
    return s


def _groups(chunk, total, hq):
    by = {}
    for b, c in enumerate(chunk):
        by.setdefault(c, []).append(b)
    out = []
    for c, members in sorted(by.items()):
        members.sort(key=lambda b: total[b])
        most = max(1, (1 << 29) // (hq * c * total[members[-1]]))
        out += [(c, members[i:i + most], _ints(members[i:i + most]).long()) for i in range(0, len(members), most)]
    return out


# ----------------------------------------------------------------------------------------------- passes
def run(state):
    return {"attn": _attn, "rope": _rope, "fork": _fork, "compact": _compact}[state["case"]["op"]](state)


def _attn(s):
    if own:
        s["ctx"].tts_chunk_attn(s["q"], s["q"].stride(0), s["k"], s["v"], s["table"], s["prefix"], s["lens"], s["row_start"], s["n"],
                                s["rows"], s["out"], s["lse"])
    else:
        # a loop over batches of equal chunks and, where one batch's scores would not fit, over its KV heads
        for c, members, index in s["groups"]:
            most = max(s["total"][b] for b in members)
            heads = s["hkv"] if len(members) * s["hq"] * c * most <= 1 << 29 else 1
            first = s["row_start"].long()[index]
            at = (first[:, None] + torch.arange(c, device="cuda")).reshape(-1)
            q = s["q"][at].float().reshape(len(members), c, s["hkv"], -1, DIM).permute(0, 2, 3, 1, 4)      # member, KV head, group, row
            pages = s["table"].long()[index, :-(-most // PAGE)].clamp_min(0)
            total = s["lens"].long()[index] + s["prefix"]
            limit = (total - c)[:, None] + torch.arange(1, c + 1, device="cuda")                            # keys that a row sees
            key = torch.arange(pages.shape[1] * PAGE, device="cuda")
            hidden = (key >= limit[:, :, None])[:, None, None]
            past = (key >= total[:, None])[:, None, :, None]                                               # nothing is stored there
            for h in range(0, s["hkv"], heads):
                k, v = (x[0][:, h:h + heads][pages].permute(0, 2, 1, 3, 4).reshape(len(members), heads, -1, DIM).float().masked_fill(past, 0) for x in (s["k"], s["v"]))
                score = torch.matmul(q[:, h:h + heads].reshape(len(members), heads, -1, DIM), k.transpose(-1, -2)) / math.sqrt(DIM)
                score = score.view(len(members), heads, -1, c, key.numel()).masked_fill_(hidden, -math.inf)
                top = score.amax(-1, keepdim=True)
                score = score.sub_(top).exp_()
                total_p = score.sum(-1, keepdim=True)
                o = torch.matmul(score.view(len(members), heads, -1, key.numel()), v).view(len(members), heads, -1, c, DIM) / total_p
                cols = slice(h * (s["hq"] // s["hkv"]), (h + heads) * (s["hq"] // s["hkv"]))
                s["out"][at, cols] = o.permute(0, 3, 1, 2, 4).reshape(at.numel(), -1, DIM).to(torch.bfloat16)
                if s["lse"] is not None:
                    s["lse"][at, cols] = (top + total_p.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(at.numel(), -1)
    return {"out": s["out"]} | ({"lse": s["lse"]} if s["lse"] is not None else {})


def _turn(x, cos, sin, pairs, interleaved):
    """x rotated by the angles of its first `pairs` pairs; the dims past them stay."""
    x = x.float()
    turned, rest = x[..., :2 * pairs], x[..., 2 * pairs:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else (turned[..., :pairs], turned[..., pairs:])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1)
    return torch.cat((turned, rest), -1).to(torch.bfloat16)


def _rope(s):
    case = s["case"]
    if own:
        s["ctx"].tts_kv_append_rope(s["rope"], s["q"], s["q"].stride(0), s["k_new"], s["v_new"], s["k_new"].stride(0), s["positions"],
                                    s["k"], s["v"], s["table"], s["prefix"], s["lens"], s["row_start"], s["n"], s["rows"], s["out"])
    else:
        freq = torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
        angle = s["positions"].double()[torch.tensor(s["axis"], device="cuda")].T * freq                    # row, pair; in 64 bits: positions are far
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        s["out"].copy_(_turn(s["q"], cos, sin, case["pairs"], case["interleaved"]))
        page, slot = s["table"].long()[s["branch"], s["place"] // PAGE], s["place"] % PAGE
        s["k"][0][page, :, slot] = _turn(s["k_new"], cos, sin, case["pairs"], case["interleaved"])
        s["v"][0][page, :, slot] = s["v_new"]
    return {"q": s["out"], "k_pages": s["k"], "v_pages": s["v"]}


def _count(table, like):
    held = torch.where(table >= 0, table, like.numel()).reshape(-1).long()
    return torch.zeros(like.numel() + 1, dtype=torch.int32, device="cuda").index_add_(0, held, torch.ones_like(held, dtype=torch.int32))[:-1]


def _lowest_free(refs, wanted):
    """For each true place of `wanted`, in order, the next lowest page that nothing refers to."""
    free = torch.sort(torch.where(refs == 0, 0, 1), stable=True).indices
    return free[(wanted.reshape(-1).long().cumsum(0) - 1).clamp_min(0)].reshape(wanted.shape)


def _fork(s):
    if own:
        s["ctx"].tts_kv_fork(s["pools"], s["table"], s["prefix"], s["lens"], s["n"], s["parents"], s["parents"].numel(), s["refs"],
                             s["new_table"], s["new_lens"], s["new_refs"])
        s["ctx"].tts_kv_grow(s["new_table"], s["prefix"], s["new_lens"], s["more"], s["parents"].numel(), s["new_refs"])
    else:
        parent = s["parents"].long()
        first = (parent[:, None] == parent[None, :]).int().argmax(1) == torch.arange(parent.numel(), device="cuda")
        tokens = s["lens"].long()[parent] + s["prefix"]
        full, partial = tokens // PAGE, (tokens % PAGE != 0) & ~first
        column = torch.arange(s["table"].shape[1], device="cuda")
        old = s["table"].long()[parent]
        new = torch.where(first[:, None] | (column < full[:, None]), old, -1)
        page = _lowest_free(s["refs"], partial)
        source = old.gather(1, full[:, None].clamp_max(column.numel() - 1))[:, 0]
        new = torch.where(partial[:, None] & (column == full[:, None]), page[:, None], new)
        s["k"][:, page[partial]] = s["k"][:, source[partial]]
        s["v"][:, page[partial]] = s["v"][:, source[partial]]
        refs = s["refs"] - _count(s["table"], s["refs"]) + _count(new, s["refs"])
        # room for the next rows
        after = tokens + s["more"]
        wanted = (new < 0) & (column < ((after + PAGE - 1) // PAGE)[:, None])
        new = torch.where(wanted, _lowest_free(refs, wanted), new)
        s["new_table"].copy_(new)
        s["new_lens"].copy_(after - s["prefix"])
        s["new_refs"].copy_(refs - _count(torch.where(wanted, -1, new), refs) + _count(new, refs))
    return {"k_pages": s["k"], "v_pages": s["v"], "table": s["new_table"], "lens": s["new_lens"], "refs": s["new_refs"]}


def _compact(s):
    if own:
        s["ctx"].tts_kv_compact(s["pools"], s["table"], s["n"], s["refs"], s["new_table"], s["new_refs"], s["page_map"], s["n_used"])
    else:
        used = s["refs"] > 0
        count = used.sum()
        page = torch.arange(used.numel(), device="cuda")
        moves, hole = used & (page >= count), ~used & (page < count)
        source, target = page[moves], page[hole]
        mapped = torch.where(used, page, -1)
        mapped[source] = target
        s["k"][:, target] = s["k"][:, source]
        s["v"][:, target] = s["v"][:, source]
        s["page_map"].copy_(mapped)
        s["new_table"].copy_(torch.where(s["table"] >= 0, mapped[s["table"].long().clamp_min(0)], -1))
        s["new_refs"].zero_()
        s["new_refs"][mapped[used]] = s["refs"][used]
        s["n_used"].copy_(count)
    return {"k_pages": s["k"], "v_pages": s["v"], "table": s["new_table"], "refs": s["new_refs"], "page_map": s["page_map"], "n_used": s["n_used"]}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """From the definitions: every branch by itself, in 64 bits; copies of pages are exact in their own type."""
    s = prepare(case, seed)
    return {"attn": _exact_attn, "rope": _exact_rope, "fork": _exact_fork, "compact": _exact_compact}[case["op"]](s)


def _exact_attn(s):
    group = s["hq"] // s["hkv"]
    out = torch.zeros(s["rows"], s["hq"], DIM, device="cuda", dtype=torch.float64)
    lse = torch.zeros(s["rows"], s["hq"], device="cuda", dtype=torch.float64)
    for b in range(s["n"]):
        total, c, r0 = s["total"][b], s["chunk"][b], s["starts"][b]
        pages = s["table"][b, :(total + PAGE - 1) // PAGE].long()
        for h in range(s["hq"]):
            k = s["k"][0, pages, h // group].reshape(-1, DIM)[:total].double()
            v = s["v"][0, pages, h // group].reshape(-1, DIM)[:total].double()
            z = s["q"][r0:r0 + c, h].double() @ k.T * DIM ** -0.5
            late = torch.arange(total, device="cuda")[None, :] > torch.arange(total - c, total, device="cuda")[:, None]
            z = z.masked_fill_(late, -math.inf)
            lse[r0:r0 + c, h] = torch.logsumexp(z, 1)
            out[r0:r0 + c, h] = torch.softmax(z, 1) @ v
    return {"out": out} | ({"lse": lse} if s["lse"] is not None else {})


def _exact_rope(s):
    case = s["case"]
    turn = s["positions"].double()[torch.tensor(s["axis"], device="cuda")].T * torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]

    def turned(x):
        x, n = x.double(), case["pairs"]
        lo = (torch.arange(n, device="cuda") * 2) if case["interleaved"] else torch.arange(n, device="cuda")
        hi = lo + 1 if case["interleaved"] else lo + n
        z = torch.complex(x[..., lo], x[..., hi]) * turn
        y = x.clone()
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    k, v = s["k"].double(), s["v"].double()
    row = s["table"].long()[s["branch"]].gather(1, (s["place"] // PAGE)[:, None])[:, 0]
    k[0, row, :, s["place"] % PAGE] = turned(s["k_new"])
    v[0, row, :, s["place"] % PAGE] = s["v_new"].double()
    return {"q": turned(s["q"]), "k_pages": k, "v_pages": v}


def _exact_fork(s):
    refs, prefix = s["refs"].tolist(), s["prefix"]
    free = [p for p, n in enumerate(refs) if n == 0]
    table, lens = s["table"].tolist(), s["lens"].tolist()
    seen, at = set(), 0
    for p in s["parents"].tolist():
        full, rest = divmod(prefix + lens[p], PAGE)
        if p in seen and rest:
            for pool in (s["k"], s["v"]):
                pool[:, free[at]] = pool[:, table[p][full]]
            at += 1
        seen.add(p)
    return {"k_pages": s["k"], "v_pages": s["v"], "table": None, "lens": None, "refs": None}


def _exact_compact(s):
    refs = s["refs"].tolist()
    used = [p for p, n in enumerate(refs) if n]
    holes = [p for p in range(len(used)) if refs[p] == 0]
    for p, hole in zip([p for p in used if p >= len(used)], holes):
        for pool in (s["k"], s["v"]):
            pool[:, hole] = pool[:, p]
    return {"k_pages": s["k"], "v_pages": s["v"], "table": None, "refs": None, "page_map": None, "n_used": None}
