"""A search over many branches on an 8-bit cache, as it is measured: keys and values quantised on their way into the
cache and read back, attention of chains and trees of drafted tokens over that cache, the selection of the best
continuations of all beams, and the reordering of the beams' states.

Every case is a dict of plain values.  `prepare` makes its inputs, `run` is one pass through the operator: in plain
torch operations where `own` is false, through the library's entry points where it is true.
"""
import math
import random

import torch

own = False

PAGE, DIM = 16, 128
RECORD = 2 * PAGE * DIM + 2 * PAGE * 4      # bytes of one page of one KV head: codes of K, codes of V, a scale of each for every token
ROPE_BASE = 1.0e6          # the usual base of long-context rotary embeddings; any positive number would do
E4M3, INT8 = 0, 1
LARGEST = (448.0, 127.0)   # the largest code of either format
LEAST = 2.0 ** -120        # the smallest scale


# ------------------------------------------------------------------------------------------------ cases
def listed():
    """The head shapes are those of the repository's workloads: 8 / 2 (tiny), 16 / 2 (3B), 40 / 8 (32B); so are the vocabularies."""
    return [
        # the verify step's rows (gamma 3, 16 branches) on their way into the cache: latency
        {"name": "append_verify_rows", "op": "append", "format": E4M3, "hq": 40, "hkv": 8, "prefix": 512, "n": 16, "rows_lo": 4, "rows_hi": 4,
         "ctx_lo": 300, "ctx_hi": 2048, "rope": True, "pairs": 64, "interleaved": False, "layout": 1},
        # a batch of long prompts enters the cache: bandwidth
        {"name": "append_prompts", "op": "append", "format": INT8, "hq": 40, "hkv": 8, "prefix": 0, "n": 11, "rows_lo": 700, "rows_hi": 1900,
         "ctx_lo": 0, "ctx_hi": 500, "rope": True, "pairs": 64, "interleaved": False, "layout": 2},
        # one prompt below 800 tokens is read back, small model: latency
        {"name": "read_one_prompt", "op": "read", "format": INT8, "hq": 16, "hkv": 2, "pages": 47, "spare": 10, "layout": 3},
        # the branches of a whole question are read back ahead of a long chunk: bandwidth
        {"name": "read_branches", "op": "read", "format": E4M3, "hq": 40, "hkv": 8, "pages": 4128, "spare": 33, "layout": 4},
        # the smallest call: one new token for each of four short branches; its time is latency
        {"name": "attn_one_token_small", "op": "attn", "format": E4M3, "hq": 8, "hkv": 2, "prefix": 256, "n": 4, "rows": 1, "tree": False,
         "len_lo": 200, "len_hi": 256, "lse": False, "layout": 5},
        # the verify step of the 32B shape: 16 branches, three drafted tokens each
        {"name": "attn_verify_32b", "op": "attn", "format": E4M3, "hq": 40, "hkv": 8, "prefix": 512, "n": 16, "rows": 4, "tree": False,
         "len_lo": 3500, "len_hi": 4600, "lse": False, "layout": 6},
        # plain decoding of 64 branches of different questions, ragged: bandwidth
        {"name": "attn_one_token_64", "op": "attn", "format": INT8, "hq": 40, "hkv": 8, "prefix": 0, "n": 64, "rows": 1, "tree": False,
         "len_lo": 1024, "len_hi": 8192, "lse": True, "layout": 7},
        # draft trees of 60 nodes in 8 branches: 300 rows for each key
        {"name": "attn_trees_60", "op": "attn", "format": E4M3, "hq": 40, "hkv": 8, "prefix": 512, "n": 8, "rows": 60, "tree": True,
         "len_lo": 7000, "len_hi": 7800, "lse": False, "layout": 8},
        # one question's four beams, the 3B shape's vocabulary: latency
        {"name": "select_4_beams", "op": "select", "groups": 1, "beams": 4, "select": 4, "vocab": 151936, "bf16": True, "done": 0, "layout": 9},
        # sixteen questions of sixteen beams, some of them finished, the 32B shape's vocabulary: bandwidth
        {"name": "select_16_x_16", "op": "select", "groups": 16, "beams": 16, "select": 16, "vocab": 152064, "bf16": True, "done": 20, "layout": 10},
        # token histories, running figures and last hidden states of 16 beams: few bytes, odd rows
        {"name": "reorder_small", "op": "reorder", "n": 16, "children": 16, "arrays": 5, "bytes_lo": 12, "bytes_hi": 33000, "layout": 11},
        # the dense caches of a small draft model, K and V of 24 layers: bandwidth
        {"name": "reorder_draft_caches", "op": "reorder", "n": 16, "children": 16, "arrays": 48, "bytes_lo": 524288, "bytes_hi": 524288, "layout": 12},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "read", "attn", "attn", "attn", "select", "reorder"])
    layout, fmt = rng.randrange(100, 1 << 20), rng.choice([E4M3, INT8])
    hq, hkv = rng.choice([(8, 2), (16, 2), (40, 8), (8, 8), (12, 1), (28, 4), (32, 8)])
    if kind == "append":
        n = _spread(rng, 1, 64)
        hi = _spread(rng, 1, 14000 // n)
        return {"op": "append", "format": fmt, "hq": hq, "hkv": hkv, "prefix": 16 * rng.choice([0, _spread(rng, 1, 64)]), "n": n,
                "rows_lo": max(1, hi // 3), "rows_hi": hi, "ctx_lo": 0, "ctx_hi": _spread(rng, 1, 60000 // n), "rope": rng.random() < 0.75,
                "pairs": rng.choice([64, 64, 32, 48, 20]), "interleaved": rng.random() < 0.5, "layout": layout}
    if kind == "read":
        return {"op": "read", "format": fmt, "hq": hq, "hkv": hkv, "pages": _spread(rng, 1, 4000), "spare": rng.randrange(100), "layout": layout}
    if kind == "attn":
        rows = rng.choice([1, 1, rng.randrange(2, 9), _spread(rng, 2, 64)])
        n = _spread(rng, 1, max(1, min(64, 400 // rows)))
        hi = max(rows, _spread(rng, 16, min(32000, 240000 // n)))
        return {"op": "attn", "format": fmt, "hq": hq, "hkv": hkv, "prefix": 16 * rng.choice([0, 0, _spread(rng, 1, 64)]), "n": n, "rows": rows,
                "tree": rows > 1 and rng.random() < 0.5, "len_lo": max(rows, hi // rng.choice([1, 2, 8])), "len_hi": hi, "lse": rng.random() < 0.5,
                "layout": layout}
    if kind == "select":
        groups, beams = _spread(rng, 1, 16), _spread(rng, 1, 16)
        vocab = rng.choice([1024, 32000, 50257, 151936, 152064, _spread(rng, 200, 150000)])
        return {"op": "select", "groups": groups, "beams": beams, "select": min(vocab, _spread(rng, 1, 64)), "vocab": vocab, "bf16": rng.random() < 0.7,
                "done": rng.choice([0, rng.randrange(0, groups * beams)]), "layout": layout}
    n = _spread(rng, 1, 64)
    arrays = _spread(rng, 1, 64)
    hi = _spread(rng, 16, 400000000 // (n * arrays))
    return {"op": "reorder", "n": n, "children": _spread(rng, 1, n), "arrays": arrays, "bytes_lo": max(1, hi // 4), "bytes_hi": hi, "layout": layout}


# ----------------------------------------------------------------- what a case fixes, whatever the seed is
def _plan(case):
    """Lengths, page tables, trees and sizes of a case, on the host: they belong to the case, so that work() knows them."""
    r = random.Random(case["layout"])
    op = case["op"]
    if op == "read":
        total = case["pages"] + case["spare"]
        return {"src": r.sample(range(total), case["pages"]), "dst": r.sample(range(case["pages"]), case["pages"]), "pages": total}
    if op == "select":
        rows = case["groups"] * case["beams"]
        return {"done": sorted(r.sample(range(rows), min(case["done"], rows)))}
    if op == "reorder":
        return {"bytes": [r.randint(case["bytes_lo"], case["bytes_hi"]) for _ in range(case["arrays"])],
                "parents": sorted(r.randrange(case["n"]) for _ in range(case["children"]))}
    if op == "append":
        chunk = [r.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["n"])]
        lens = [c + r.randint(case["ctx_lo"], case["ctx_hi"]) for c in chunk]
    else:
        chunk = [case["rows"]] * case["n"]
        lens = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["n"])]
    shared = case["prefix"] // PAGE
    need = [-(-x // PAGE) for x in lens]
    pages = list(range(shared + sum(need) + 3))
    r.shuffle(pages)
    at, rows = shared, []
    for n in need:
        rows.append(pages[:shared] + pages[at:at + n])
        at += n
    plan = {"chunk": chunk, "lens": lens, "rows": rows, "pages": len(pages)}
    if op == "append":      # the pages that take a new token
        plan["touched"] = [row[i] for row, c, n in zip(rows, chunk, lens) for i in range((case["prefix"] + n - c) // PAGE, len(row))]
    elif case["tree"]:      # a node's parent is a node before it, or none: depths as drafts have them
        plan["parents"] = [[max(-1, i - 1 - r.randrange(0, 12)) for i in range(case["rows"])] for _ in range(case["n"])]
    return plan


def _inv_freq(case):
    return [ROPE_BASE ** (-i / case["pairs"]) for i in range(case["pairs"])]


def _seen(case, plan):
    """How many of its branch's last rows each row sees, summed over the rows of a branch."""
    rows = case["rows"]
    if not case["tree"]:
        return [rows * (rows + 1) // 2] * case["n"]
    out = []
    for parents in plan["parents"]:
        depth = []
        for p in parents:
            depth.append(1 + (depth[p] if p >= 0 else 0))
        out.append(sum(depth))
    return out


def work(case):
    plan, op = _plan(case), case["op"]
    if op == "append":
        rows, hq, hkv = sum(plan["chunk"]), case["hq"], case["hkv"]
        rotary = rows * (hq * DIM * 4 + 4) if case["rope"] else 0
        return {"bytes": rotary + rows * hkv * (2 * DIM * 2 + 2 * (DIM + 4)) + len(plan["touched"]) * hkv * (RECORD + PAGE * DIM * 4),
                "flops": rows * (hq + hkv) * case["pairs"] * 6 if case["rope"] else 0}
    if op == "read":
        return {"bytes": case["pages"] * case["hkv"] * (RECORD + PAGE * DIM * 4), "flops": 0}
    if op == "attn":
        keys = sum(plan["lens"]) + case["prefix"]                       # every cached token once, the shared ones once
        rows = sum(plan["chunk"])
        seen = sum(case["rows"] * (case["prefix"] + n - case["rows"]) + s for n, s in zip(plan["lens"], _seen(case, plan)))
        return {"bytes": keys * case["hkv"] * (2 * DIM + 8) + rows * case["hq"] * (DIM * 4 + (4 if case["lse"] else 0)), "flops": 4 * DIM * case["hq"] * seen}
    if op == "select":
        rows = case["groups"] * case["beams"] - len(plan["done"])
        return {"bytes": rows * case["vocab"] * (2 if case["bf16"] else 4), "flops": 3 * rows * case["vocab"]}
    children, sources = len(plan["parents"]), len(set(plan["parents"]))
    return {"bytes": sum(plan["bytes"]) * (children + sources), "flops": 0}


# ------------------------------------------------------------------------------------- the 8-bit cache, plainly
def _place():
    """[16][8]: where the 16-byte chunk c of token t lies among the eight of its row."""
    t = torch.arange(PAGE, device="cuda")[:, None]
    return torch.arange(8, device="cuda")[None, :] ^ ((t & 1) | (t >> 2 << 1))


def _quantised(x, fmt):
    """Codes (bytes) and scales of the vectors x [...][128]: a scale for each vector."""
    top = torch.full((), LARGEST[fmt], device="cuda")                   # (a tensor: the division is one rounding on the GPU too)
    scale = (x.abs().amax(-1, keepdim=True) / top).clamp_min(LEAST)
    y = x / scale
    code = y.clamp(-LARGEST[fmt], LARGEST[fmt]).to(torch.float8_e4m3fn) if fmt == E4M3 else y.round().clamp(-127, 127).to(torch.int8)
    return code.view(torch.uint8), scale[..., 0]


def _records(k, v, fmt):
    """Records of whole pages k, v [pages][heads][16][128]."""
    parts, scales = [], []
    for x in (k, v):
        code, scale = _quantised(x, fmt)
        code = code.view(*code.shape[:3], 8, 16)
        parts.append(torch.gather(code, 3, _place()[:, :, None].expand(code.shape)).flatten(2))      # (the exchange is its own inverse)
        scales.append(scale.contiguous().view(torch.uint8))
    return torch.cat(parts + scales, -1)


def _values(records, fmt, dtype=torch.float32):
    """(k, v) [...][16][128] of records [...][4224]."""
    code = records[..., :2 * PAGE * DIM].unflatten(-1, (2, PAGE, 8, 16))
    code = torch.gather(code, -2, _place()[:, :, None].expand(code.shape)).flatten(-2)
    code = code.view(torch.float8_e4m3fn if fmt == E4M3 else torch.int8).to(dtype)
    scale = records[..., 2 * PAGE * DIM:].contiguous().view(torch.float32).unflatten(-1, (2, PAGE)).to(dtype)
    x = code * scale[..., None]
    return x.unbind(-3)


# ----------------------------------------------------------------------------------------------- inputs
def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    plan, op = _plan(case), case["op"]
    gen = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    s = {"case": case}
    if op == "select":
        rows = case["groups"] * case["beams"]
        s["logits"] = (normal(rows, case["vocab"], dtype=torch.float32) * 3).to(torch.bfloat16 if case["bf16"] else torch.float32)
        s["scores"] = torch.rand(rows, generator=gen, device="cuda") * -8 - 4      # beams of one question stay close together
        s["finished"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s["finished"][_ints(plan["done"]).long()] = 1
        shape = (case["groups"], case["select"])
        s["parents"], s["tokens"], s["new_scores"] = (torch.empty(shape, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32))
    elif op == "reorder":
        n = case["n"]
        s["src"] = [torch.randint(0, 256, (n, b), generator=gen, device="cuda", dtype=torch.uint8) for b in plan["bytes"]]
        s["dst"] = [torch.zeros(case["children"], b, device="cuda", dtype=torch.uint8) for b in plan["bytes"]]
        s["parents"], s["bytes"] = _ints(plan["parents"]), plan["bytes"]
    else:
        hkv, fmt = case["hkv"], case["format"]
        # tokens and heads differ in size, and the first of a sequence is larger than the others, as in trained models
        size = (normal(plan["pages"], hkv, PAGE, 1, dtype=torch.float32) * 0.3).exp()
        s["pool"] = _records(normal(plan["pages"], hkv, PAGE, DIM, dtype=torch.float32) * size, normal(plan["pages"], hkv, PAGE, DIM, dtype=torch.float32) * size.flip(2), fmt)
        if op == "read":
            s["src"], s["dst"] = _ints(plan["src"]), _ints(plan["dst"])
        else:
            width = max(1, max(len(row) for row in plan["rows"]))
            s["table"] = _ints([row + [-1] * (width - len(row)) for row in plan["rows"]])
            s["lens"], s["n"] = _ints(plan["lens"]), case["n"]
        if op == "append":
            starts = [0]
            for c in plan["chunk"]:
                starts.append(starts[-1] + c)
            rows = starts[-1]
            s |= {"row_start": _ints(starts), "rows": rows, "src": _ints(plan["touched"]), "dst": torch.arange(len(plan["touched"]), dtype=torch.int32, device="cuda")}
            qkv = normal(rows, case["hq"] + 2 * hkv, DIM)               # the projection's result: q, k and v side by side
            s["q"], s["k_new"], s["v_new"] = qkv[:, :case["hq"]], qkv[:, case["hq"]:case["hq"] + hkv], qkv[:, case["hq"] + hkv:]
            s["q_out"] = torch.empty(rows, case["hq"], DIM, device="cuda", dtype=torch.bfloat16)
            chunk = _ints(plan["chunk"]).long()
            s["branch"] = torch.repeat_interleave(torch.arange(s["n"], device="cuda"), chunk, output_size=rows)
            # each row's place in its sequence
            s["place"] = torch.arange(rows, device="cuda") - s["row_start"].long()[s["branch"]] + (s["lens"].long() - chunk)[s["branch"]] + case["prefix"]
            s["positions"] = s["place"].to(torch.int32)[None].contiguous()
            s["inv_freq"] = _inv_freq(case)
        if op == "attn":
            s["q"] = normal(case["n"] * case["rows"], case["hq"], DIM)
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(s["q"].shape[:2], device="cuda") if case["lse"] else None
            s["parents"] = _ints(plan["parents"]) if case["tree"] else None
        else:
            s["k"], s["v"] = (torch.empty(s["dst"].numel(), hkv, PAGE, DIM, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    if own:
        # the handle that a server keeps: a context for this model and pool
        import paper_2505_19634_b200 as tts
        rows = case["groups"] * case["beams"] if op == "select" else case.get("n", 1)
        s["ctx"] = tts.TtsContext(case.get("hq", 8), case.get("hkv", 2), rows, case.get("rows", 1), s["table"].shape[1] if "table" in s else 1, plan.get("pages", 1))
        if op == "select":
            s["ctx"].tts_beam_reserve(rows, case["select"])
        elif op == "reorder":
            s["states"] = tts.TtsStates(s["src"], s["dst"], s["bytes"])
        elif op == "append" and case["rope"]:
            s["rope"] = tts.TtsRope([0] * case["pairs"], s["inv_freq"], case["interleaved"])
    return s


# ----------------------------------------------------------------------------------------------- passes
def run(state):
    return {"append": _append, "read": _read, "attn": _attn, "select": _select, "reorder": _reorder}[state["case"]["op"]](state)


def _turn(x, cos, sin, pairs, interleaved):
    """x rotated by the angles of its first `pairs` pairs, in 32 bits; the dims past them stay."""
    x = x.float()
    turned, rest = x[..., :2 * pairs], x[..., 2 * pairs:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else (turned[..., :pairs], turned[..., pairs:])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1)
    return torch.cat((turned, rest), -1)


def _append(s):
    """Rows into the cache, and their pages read back, as a chunk that is to attend to them does."""
    case = s["case"]
    fmt, rotary = case["format"], case["rope"]
    if own:
        ctx = s["ctx"]
        if rotary:
            ctx.tts_kv8_append(fmt, s["rope"], s["q"], s["q"].stride(0), s["k_new"], s["v_new"], s["k_new"].stride(0), s["positions"], s["pool"], s["table"],
                               case["prefix"], s["lens"], s["row_start"], s["n"], s["rows"], s["q_out"])
        else:
            ctx.tts_kv8_append(fmt, None, None, 0, s["k_new"], s["v_new"], s["k_new"].stride(0), None, s["pool"], s["table"], case["prefix"], s["lens"],
                               s["row_start"], s["n"], s["rows"], None)
        ctx.tts_kv8_read(fmt, s["pool"], s["src"], s["dst"], s["src"].numel(), s["k"], s["v"], s["k"].shape[0])
    else:
        k, v = s["k_new"].float(), s["v_new"].float()
        if rotary:
            freq = torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
            angle = s["positions"][0].double()[:, None] * freq                  # row, pair; in 64 bits: positions are far
            cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
            s["q_out"].copy_(_turn(s["q"], cos, sin, case["pairs"], case["interleaved"]))
            k = _turn(s["k_new"], cos, sin, case["pairs"], case["interleaved"])
        page, slot = s["table"].long()[s["branch"], s["place"] // PAGE][:, None, None], (s["place"] % PAGE)[:, None, None]
        head, kv = torch.arange(case["hkv"], device="cuda"), torch.arange(2, device="cuda")[:, None]
        code, scale = _quantised(torch.stack((k, v), 1), fmt)                   # row, K or V, head
        scales = s["pool"][..., 2 * PAGE * DIM:].unflatten(-1, (2, PAGE, 4))
        scales[page, head, kv, slot] = scale.contiguous()[..., None].view(torch.uint8)
        codes = s["pool"][..., :2 * PAGE * DIM].unflatten(-1, (2, PAGE, 8, 16))
        codes[page[..., None], head[:, None], kv[..., None], slot[..., None], _place()[slot]] = code.unflatten(-1, (8, 16))
        _read(s)
    return {"k": s["k"], "v": s["v"]} | ({"q": s["q_out"]} if rotary else {})


def _read(s):
    if own:
        s["ctx"].tts_kv8_read(s["case"]["format"], s["pool"], s["src"], s["dst"], s["src"].numel(), s["k"], s["v"], s["k"].shape[0])
    else:
        k, v = _values(s["pool"][s["src"].long()], s["case"]["format"])
        s["k"][s["dst"].long()] = k.to(torch.bfloat16)
        s["v"][s["dst"].long()] = v.to(torch.bfloat16)
    return {"k": s["k"], "v": s["v"]}


def _visible(s, width):
    """[branch][row][key]: what each row sees of its branch's tokens."""
    case = s["case"]
    rows, total = case["rows"], s["lens"].long() + case["prefix"]
    key = torch.arange(width, device="cuda")
    tail = key - (total - rows)[:, None]                                        # a key's place among the last rows
    if case["tree"]:
        # ancestors by repeated squaring of "is itself or its parent"
        parent = s["parents"].long()
        reach = torch.eye(rows, device="cuda").repeat(case["n"], 1, 1)
        reach[torch.arange(case["n"], device="cuda")[:, None], torch.arange(rows, device="cuda"), parent.clamp_min(0)] += (parent >= 0).float()
        for _ in range(6):
            reach = (reach @ reach).clamp_max(1)
        mine = reach > 0
    else:
        mine = torch.ones(rows, rows, dtype=torch.bool, device="cuda").tril().expand(case["n"], -1, -1)
    inside = (tail >= 0) & (tail < rows)
    late = torch.gather(mine, 2, tail.clamp(0, rows - 1)[:, None].expand(-1, rows, -1))
    return (tail < 0)[:, None] | (inside[:, None] & late)


def _attn(s):
    case = s["case"]
    n, rows, hq, hkv = case["n"], case["rows"], case["hq"], case["hkv"]
    if own:
        s["ctx"].tts_kv8_attn(case["format"], s["q"], s["q"].stride(0), s["pool"], s["table"], case["prefix"], s["lens"], s["parents"], n, rows, s["out"], s["lse"])
    else:
        k, v = (x.permute(0, 2, 1, 3, 4).flatten(2, 3) for x in _values(s["pool"][s["table"].long().clamp_min(0)], case["format"]))     # branch, head, key
        q = s["q"].float().view(n, rows, hkv, hq // hkv, DIM).permute(0, 2, 3, 1, 4).flatten(2, 3)                                    # branch, head, (group, row)
        seen = _visible(s, k.shape[2])[:, None, None]
        score = torch.matmul(q, k.transpose(-1, -2)).mul_(DIM ** -0.5).unflatten(2, (hq // hkv, rows)).masked_fill_(~seen, -math.inf)
        top = score.amax(-1, keepdim=True)
        score = score.sub_(top).exp_()
        total = score.sum(-1, keepdim=True)
        o = torch.matmul(score.flatten(2, 3), v).unflatten(2, (hq // hkv, rows)) / total
        s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(n * rows, hq, DIM))
        if s["lse"] is not None:
            s["lse"].copy_((top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(n * rows, hq))
    return {"out": s["out"]} | ({"lse": s["lse"]} if s["lse"] is not None else {})


def _select(s):
    case = s["case"]
    if own:
        s["ctx"].tts_beam_select(s["logits"], 0 if case["bf16"] else 1, case["vocab"], case["vocab"], s["scores"], s["finished"], 0, case["groups"], case["beams"], case["select"],
                                 s["parents"], s["tokens"], s["new_scores"])
    else:
        # in 64 bits: whether one candidate is better than another must not hang on a rounding
        x = s["logits"].double()
        top = x.amax(-1, keepdim=True)
        x = s["scores"].double()[:, None] + (x - (top + (x - top).exp().sum(-1, keepdim=True).log()))
        alone = torch.full_like(x[:1], -math.inf)
        alone[0, 0] = 0                                                         # a finished beam goes on as it is, with the filling token 0
        x = torch.where(s["finished"][:, None] != 0, s["scores"].double()[:, None] + alone, x)
        best, index = x.view(case["groups"], -1).sort(dim=-1, descending=True, stable=True)          # ties: lowest beam, then token
        best, index = best[:, :case["select"]], index[:, :case["select"]]
        none = best == -math.inf
        first = torch.arange(case["groups"], device="cuda")[:, None] * case["beams"]
        s["parents"].copy_(torch.where(none, -1, first + index // case["vocab"]))
        s["tokens"].copy_(torch.where(none, -1, index % case["vocab"]))
        s["new_scores"].copy_(best)
    return {"parents": s["parents"], "tokens": s["tokens"], "scores": s["new_scores"]}


def _wide(a):
    """Rows of bytes as rows of 64-bit words, where they are."""
    return a.view(torch.int64) if a.shape[1] % 8 == 0 else a


def _reorder(s):
    if own:
        s["ctx"].tts_beam_reorder(s["states"], s["parents"], s["case"]["n"], s["parents"].numel())
    else:
        parent = s["parents"].long()
        [torch.index_select(_wide(a), 0, parent, out=_wide(b)) for a, b in zip(s["src"], s["dst"])]
    return s["dst"]


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """From the definitions, in 64 bits: branch by branch, row by row."""
    s = prepare(case, seed)
    return {"append": _exact_append, "read": _exact_read, "attn": _exact_attn, "select": _exact_select, "reorder": _exact_reorder}[case["op"]](s)


def _exact_pages(s, pages):
    """(k, v) of the pages, token by token of a page."""
    fmt = s["case"]["format"]
    rec = s["pool"][pages.long()]
    out = torch.empty(2, *rec.shape[:2], PAGE, DIM, dtype=torch.float64, device="cuda")
    scale = rec[..., 2 * PAGE * DIM:].contiguous().view(torch.float32).double()
    for kv in range(2):
        for t in range(PAGE):
            for c in range(8):
                at = (kv * PAGE + t) * DIM + 16 * (c ^ ((t & 1) | (t // 4 * 2)))
                code = rec[..., at:at + 16].contiguous().view(torch.float8_e4m3fn if fmt == E4M3 else torch.int8)
                out[kv, :, :, t, 16 * c:16 * c + 16] = code.double() * scale[..., kv * PAGE + t, None]
    return out[0], out[1]


def _exact_read(s):
    k, v = _exact_pages(s, s["src"])
    back = s["dst"].long().argsort()
    return {"k": k[back], "v": v[back]}


def _nearest(x, fmt):
    """The values that codes and a 32-bit scale can hold next to the vectors x, in 64 bits."""
    scale = (x.abs().amax(-1, keepdim=True) / LARGEST[fmt]).clamp_min(LEAST).float().double()
    y = (x / scale).clamp(-LARGEST[fmt], LARGEST[fmt])
    # e4m3: three bits behind the leading one, down to steps of 2^-9
    step = torch.exp2((torch.frexp(y).exponent - 4).clamp_min(-9).double()) if fmt == E4M3 else torch.ones_like(y)
    return (y / step).round() * step * scale


def _exact_append(s):
    case = s["case"]
    k, v = _exact_pages(s, s["src"])
    q, k_new = s["q"].double(), s["k_new"].double()
    if case["rope"]:
        turn = s["positions"][0].double()[:, None] * torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.ones_like(turn), turn)[:, None]
        m = case["pairs"]
        lo = (torch.arange(m, device="cuda") * 2) if case["interleaved"] else torch.arange(m, device="cuda")
        hi = lo + 1 if case["interleaved"] else lo + m
        for x in (q, k_new):
            z = torch.complex(x[..., lo], x[..., hi]) * turn
            x[..., lo], x[..., hi] = z.real, z.imag
    index = torch.full((s["pool"].shape[0],), -1, device="cuda")
    index[s["src"].long()] = torch.arange(s["src"].numel(), device="cuda")
    page = index[s["table"].long()[s["branch"], s["place"] // PAGE]]
    k[page, :, s["place"] % PAGE] = _nearest(k_new, case["format"])
    v[page, :, s["place"] % PAGE] = _nearest(s["v_new"].double(), case["format"])
    return {"k": k, "v": v} | ({"q": q} if case["rope"] else {})


def _exact_attn(s):
    case = s["case"]
    rows, hq, hkv = case["rows"], case["hq"], case["hkv"]
    out = torch.zeros(case["n"], rows, hq, DIM, device="cuda", dtype=torch.float64)
    lse = torch.zeros(case["n"], rows, hq, device="cuda", dtype=torch.float64)
    for b, n in enumerate(s["lens"].tolist()):
        total = n + case["prefix"]
        k, v = (x.transpose(0, 1).flatten(1, 2)[:, :total] for x in _exact_pages(s, s["table"][b, :-(-total // PAGE)]))
        hidden = torch.zeros(rows, total, dtype=torch.bool, device="cuda")
        parents = s["parents"][b].tolist() if case["tree"] else list(range(-1, rows - 1))
        hidden[:, total - rows:] = True
        sees = []
        for i, p in enumerate(parents):
            sees.append([i] + (sees[p] if p >= 0 else []))
            hidden[i, [total - rows + a for a in sees[i]]] = False
        for h in range(hq):
            z = (s["q"].view(-1, rows, hq, DIM)[b, :, h].double() @ k[h * hkv // hq].T / math.sqrt(DIM)).masked_fill_(hidden, -math.inf)
            lse[b, :, h] = torch.logsumexp(z, 1)
            out[b, :, h] = torch.softmax(z, 1) @ v[h * hkv // hq]
    return {"out": out.flatten(0, 1)} | ({"lse": lse.flatten(0, 1)} if s["lse"] is not None else {})


def _exact_select(s):
    case = s["case"]
    best = []
    for r in range(case["groups"] * case["beams"]):
        if s["finished"][r]:
            best.append(s["scores"][r:r + 1].double())
        else:
            best.append(torch.log_softmax(s["logits"][r].double(), 0).topk(case["select"]).values + s["scores"][r].double())
    per = case["beams"]
    rows = [torch.cat(best[g * per:(g + 1) * per]).sort(descending=True).values for g in range(case["groups"])]
    scores = torch.full((case["groups"], case["select"]), -math.inf, dtype=torch.float64, device="cuda")
    for g, x in enumerate(rows):
        scores[g, :min(case["select"], x.numel())] = x[:case["select"]]
    return {"parents": None, "tokens": None, "scores": scores}


def _exact_reorder(s):
    return [torch.stack([a[p] for p in s["parents"].tolist()]) for a in s["src"]]
