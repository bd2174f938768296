"""Plain implementations, in 64 bits or in whole numbers, of the 8-bit cache and of beam selection.  Nothing here calls the
library.  Works on CPU and GPU tensors alike."""
from __future__ import annotations

import math
import random

import torch

PAGE, DIM, RECORD = 16, 128, 4224
E4M3, INT8 = 0, 1
LARGEST = (448.0, 127.0)


def table(fmt, device="cpu"):
    """The value of every code 0 .. 255 in 64 bits; NaN where a code has none."""
    if fmt == INT8:
        return torch.arange(256, dtype=torch.float64, device=device).sub(256 * (torch.arange(256, device=device) > 127))
    out = []
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v = math.ldexp(f, -9) if e == 0 else math.ldexp(8 + f, e - 10)
        out.append(math.nan if c & 127 == 127 else -v if c >> 7 else v)
    return torch.tensor(out, dtype=torch.float64, device=device)


def scales(x, fmt):
    """fp32 scales of the fp32 vectors x [..][128]."""
    return (x.abs().amax(-1) / torch.full((), LARGEST[fmt], device=x.device)).clamp_min(2.0 ** -120)


def codes(x, scale, fmt):
    """The codes nearest to x / scale (an fp32 quotient), ties to the even code, by comparing with all of them."""
    y = (x / scale[..., None]).double()
    values = table(fmt, x.device)
    order = values.nan_to_num(math.inf).argsort(stable=True)
    order = order[~values[order].isnan()]
    if fmt == E4M3:
        order = order[order != 128]                                 # (-0 is told from 0 below)
    sorted_values = values[order]
    hi = torch.searchsorted(sorted_values, y.contiguous()).clamp(1, order.numel() - 1)
    lo = hi - 1
    below, above = y - sorted_values[lo], sorted_values[hi] - y
    even = (order[lo] & 1) == 0
    pick = torch.where((below < above) | ((below == above) & even), order[lo], order[hi])
    if fmt == E4M3:
        pick = torch.where((pick == 0) & (torch.signbit(y)), 128, pick)
    return pick.to(torch.uint8)


def place(t, c):
    return c ^ ((t & 1) | (t >> 2 << 1))


def pack(code_k, code_v, scale_k, scale_v):
    """Records [..][4224] of codes [..][16][128] and scales [..][16]."""
    out = torch.zeros(*code_k.shape[:-2], RECORD, dtype=torch.uint8, device=code_k.device)
    for kv, code in enumerate((code_k, code_v)):
        for t in range(PAGE):
            for c in range(8):
                at = (kv * PAGE + t) * DIM + 16 * place(t, c)
                out[..., at:at + 16] = code[..., t, 16 * c:16 * c + 16]
    for kv, s in enumerate((scale_k, scale_v)):
        out[..., 4096 + 64 * kv:4160 + 64 * kv] = s.contiguous().view(torch.uint8)
    return out


def unpack(records):
    """(codes, scales) of K and V: [..][2][16][128] bytes, [..][2][16] fp32."""
    code = torch.zeros(*records.shape[:-1], 2, PAGE, DIM, dtype=torch.uint8, device=records.device)
    for kv in range(2):
        for t in range(PAGE):
            for c in range(8):
                at = (kv * PAGE + t) * DIM + 16 * place(t, c)
                code[..., kv, t, 16 * c:16 * c + 16] = records[..., at:at + 16]
    return code, records[..., 4096:].contiguous().view(torch.float32).unflatten(-1, (2, PAGE))


def values(records, fmt):
    """(K, V) [..][16][128] in 64 bits."""
    code, scale = unpack(records)
    x = table(fmt, records.device)[code.long()] * scale.double()[..., None]
    return x[..., 0, :, :], x[..., 1, :, :]


class Cache8:
    """An 8-bit paged cache: tables, lengths, one pool; NaN codes and scales in every slot that holds no token."""

    def __init__(self, fmt, hkv, lens, prefix=0, seed=0, device="cuda", spare=3, extra_blocks=0, num_pages=None, spread=0.3, poison=True):
        r = random.Random(seed)
        gen = torch.Generator().manual_seed(seed)
        self.fmt, self.hkv, self.prefix, self.lens, self.n = fmt, hkv, prefix, list(lens), len(lens)
        shared, need = prefix // PAGE, [-(-max(0, x) // PAGE) for x in lens]
        total = shared + sum(need) + spare
        self.num_pages = num_pages or total
        # with a given number of pages the used ones are the pool's last, behind what 32-bit offsets reach
        ids = r.sample(range(total), total) if num_pages is None else [num_pages - 1 - i for i in r.sample(range(total), total)]
        at, self.rows = shared, []
        for n in need:
            self.rows.append(ids[:shared] + ids[at:at + n])
            at += n
        self.width = max(1, max(len(x) for x in self.rows)) + extra_blocks
        self.table = torch.tensor([x + [-1] * (self.width - len(x)) for x in self.rows], dtype=torch.int32, device=device)
        self.branch_lens = torch.tensor(lens, dtype=torch.int32, device=device)
        k, v = (torch.randn(total, hkv, PAGE, DIM, generator=gen) * torch.exp(spread * torch.randn(total, hkv, PAGE, 1, generator=gen)) for _ in range(2))
        rec = pack(codes(k, scales(k, fmt), fmt), codes(v, scales(v, fmt), fmt), scales(k, fmt), scales(v, fmt))
        if poison:
            code, scale = unpack(rec)
            used = torch.zeros(total, PAGE, dtype=torch.bool)
            index = {p: i for i, p in enumerate(sorted(ids))}
            for b, row in enumerate(self.rows):
                for i, page in enumerate(row):
                    used[index[page], :max(0, min(PAGE, prefix + lens[b] - i * PAGE))] = True
            code.permute(0, 3, 1, 2, 4)[~used] = 127                # NaN of e4m3
            scale.permute(0, 3, 1, 2)[~used] = math.nan
            rec = pack(code[..., 0, :, :], code[..., 1, :, :], scale[..., 0, :], scale[..., 1, :])
        self.first = min(ids)
        if num_pages is None:
            self.pool = rec.to(device)
        else:
            self.pool = torch.empty(num_pages, hkv, RECORD, dtype=torch.uint8, device=device)
            self.pool[self.first:] = rec.to(device)

    def kv(self, b):
        """(K, V) [heads][tokens][128] of branch b in 64 bits."""
        total = self.prefix + self.lens[b]
        pages = torch.tensor(self.rows[b], dtype=torch.long, device=self.pool.device)
        return tuple(x.transpose(0, 1).flatten(1, 2)[:, :total] for x in values(self.pool[pages], self.fmt))


def sees(rows, total, parents=None):
    """[rows][total]: what each row sees of a branch of `total` tokens whose last `rows` are a chain, or a tree."""
    out = torch.zeros(rows, total, dtype=torch.bool)
    out[:, :max(0, total - rows)] = True
    for i in range(rows):
        a = i
        while a >= 0:
            if total - rows + a >= 0:
                out[i, total - rows + a] = True
            a = a - 1 if parents is None else parents[a]
    return out


def attention(c: Cache8, q, rows, parents=None, scale=None):
    """(out, lse, bound): in 64 bits, and how far an element and a logarithm may be off, from the formula: probabilities times V's
    scale are rounded to fp16 (2^-11 of the softmax mean of |V|; below 2^-14 of their unit an absolute 2^-25 of it, the unit being at
    most 2^-5 of the largest scale of V), scores are sums of 128 exact products in fp32, whose additions lose at most 2^-23 of the
    sum of magnitudes each, and the exponential is good to 2^-22."""
    scale = scale or DIM ** -0.5
    n_rows, hq, _ = q.shape
    group = hq // c.hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    bound, lse, lse_bound = torch.zeros_like(out), torch.full((n_rows, hq), -math.inf, dtype=torch.float64, device=q.device), torch.zeros(n_rows, hq, dtype=torch.float64, device=q.device)
    for b in range(c.n):
        total = c.prefix + c.lens[b]
        if total <= 0:
            continue
        k, v = (x.repeat_interleave(group, 0) for x in c.kv(b))
        at = slice(b * rows, (b + 1) * rows)
        x = q[at].double().transpose(0, 1)
        hidden = ~sees(rows, total, parents[b] if parents is not None else None).to(q.device)
        s = (x @ k.transpose(1, 2) * scale).masked_fill(hidden, -math.inf)
        l = torch.logsumexp(s, -1)
        p = torch.exp(s - torch.where(l == -math.inf, 0.0, l)[..., None])
        off = (x.abs() @ k.abs().transpose(1, 2) * scale).nan_to_num(0).masked_fill(hidden, 0).amax(-1) * 128 * 2.0 ** -23 + 2.0 ** -21
        out[at] = (p @ v).transpose(0, 1)
        mean = p @ v.abs()
        bound[at] = (mean * (2.0 ** -11 + 3 * off[..., None]) + total * 2.0 ** -29 * v.abs().amax(dim=(1, 2))[:, None, None]).transpose(0, 1)
        lse[at], lse_bound[at] = l.T, off.T + l.T.abs().nan_to_num(0, 0, 0) * 2.0 ** -22
    return out, lse, bound, lse_bound


def assert_attention(c, q, rows, out, lse=None, parents=None, scale=None):
    want, want_lse, bound, lse_bound = attention(c, q, rows, parents, scale)
    step = torch.finfo(out.dtype).eps / 2
    over = (out.double() - want).abs() - bound - want.abs() * step - torch.finfo(torch.float32).tiny
    assert torch.isfinite(out).all()
    assert over.max() <= 0, f"element {over.argmax().item()} over its bound by {over.max().item():.3e}"
    if lse is not None:
        none = want_lse == -math.inf
        assert torch.equal(none, lse == -math.inf)
        assert ((lse.double() - want_lse).abs()[~none] <= lse_bound[~none]).all()


# ------------------------------------------------------------------------------------------------ beams
def select(logits, scores, finished, pad, groups, beams, k):
    """[(parent, token, score in 64 bits)] per question, from the definition."""
    x = logits.double().cpu()
    out = []
    for g in range(groups):
        every = []
        for b in range(beams):
            r = g * beams + b
            before = float(scores[r])
            if not math.isfinite(before):
                continue
            if finished is not None and int(finished[r]):
                every.append((-before, b, pad))
                continue
            z = torch.logsumexp(x[r], 0)
            if not torch.isfinite(z) or x[r].isnan().any():
                continue
            s = before + (x[r] - z)
            # a row's candidates beyond its k best by (score, token) cannot be among the question's
            best = torch.sort(-s, stable=True)
            every += [(float(v), b, int(t)) for v, t in zip(best.values[:k], best.indices[:k]) if v < math.inf]
        every.sort()
        got = [(g * beams + b, t, -v) for v, b, t in every[:k]]
        out.append(got + [(-1, -1, -math.inf)] * (k - len(got)))
    return out
