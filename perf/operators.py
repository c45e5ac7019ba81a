"""Timed cases of the operators around a cache held in pages of 8-bit rows: rotary positions, the compaction that quantises into
pages, the append of new tokens' rows, the attention over the pages, and the pages' own management.

A case is a plain dict; `op` names the operator:

    rotate   queries and keys of the same tokens are rotated by their positions (part of the head, both pairings, scalings)
    store    the compaction of selected rows and window rows of several layers, quantised into pages
    append   the rows of new tokens of one layer, quantised behind the rows that the pages hold
    attend   attention of one new token per sequence over the pages, one layer or several
    pages    a step of beams: sequences take over others' pages, grow by a row (a shared last page is copied first) and give the
             row back (a rejected draft)

Sizes are those of workloads.py's configurations, or generic. With `own` false the operators are computed from elementary torch
operations; with `own` true by the package.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LOWEST, HIGHEST = -100, 100        # exponents of a page's scale


# ---------------------------------------------------------------------------------------------------------------- cases
def _rotate(name, n_seqs, tokens, Hq, Hkv, d, rot, dtype="bf16", interleaved=False, scaling="plain", first=0):
    return {"name": name, "op": "rotate", "n_seqs": n_seqs, "tokens": tokens, "Hq": Hq, "Hkv": Hkv, "d": d, "rot": rot,
            "dtype": dtype, "interleaved": interleaved, "scaling": scaling, "first": first}


def _store(name, n_seqs, L, Hkv, d, tokens, w, lo, hi, page_rows, dtype="bf16"):
    return {"name": name, "op": "store", "n_seqs": n_seqs, "L": L, "Hq": Hkv, "Hkv": Hkv, "d": d, "tokens": tokens, "w": w,
            "lo": lo, "hi": hi, "page_rows": page_rows, "dtype": dtype}


def _append(name, n_seqs, Hkv, d, new, lo, hi, page_rows, dtype="bf16"):
    return {"name": name, "op": "append", "n_seqs": n_seqs, "L": 1, "Hq": Hkv, "Hkv": Hkv, "d": d, "new": new, "lo": lo,
            "hi": hi, "page_rows": page_rows, "dtype": dtype}


def _attend(name, n_seqs, L, Hq, Hkv, d, lo, hi, page_rows, dtype="bf16"):
    return {"name": name, "op": "attend", "n_seqs": n_seqs, "L": L, "Hq": Hq, "Hkv": Hkv, "d": d, "lo": lo, "hi": hi,
            "page_rows": page_rows, "dtype": dtype}


def _pages(name, n_seqs, L, Hkv, d, lo, hi, page_rows, width):
    return {"name": name, "op": "pages", "n_seqs": n_seqs, "L": L, "Hq": Hkv, "Hkv": Hkv, "d": d, "lo": lo, "hi": hi,
            "page_rows": page_rows, "width": width, "dtype": "bf16"}


def listed():
    return [
        # one new token of one sequence, once per layer of a decoder: the smallest call
        _rotate("rotate_token", 1, 1, 32, 8, 128, 128, first=32768),
        # fp32, the first half of each head, neighbouring elements paired, a ragged number of tokens of several sequences
        _rotate("rotate_f32_partial", 8, 1001, 4, 2, 64, 32, "f32", True, "bands", 5000),
        # one layer's queries and keys of a 32K prompt that starts far out in a long context
        _rotate("rotate_prompt_32k", 1, 32768, 32, 8, 128, 128, scaling="ramp", first=98304),
        # four layers of a 1K prompt in fp32
        _store("store_f32_1k", 1, 4, 2, 64, 1024, 16, 100, 256, 16, "f32"),
        # all layers of a 32K prompt: window rows and the rows the budgets left, 64 to 2048 a layer
        _store("store_32k", 1, 32, 8, 128, 32768, 32, 64, 960, 64),
        # one new token of one sequence, once per layer of a decoder
        _append("append_token", 1, 8, 128, 1, 576, 576, 64),
        # 33 tokens each of 64 sequences (a chunk of a prompt that goes on, drafted tokens)
        _append("append_chunk", 64, 8, 128, 33, 40, 2080, 64),
        # a decoder's call: one layer of one compressed 32K prompt
        _attend("attend_layer", 1, 1, 32, 8, 128, 544, 544, 64),
        # the compressed cache of all layers in one call
        _attend("attend_layers", 1, 32, 32, 8, 128, 96, 992, 64),
        # a serving batch over long caches that were not compressed, seven query heads per KV head
        _attend("attend_long", 16, 1, 28, 4, 128, 8192, 32768, 64),
        # four beams of a small model: latency
        _pages("pages_beams4", 4, 4, 2, 64, 40, 260, 16, 2),
        # eight beams each of four requests, 28 layers of a small budget
        _pages("pages_beams32", 32, 28, 4, 128, 64, 288, 64, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "store", "append", "attend", "attend", "attend", "pages"])
    d, dtype = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    Hkv, page_rows = rng.choice([1, 2, 4, 5, 8, 8]), rng.choice([16, 32, 64, 64, 128])
    if op == "rotate":
        G = rng.choice([1, 2, 4, 7, 8])
        rot = rng.choice([d, d, d // 2, d // 4, 3 * d // 4, 20])
        n_seqs = rng.choice([1, 1, 3, 8, 64])
        most = 32768 * 40 * 128 // (n_seqs * Hkv * (G + 1) * d * (2 if dtype == "f32" else 1))
        c = _rotate("", n_seqs, max(1, min(_log(rng, 1, 40000), most)), Hkv * G, Hkv, d, rot, dtype, rng.random() < 0.4,
                    rng.choice(["plain", "linear", "bands", "ramp"]), rng.choice([0, 7, 4095, 131072, 1000000]))
    elif op == "store":
        n_seqs, L, w = rng.choice([1, 1, 2, 5]), rng.choice([1, 2, 4, 7, 16, 32]), rng.choice([8, 16, 32, 64])
        most = 32 * 8 * 32768 * 128 // (n_seqs * L * Hkv * d * (2 if dtype == "f32" else 1))
        tokens = max(300, min(_log(rng, 300, 65536), most))
        hi = min(_log(rng, 16, 2048), tokens - w)
        hi = max(8, min(hi, 32 * 8 * 512 * 128 // (n_seqs * L * Hkv * d) - w))
        c = _store("", n_seqs, L, Hkv, d, tokens, w, rng.randint(0, hi), hi, page_rows, dtype)
    elif op == "append":
        new = rng.choice([1, 1, 1, 2, 5, _log(rng, 2, 160)])
        n_seqs = min(_log(rng, 1, 256), 64 * 33 // new)
        hi = new + _log(rng, 1, 4000)
        c = _append("", max(1, n_seqs), Hkv, d, new, rng.randint(new, hi), hi, page_rows, dtype)
    elif op == "attend":
        G = rng.choice([1, 2, 4, 4, 7, 8, 16])
        n_seqs, L = _log(rng, 1, 64), rng.choice([1, 1, 1, 4, 8, 32])
        hi = _log(rng, 1, 65536)
        hi = max(1, min(hi, 16 * 4 * 20000 * 128 // (n_seqs * L * Hkv * d)))
        c = _attend("", n_seqs, L, Hkv * G, Hkv, d, rng.randint(hi // 8, hi), hi, page_rows, dtype)
    else:
        width = rng.choice([1, 2, 4, 5])
        n_seqs, L = width * rng.choice([1, 2, 4]), rng.choice([1, 4, 8, 28])
        hi = _log(rng, 20, 1000)
        hi = max(20, min(hi, 32 * 28 * 4 * 288 * 128 // (n_seqs * L * Hkv * d)))
        c = _pages("", n_seqs, L, Hkv, d, rng.randint(1, hi), hi, page_rows, width)
    del c["name"]
    return c


# --------------------------------------------------------------------------------------------------------------- inputs
def _rows(case):
    """Rows of every (sequence, layer): spread over lo .. hi, the same for every seed."""
    i = np.arange(case["n_seqs"] * case["L"], dtype=np.int64) + 1
    at = (i * 2654435761 % (1 << 32)) / float(1 << 32)
    return (case["lo"] + np.floor(at * (case["hi"] - case["lo"] + 1))).astype(np.int64).reshape(case["n_seqs"], case["L"])


def _table_len(case):
    more = {"store": case.get("w", 0), "append": 0, "attend": 0, "pages": 1}[case["op"]]
    return -(-(case["hi"] + more) // case["page_rows"])


def _frequencies(case):
    """(radians per position of every pair, in 64 bits; the factor of the rotated elements)."""
    r = case["rot"]
    f = 10000.0 ** (-2.0 * np.arange(r // 2) / r)
    if case["scaling"] == "plain":
        return f, 1.0
    if case["scaling"] == "linear":
        return f / 4.0, 1.0
    if case["scaling"] == "bands":          # by wavelength: short ones stay, long ones are stretched, in between a blend
        factor, original, low, high = 8.0, 8192.0, 1.0, 4.0
        turns = original * f / (2.0 * math.pi)
        blend = np.clip((turns - low) / (high - low), 0.0, 1.0)
        return f * ((1.0 - blend) / factor + blend), 1.0
    factor, original, slow, fast = 16.0, 4096.0, 1.0, 32.0       # "ramp": by the pair's index
    pair = lambda n: r * math.log(original / (n * 2.0 * math.pi)) / (2.0 * math.log(10000.0))  # noqa: E731
    lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), r - 1)
    ramp = np.clip((np.arange(r // 2) - lo) / max(hi - lo, 0.001), 0.0, 1.0)
    return f * (ramp / factor + 1.0 - ramp), 0.1 * math.log(factor) + 1.0


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _pool(case, gen, in_use):
    """Pages, their scales and the table: `in_use` [n_seqs][L] pages each, in a random order, a quarter more pages than are used."""
    n_seqs, L, Hkv, d, pr = case["n_seqs"], case["L"], case["Hkv"], case["d"], case["page_rows"]
    used = int(in_use.sum())
    n_pages = used + used // 4 + n_seqs * L * 2 + 3
    codes = lambda *shape: (torch.randn(shape, generator=gen, device="cuda") * 112.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: _power_of_two(torch.randint(-8, -5, (n_pages, Hkv), generator=gen, device="cuda"))  # noqa: E731
    order = torch.randperm(n_pages, generator=gen, device="cuda").int()
    table = torch.full((n_seqs, L, _table_len(case)), -1, dtype=torch.int32, device="cuda")
    mask = torch.arange(table.shape[2], device="cuda") < torch.from_numpy(in_use).cuda()[..., None]
    table[mask] = order[:used]
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[order[:used].long()] = 1
    empty = case["op"] == "store"
    k = torch.zeros((n_pages, Hkv, pr, d), dtype=torch.float8_e4m3fn, device="cuda") if empty else codes(n_pages, Hkv, pr, d)
    v = torch.zeros((n_pages, Hkv, d, pr), dtype=torch.float8_e4m3fn, device="cuda") if empty else codes(n_pages, Hkv, d, pr)
    return {"k": k, "v": v, "k_scale": scale(), "v_scale": scale(), "table": table, "refs": refs,
            "missing": torch.zeros(1, dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, s = _type(case), {"case": dict(case)}
    n_seqs, Hq, Hkv, d = case["n_seqs"], case["Hq"], case["Hkv"], case["d"]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=t)  # noqa: E731
    if case["op"] == "rotate":
        n = case["tokens"]
        f, s["factor"] = _frequencies(case)
        s["f"] = torch.from_numpy(f).cuda()
        # prompts keep their keys by head, a decoder's new token has its heads side by side
        s["q"], s["k"] = randn(n_seqs, n, Hq, d), randn(n_seqs, Hkv, n, d).transpose(1, 2)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        start = case["first"] + torch.randint(0, 100, (n_seqs, 1), generator=gen, device="cuda")
        s["positions"] = (start + torch.arange(n, device="cuda")).int()
        return s
    pr, L, rows = case["page_rows"], case["L"], _rows(case)
    if case["op"] == "store":
        T, w, counts = case["tokens"], case["w"], rows
        s |= _pool(case, gen, -(-(counts + w) // pr))
        s["rows"] = torch.from_numpy(counts + w).int().cuda()
        s["counts"] = torch.from_numpy(counts).int().cuda()
        s["cu"] = torch.arange(0, (n_seqs + 1) * T, T, device="cuda").int()
        s["ks"], s["vs"] = randn(L, Hkv, n_seqs * T, d), randn(L, Hkv, n_seqs * T, d)
        # positions in the order of random scores, as the selection leaves them
        order = torch.rand((L * n_seqs * Hkv, T - w), generator=gen, device="cuda").topk(case["hi"], dim=1).indices.int()
        s["idx"] = order.reshape(L, n_seqs, Hkv, case["hi"]).contiguous()
        return s
    s |= _pool(case, gen, -(-rows // pr))
    s["rows"] = torch.from_numpy(rows).int().cuda()
    if case["op"] == "append":
        s["k_new"], s["v_new"] = 4.0 * randn(n_seqs, case["new"], Hkv, d), randn(n_seqs, case["new"], Hkv, d)
    elif case["op"] == "attend":
        s["q"] = 2.0 * randn(L, n_seqs, Hq, d)
        s["out"] = torch.empty((L, n_seqs, Hq, d), dtype=torch.float32, device="cuda")
        s["lse"] = torch.empty((L, n_seqs, Hq), dtype=torch.float32, device="cuda")
        s["of_layer"] = (s["q"][0], s["out"][0], s["lse"][0])        # a decoder's tensors of one layer
    else:
        width = case["width"]               # beams of a request; half of them go on from one of the others that stay
        beam, first = torch.arange(n_seqs, device="cuda") % width, torch.arange(n_seqs, device="cuda") // width * width
        stay = (width + 1) // 2
        parent = (torch.rand(n_seqs, generator=gen, device="cuda") * stay).long().clamp_max(stay - 1)
        s["parents"] = torch.where(beam < stay, beam + first, parent + first).int()
    return s


# ---------------------------------------------------------------------------------------------------------- plain forms
def _power_of_two(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _scale_exponent(amax):
    """The smallest e with amax <= 448 * 2^e, from amax = m * 2^x with m in [1/2, 1)."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8)
    return torch.where(amax == 0, torch.full_like(e, LOWEST), e).clamp(LOWEST, HIGHEST).int()


def _to_codes(x, e):
    return (x * _power_of_two(-e)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _plain_rotate(s, x):
    c = s["case"]
    r = c["rot"]
    angle = (s["positions"].double()[..., None] * s["f"])[:, :, None, :]
    cos, sin = (torch.cos(angle) * s["factor"]).float(), (torch.sin(angle) * s["factor"]).float()
    y = x.float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(turned, -1).flatten(-2) if c["interleaved"] else torch.cat(turned, -1)
    return torch.cat((turned, y[..., r:]), -1).to(x.dtype)


def _plain_store(s):
    c = s["case"]
    L, n_seqs, Hkv, d, pr, w, T = c["L"], c["n_seqs"], c["Hkv"], c["d"], c["page_rows"], c["w"], c["tokens"]
    pages = s["table"].shape[2]
    r = torch.arange(pages * pr, device="cuda")
    length = s["cu"][1:] - s["cu"][:-1]
    kept = s["idx"][..., (r - w).clamp(0, s["idx"].shape[3] - 1)]
    token = torch.where(r < w, (length[:, None] - w + r)[None, :, None, :], kept) + s["cu"][:-1][None, :, None, None]
    valid = (r < (w + s["counts"].t())[..., None])[:, :, None, :]
    row = torch.arange(L * Hkv, device="cuda").reshape(L, 1, Hkv, 1) * (n_seqs * T) + torch.where(valid, token, 0)
    held = torch.arange(pages, device="cuda") < (-(-s["rows"] // pr))[..., None]                    # [n_seqs][L][pages]
    ids = s["table"][held].long()

    def quantise(x, transpose):
        y = x.reshape(-1, d)[row].float() * valid[..., None]
        y = y.reshape(L, n_seqs, Hkv, pages, pr, d).permute(1, 0, 3, 2, 4, 5)[held]                 # [used][Hkv][pr][d]
        e = _scale_exponent(y.abs().amax((2, 3)))
        codes = _to_codes(y, e[..., None, None])
        return (codes.transpose(2, 3) if transpose else codes).contiguous(), _power_of_two(e)

    for_k, for_v = quantise(s["ks"], False), quantise(s["vs"], True)
    s["k"].view(torch.uint8)[ids], s["k_scale"][ids] = for_k[0].view(torch.uint8), for_k[1]
    s["v"].view(torch.uint8)[ids], s["v_scale"][ids] = for_v[0].view(torch.uint8), for_v[1]


def _plain_append(s):
    c = s["case"]
    n_seqs, Hkv, d, pr, new = c["n_seqs"], c["Hkv"], c["d"], c["page_rows"], c["new"]
    rows = s["rows"][:, 0].long()
    first = (rows - new) // pr
    page = first[:, None] + torch.arange((new + pr - 2) // pr + 1, device="cuda")                   # [n_seqs][pages]
    touched = page * pr < rows[:, None]
    ids = torch.gather(s["table"][:, 0], 1, page.clamp_max(s["table"].shape[2] - 1))[touched].long()
    g = page[..., None] * pr + torch.arange(pr, device="cuda")                                      # [n_seqs][pages][pr]
    at = g - (rows - new)[:, None, None]
    is_new, is_old = ((at >= 0) & (at < new))[touched], (at < 0)[touched]                           # [used][pr]
    seq = torch.arange(n_seqs, device="cuda")[:, None, None].expand_as(at)[touched]
    at = at.clamp(0, new - 1)[touched]

    def quantise(x, codes, scales, transpose):
        fresh = x[seq, at].float().permute(0, 2, 1, 3)                                              # [used][Hkv][pr][d]
        mask_new, mask_old = is_new[:, None, :, None], is_old[:, None, :, None]
        before = codes[ids].transpose(2, 3) if transpose else codes[ids]
        e_old = torch.frexp(scales[ids])[1].int() - 1
        e = _scale_exponent((fresh.abs() * mask_new).amax((2, 3)))
        e = torch.where(is_old.any(1)[:, None], torch.maximum(e, e_old), e)
        moved = _to_codes(before.float(), (e - e_old)[..., None, None])
        y = torch.where(mask_old, moved.view(torch.uint8), before.view(torch.uint8))
        y = torch.where(mask_new, _to_codes(fresh, e[..., None, None]).view(torch.uint8), y)
        codes.view(torch.uint8)[ids] = y.transpose(2, 3) if transpose else y
        scales[ids] = _power_of_two(e)

    quantise(s["k_new"], s["k"], s["k_scale"], False)
    quantise(s["v_new"], s["v"], s["v_scale"], True)


def _plain_attend(s):
    c = s["case"]
    L, n_seqs, Hq, Hkv, d, pr = c["L"], c["n_seqs"], c["Hq"], c["Hkv"], c["d"], c["page_rows"]
    G, pages = Hq // Hkv, s["table"].shape[2]
    R = pages * pr
    ids = s["table"].clamp_min(0).long()                                                            # [n_seqs][L][pages]
    k = (s["k"][ids].float() * s["k_scale"][ids][..., None, None]).permute(0, 1, 3, 2, 4, 5).reshape(-1, R, d)
    q = s["q"].float().transpose(0, 1).reshape(-1, G, d).transpose(1, 2).contiguous()               # [n_seqs*L*Hkv][d][G]
    x = torch.matmul(k, q).reshape(n_seqs, L, Hkv, R, G) / math.sqrt(d)
    x = x.masked_fill((torch.arange(R, device="cuda") >= s["rows"][..., None])[:, :, None, :, None], -math.inf)
    top = x.amax(3, keepdim=True)
    p = torch.exp(x - top.clamp_min(-3.0e38))
    total = p.sum(3, keepdim=True)
    lse = (top + torch.log(total)).squeeze(3).permute(1, 0, 2, 3).reshape(L, n_seqs, Hq)
    p = p / total.clamp_min(1e-30)
    v = (s["v"][ids].float() * s["v_scale"][ids][..., None, None]).permute(0, 1, 3, 4, 2, 5).reshape(-1, d, R)
    out = torch.matmul(v, p.reshape(-1, R, G)).transpose(1, 2).reshape(n_seqs, L, Hq, d).transpose(0, 1)
    return {"out": out.contiguous(), "lse": lse}


def _plain_fork(s):
    parents = s["parents"].long()
    moved = (parents != torch.arange(parents.numel(), device="cuda"))[:, None, None]
    count = lambda ids, m: torch.zeros_like(s["refs"]).index_add_(0, ids.clamp_min(0).flatten().long(), (m & (ids >= 0)).flatten().int())  # noqa: E731
    after = s["table"][parents]
    s["refs"] += count(after, moved.expand_as(after)) - count(s["table"], moved.expand_as(after))
    s["table"].copy_(after)
    s["rows"].copy_(s["rows"][parents])


def _plain_resize(s, extra):
    """Every (sequence, layer) to its rows + extra: pages behind the end are given back; then the lowest free pages are granted,
    for a shared last page that is not full as well (it is copied), to all or to none."""
    pr = s["case"]["page_rows"]
    table, refs = s["table"].reshape(-1, s["table"].shape[2]), s["refs"]
    old = s["rows"].flatten().long()
    target = (old + extra).clamp_min(0)
    held, want = -(-old // pr), -(-target // pr)
    j = torch.arange(table.shape[1], device="cuda")
    gone = (j >= want[:, None]) & (j < held[:, None])
    refs.index_add_(0, table[gone].long(), torch.full_like(table[gone], -1))
    table.masked_fill_(gone, -1)
    s["rows"].copy_(torch.minimum(old, target).reshape(s["rows"].shape))
    tail = torch.gather(table, 1, (held - 1).clamp_min(0)[:, None])[:, 0].clamp_min(0).long()
    copied = (target > old) & (old % pr != 0) & (refs[tail] > 1)
    need = (want - held).clamp_min(0) + copied
    start, total = torch.cumsum(need, 0) - need, need.sum()
    free = torch.cumsum((refs == 0).int(), 0)
    beyond = (want - table.shape[1]).clamp_min(0).sum()
    lacking = (total - free[-1]).clamp_min(0) + beyond
    s["missing"].copy_(lacking[None])
    granted = lacking == 0
    place = start[:, None] + (j - held[:, None]) + copied[:, None]
    fresh = (j >= held[:, None]) & (j < want[:, None]) & granted
    page = torch.searchsorted(free, torch.where(fresh, place, 0) + 1).int()
    copied = copied & granted
    source, copy = tail[copied], torch.searchsorted(free, start[copied] + 1).int()
    table.copy_(torch.where(fresh, page, table))
    table[copied.nonzero()[:, 0], held[copied] - 1] = copy
    refs.index_add_(0, source, torch.full_like(copy, -1))
    refs.index_add_(0, table[fresh].long(), torch.ones_like(table[fresh]))
    refs.index_add_(0, copy.long(), torch.ones_like(copy))
    s["rows"].copy_(torch.where(granted, target, torch.minimum(old, target)).reshape(s["rows"].shape))
    s["k"].view(torch.uint8)[copy.long()], s["v"].view(torch.uint8)[copy.long()] = s["k"].view(torch.uint8)[source], s["v"].view(torch.uint8)[source]
    s["k_scale"][copy.long()], s["v_scale"][copy.long()] = s["k_scale"][source], s["v_scale"][source]


# ------------------------------------------------------------------------------------------------------------------ run
_POOL = ("k", "v", "k_scale", "v_scale")
_HELD = ("table", "rows", "refs", "missing")


def _handle(s):
    """What a user's program builds once: the package's rotation, or its cache over the pages."""
    from paper_2412_14838_amd import dkv
    from paper_2412_14838_amd.pages import PagedCache
    from paper_2412_14838_amd.rotary import Rotary
    c = s["case"]
    dtype = dkv.DKV_BF16 if c["dtype"] == "bf16" else dkv.DKV_F32
    if c["op"] == "rotate":
        scaling = {"plain": None, "linear": dict(kind="linear", factor=4.0),
                   "bands": dict(kind="bands", factor=8.0, original=8192, low=1.0, high=4.0),
                   "ramp": dict(kind="ramp", factor=16.0, original=4096, low=1.0, high=32.0)}[c["scaling"]]
        return Rotary(c["d"], rot_dim=c["rot"], base=10000.0, interleaved=c["interleaved"], scaling=scaling, dtype=dtype)
    T = c.get("tokens", 1)
    desc = dkv.make_desc(n_layers=c["L"], n_q_heads=c["Hq"], n_kv_heads=c["Hkv"], head_dim=c["d"], window=c.get("w", 1),
                         pool_kernel=7, layer_max=c["hi"] if c["op"] == "store" else 1, mean_budget=1, interval=1, dtype=dtype,
                         n_seqs=c["n_seqs"], total_tokens=c["n_seqs"] * T, max_seq_len=T)
    return PagedCache(desc, n_pages=s["refs"].numel(), page_rows=c["page_rows"], max_rows=s["table"].shape[2] * c["page_rows"],
                      **{name: s[name] for name in _POOL + _HELD})


def run(state):
    s, c = state, state["case"]
    if own and "handle" not in s:
        s["handle"] = _handle(s)
    if c["op"] == "rotate":
        if own:
            s["handle"].rotate(s["positions"], s["q"], s["k"], s["q_out"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        return {"q": _plain_rotate(s, s["q"]), "k": _plain_rotate(s, s["k"])}
    if c["op"] == "attend":
        if own:
            if c["L"] == 1:
                s["handle"].attention(0, *s["of_layer"], expected_rows=(c["lo"] + c["hi"]) // 2)
            else:
                s["handle"].attention_layers(0, c["L"], s["q"], s["out"], s["lse"], expected_rows=(c["lo"] + c["hi"]) // 2)
            return {"out": s["out"], "lse": s["lse"]}
        return _plain_attend(s)
    if c["op"] == "store":
        if own:
            s["handle"].store_layers(0, list(s["ks"]), list(s["vs"]), s["cu"], s["idx"], s["counts"])
        else:
            _plain_store(s)
    elif c["op"] == "append":
        if own:
            s["handle"].append(0, s["k_new"], s["v_new"])
        else:
            _plain_append(s)
    else:
        if own:
            s["handle"].fork(s["parents"])
            s["handle"].resize(s["rows"], 1)
            s["handle"].resize(s["rows"], -1)
        else:
            _plain_fork(s)
            _plain_resize(s, 1)
            _plain_resize(s, -1)
        return {name: s[name] for name in _POOL + _HELD}
    return {name: s[name] for name in _POOL}


# ----------------------------------------------------------------------------------------------------------------- work
def work(case):
    elt = 2 if case["dtype"] == "bf16" else 4
    n_seqs, Hq, Hkv, d = case["n_seqs"], case["Hq"], case["Hkv"], case["d"]
    if case["op"] == "rotate":
        n = n_seqs * case["tokens"]
        return {"bytes": 2 * n * (Hq + Hkv) * d * elt + 4 * n, "flops": 3 * n * (Hq + Hkv) * case["rot"]}
    rows, pr = _rows(case), case["page_rows"]
    if case["op"] == "store":
        kept = int((rows + case["w"]).sum()) * Hkv
        return {"bytes": 2 * kept * d * (elt + 1) + 4 * int(rows.sum()) * Hkv, "flops": 4 * kept * d}
    if case["op"] == "append":
        new = n_seqs * case["new"] * Hkv * d
        return {"bytes": 2 * new * (elt + 1), "flops": 4 * new}
    if case["op"] == "attend":
        held, heads = int(rows.sum()), n_seqs * case["L"] * Hq
        return {"bytes": 2 * held * Hkv * d + heads * (d * (elt + 4) + 4), "flops": 4 * held * Hq * d}
    width = case["width"]                    # a beam that goes on from another makes one copy of its last page necessary
    beam = np.arange(n_seqs) % width
    origin = np.where(beam < (width + 1) // 2, np.arange(n_seqs), np.arange(n_seqs) // width * width)
    moved = beam >= (width + 1) // 2
    copies = int(((rows[origin] % pr != 0) & moved[:, None]).sum())
    return {"bytes": 4 * copies * Hkv * d * pr + 2 * 4 * n_seqs * case["L"] * (_table_len(case) + 1), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------- exact
def _e4m3(x):
    """The nearest value of four exponent and three mantissa bits (ties to even), in 64 bits."""
    a = x.abs().clamp_max(448.0)
    step = torch.exp2((torch.frexp(a)[1].double() - 1.0).clamp_min(-6.0) - 3.0)
    return torch.sign(x) * torch.round(a / step) * step


def _exact_scale(x):
    top = float(x.abs().max()) if x.numel() else 0.0
    e = LOWEST if top == 0.0 else math.ceil(math.log2(top / 448.0))
    while e > LOWEST and top <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    while e < HIGHEST and top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** min(max(e, LOWEST), HIGHEST)


def _exact_rotate(s, x):
    c = s["case"]
    r = c["rot"]
    turn = torch.polar(torch.full_like(s["f"], s["factor"])[None, None], s["positions"].double()[..., None] * s["f"])[:, :, None]
    y = x.double().clone()
    pairs = [slice(0, r, 2), slice(1, r, 2)] if c["interleaved"] else [slice(0, r // 2), slice(r // 2, r)]
    z = torch.complex(y[..., pairs[0]], y[..., pairs[1]]) * turn
    y[..., pairs[0]], y[..., pairs[1]] = z.real, z.imag
    return y


def _exact_attend(s):
    c = s["case"]
    L, n_seqs, Hq, Hkv, d = c["L"], c["n_seqs"], c["Hq"], c["Hkv"], c["d"]
    out = torch.zeros((L, n_seqs, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((L, n_seqs, Hq), -math.inf, dtype=torch.float64, device="cuda")
    rows = s["rows"].tolist()
    for l in range(L):
        for b in range(n_seqs):
            n = rows[b][l]
            if n == 0:
                continue
            ids = s["table"][b, l, :-(-n // c["page_rows"])].long()
            k = (s["k"][ids].double() * s["k_scale"][ids].double()[..., None, None]).transpose(0, 1).reshape(Hkv, -1, d)[:, :n]
            v = (s["v"][ids].double() * s["v_scale"][ids].double()[..., None, None]).permute(1, 0, 3, 2).reshape(Hkv, -1, d)[:, :n]
            x = torch.matmul(s["q"][l, b].double().reshape(Hkv, -1, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
            lse[l, b] = torch.logsumexp(x, -1).flatten()
            out[l, b] = torch.matmul(torch.softmax(x, -1), v).reshape(Hq, d)
    return {"out": out, "lse": lse}


def _exact_store(s):
    c = s["case"]
    w, pr, Hkv = c["w"], c["page_rows"], c["Hkv"]
    r = {name: s[name].double() for name in _POOL}
    counts, cu, table = s["counts"].tolist(), s["cu"].tolist(), s["table"].tolist()
    for l in range(c["L"]):
        for b in range(c["n_seqs"]):
            n = counts[b][l]
            window = torch.arange(cu[b + 1] - w, cu[b + 1], device="cuda").expand(Hkv, w)
            token = torch.cat((window, s["idx"][l, b, :, :n] + cu[b]), 1).long()
            for name, source in (("k", s["ks"]), ("v", s["vs"])):
                x = torch.gather(source[l], 1, token[..., None].expand(-1, -1, c["d"])).double()
                x = torch.nn.functional.pad(x, (0, 0, 0, -(w + n) % pr)).reshape(Hkv, -1, pr, c["d"]).transpose(0, 1)
                top = x.abs().amax((2, 3))
                e = torch.ceil(torch.log2(top / 448.0))
                e = torch.where(top <= 448.0 * torch.exp2(e - 1.0), e - 1.0, e)
                e = torch.where(top > 448.0 * torch.exp2(e), e + 1.0, e).clamp(LOWEST, HIGHEST)
                codes = _e4m3(x / torch.exp2(e)[..., None, None])
                ids = torch.tensor(table[b][l][:x.shape[0]], device="cuda")
                r[name][ids] = codes.transpose(2, 3) if name == "v" else codes
                r[name + "_scale"][ids] = torch.exp2(e)
    return r


def _exact_append(s):
    c = s["case"]
    pr, new = c["page_rows"], c["new"]
    r = {name: s[name].double() for name in _POOL}
    for b in range(c["n_seqs"]):
        n = int(s["rows"][b, 0])
        for page in range((n - new) // pr, -(-n // pr)):
            i = int(s["table"][b, 0, page])
            lo, hi = max(n - new, page * pr), min(n, (page + 1) * pr)
            a, z = lo - page * pr, hi - page * pr
            for name, source in (("k", s["k_new"]), ("v", s["v_new"])):
                x = source[b, lo - (n - new):hi - (n - new)].double().transpose(0, 1)                # [Hkv][new rows][d]
                for h in range(c["Hkv"]):
                    codes = r[name][i, h] if name == "k" else r[name][i, h].t()
                    before, scale = float(r[name + "_scale"][i, h]), _exact_scale(x[h])
                    scale = max(scale, before) if a > 0 else scale
                    codes[:a] = _e4m3(codes[:a] * (before / scale))
                    codes[a:z] = _e4m3(x[h] / scale)
                    r[name + "_scale"][i, h] = scale
    return r


def _exact_pages(s):
    """The step one (sequence, layer) after the other, on the host."""
    pr = s["case"]["page_rows"]
    table, rows, refs, parents = (s[name].tolist() for name in ("table", "rows", "refs", "parents"))
    r = {name: s[name].double() for name in _POOL}
    n_seqs, L, most = len(rows), len(rows[0]), len(table[0][0])
    before = [[list(t) for t in of] for of in table]
    had = [list(x) for x in rows]
    for b, p in enumerate(parents):
        if p == b:
            continue
        for l in range(L):
            for i in before[b][l]:
                refs[i] -= i >= 0
            for i in before[p][l]:
                refs[i] += i >= 0
            table[b][l], rows[b][l] = list(before[p][l]), had[p][l]
    free = [i for i, x in enumerate(refs) if x == 0]
    shared = [[rows[b][l] % pr != 0 and refs[table[b][l][(rows[b][l] - 1) // pr]] > 1 for l in range(L)] for b in range(n_seqs)]
    for b in range(n_seqs):
        for l in range(L):
            n = rows[b][l]
            if shared[b][l]:
                i, j = table[b][l][n // pr], free.pop(0)
                for name in _POOL:
                    r[name][j] = r[name][i]
                refs[i] -= 1
                refs[j], table[b][l][n // pr] = 1, j
            elif n % pr == 0 and n // pr < most:
                free.pop(0)                  # granted for the row, given back with it
    held = {"table": table, "rows": rows, "refs": refs, "missing": [0]}
    return r | {name: torch.tensor(x, dtype=torch.int32) for name, x in held.items()}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return {"q": _exact_rotate(s, s["q"]), "k": _exact_rotate(s, s["k"])}
    return {"store": _exact_store, "append": _exact_append, "attend": _exact_attend, "pages": _exact_pages}[case["op"]](s)
