"""What a program that serves a model from a 4-bit K/V cache has the library do:
attention over the cache, writing tokens into it, the upkeep of its pages, and
products with the 4-bit weights of the projections that stay out of ternary.

listed() names the cases, draw() makes more of the same ranges, prepare() /
run() execute one (elementary torch operations, or the library's entry points
where `own` is true), work() counts what a pass cannot do without and exact()
states its result in 64-bit arithmetic.

The cache.  A page holds 64 tokens; data is [layers][pages][heads][block], a
block the bytes of one head's page: K codes [64][D / 2] (dimension 2 b in the
low half of byte b), V codes, K parameters [D / 64][64] and V parameters, 16
bits each.  A parameter is an fp16 scale s whose four low bits are replaced by
the zero z; a code c stands for s (c - z).  table[slot][i] is the page of a
sequence's tokens 64 i .., length[slot] its tokens, refs[page] how many
sequences hold the page.
4-bit weights: W[n][k] = scale[n][g] c[n][k] + minimum[n][g], g = k / 128.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE, GROUP, WGROUP = 64, 64, 128


def listed():
    return [
        # One user, a short context, one token: latency.  Heads as in the benchmark's models (32 queries, 8 keys of 128).
        {"name": "attend_1x700", "kind": "attend", "B": 1, "lo": 700, "hi": 700, "nq_lo": 1, "nq_hi": 1, "hkv": 8,
         "group": 4, "D": 128, "window": 0, "dtype": "fp16", "layers": 2, "ragged": 1},
        # A decode batch of a server: 48 sequences of 1000 to 8000 tokens, one token each.
        {"name": "attend_48_ragged", "kind": "attend", "B": 48, "lo": 1000, "hi": 8000, "nq_lo": 1, "nq_hi": 1, "hkv": 8,
         "group": 4, "D": 128, "window": 0, "dtype": "fp16", "layers": 2, "ragged": 2},
        # Two very long contexts, one token each.
        {"name": "attend_2x130k_bf16", "kind": "attend", "B": 2, "lo": 126001, "hi": 131072, "nq_lo": 1, "nq_hi": 1,
         "hkv": 8, "group": 4, "D": 128, "window": 0, "dtype": "bf16", "layers": 1, "ragged": 3},
        # Checking a draft: a few tokens for each of 16 sequences, smaller heads, a sliding window.
        {"name": "attend_verify_window", "kind": "attend", "B": 16, "lo": 900, "hi": 5000, "nq_lo": 3, "nq_hi": 6, "hkv": 4,
         "group": 6, "D": 64, "window": 1023, "dtype": "fp16", "layers": 2, "ragged": 4},
        # Prompts in pieces: three sequences, 700 to 2048 tokens on top of what they have already.
        {"name": "attend_prompt", "kind": "attend", "B": 3, "lo": 4100, "hi": 6144, "nq_lo": 700, "nq_hi": 2048, "hkv": 8,
         "group": 4, "D": 128, "window": 0, "dtype": "fp16", "layers": 1, "ragged": 5},
        # One token of 64 sequences into the cache.
        {"name": "append_64x1", "kind": "append", "B": 64, "n_lo": 1, "n_hi": 1, "lo": 0, "hi": 3000, "hkv": 8, "group": 4,
         "D": 128, "dtype": "fp16", "layers": 2, "ragged": 6},
        # A prompt's tokens into the cache, three sequences at once.
        {"name": "append_prompts", "kind": "append", "B": 3, "n_lo": 1500, "n_hi": 4096, "lo": 0, "hi": 500, "hkv": 8,
         "group": 4, "D": 128, "dtype": "bf16", "layers": 2, "ragged": 7},
        # Sampling several continuations: each prompt forked, a token for each child (its shared last page is copied), the
        # children freed again.
        {"name": "fork_8x4", "kind": "fork", "parents": 8, "children": 4, "lo": 300, "hi": 2000, "new": 1, "hkv": 8, "D": 128,
         "layers": 36, "spare": 60, "ragged": 8},
        # Closing the gaps that finished sequences left.
        {"name": "compact_900", "kind": "compact", "pages": 900, "used": 0.45, "slots": 24, "hkv": 8, "D": 128, "layers": 12,
         "ragged": 9},
        # A projection of the benchmark's larger model kept at 4 bits, one token.
        {"name": "w4_4096x4096_m1", "kind": "w4", "M": 1, "N": 4096, "K": 4096, "f32": False},
        # The output head, one token, logits in 32 bits.
        {"name": "w4_head_131072x4096_m1", "kind": "w4", "M": 1, "N": 131072, "K": 4096, "f32": True},
        # A few tokens, odd sizes.
        {"name": "w4_9725x2560_m13", "kind": "w4", "M": 13, "N": 9725, "K": 2560, "f32": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "verify", "prompt", "append", "fork", "compact", "w4", "w4"])
    heads = {"hkv": rng.choice([1, 2, 4, 8]), "group": rng.choice([1, 2, 4, 5, 8]), "D": rng.choice([64, 128, 128])}
    ragged = rng.randrange(1 << 20)
    dtype = rng.choice(["fp16", "fp16", "bf16"])
    if kind in ("decode", "verify"):
        B = _log(rng, 1, 64)
        hi = _log(rng, 1, min(131072, 262144 // B))
        nq = 1 if kind == "decode" else rng.randint(2, 9)
        return {"kind": "attend", "B": B, "lo": max(1, hi // rng.choice([1, 2, 6])), "hi": hi, "nq_lo": 1, "nq_hi": nq, **heads,
                "window": rng.choice([0, 0, 0, _log(rng, 1, hi)]), "dtype": dtype, "layers": 2, "ragged": ragged}
    if kind == "prompt":
        B = rng.randint(1, 4)
        nq = _log(rng, 10, 2048 // B)
        hi = nq + _log(rng, 1, 4096)
        return {"kind": "attend", "B": B, "lo": max(nq, hi // 2), "hi": hi, "nq_lo": max(1, nq // rng.choice([1, 3])),
                "nq_hi": nq, **heads, "window": rng.choice([0, 0, _log(rng, 16, hi)]), "dtype": dtype, "layers": 1,
                "ragged": ragged}
    if kind == "append":
        B = _log(rng, 1, 64)
        n = _log(rng, 1, 8192 // B)
        return {"kind": "append", "B": B, "n_lo": max(1, n // 3), "n_hi": n, "lo": 0, "hi": _log(rng, 1, 1000), **heads,
                "dtype": dtype, "layers": 2, "ragged": ragged}
    if kind == "fork":
        parents = _log(rng, 1, 8)
        return {"kind": "fork", "parents": parents, "children": rng.randint(1, 4), "lo": 1, "hi": _log(rng, 64, 2000),
                "new": rng.choice([1, 1, 2, 70]), "hkv": heads["hkv"], "D": heads["D"], "layers": _log(rng, 2, 36),
                "spare": rng.randint(0, 99), "ragged": ragged}
    if kind == "compact":
        return {"kind": "compact", "pages": _log(rng, 40, 900), "used": round(rng.uniform(0.1, 0.8), 3),
                "slots": rng.randint(3, 40), "hkv": heads["hkv"], "D": heads["D"], "layers": _log(rng, 2, 12),
                "ragged": ragged}
    return {"kind": "w4", "M": _log(rng, 1, 40), "N": _log(rng, 100, 60000), "K": WGROUP * _log(rng, 4, 64),
            "f32": rng.random() < 0.3}


# ------------------------------------------------------------------- inputs
def _gen(seed, *ids):
    s = seed
    for i in ids:
        s = (s * 1000003 + i + 1) % (1 << 62)
    g = torch.Generator(device="cuda")
    g.manual_seed(s)
    return g


def _randn(shape, g):
    return torch.randn(shape, generator=g, device="cuda")


def _dtype(case):
    return {"fp16": torch.float16, "bf16": torch.bfloat16}[case["dtype"]]


def _block(D):
    return PAGE * D + 2 * (D // GROUP) * PAGE * 2


def _lengths(case):
    """(tokens in the cache, new tokens) of each sequence, as the case alone gives them."""
    r = random.Random(case["ragged"])
    if case["kind"] == "attend":
        n = [r.randint(case["nq_lo"], case["nq_hi"]) for _ in range(case["B"])]
        return [max(r.randint(case["lo"], case["hi"]), k) for k in n], n
    if case["kind"] == "append":
        n = [r.randint(case["n_lo"], case["n_hi"]) for _ in range(case["B"])]
        return [r.randint(case["lo"], case["hi"]) + k for k in n], n
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["parents"])], []


def _pool(layers, pages, heads, D, seed):
    """A cache's bytes: codes around the middle, scales around a third, as normalised keys and values give them."""
    g = _gen(seed, 1)
    data = torch.empty((layers, pages, heads, _block(D)), dtype=torch.uint8, device="cuda")
    for layer in range(layers):
        lo, hi = ((_randn((pages, heads, PAGE * D), g) * 3 + 7.5).round_().clamp_(0, 15).to(torch.uint8) for _ in "lh")
        data[layer, :, :, :PAGE * D] = lo | hi << 4
        n = (pages, heads, 2 * (D // GROUP) * PAGE)
        s = torch.exp(_randn(n, g) * 0.3 - 1.1).half().view(torch.int16)
        z = torch.randint(6, 10, n, generator=g, device="cuda", dtype=torch.int16)
        data[layer, :, :, PAGE * D:] = ((s & -16) | z).view(torch.uint8)
    return data


def _tables(lengths, pages, slots, seed, order=None):
    """table, length, refs of sequences in slots 0 .., their pages anywhere in the pool."""
    g = _gen(seed, 2)
    ids = torch.randperm(pages, generator=g, device="cuda").cpu().tolist() if order is None else list(order)
    need = [-(-n // PAGE) for n in lengths]
    table = np.full((slots, max(need + [1]) + 2), -1, np.int32)
    refs = np.zeros(pages, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        refs[ids[at:at + n]] = 1
        at += n
    length = np.zeros(slots, np.int32)
    length[:len(lengths)] = lengths
    return tuple(torch.from_numpy(a).cuda() for a in (table, length, refs))


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _indptr(n):
    return _int(np.concatenate([[0], np.cumsum(n)]).tolist())


def _where(table, lengths, n):
    """page * 64 + offset of each sequence's last n tokens."""
    t = table.cpu().numpy()
    pos = [np.arange(L - k, L) for L, k in zip(lengths, n)]
    return _int(np.concatenate([t[b, p // PAGE].astype(np.int64) * PAGE + p % PAGE for b, p in enumerate(pos)]).tolist())


def _fork_lists(case):
    P, C = case["parents"], case["children"]
    return [i // C for i in range(P * C)], [P + i for i in range(P * C)]


def _used_pages(case):
    """The sequences of a cache with gaps: how many pages each holds, and which."""
    r = random.Random(case["ragged"])
    live = r.sample(range(case["pages"]), max(1, int(case["pages"] * case["used"])))
    cuts = sorted(r.randint(0, len(live)) for _ in range(case["slots"] - 1))
    counts = [b - a for a, b in zip([0] + cuts, cuts + [len(live)])]
    return counts, live, [max(0, c * PAGE - r.randint(0, PAGE - 1)) for c in counts]


def prepare(case, seed):
    s = {"case": case, "kind": case["kind"]}
    if case["kind"] == "w4":
        g, G = _gen(seed, 3), case["K"] // WGROUP
        s["codes"] = (_randn((case["N"], case["K"]), g) * 3 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
        s["scale"] = torch.exp(_randn((case["N"], G), g) * 0.4 - 5.0).half()
        s["minimum"] = (s["scale"].float() * (_randn((case["N"], G), g) * 0.5 - 7.5)).half()
        s["x"] = _randn((case["M"], case["K"]), g).half()
        if own:
            from paper_2609_09240_gb300 import tq
            s["w"] = tq.pack_w4(s["codes"], s["scale"], s["minimum"])
        return s
    D, H, layers = case["D"], case["hkv"], case["layers"]
    s["D"], s["layer"] = D, layers - 1
    if case["kind"] == "compact":
        counts, live, lengths = _used_pages(case)
        pages = case["pages"]
        s["table"], s["length"], s["refs"] = _tables(lengths, pages, case["slots"], seed, order=live)
        s["table_out"], s["refs_out"] = torch.empty_like(s["table"]), torch.empty_like(s["refs"])
    elif case["kind"] == "fork":
        lengths, _ = _lengths(case)
        src, dst = _fork_lists(case)
        grow = -(-case["new"] // PAGE) + 1
        pages = sum(-(-n // PAGE) for n in lengths) + len(dst) * grow + case["spare"]
        s["table"], s["length"], s["refs"] = _tables(lengths, pages, case["parents"] + len(dst), seed)
        s["src"], s["dst"], s["new"], s["tokens"] = _int(src), _int(dst), _int([case["new"]] * len(dst)), case["new"] * len(dst)
    else:
        lengths, n = _lengths(case)
        pages = sum(-(-k // PAGE) for k in lengths) + 3
        s["table"], s["length"], s["refs"] = _tables(lengths, pages, case["B"], seed)
        s["slots"], s["indptr"] = _int(list(range(case["B"]))), _indptr(n)
        s["max_q"], s["max_len"] = max(n), max(lengths)
        g, T, Hq = _gen(seed, 4), sum(n), H * case["group"]
        if case["kind"] == "append":
            # keys and values as they leave the projection: columns of its output
            qkv = (_randn((T, (Hq + 2 * H) * D), g) * torch.exp(0.5 * _randn((T, 1), g))).to(_dtype(case))
            s["qkv"] = qkv
            s["k"] = qkv[:, Hq * D:(Hq + H) * D].unflatten(1, (H, D))
            s["v"] = qkv[:, (Hq + H) * D:].unflatten(1, (H, D))
            s["where"] = _where(s["table"], lengths, n)
        else:
            s["q"] = (_randn((T, Hq, D), g) * 1.5).to(_dtype(case))
            s["scale"], s["window"] = 1.0 / math.sqrt(D), case["window"]
    s["data"] = _pool(layers, pages, H, D, seed)
    if own:
        from paper_2609_09240_gb300 import tq
        s["cache"] = tq.Kv4Cache(s["data"], s["table"], s["length"], s["refs"], D)
    return s


# -------------------------------------------------------------- plain forms
def _values(codes, params, D):
    """codes [.., 64 D / 2] bytes, params [.., (D / 64) 64 2] bytes -> [.., 64, D] in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).float().unflatten(-2, (PAGE, D // 2)).flatten(-2)
    p = params.contiguous().view(torch.int16).unflatten(-1, (D // GROUP, PAGE)).transpose(-1, -2)
    s, z = (p & -16).view(torch.float16).float(), (p & 15).float()
    return (s[..., None] * (c.unflatten(-1, (D // GROUP, GROUP)) - z[..., None])).flatten(-2)


def _kv(blocks, D):
    h, q = PAGE * D // 2, (D // GROUP) * PAGE * 2
    k, v, pk, pv = blocks.split([h, h, q, q], -1)
    return _values(k, pk, D), _values(v, pv, D)


def _attend(s):
    D, q, length = s["D"], s["q"], s["length"][s["slots"].long()].long()
    B, H = length.shape[0], s["data"].shape[2]
    npages = -(-s["max_len"] // PAGE)
    pages = s["table"][s["slots"].long(), :npages].long().clamp_min(0)
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in _kv(s["data"][s["layer"]][pages], D))  # [B][H][L][D]
    n = (s["indptr"][1:] - s["indptr"][:-1]).long()
    i = torch.arange(s["max_q"], device=q.device)
    token = (s["indptr"][:-1].long()[:, None] + i).clamp_max(q.shape[0] - 1)
    there = i < n[:, None]
    pos = length[:, None] - n[:, None] + i  # [B][nq]
    qs = q[token].float().unflatten(2, (H, -1)).permute(0, 2, 1, 3, 4)  # [B][H][nq][g][D]
    a = (qs.flatten(2, 3) @ k.transpose(-1, -2)) * s["scale"]
    t = torch.arange(k.shape[2], device=q.device)
    seen = t <= pos[..., None]
    if s["window"]:
        seen &= t > pos[..., None] - s["window"]
    seen = seen.repeat_interleave(qs.shape[3], 1)[:, None]  # [B][1][nq g][L]
    a = a.masked_fill(~seen, -math.inf)
    top = a.amax(-1, keepdim=True)
    e = torch.exp(a - torch.where(torch.isfinite(top), top, 0.0))
    o = (e @ v) / e.sum(-1, keepdim=True).clamp_min(1e-30)
    o = o.unflatten(2, (s["max_q"], -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B][nq][Hq][D]
    return o[there].to(q.dtype)


def _encode(x):
    """x [T][H][D] -> codes (bytes, two values each) and params [T][H][D / 64]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1).clamp_max(0.0), x.amax(-1).clamp_min(0.0)
    bits = (((hi - lo) / 15).half().view(torch.int16) + 15) & -16
    sc = bits.view(torch.float16).float()
    safe = torch.where(sc > 0, sc, 1.0)
    z = torch.round(-lo / safe).clamp(0, 15)
    c = (torch.round(x / safe[..., None]) + z[..., None]).clamp(0, 15).to(torch.uint8).flatten(-2)
    return c[..., 0::2] | c[..., 1::2] << 4, bits | z.to(torch.int16)


def _append(s):
    D, data = s["D"], s["data"][s["layer"]]
    H, G = data.shape[1], D // GROUP
    page, off = s["where"].long() // PAGE, s["where"].long() % PAGE
    h = PAGE * D // 2
    heads = torch.arange(H, device=page.device)[None, :, None]
    halves = torch.arange(D // 2, device=page.device)
    groups = torch.arange(2 * G, device=page.device)
    ck, pk = _encode(s["k"])
    cv, pv = _encode(s["v"])
    row = page[:, None, None], heads
    at = off[:, None, None]
    data[(*row, at * (D // 2) + halves)] = ck
    data[(*row, h + at * (D // 2) + halves)] = cv
    at = 2 * h + (groups // 2 * PAGE + at) * 2 + groups % 2
    data[(*row, at)] = pk.contiguous().view(torch.uint8)
    data[(*row, at + G * PAGE * 2)] = pv.contiguous().view(torch.uint8)
    k, v = (x[torch.arange(page.shape[0], device=page.device), :, off] for x in _kv(data[page], D))
    return [k.to(s["k"].dtype), v.to(s["v"].dtype)]


def _held(s, slots):
    """The pages of the listed sequences, and which table entries they are."""
    table = s["table"][slots]
    in_use = torch.arange(table.shape[1], device=table.device) < ((s["length"][slots] + PAGE - 1) // PAGE)[:, None]
    return table[in_use].long(), in_use


def _fork(s):
    table, length, refs, data = s["table"], s["length"], s["refs"], s["data"]
    src, dst, new = s["src"].long(), s["dst"].long(), s["new"].long()
    # fork
    pages, in_use = _held(s, src)
    refs.index_add_(0, pages, torch.ones_like(pages, dtype=torch.int32))
    table[dst] = torch.where(in_use, table[src], -1)
    length[dst] = length[src]
    # extend
    L = length[dst].long()
    have, want = (L + PAGE - 1) // PAGE, (L + new + PAGE - 1) // PAGE
    last = table[dst, (L // PAGE).clamp_max(table.shape[1] - 1)].long().clamp_min(0)
    copy = (new > 0) & (L % PAGE != 0) & (refs[last] > 1)
    need = want - have + copy
    free = torch.nonzero(refs == 0).flatten()[: int(need.sum())]
    seq = torch.repeat_interleave(torch.arange(dst.shape[0], device=L.device), need)
    j = torch.arange(seq.shape[0], device=L.device) - (torch.cumsum(need, 0) - need)[seq]
    copied = copy[seq] & (j == 0)
    data[:, free[copied]] = data[:, last[seq[copied]]]
    refs[free] = 1
    refs.index_add_(0, last[copy], torch.full_like(last[copy], -1, dtype=torch.int32))
    table[dst[seq], torch.where(copied, L[seq] // PAGE, have[seq] + j - copy[seq].long())] = free.int()
    length[dst] = (L + new).int()
    indptr = torch.cat([torch.zeros(1, dtype=torch.int64, device=L.device), torch.cumsum(new, 0)])
    seq = torch.repeat_interleave(torch.arange(dst.shape[0], device=L.device), new)
    pos = L[seq] + torch.arange(seq.shape[0], device=L.device) - indptr[seq]
    where = table[dst[seq], pos // PAGE].long() * PAGE + pos % PAGE
    # free
    pages, _ = _held(s, dst)
    refs.index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    table[dst] = -1
    length[dst] = 0
    return [indptr.int(), where.int(), table, length, refs, data]


def _compact(s):
    table, refs, data = s["table"], s["refs"], s["data"]
    ids = torch.arange(refs.shape[0], device=refs.device)
    live = refs > 0
    n = live.sum()
    holes, movers = ids[~live & (ids < n)], ids[live & (ids >= n)]
    remap = torch.where(live, ids, -1)
    remap[movers] = holes
    data[:, holes] = data[:, movers]
    held = torch.arange(table.shape[1], device=refs.device) < ((s["length"] + PAGE - 1) // PAGE)[:, None]
    s["table_out"].copy_(torch.where(held, remap[table.long().clamp_min(0)], -1))
    s["refs_out"].zero_()
    s["refs_out"][remap[live]] = refs[live]
    return [s["table_out"], s["refs_out"], remap.int(), n.int().reshape(1), data]


def _w4(s):
    N, K = s["codes"].shape
    w = s["codes"].float().view(N, -1, WGROUP) * s["scale"].float()[..., None] + s["minimum"].float()[..., None]
    y = s["x"].float() @ w.view(N, K).t()
    return y if s["case"]["f32"] else y.half()


def run(s):
    if not own:
        return {"attend": _attend, "append": _append, "fork": _fork, "compact": _compact, "w4": _w4}[s["kind"]](s)
    from paper_2609_09240_gb300 import tq

    if s["kind"] == "w4":
        return tq.tq_w4_linear(s["x"], s["w"], f32=s["case"]["f32"])
    c = s["cache"]
    if s["kind"] == "attend":
        return tq.tq_kv4_attention(s["q"], c, s["layer"], s["slots"], s["indptr"], max_q=s["max_q"], scale=s["scale"],
                                   window=s["window"])
    if s["kind"] == "append":
        tq.tq_kv4_append(s["k"], s["v"], c, s["layer"], s["where"])
        return list(tq.tq_kv4_read(c, s["layer"], s["where"], dtype=s["k"].dtype))
    if s["kind"] == "fork":
        tq.tq_kv4_fork(c, s["src"], s["dst"])
        indptr, where = tq.tq_kv4_extend(c, s["dst"], s["new"], s["tokens"])
        tq.tq_kv4_free(c, s["dst"])
        return [indptr, where, c.table, c.length, c.refs, c.data]
    remap, live = tq.tq_kv4_compact(c, table_out=s["table_out"], refs_out=s["refs_out"])
    return [s["table_out"], s["refs_out"], remap, live, c.data]


# ---------------------------------------------------------------- the floor
def work(case):
    if case["kind"] == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K // 2 + N * (K // WGROUP) * 4 + M * K * 2 + M * N * (4 if case["f32"] else 2),
                "flops": 2 * M * N * K}
    D, H = case["D"], case["hkv"]
    token = H * (D + 4 * (D // GROUP))  # bytes of a token's keys and values in one layer
    block = _block(D) * H * case["layers"]
    if case["kind"] == "attend":
        lengths, n = _lengths(case)
        W, Hq = case["window"], H * case["group"]
        first = [max(0, L - k - W + 1) if W else 0 for L, k in zip(lengths, n)]
        seen = sum(min(p + 1, W or p + 1) for L, k in zip(lengths, n) for p in range(L - k, L))
        return {"bytes": sum(L - f for L, f in zip(lengths, first)) * token + sum(n) * Hq * D * 4, "flops": 4 * D * Hq * seen}
    if case["kind"] == "append":
        T = sum(_lengths(case)[1])
        return {"bytes": T * (2 * H * D * 2 * 2 + 2 * token), "flops": T * H * D * 2 * 8}
    if case["kind"] == "fork":
        lengths, _ = _lengths(case)
        src, dst = _fork_lists(case)
        copied = sum(1 for p in src if lengths[p] % PAGE)
        held = sum(-(-lengths[p] // PAGE) for p in src)
        return {"bytes": 2 * copied * block + held * 4 * 6 + len(dst) * 40, "flops": 0}
    counts, live, _ = _used_pages(case)
    moved = sum(1 for p in live if p >= len(live))
    return {"bytes": 2 * moved * block + case["pages"] * 12 + len(live) * 8, "flops": 0}


# -------------------------------------------------------- the definition, 64 bits
def _decode64(raw, params, D):
    """One head's codes [T][D / 2] and parameters [T][D / 64] (16 bits each) -> [T][D] in 64 bits."""
    out = torch.empty((raw.shape[0], D), dtype=torch.float64, device=raw.device)
    out[:, 0::2] = (raw % 16).double()
    out[:, 1::2] = (raw // 16).double()
    bits = params.long() & 0xFFFF
    zero, e, m = bits % 16, bits // 1024 % 32, (bits % 1024) // 16 * 16
    scale = torch.where(e > 0, (1024 + m).double() * torch.exp2(e.double() - 25), m.double() * 2.0 ** -24)
    return scale.repeat_interleave(GROUP, 1) * (out - zero.double().repeat_interleave(GROUP, 1))


def _exact_attend(case, s):
    D, H, g = case["D"], case["hkv"], case["group"]
    lengths, n = _lengths(case)
    table, pool = s["table"].cpu().tolist(), s["data"][s["layer"]]
    half, par = PAGE * D // 2, D // GROUP * PAGE * 2
    out = torch.zeros((sum(n), H * g, D), dtype=torch.float64, device="cuda")
    at = 0
    for b, (L, k) in enumerate(zip(lengths, n)):
        blocks = pool[torch.tensor(table[b][:-(-L // PAGE)], device="cuda")]
        for h in range(H):
            one = blocks[:, h]
            ints = one[:, 2 * half:].contiguous().view(torch.int16).view(-1, 2, D // GROUP, PAGE).transpose(2, 3)
            keys = _decode64(one[:, :half].reshape(-1, D // 2), ints[:, 0].reshape(-1, D // GROUP), D)[:L]
            vals = _decode64(one[:, half:2 * half].reshape(-1, D // 2), ints[:, 1].reshape(-1, D // GROUP), D)[:L]
            for i in range(0, k, 256):
                m = min(256, k - i)
                q = s["q"][at + i:at + i + m, h * g:(h + 1) * g].double()
                z = torch.einsum("mgd,td->mgt", q, keys) / math.sqrt(D)
                last = torch.arange(L - k + i, L - k + i + m, device="cuda")[:, None, None]
                t = torch.arange(L, device="cuda")
                hidden = (t > last) | ((t <= last - case["window"]) if case["window"] else False)
                w = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
                out[at + i:at + i + m, h * g:(h + 1) * g] = torch.einsum("mgt,td->mgd", w, vals)
        at += k
    return out


def _exact_values(x):
    """What the cache holds of x [T][H][D]: per 64 values the scale's seven bits and the nearest step."""
    x = x.double().reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = x.amin(-1).clamp(max=0), x.amax(-1).clamp(min=0)
    step = ((hi - lo) / 15).to(torch.float16)
    e = torch.floor(torch.log2(step.double().clamp(min=2.0 ** -14)))
    ulp = torch.exp2(e - 6)  # of a number with seven significant bits
    step = torch.ceil(step.double() / ulp) * ulp
    step1 = torch.where(step > 0, step, torch.ones_like(step))
    zero = torch.round(-lo / step1).clamp(0, 15)
    code = (torch.round(x / step1[..., None]) + zero[..., None]).clamp(0, 15)
    return (step[..., None] * (code - zero[..., None])).flatten(-2)


def _exact_fork(case, s):
    table, length, refs = (s[k].cpu().numpy().copy() for k in ("table", "length", "refs"))
    src, dst = _fork_lists(case)
    before = [a.copy() for a in (table, length, refs)]
    for a, b in zip(src, dst):
        n = -(-int(length[a]) // PAGE)
        table[b, :n], length[b] = table[a, :n], length[a]
        refs[table[a, :n]] += 1
    free, where = list(np.flatnonzero(refs == 0)), []
    for b in dst:
        L = int(length[b])
        if L % PAGE:  # a child's last page is its parent's too
            table[b, L // PAGE] = free.pop(0)
        for i in range(-(-L // PAGE), -(-(L + case["new"]) // PAGE)):
            table[b, i] = free.pop(0)
        where += [int(table[b, p // PAGE]) * PAGE + p % PAGE for p in range(L, L + case["new"])]
    # the children are gone again: what is left is what was there
    return [np.arange(len(dst) + 1, dtype=np.int32) * np.int32(case["new"]), np.array(where, np.int32), *before, None]


def _exact_compact(case, s):
    table, length, refs = (s[k].cpu().numpy() for k in ("table", "length", "refs"))
    live = [p for p in range(len(refs)) if refs[p] > 0]
    n = len(live)
    new = {p: p for p in live if p < n}
    new.update(zip([p for p in live if p >= n], [p for p in range(n) if refs[p] == 0]))
    out, held = np.full_like(table, -1), np.zeros_like(refs)
    for b in range(table.shape[0]):
        for i in range(-(-int(length[b]) // PAGE)):
            out[b, i] = new[int(table[b, i])]
    for p, q in new.items():
        held[q] = refs[p]
    return [out, held, np.array([new.get(p, -1) for p in range(len(refs))], np.int32), np.array([n], np.int32), None]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(case, s)
    if case["kind"] == "append":
        return [_exact_values(s["k"]), _exact_values(s["v"])]
    if case["kind"] == "fork":
        return _exact_fork(case, s)
    if case["kind"] == "compact":
        return _exact_compact(case, s)
    x, y = s["x"].double(), torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda")
    for a in range(0, case["N"], 8192):
        c, sc, mn = (s[k][a:a + 8192].double() for k in ("codes", "scale", "minimum"))
        y[:, a:a + 8192] = x @ (c * sc.repeat_interleave(WGROUP, 1) + mn.repeat_interleave(WGROUP, 1)).t()
    return y
