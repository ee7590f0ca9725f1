"""Operators around the paged mixed-precision KV cache: what a decode or prefill step of a batch of agents calls beside
append and decode attention, at the sizes that it meets.

  rope    queries and keys normed per head and rotated to their positions (one axis, or time, height and width), the
          values moved out of the packed projection: what append and decode attention take
  table   the page tables kept on the GPU: sequences are cut back to what they keep (rejected draft tokens, a request that
          ends), newly arriving tokens get their slots, pages, positions and the work list of the append kernel
  shared  decode attention for groups of sequences that share a long prefix

`own` false: elementary torch operations.  `own` true: the calls of paper_2605_17170_amd.tkv.
"""
import math

import numpy as np
import torch

own = False

D, GROUP, PAGE = 128, 32, 64
EPS = 1e-6
DEV = torch.device("cuda" if torch.cuda.is_available() else "cpu")
MOST_ROPE = 16384 * (64 + 2 * 8)          # tokens x heads of the largest listed case
MOST_TABLE = 65536                        # arriving tokens
MOST_SHARED = 32 * 64 * 33600             # query heads x tokens attended to


# ------------------------------------------------------------------ cases
def _rope(name, tokens, q_heads, kv_heads, axes="", interleaved=False, adjacent=False, rotary=128, norm=True, packed=True,
          first=0, theta=1e6):
    """`axes`: pairs of channels of each axis, "" for one axis; `packed`: q, k and v are parts of one projection's rows;
    `first`: position of the first token."""
    c = {"op": "rope", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "axes": axes, "interleaved": interleaved,
         "adjacent": adjacent, "rotary": rotary, "norm": norm, "packed": packed, "first": first, "theta": theta}
    return dict(c, name=name) if name else c


def _table(name, seqs, shortest, longest, keep, new_least, new_most, channel_keys=False, spare=0, shape=0):
    """`seqs` sequences of `shortest` .. `longest` tokens, of which the last up to `keep` are cut off (-1: all of them);
    then each gets `new_least` .. `new_most` tokens; `spare`: tokens of the padded batch behind the last sequence."""
    c = {"op": "table", "seqs": seqs, "shortest": shortest, "longest": longest, "cut": keep, "new_least": new_least,
         "new_most": new_most, "channel_keys": channel_keys, "spare": spare, "shape": shape}
    return dict(c, name=name) if name else c


def _shared(name, kv_heads, group, groups, seqs, prefix, shortest, longest, channel_keys=False, shape=0):
    """`groups` groups of up to `seqs` sequences each; about `prefix` shared tokens per group; `shortest` .. `longest`
    tokens of their own per sequence."""
    c = {"op": "shared", "kv_heads": kv_heads, "group": group, "groups": groups, "seqs": seqs, "prefix": prefix,
         "shortest": shortest, "longest": longest, "channel_keys": channel_keys, "shape": shape}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one generated token for each of 32 sequences, far into their contexts: the call is all latency
        _rope("rope_32x1", 32, 64, 8, first=120001),
        # a screenshot between text, positions by time, height and width, axes dealt out in turn
        _rope("rope_2501_three_axes", 2501, 32, 8, axes="24,20,20", interleaved=True, theta=5e6),
        # a tool result for a model of adjacent pairs, half of the head rotated, no norms, tensors of their own
        _rope("rope_701_adjacent_half", 701, 16, 2, adjacent=True, rotary=64, norm=False, packed=False, first=4000, theta=1e4),
        # a long prompt in one piece
        _rope("rope_16384", 16384, 64, 8, axes="16,24,24"),
        # one generated token for each of 32 sequences, nothing cut off
        _table("table_32x1", 32, 300, 30000, 0, 1, 1, shape=1),
        # 200 sequences with draft tokens: up to seven rejected, five more drafted, a batch padded to a round size
        _table("table_200x5_drafts", 200, 97, 3001, 7, 5, 5, spare=24, shape=2),
        # tool results behind open pages, per-channel INT2 keys
        _table("table_12_ragged_channel_keys", 12, 33, 2999, 0, 1, 1501, channel_keys=True, shape=3),
        # requests that have ended make room for prompts of 64K tokens in all
        _table("table_6_prompts", 6, 5000, 20000, -1, 10000, 10922, shape=4),
        # a small agent, four attempts side by side, one kv head
        _shared("shared_4_prefix_1500_1head", 1, 4, 1, 4, 1500, 3, 201, shape=5),
        # eight function-calling agents behind one system prompt with its tools
        _shared("shared_8_prefix_11000", 8, 8, 1, 8, 11000, 97, 1501, shape=6),
        # three applications with a prompt each, per-channel INT2 keys
        _shared("shared_3x6_prefix_5000_channel_keys", 4, 4, 3, 6, 5000, 0, 2001, channel_keys=True, shape=7),
        # 32 samples from one long document
        _shared("shared_32_prefix_32768", 8, 8, 1, 32, 32768, 64, 1024, shape=8),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["rope", "table", "shared", "shared"])
    shape = rng.randint(100, 1 << 30)
    if op == "rope":
        kv = rng.choice([1, 2, 4, 8])
        q = kv * rng.choice([1, 2, 4, 5, 8])
        rotary = rng.choice([128, 128, 96, 64, 32])
        axes = ""
        if rng.random() < 0.5:
            a = rng.randint(1, rotary // 6)
            b = rng.randint(1, rotary // 6)
            axes = "%d,%d,%d" % (rotary // 2 - a - b, a, b)
        return _rope(None, _log_uniform(rng, 1, MOST_ROPE // (q + 2 * kv)) if rng.random() < 0.8 else _log_uniform(rng, 1, 64), q, kv, axes,
                     rng.random() < 0.5, rng.random() < 0.4, rotary, rng.random() < 0.8, rng.random() < 0.6,
                     _log_uniform(rng, 1, 1000000), rng.choice([1e4, 5e5, 1e6, 5e6]))
    if op == "table":
        seqs = _log_uniform(rng, 1, 512)
        most = max(1, MOST_TABLE // seqs)
        new = _log_uniform(rng, 1, min(most, 16384))
        longest = _log_uniform(rng, 1, max(2, min(30000, 1000000 // seqs)))
        return _table(None, seqs, max(1, longest // rng.randint(1, 40)), longest, rng.choice([0, 0, 3, 500, -1]),
                      rng.choice([new, max(1, new // 10), 1]), new, rng.random() < 0.3, rng.choice([0, 0, 7, 100]), shape)
    kv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 4, 4, 8, 8])
    groups = rng.choice([1, 1, 1, 2, 4])
    seqs = _log_uniform(rng, 1, 32 // groups)
    most = min(32768, MOST_SHARED // (kv * group * groups * seqs))
    prefix = _log_uniform(rng, 1, most)
    longest = _log_uniform(rng, 1, min(4096, max(1, most - prefix)))
    return _shared(None, kv, group, groups, seqs, prefix, rng.choice([0, 1, longest // 3, longest]), longest, rng.random() < 0.3, shape)


# ------------------------------------------------------------------ widths of tokens
def _trace(rng, n, recent=0):
    """u8[n]: the width of every token of one context: runs of lognormal length at INT2 or INT4, the last ones at INT4."""
    runs = np.clip(np.round(rng.lognormal(math.log(200.0), 1.0, n // 16 + 1)), 16, 4096).astype(np.int64)
    bits = np.repeat(np.where(rng.random(runs.size) < 0.3, 4, 2), runs)[:n].astype(np.uint8)
    bits[max(n - recent, 0):] = 4
    return bits


def _route(bits):
    """Per-channel INT2 keys come in whole blocks of 32 tokens: the last INT2 tokens that fill none are INT4."""
    at = np.flatnonzero(bits == 2)
    out = bits.copy()
    out[at[at.size - at.size % GROUP:]] = 4
    return out


def _lengths(rng, n, lo, hi):
    if lo <= 0:
        return rng.integers(0, hi + 1, n)
    return np.round(np.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)), n))).astype(np.int64)


def _generator(seed, part):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + part)
    return g


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


# ------------------------------------------------------------------ rope
def _axis_of_pair(case):
    """Which axis each pair of channels turns with."""
    pairs = case["rotary"] // 2
    if not case["axes"]:
        return np.zeros(pairs, np.int64)
    sections = [int(x) for x in case["axes"].split(",")]
    if not case["interleaved"]:
        return np.repeat(np.arange(len(sections)), sections)
    i = np.arange(pairs)   # dealt out in turn; the turn of an axis whose pairs are used up goes to the first
    a = i % len(sections)
    return np.where(i // len(sections) < np.array(sections)[a], a, 0)


def _rope_sections(case):
    """Pairs of each axis as _axis_of_pair deals them out (the first axis has what the others leave)."""
    return [int(x) for x in np.bincount(_axis_of_pair(case), minlength=len(case["axes"].split(",")) if case["axes"] else 1)]


def _rope_inputs(case, seed):
    t, hq, hk = case["tokens"], case["q_heads"], case["kv_heads"]
    g = _generator(seed, 1)
    # a few channels of the projection are far larger than the others
    loud = torch.where(torch.rand((hq + 2 * hk, D), device=DEV, generator=g) < 0.03, 20.0, 1.0)
    rows = (torch.randn((t, hq + 2 * hk, D), device=DEV, generator=g) * loud).to(torch.bfloat16)
    parts = list(torch.split(rows, [hq, hk, hk], 1))
    if not case["packed"]:
        parts = [p.contiguous() for p in parts]
    weights = [(1.0 + 0.2 * torch.randn((D,), device=DEV, generator=g)).to(torch.bfloat16) if case["norm"] else None for _ in range(2)]
    i = torch.arange(t, device=DEV)
    pos = case["first"] + seed % 97 + i
    if case["axes"]:   # text, an image of rows of 37 patches, text
        a, b = t // 4, t - t // 4
        inside = (i >= a) & (i < b)
        start = case["first"] + seed % 97 + a
        pos = torch.stack([torch.where(inside, start, pos), torch.where(inside, start + (i - a) // 37, pos),
                           torch.where(inside, start + (i - a) % 37, pos)])
    else:
        pos = pos[None]
    return parts, weights, pos.to(torch.int32).contiguous()


def _rope_plain(s):
    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
        angle = s["pos"].double()[s["axis"]].t() * s["freq"]
        c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
        a, b = x[..., s["first"]], x[..., s["second"]]
        out = x.clone()
        out[..., s["first"]] = a * c - b * n
        out[..., s["second"]] = a * n + b * c
        return out.to(torch.bfloat16)
    q, k, v = s["parts"]
    return [turned(q, s["weights"][0]), turned(k, s["weights"][1]), v.clone(memory_format=torch.contiguous_format)]


def _pair_channels(case):
    i = np.arange(case["rotary"] // 2)
    return (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + case["rotary"] // 2)


def _rope_exact(case, seed):
    parts, weights, pos = _rope_inputs(case, seed)
    axis, half = _axis_of_pair(case), case["rotary"] // 2
    outs = []
    for x, w in zip(parts[:2], weights):
        y = x.double()
        if w is not None:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + EPS) * w.double()
        z = y.clone()
        first, second = _pair_channels(case)
        for i in range(half):
            angle = pos[axis[i]].double() * case["theta"] ** (-2.0 * i / case["rotary"])
            turn = torch.polar(torch.ones_like(angle), angle)[:, None]
            p = torch.complex(y[..., first[i]], y[..., second[i]]) * turn
            z[..., first[i]], z[..., second[i]] = p.real, p.imag
        outs.append(z)
    return outs + [parts[2].double()]


# ------------------------------------------------------------------ table
def _table_shape(case):
    """Widths of the tokens that each sequence holds and gets, and how many of each width it keeps."""
    rng = np.random.default_rng([case["shape"], 31])
    n = case["seqs"]
    held = [_trace(rng, int(x), 200) for x in _lengths(rng, n, case["shortest"], case["longest"])]
    new = rng.integers(case["new_least"], case["new_most"] + 1, n)
    arriving = [np.full(int(x), 4, np.uint8) if case["new_most"] <= 16 else _trace(rng, int(x)) for x in new]
    if case["channel_keys"]:
        held, arriving = [_route(b) for b in held], [_route(b) for b in arriving]
    have = np.array([[(b == 2).sum(), (b == 4).sum()] for b in held], np.int64)
    keep = have.copy()
    if case["cut"] < 0:
        keep[:] = 0
    else:
        keep[:, 1] -= np.minimum(keep[:, 1], rng.integers(0, case["cut"] + 1, n))
    return have, keep, arriving


def _pages(n):
    return -(-n // PAGE)


def _table_inputs(case, seed):
    have, keep, arriving = _table_shape(case)
    n = case["seqs"]
    after = keep + np.array([[(b == 2).sum(), (b == 4).sum()] for b in arriving], np.int64)
    stride = int(max(_pages(have).sum(1).max(), _pages(after).sum(1).max())) + 3
    # as many pages again as the sequences hold or will hold, and a few more
    p2, p4 = (int(2 * max(_pages(have)[:, k].sum(), _pages(after)[:, k].sum())) + 8 for k in range(2))
    rng = np.random.default_rng([seed, 37])
    order = [rng.permutation(p2), p2 + rng.permutation(p4)]
    rows = np.full((n, stride), -1, np.int32)
    at = [0, 0]
    for b in range(n):
        for k in range(2):
            m = int(_pages(have[b, k]))
            lead = int(_pages(have[b, 0])) if k else 0
            rows[b, lead:lead + m] = order[k][at[k]:at[k] + m]
            at[k] += m
    free = np.full(p2 + p4, -1, np.int32)
    free[:p2 - at[0]], free[p2:p2 + p4 - at[1]] = order[0][at[0]:], order[1][at[1]:]
    tags = np.concatenate(arriving + [np.full(case["spare"], 4, np.uint8)])
    lens = np.array([b.size for b in arriving], np.int32)
    work = int(sum(_pages(b.size) + 2 for b in arriving)) if case["new_most"] > 16 else int(sum(min(b.size, 2) for b in arriving))
    return {"have": have.astype(np.int32), "keep": keep.astype(np.int32), "tags": tags, "lens": lens, "rows": rows, "free": free,
            "n_free": np.array([p2 - at[0], p4 - at[1]], np.int32), "pages": (p2, p4), "work": max(1, work)}


def _table_state(case, seed):
    x = _table_inputs(case, seed)
    n, t = case["seqs"], x["tags"].size
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=DEV)  # noqa: E731
    return {"p2": x["pages"][0], "p4": x["pages"][1], "tags": _dev(x["tags"]), "lens": _dev(x["lens"]),
            "keep2": _dev(x["keep"][:, 0]), "keep4": _dev(x["keep"][:, 1]), "n2": _dev(x["have"][:, 0]), "n4": _dev(x["have"][:, 1]),
            "rows": _dev(x["rows"]), "free": _dev(x["free"]), "n_free": _dev(x["n_free"]),
            "indptr": i32(n + 1), "positions": i32(t), "slots": i32(t), "work_pages": i32(x["work"]), "work_src": i32(x["work"], PAGE),
            "n_work": i32(1)}


TABLE_OUT = ["indptr", "positions", "slots", "work_pages", "work_src", "n_work", "n2", "n4", "rows", "free", "n_free"]


def _ragged(counts):
    """(owner, index within the owner) of sum(counts) entries."""
    owner = torch.repeat_interleave(torch.arange(counts.numel(), device=DEV), counts)
    return owner, torch.arange(owner.numel(), device=DEV) - (counts.cumsum(0) - counts)[owner]


def _table_plain(s):
    p2, n, t = s["p2"], s["lens"].numel(), s["tags"].numel()
    lens, n2, n4 = s["lens"].long(), s["n2"].long(), s["n4"].long()
    keep2, keep4 = torch.minimum(s["keep2"].long(), n2), torch.minimum(s["keep4"].long(), n4)
    indptr = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), lens.cumsum(0)])
    seq, rank = _ragged(lens)
    total = seq.numel()
    wide = (s["tags"][:total] == 4).long()
    before4 = wide.cumsum(0) - wide
    first4 = torch.cat([before4, wide.sum()[None]])[indptr[:-1]] if total else torch.zeros_like(lens)
    rank4 = before4 - first4[seq]
    place = torch.where(wide == 1, keep4[seq] + rank4, keep2[seq] + rank - rank4)   # place in the stream of its width
    new4 = torch.zeros_like(lens).scatter_add_(0, seq, wide)
    new2 = lens - new4
    free, rows = s["free"].clone(), s["rows"].clone()
    n_free = s["n_free"].long().clone()
    widest = torch.arange(rows.shape[1], device=DEV)[None]
    had2, had4 = _pages(n2), _pages(n4)
    kept2, kept4 = _pages(keep2), _pages(keep4)
    np2, np4 = _pages(keep2 + new2), _pages(keep4 + new4)
    # the pages that are given back, the first of them on top of the free list, and those that are taken from its top
    got = []
    for w, lo, had, kept, now, lead in ((0, 0, had2, kept2, np2, torch.zeros_like(had2)), (1, p2, had4, kept4, np4, had2)):
        b, i = _ragged(had - kept)
        dropped = rows[b, lead[b] + kept[b] + i]
        top = n_free[w] + dropped.numel()
        free[lo + top - 1 - torch.arange(dropped.numel(), device=DEV)] = dropped
        b, i = _ragged(now - kept)
        taken = free[lo + top - 1 - torch.arange(b.numel(), device=DEV)]
        n_free[w] = top - b.numel()
        got.append((b, kept[b] + i, taken))
    out = torch.full_like(rows, -1)
    b, i = (widest < kept2[:, None]).nonzero(as_tuple=True)
    out[b, i] = rows[b, i]
    b, i = (widest < kept4[:, None]).nonzero(as_tuple=True)
    out[b, np2[b] + i] = rows[b, had2[b] + i]
    out[got[0][0], got[0][1]] = got[0][2]
    out[got[1][0], np2[got[1][0]] + got[1][1]] = got[1][2]
    # the pages that receive tokens: of every sequence those at INT2, then those at INT4
    first2, first4p = keep2 // PAGE, keep4 // PAGE
    touch2, touch4 = torch.where(new2 > 0, np2 - first2, 0), torch.where(new4 > 0, np4 - first4p, 0)
    base = (touch2 + touch4).cumsum(0) - touch2 - touch4
    work_pages = torch.zeros_like(s["work_pages"])
    b, i = _ragged(touch2)
    work_pages[base[b] + i] = out[b, first2[b] + i]
    b, i = _ragged(touch4)
    work_pages[base[b] + touch2[b] + i] = out[b, np2[b] + first4p[b] + i]
    index = place // PAGE
    page = out[seq, index + wide * np2[seq]]
    entry = base[seq] + torch.where(wide == 1, touch2[seq] + index - first4p[seq], index - first2[seq])
    work_src = torch.full_like(s["work_src"], -1)
    work_src.view(-1)[entry * PAGE + place % PAGE] = torch.arange(total, dtype=torch.int32, device=DEV)
    behind = torch.full((t - total,), -1, dtype=torch.int32, device=DEV)
    s["indptr"].copy_(indptr)
    s["positions"].copy_(torch.cat([(keep2 + keep4)[seq] + rank, behind]))
    s["slots"].copy_(torch.cat([page * PAGE + place % PAGE, behind]))
    s["work_pages"].copy_(work_pages)
    s["work_src"].copy_(work_src)
    s["n_work"].copy_((touch2 + touch4).sum()[None])
    s["n2"].copy_(keep2 + new2)
    s["n4"].copy_(keep4 + new4)
    s["rows"].copy_(out)
    s["free"].copy_(free)
    s["n_free"].copy_(n_free)
    return [s[k] for k in TABLE_OUT]


def _table_exact(case, seed):
    """One token after the other, with lists."""
    x = _table_inputs(case, seed)
    p2 = x["pages"][0]
    free = x["free"].copy()
    top = [int(v) for v in x["n_free"]]
    lead = [0, p2]
    n = case["seqs"]
    lists = []
    for b in range(n):
        a, c = (int(_pages(int(v))) for v in x["have"][b])
        lists.append([list(x["rows"][b, :a]), list(x["rows"][b, a:a + c])])
    count = [[min(int(x["have"][b, w]), int(x["keep"][b, w])) for w in range(2)] for b in range(n)]
    for b in reversed(range(n)):     # the last page of the last sequence goes back first
        for w in range(2):
            while len(lists[b][w]) > _pages(count[b][w]):
                free[lead[w] + top[w]] = lists[b][w].pop()
                top[w] += 1
    t = x["tags"].size
    positions, slots = np.full(t, -1, np.int32), np.full(t, -1, np.int32)
    work_pages, work_src = np.zeros(x["work"], np.int32), np.full((x["work"], PAGE), -1, np.int32)
    indptr, done, n_work = [0], 0, 0
    for b in range(n):
        tags = x["tags"][done:done + int(x["lens"][b])]
        entry = {}
        for w, bits in ((0, 2), (1, 4)):   # INT2 tokens first
            for i in np.flatnonzero(tags == bits):
                at = count[b][w]
                if at // PAGE == len(lists[b][w]):
                    top[w] -= 1
                    lists[b][w].append(free[lead[w] + top[w]])
                page = int(lists[b][w][at // PAGE])
                if page not in entry:
                    entry[page] = n_work
                    work_pages[n_work] = page
                    n_work += 1
                work_src[entry[page], at % PAGE] = done + i
                slots[done + i] = page * PAGE + at % PAGE
                count[b][w] = at + 1
        held = sum(min(int(x["have"][b, w]), int(x["keep"][b, w])) for w in range(2))
        positions[done:done + tags.size] = held + np.arange(tags.size)
        done += tags.size
        indptr.append(done)
    rows = np.full_like(x["rows"], -1)
    for b in range(n):
        ids = lists[b][0] + lists[b][1]
        rows[b, :len(ids)] = ids
    count = np.array(count, np.int32)
    return [torch.from_numpy(np.ascontiguousarray(v)) for v in
            (np.array(indptr, np.int32), positions, slots, work_pages, work_src, np.array([n_work], np.int32), count[:, 0], count[:, 1],
             rows, free, np.array(top, np.int32))]


# ------------------------------------------------------------------ shared: the packed cache
def _code_places(bits):
    """(word, first bit) of the K code and of the V code of every (slot, channel) of a record's planes, and the places of
    the K and the V metadata of every (slot, group of channels)."""
    t, c = np.meshgrid(np.arange(PAGE), np.arange(D), indexing="ij")
    tile, row, quad, j = t // 16, t % 16, (t % 16) // 4, 4 * ((t // 16) % 2) + t % 4
    per = 32 // bits
    kw, kb = ((tile * bits + (c % 32) // per) * 16 + row) * 4 + c // 32, bits * (c % per)
    if bits == 4:
        vw, vb = (((t // 32 * 2 + c // 64) * 4 + quad) * 16 + c % 16) * 4 + (c // 16) % 4, 4 * ((j % 2) * 4 + j // 2)
    else:
        vw, vb = ((c // 64 * 4 + quad) * 16 + c % 16) * 4 + (c // 16) % 4, 2 * (4 * (t // 32) + j // 2 + 8 * (j % 2))
    t, g = np.meshgrid(np.arange(PAGE), np.arange(4), indexing="ij")
    km, vm = 4 * t + g, ((t // 32 * 4 + (t % 16) // 4) * 4 + g) * 8 + 4 * ((t // 16) % 2) + t % 4
    return [_dev(a.astype(np.int64)) for a in (kw, kb, vw, vb, km, vm)]


def _channel_places():
    """Place of the metadata of every (block of 32 slots, channel) of per-channel INT2 keys."""
    b, c = np.meshgrid(np.arange(2), np.arange(D), indexing="ij")
    r = c % 32
    return _dev((((b * 4 + c // 32) * 4 + 2 * (r // 16) + (r % 8) // 4) * 8 + 2 * (r % 4) + (r % 16) // 8).astype(np.int64))


def _grid(x, bits, dim):
    """Codes, scale and zero-point (fp16) of x quantised by groups along `dim`."""
    f = x.float()
    lo, hi = f.amin(dim, keepdim=True), f.amax(dim, keepdim=True)
    scale, zero = ((hi - lo) / float(2 ** bits - 1)).half(), (lo + 0.0).half()
    s = scale.float()
    code = torch.where(s > 0, torch.round((f - zero.float()) * torch.where(s > 0, 1.0 / s, 0.0)), 0.0).clamp(0, 2 ** bits - 1)
    return code.int(), scale, zero


def _words(code, word, bit, n):
    """Codes [records, 64, 128] to words [records, n]."""
    out = torch.zeros((code.shape[0], n), dtype=torch.int32, device=DEV)
    shifted = code << bit.int()
    return out.scatter_add_(1, word.reshape(1, -1).expand(code.shape[0], -1), shifted.reshape(code.shape[0], -1))


def _records(K, V, valid, bits, channel_keys):
    """Packs K, V [pages, heads, 64, 128] of which the slots `valid` [pages, 64] are written: bytes [pages, heads, record], and
    the values that they stand for, in 64 bits.  What was never written holds patterns of NaN."""
    n, h = K.shape[0], K.shape[1]
    kw, kb, vw, vb, km, vm = _code_places(bits)
    words = PAGE * D * bits // 32
    nan = torch.full((), float("nan"), dtype=torch.half, device=DEV)
    alive = valid[:, None, :, None].expand(n, h, PAGE, 4)

    def by_token(x):
        code, scale, zero = _grid(x.reshape(n, h, PAGE, 4, GROUP), bits, -1)
        value = code.double() * scale.double() + zero.double()
        return code.reshape(n * h, PAGE, D), torch.where(alive, scale[..., 0], nan), torch.where(alive, zero[..., 0], nan), value.reshape(n, h, PAGE, D)

    def plane(x, at):
        out = torch.empty((n * h, PAGE * 4), dtype=torch.half, device=DEV)
        out[:, at.reshape(-1)] = x.reshape(n * h, -1)
        return out.view(torch.uint8)

    if channel_keys and bits == 2:
        code, scale, zero = _grid(K.reshape(n, h, 2, 32, D), bits, 3)
        k_value = (code.double() * scale.double() + zero.double()).reshape(n, h, PAGE, D)
        whole = valid.reshape(n, 1, 2, 32, 1).all(3).expand(n, h, 2, D)
        at = _channel_places()
        k_code, k_meta = code.reshape(n * h, PAGE, D), [plane(torch.where(whole, x[..., 0, :], nan), at) for x in (scale, zero)]
    else:
        k_code, scale, zero, k_value = by_token(K)
        k_meta = [plane(x, km) for x in (scale, zero)]
    v_code, scale, zero, v_value = by_token(V)
    rec = torch.cat([_words(k_code, kw, kb, words).view(torch.uint8)] + k_meta +
                    [_words(v_code, vw, vb, words).view(torch.uint8), plane(scale, vm), plane(zero, vm)], 1)
    return rec.reshape(n, h, -1), k_value, v_value


def _unpack(rec, bits, places, channel_places):
    """K and V [pages, heads, 64, 128] in 32 bits of records [pages, heads, bytes]."""
    n, h, codes = rec.shape[0], rec.shape[1], PAGE * D * bits // 8
    kw, kb, vw, vb, km, vm = places
    part = lambda a, b, t: rec[..., a:b].contiguous().view(t)  # noqa: E731
    code = lambda w, word, bit: ((w[..., word] >> bit.int()) & (2 ** bits - 1)).float()  # noqa: E731
    spread = lambda x: x.float().repeat_interleave(GROUP, -1)  # noqa: E731
    planes = [part(a, a + 512, torch.half) for a in (codes, codes + 512, 2 * codes + 1024, 2 * codes + 1536)]
    if channel_places is not None and bits == 2:
        scale, zero = (p[..., channel_places].float().repeat_interleave(32, -2) for p in planes[:2])
    else:
        scale, zero = (spread(p[..., km]) for p in planes[:2])
    K = code(part(0, codes, torch.int32), kw, kb) * scale + zero
    V = code(part(codes + 1024, 2 * codes + 1024, torch.int32), vw, vb) * spread(planes[2][..., vm]) + spread(planes[3][..., vm])
    return K, V


# ------------------------------------------------------------------ shared
def _shared_shape(case):
    """Per list of pages (the groups' prefixes, then the sequences' own): tokens of either width; the group of every sequence."""
    rng = np.random.default_rng([case["shape"], 41])
    sizes = [case["seqs"]] * case["groups"] if case["groups"] == 1 else [int(x) for x in rng.integers(1, case["seqs"] + 1, case["groups"])]
    member = np.repeat(np.arange(case["groups"]), sizes)
    member = member[rng.permutation(member.size)]     # sequences of a group stand anywhere in the batch
    prefix = [case["prefix"]] * case["groups"] if case["groups"] == 1 else _lengths(rng, case["groups"], max(1, case["prefix"] // 2), case["prefix"])
    lists = [_trace(rng, int(x)) for x in prefix] + [_trace(rng, int(x), 64) for x in _lengths(rng, member.size, case["shortest"], case["longest"])]
    if case["channel_keys"]:
        lists = [_route(b) for b in lists]
    return np.array([[(b == 2).sum(), (b == 4).sum()] for b in lists], np.int64).reshape(-1, 2), member


def _shared_cache(case, seed):
    """The packed pool, page lists, and the values that stand in it: K, V [list tokens, heads, 128] in 64 bits, lists one behind
    the other, INT2 tokens first."""
    tokens, member = _shared_shape(case)
    h = case["kv_heads"]
    pages = _pages(tokens)
    n2, n4 = int(pages[:, 0].sum()), int(pages[:, 1].sum())
    p2, p4 = n2 + 3, n4 + 3
    g = _generator(seed, 2)
    loud = torch.ones((2, h, 1, D), device=DEV)      # four channels of a head are 20 times the others
    loud.scatter_(3, torch.rand((2, h, 1, D), device=DEV, generator=g).argsort(-1)[..., :4], 20.0)
    pool, ids, values = [], [], []
    for w, bits, n, p in ((0, 2, n2, p2), (1, 4, n4, p4)):
        fill = torch.arange(PAGE, device=DEV)[None]
        left = np.concatenate([np.clip(tokens[i, w] - PAGE * np.arange(pages[i, w]), 0, PAGE) for i in range(len(tokens))]) if n else np.zeros(0, np.int64)
        valid = fill < _dev(left)[:, None]
        K, V = ((torch.randn((n, h, PAGE, D), device=DEV, generator=g) * loud[k]).to(torch.bfloat16) for k in range(2))
        rec, k_value, v_value = _records(K, V, valid, bits, case["channel_keys"]) if n else (None, K.double(), V.double())
        at = torch.randperm(p, device=DEV, generator=g)[:n]
        arena = torch.full((p, h, 2 * (PAGE * D * bits // 8) + 2048), 255, dtype=torch.uint8, device=DEV)
        if n:
            arena[at] = rec
        pool.append(arena.reshape(-1))
        ids.append((at + w * p2).int())
        values.append((k_value, v_value, valid))
    lists = []   # INT2 pages, then INT4 pages of every list
    at = np.concatenate([[[0, 0]], np.cumsum(pages, 0)])
    for i in range(len(tokens)):
        lists += [ids[w][int(at[i, w]):int(at[i + 1, w])] for w in range(2)]
    bit_map = torch.zeros(p2 + p4, dtype=torch.uint8, device=DEV)
    bit_map[ids[0].long()], bit_map[ids[1].long()] = 2, 4
    return {"tokens": tokens, "member": member, "pages": pages, "p2": p2, "p4": p4, "pool": torch.cat(pool), "bit_map": bit_map,
            "page_ids": torch.cat(lists) if lists else torch.zeros(0, dtype=torch.int32, device=DEV), "values": values, "at": at}


def _shared_q(case, seed, batch):
    return torch.randn((batch, case["kv_heads"] * case["group"], D), device=DEV, generator=_generator(seed, 3)).to(torch.bfloat16)


def _shared_state(case, seed):
    c = _shared_cache(case, seed)
    groups, batch = case["groups"], c["member"].size
    counts = c["pages"].sum(1)
    indptr = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    order = np.argsort(c["member"], kind="stable").astype(np.int32)
    s = {"pool": c["pool"], "bit_map": c["bit_map"], "page_ids": c["page_ids"], "p2": c["p2"], "p4": c["p4"], "q": _shared_q(case, seed, batch),
         "n2": _dev(c["tokens"][:, 0].astype(np.int32)), "n4": _dev(c["tokens"][:, 1].astype(np.int32)), "indptr": _dev(indptr),
         "group_of": _dev(c["member"].astype(np.int32)), "groups": groups,
         "places": {bits: _code_places(bits) for bits in (2, 4)}, "channel_places": _channel_places() if case["channel_keys"] else None}
    if own:
        _shared_plan(case, s, c, groups, batch, indptr, order)
    return s


def _shared_plan(case, s, c, groups, batch, indptr, order):
    from paper_2605_17170_amd import harness, tkv
    desc = tkv.tkv_desc.make(case["kv_heads"], c["p2"], c["p4"], int2_key_axis=1 if case["channel_keys"] else 0)
    tokens = c["tokens"].astype(np.int32)
    heads = case["kv_heads"] * case["group"]
    target = harness.default_target_items(case["kv_heads"])
    items, slots = tkv.tkv_plan_decode(desc, indptr[groups:] - indptr[groups], tokens[groups:, 0], tokens[groups:, 1], target)
    member_indptr = np.concatenate([[0], np.cumsum(np.bincount(c["member"], minlength=groups))]).astype(np.int32)
    plan = tkv.tkv_plan_decode_shared(desc, batch, heads, tokens[:groups, 0], tokens[:groups, 1], member_indptr, order, harness.default_shared_units(),
                                      items, slots)
    prefix = tkv.tkv_prefix.make(s["indptr"][:groups + 1], s["page_ids"], s["n2"][:groups], s["n4"][:groups], _dev(member_indptr), _dev(order),
                                 _dev(plan.member_slots), _dev(plan.prefix_items), plan.max_members)
    out = torch.empty((batch, heads, D), dtype=torch.bfloat16, device=DEV)
    workspace = torch.empty(max(16, tkv.tkv_decode_workspace_bytes(desc, plan.n_slots, heads)), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    s["out"] = out
    s["call"] = tkv.tkv_decode_attention_shared(desc, s["pool"], s["bit_map"], s["q"], s["indptr"][groups:], s["page_ids"], s["n2"][groups:], s["n4"][groups:],
                                                _dev(plan.items), prefix, _dev(plan.seq_item_indptr), plan.n_slots, 1.0 / math.sqrt(D), out, workspace,
                                                status, prepare=True)


def _shared_plain(s, case):
    h, r, groups = case["kv_heads"], case["group"], s["groups"]
    counts = s["indptr"].long().diff()
    owner, i = _ragged(counts)      # list of every page, and the page's place in it
    lead = _pages(s["n2"].long())
    wide = i >= lead[owner]
    cut = s["p2"] * h * 6144
    ids = s["page_ids"].long()
    arena2, arena4 = s["pool"][:cut].view(s["p2"], h, 6144), s["pool"][cut:].view(s["p4"], h, 10240)
    parts = []
    for w, bits, arena, lo, n, begin in ((False, 2, arena2, 0, s["n2"], torch.zeros_like(lead)), (True, 4, arena4, s["p2"], s["n4"], lead)):
        at = (wide == w).nonzero()[:, 0]
        K, V = _unpack(arena[ids[at] - lo], bits, s["places"][bits], s["channel_places"])
        left = n.long()[owner[at]] - PAGE * (i[at] - begin[owner[at]])
        valid = torch.arange(PAGE, device=DEV)[None] < left[:, None]
        page, slot = valid.nonzero(as_tuple=True)
        parts.append((K[page, :, slot], V[page, :, slot], owner[at][page]))
    K, V, owner = (torch.cat([p[k] for p in parts]) for k in range(3))      # [tokens, heads, 128], list of every token
    b = s["q"].shape[0]
    sees = (owner[None] == s["group_of"].long()[:, None]) | (owner[None] == groups + torch.arange(b, device=DEV)[:, None])
    q = s["q"].float().view(b, h, r, D).permute(1, 0, 2, 3).reshape(h, b * r, D)
    logits = torch.bmm(q, K.permute(1, 2, 0).contiguous()) / math.sqrt(D)
    logits = torch.where(sees.repeat_interleave(r, 0)[None], logits, float("-inf"))
    top = logits.amax(-1, keepdim=True)
    weight = torch.exp(logits - torch.where(torch.isfinite(top), top, 0.0))
    total = weight.sum(-1, keepdim=True)
    out = torch.bmm(weight, V.permute(1, 0, 2).contiguous()) / torch.where(total > 0, total, 1.0)
    return out.view(h, b, r, D).permute(1, 0, 2, 3).reshape(b, h * r, D).to(torch.bfloat16)


def _shared_exact(case, seed):
    c = _shared_cache(case, seed)
    h, r, groups = case["kv_heads"], case["group"], case["groups"]
    q = _shared_q(case, seed, c["member"].size).double()

    def rows(i, which):
        """Values of list i, one head after the other: [heads, tokens, 128]."""
        got = []
        for w in range(2):
            a, e = int(c["at"][i, w]), int(c["at"][i + 1, w])
            value, valid = c["values"][w][which][a:e], c["values"][w][2][a:e]
            got.append(value.permute(1, 0, 2, 3).reshape(h, -1, D)[:, valid.reshape(-1)])
        return torch.cat(got, 1)

    prefix = [(rows(i, 0), rows(i, 1)) for i in range(groups)]
    out = torch.zeros((q.shape[0], h * r, D), dtype=torch.float64, device=DEV)
    for b in range(q.shape[0]):
        K, V = (torch.cat([prefix[c["member"][b]][k], rows(groups + b, k)], 1) for k in range(2))
        if K.shape[1]:
            p = torch.softmax(torch.matmul(q[b].view(h, r, D), K.transpose(1, 2).contiguous()) * D ** -0.5, -1)
            out[b] = torch.matmul(p, V).reshape(h * r, D)
    return out


# ------------------------------------------------------------------ what is measured
def prepare(case, seed):
    if case["op"] == "shared":
        return dict(_shared_state(case, seed), case=case)
    if case["op"] == "table":
        s = dict(_table_state(case, seed), case=case)
        if own:
            from paper_2605_17170_amd import tkv
            n, t = s["lens"].numel(), s["tags"].numel()
            desc = tkv.tkv_desc.make(8, s["p2"], s["p4"], int2_key_axis=1 if case["channel_keys"] else 0)
            table = tkv.tkv_table.make(s["rows"], s["n2"], s["n4"], s["free"], s["n_free"])
            workspace = torch.empty(tkv.tkv_table_workspace_bytes(n, t), dtype=torch.uint8, device=DEV)
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            s["call"] = tkv.tkv_table_append(desc, table, s["keep2"], s["keep4"], s["lens"], s["tags"], s["indptr"], s["positions"], s["slots"],
                                             s["work_pages"], s["work_src"], s["n_work"], workspace, status, prepare=True)
        return s
    parts, weights, pos = _rope_inputs(case, seed)
    first, second = (_dev(np.asarray(x)) for x in _pair_channels(case))
    freq = case["theta"] ** (-2.0 * torch.arange(case["rotary"] // 2, dtype=torch.float64, device=DEV) / case["rotary"])
    s = {"case": case, "parts": parts, "weights": weights, "pos": pos, "axis": _dev(_axis_of_pair(case)), "freq": freq, "first": first, "second": second}
    if own:
        from paper_2605_17170_amd import tkv
        s["out"] = [torch.empty(p.shape, dtype=torch.bfloat16, device=DEV) for p in parts]
        rope = tkv.tkv_rope_make(case["rotary"], case["theta"], _rope_sections(case), interleaved=case["interleaved"], adjacent=case["adjacent"])
        s["call"] = tkv.tkv_norm_rope(rope, *parts, pos, *weights, EPS, *s["out"], prepare=True)
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        state["call"]()
        return [state[k] for k in TABLE_OUT] if op == "table" else state["out"]
    if op == "rope":
        return _rope_plain(state)
    return _table_plain(state) if op == "table" else _shared_plain(state, state["case"])


def exact(case, seed):
    return {"rope": _rope_exact, "table": _table_exact, "shared": _shared_exact}[case["op"]](case, seed)


def work(case):
    if case["op"] == "rope":
        t, h = case["tokens"], case["q_heads"] + 2 * case["kv_heads"]
        axes = 3 if case["axes"] else 1
        return {"bytes": 2 * t * h * D * 2 + 4 * axes * t + (4 * D if case["norm"] else 0), "flops": t * (h - case["kv_heads"]) * D * 8}
    if case["op"] == "table":
        have, keep, arriving = _table_shape(case)
        new = sum(b.size for b in arriving) + case["spare"]
        after = keep + np.array([[(b == 2).sum(), (b == 4).sum()] for b in arriving], np.int64)
        gone = int((_pages(have) - _pages(keep)).sum())
        taken = int((_pages(after) - _pages(keep)).sum())
        entries = int(sum(_pages(b.size) + 2 for b in arriving)) if case["new_most"] > 16 else int(sum(min(b.size, 2) for b in arriving))
        # tags, slots, positions; lengths, counts and what is kept; ids that move to and from the free lists; work list
        return {"bytes": new * 9 + case["seqs"] * 4 * 8 + 8 * (gone + taken) + max(1, entries) * 4 * (PAGE + 1), "flops": 0}
    tokens, member = _shared_shape(case)
    h, hq = case["kv_heads"], case["kv_heads"] * case["group"]
    own_tokens, groups = tokens.sum(1), case["groups"]
    attended = int(own_tokens[groups:].sum()) + int(own_tokens[:groups][member].sum())
    return {"bytes": h * int((tokens * np.array([96, 160])).sum()) + member.size * hq * D * 4, "flops": 4 * D * hq * attended}
