"""Many questions about one table, as cases that can be timed: rotary positions with several axes (text, row, column), which
sequences of a batch share their first pages, and the attention of their new tokens with what they share read once for all
(mate_rope_axes, mate_cache_append_axes, mate_cache_groups, mate_attn_decode_shared), in plain torch operations and through the
library's entry points.

A case's kind is one call of a layer or of a step of a server's loop:
  "axes"    Q and K of a batch rotated by positions of several axes, or their gradients turned back
  "step"    the new token of every running sequence: Q and K rotated by several axes, K, V and ids into the pages
  "groups"  who shares how many tokens with whom, from the sequences' pages
  "shared"  the new token of every sequence against what is cached, the shared pages of a group once for all of its sequences
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_TEXT = 0x7FFFFFFF  # id of text: attends, and is attended by, everything


def _axes(name, B, N, H, Hkv, d, rot, n_axes=3, dtype="bf16", interleaved=False, mixed=False, backward=False, layout="padded"):
    return {"name": name, "kind": "axes", "B": B, "N": N, "H": H, "Hkv": Hkv, "d": d, "rot": rot, "n_axes": n_axes, "dtype": dtype,
            "interleaved": interleaved, "mixed": mixed, "backward": backward, "layout": layout}


def _cached(name, kind, groups, members, L, tail, H, Hkv, d, page, n_row, dtype="bf16", text=1.0, prefix=64, cols=8, ragged=True,
            slots_first=False, min_len=1, n_axes=3, interleaved=False, mixed=False):
    return {"name": name, "kind": kind, "groups": groups, "members": members, "L": L, "tail": tail, "H": H, "Hkv": Hkv, "d": d, "page": page,
            "n_row": n_row, "dtype": dtype, "text": text, "prefix": prefix, "cols": cols, "ragged": ragged, "slots_first": slots_first,
            "min_len": min_len, "n_axes": n_axes, "interleaved": interleaved, "mixed": mixed}


def listed():
    return [
        # one table in single precision, a head size that is no power of two, half of it rotated (a unit test, a gradient check)
        _axes("axes_one_table_f32", 1, 512, 4, 4, 40, 20, dtype="f32"),
        # a training step on medium tables: place in the cell, row and column; Q and K as views of the fused projection's output
        _axes("axes_train", 4, 2048, 12, 12, 64, 64, layout="fused", mixed=True),
        # gradients of a packed batch of long documents (time, height, width of their pictures), grouped heads
        _axes("axes_long_backward", 1, 32768, 32, 8, 128, 128, interleaved=True, backward=True, layout="packed"),
        # one step of a busy server, one layer: a token for each of 64 sequences
        _cached("axes_step", "step", 8, 8, 2048, 64, 32, 8, 128, 16, 16),
        # who shares what: eight beams of each of eight tables
        _cached("groups_beams", "groups", 8, 8, 2048, 64, 12, 12, 64, 16, 6),
        # ... and 256 questions about one very long document
        _cached("groups_questions", "groups", 1, 256, 32768, 64, 1, 1, 64, 16, 1, ragged=False, min_len=256),
        # four questions about one table: the smallest call
        _cached("shared_one_table", "shared", 1, 4, 512, 32, 12, 12, 64, 16, 6, ragged=False),
        # beam search over eight tables of every length, eight beams each
        _cached("shared_beams", "shared", 8, 8, 2048, 64, 12, 12, 64, 16, 6),
        # 64 questions about one long table, grouped heads, cache laid out slot by slot
        _cached("shared_questions", "shared", 1, 64, 8192, 128, 32, 8, 128, 16, 16, prefix=128, ragged=False, slots_first=True),
        # 256 sequences behind one long document: as many products as bytes
        _cached("shared_crowd", "shared", 1, 256, 16384, 256, 16, 4, 128, 64, 8, prefix=256, ragged=False),
        # cells of sixteen tables, six of each filled in at a time: a new token attends its row or column and the prefix
        _cached("shared_cells", "shared", 16, 6, 4096, 16, 12, 12, 64, 16, 6, text=0.0, prefix=128, cols=10),
        # single precision, odd head size and pages, row and column heads in one group, cells and text in one batch
        _cached("shared_f32", "shared", 3, 5, 1500, 40, 6, 2, 48, 24, 2, dtype="f32", text=0.5, cols=5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges of the listed ones: sizes over their logarithm, odd ones among them."""
    most = {}
    for c in listed():
        w = work(c)
        for k in ("bytes", "flops"):
            most[c["kind"], k] = max(most.get((c["kind"], k), 0), w[k])
    while True:
        kind = rng.choice(["axes", "axes", "step", "groups", "shared", "shared", "shared", "shared"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        Hkv = rng.choice([1, 2, 3, 4, 8, 12])
        H = Hkv * rng.choice([1, 1, 2, 3, 4, 8])
        if kind == "axes":
            d = rng.choice([16, 40, 64, 80, 96, 128])
            rot = rng.choice([d, d, d // 2 // 2 * 2, 8 * rng.randint(1, d // 8)])
            c = _axes("", rng.randint(1, 8), _log_int(rng, 1, 16384), H, Hkv, d, rot, rng.randint(1, 4), dtype, rng.random() < 0.5,
                      rng.random() < 0.5, rng.random() < 0.5, rng.choice(["padded", "fused", "packed"]))
            if c["layout"] == "packed":
                c["B"] = 1
        else:
            L = _log_int(rng, 1, 32768)
            c = _cached("", kind, _log_int(rng, 1, 24), _log_int(rng, 1, 256), L, _log_int(rng, 1, 512), H, Hkv,
                        rng.choice([16, 48, 64, 64, 128, 128]), rng.choice([1, 8, 16, 16, 24, 64]), rng.randint(0, H), dtype,
                        rng.choice([0.0, 0.5, 1.0, 1.0]), min(L, _log_int(rng, 1, 256)), rng.randint(2, 30), True, rng.random() < 0.5,
                        rng.choice([1, 1, 100]), rng.randint(1, 4), rng.random() < 0.5, rng.random() < 0.5)
            if sum(_sizes(c)) > 512 or 2 * _slots(c) * Hkv * c["d"] * _SIZE[dtype] > 2 << 30:
                continue
        w = work(c)
        if w["bytes"] <= most[kind, "bytes"] and w["flops"] <= most[kind, "flops"]:
            # (multiply-adds of single precision have a thirtieth of the tensor cores' rate)
            if dtype == "f32" and kind == "shared" and w["flops"] > most[kind, "flops"] // 16:
                continue
            del c["name"]
            return c


# ---------------------------------------------------------------------------------------------- sizes

def _sizes(c):
    """Sequences of every group; a ragged batch has single ones among them."""
    if not c["ragged"]:
        return [c["members"]] * c["groups"]
    rng = np.random.default_rng(c["L"] * 7 + c["members"])
    n = [int(x) for x in rng.integers(1, c["members"] + 1, c["groups"])]
    n[0] = c["members"]
    return n


def _lengths(c, seed=0):
    """Per group: the tokens of its table; per sequence: its own tokens behind the full pages of the table, which it shares.  They belong
    to the case; where they are all that an operator reads, a seed has tables of its own, up to a sixteenth shorter, in an order of its own."""
    rng = np.random.default_rng(c["L"] * 1000 + c["groups"])
    sizes, tables, tails = _sizes(c), [], []
    if c["kind"] == "groups":
        mine = np.random.default_rng(seed)
        sizes, shorter = [sizes[i] for i in mine.permutation(len(sizes))], mine.integers(0, c["L"] // 16 + 1, len(sizes))
    for g, n in enumerate(sizes):
        L = c["L"] if g == 0 or not c["ragged"] else int(math.exp(rng.uniform(math.log(max(1, c["L"] / 8)), math.log(c["L"] + 0.999))))
        if c["ragged"] and g > 0 and rng.random() < 0.1:
            L = 0  # no sequence has a token yet
        if c["kind"] == "groups":
            L = max(0, L - int(shorter[g]))
        tables.append(L)
        tails.append([L % c["page"] + (int(rng.integers(0, c["tail"] + 1)) if L else 0) for _ in range(n)])
    return tables, tails


def _slots(c):
    """Tokens that are cached."""
    tables, tails = _lengths(c)
    return sum(t + sum(s) for t, s in zip(tables, tails))


def _ids(c, rng, n):
    """Row and column ids of the n tokens of a table: prefix, then cell by cell."""
    P = min(c["prefix"], n)
    cells = rng.geometric(0.45, size=n + 1).clip(max=16)
    cell = np.repeat(np.arange(len(cells)), cells)[:n - P]
    ids = np.zeros((2, n), np.int32)
    ids[0, P:], ids[1, P:] = cell // c["cols"] + 1, cell % c["cols"] + 1
    return ids


def _new_ids(c, rng, ids):
    """The new token's ids: text, or those of a cell of the table that is being filled in."""
    if rng.random() < c["text"] or ids.shape[1] == 0:
        return np.full(2, _TEXT, np.int32)
    return ids[:, int(rng.integers(ids.shape[1]))]


def _attended(c, ids, q):
    """(2, n): the keys of a table that a new token attends, by row and by column."""
    always = (np.arange(ids.shape[1]) < c["prefix"]) | (ids[0] == _TEXT) | (q[0] == _TEXT)
    return np.stack([always | (ids[v] == q[v]) for v in (0, 1)])


def work(case):
    c = case
    size = _SIZE[c["dtype"]]
    if c["kind"] == "axes":
        values = c["B"] * c["N"] * (c["H"] + c["Hkv"]) * c["d"]
        return {"bytes": 2 * values * size + 4 * c["n_axes"] * c["B"] * c["N"], "flops": 3 * values * c["rot"] // c["d"]}
    tables, tails = _lengths(c)
    B, row = sum(_sizes(c)), c["Hkv"] * c["d"] * size
    if c["kind"] == "step":
        return {"bytes": B * (2 * (c["H"] * c["d"] * size) + 4 * row + 16), "flops": 3 * B * (c["H"] + c["Hkv"]) * c["d"]}
    if c["kind"] == "groups":
        pages = sum(L // c["page"] * len(t) for L, t in zip(tables, tails))
        return {"bytes": 4 * pages + 20 * B, "flops": 0}
    rng = np.random.default_rng(0)
    G, rows, pairs, seen = c["H"] // c["Hkv"], 0, 0, 0
    by_view = (c["n_row"], c["H"] - c["n_row"])
    for L, tail in zip(tables, tails):
        shared = L - L % c["page"]
        ids = _ids(c, rng, L)
        some = np.zeros((2, L), bool)
        for n in tail:
            mine = _attended(c, ids, _new_ids(c, rng, ids))
            some |= mine
            behind = n - L % c["page"]  # text, which everybody attends
            pairs += sum(h * (int(mine[v].sum()) + behind) for v, h in enumerate(by_view))
            rows += c["Hkv"] * n
            seen += 4 * n
        for g in range(c["Hkv"]):
            first, last = g * G < c["n_row"], (g + 1) * G - 1 < c["n_row"]
            keys = some[0] if last else some[1] if not first else some[0] | some[1]
            rows += int(keys[:shared].sum())
        seen += shared * (4 if c["text"] == 1.0 else 8)
    return {"bytes": rows * 2 * c["d"] * size + seen + B * c["H"] * (2 * c["d"] * size + 4), "flops": 4 * c["d"] * pairs}


# ---------------------------------------------------------------------------------------------- inputs

def _frequencies(rot):
    """Radians per position of every pair."""
    return 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1))


def _axis_of_pairs(c, pairs):
    """Axis of every pair: one section after the other, or the axes in turn."""
    if c["mixed"]:
        return [i % c["n_axes"] for i in range(pairs)]
    return [i * c["n_axes"] // pairs for i in range(pairs)]


def _positions(c, rng, B, N):
    """[n_axes, B, N]: place in the text or the cell; row, column (or time, height, width); the document's page."""
    place = np.arange(N)[None] + rng.integers(0, 100, (B, 1))
    row, col = np.arange(N)[None] // 40 + rng.integers(0, 100, (B, 1)), np.arange(N)[None] % 37 + rng.integers(0, 8, (B, 1))
    return np.stack([place, row, col, place // 1024])[:c["n_axes"]].astype(np.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = _DTYPES[c["dtype"]]

    def values(*shape):
        return torch.randn(shape, device="cuda", dtype=dt, generator=g) * 0.5

    s = {"c": c}
    if c["kind"] == "axes":
        B, N, H, Hkv, d = (c[k] for k in ("B", "N", "H", "Hkv", "d"))
        s["freqs"], s["axes"] = _frequencies(c["rot"]), _axis_of_pairs(c, c["rot"] // 2)
        pos = torch.from_numpy(_positions(c, rng, B, N)).cuda()
        if c["layout"] == "packed":
            s["Q"], s["K"], s["pos"] = values(H, N, d), values(Hkv, N, d), pos[:, 0].contiguous()
            return s
        if c["layout"] == "fused":
            qkv = values(B, N, H + 2 * Hkv, d)
            s["Q"], s["K"] = qkv[:, :, :H].transpose(1, 2), qkv[:, :, H:H + Hkv].transpose(1, 2)
        else:
            s["Q"], s["K"] = values(B, H, N, d), values(B, Hkv, N, d)
        s["pos"] = pos
        return s
    _cache(s, rng, values, seed)
    if own:
        import paper_2109_04312_b200 as mate
        s["cache"] = mate.Cache(s["k"], s["v"], s["row_ids"], s["col_ids"], s["table"], s["lens"], s["prefix"], s["refs"],
                                [0] * c["n_row"] + [1] * (c["H"] - c["n_row"]))
    return s


def _cache(s, rng, values, seed):
    """Pages, tables and ids of the sequences as a server has them, pages in no order, the full pages of a table once for its group;
    what the case's call takes."""
    c = s["c"]
    ps, (tables, tails) = c["page"], _lengths(c, seed)
    full = [L // ps for L in tables]
    lens = np.array([f * ps + n for f, t in zip(full, tails) for n in t], np.int64)
    B, width = len(lens), max(1, int((-(-lens // ps)).max()))
    total = sum(full) + sum(-(-n // ps) for t in tails for n in t)
    n_pages = total + 8
    wide = c["d"] if c["kind"] != "groups" else 8  # (nobody reads keys and values there)
    shape = (1, n_pages, ps, c["Hkv"], wide) if c["slots_first"] else (1, n_pages, c["Hkv"], ps, wide)
    s["k"], s["v"] = values(*shape), values(*shape)
    if c["slots_first"]:
        s["k"], s["v"] = s["k"].transpose(2, 3), s["v"].transpose(2, 3)
    order = rng.permutation(n_pages)
    table, ids = np.full((B, width), -1, np.int32), np.zeros((2, n_pages * ps), np.int32)
    refs, q_ids = np.zeros(n_pages, np.int32), np.zeros((2, B), np.int32)
    at = b = 0
    groups = np.zeros((3, B), np.int32)
    id_rng = np.random.default_rng(0)  # (ids belong to the case: work() counts by them)
    for f, L, tail in zip(full, tables, tails):
        shared, t = order[at:at + f], _ids(c, id_rng, L)
        at += f
        slot = (shared[:, None].astype(np.int64) * ps + np.arange(ps)).reshape(-1)
        ids[:, slot] = t[:, :f * ps]
        refs[shared] = len(tail)
        joined = f > 0 and len(tail) > 1 and f >= max(1, -(-c["min_len"] // ps))
        for i, n in enumerate(tail):
            q_ids[:, b] = _new_ids(c, id_rng, t)
            pages = order[at:at + -(-n // ps)]
            at += len(pages)
            refs[pages] = 1
            table[b, :f], table[b, f:f + len(pages)] = shared, pages
            own_ids = np.full((2, n), _TEXT, np.int32)
            own_ids[:, :L - f * ps] = t[:, f * ps:]
            slot = (pages[:, None].astype(np.int64) * ps + np.arange(ps)).reshape(-1)[:n]
            ids[:, slot] = own_ids
            groups[:, b] = (b - i, len(tail), f * ps) if joined else (b, 1, 0)
            b += 1

    def ints(x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()

    # the sequences' places in the cache are not the batch's order
    seqs = rng.permutation(B)
    place = np.argsort(seqs)
    s["seqs"] = ints(seqs)
    s["table"], s["lens"], s["refs"] = ints(table[place]), ints(lens[place]), ints(refs)
    s["prefix"] = ints(np.minimum(c["prefix"], lens[place]))
    s["row_ids"], s["col_ids"] = ints(ids[0]).view(n_pages, ps), ints(ids[1]).view(n_pages, ps)
    s["groups"] = ints(groups)
    # where the groups begin and what they share, as the program that made them knows it on the host
    # (and pages that the longest of its sequences has of its own)
    s["host"] = [(int(b), int(n), int(sh), max(1, -(-(int(lens[b:b + n].max()) - int(sh)) // ps))) for b, n, sh in zip(*np.unique(groups, axis=1))]
    if c["kind"] == "shared":
        s["Q"] = values(B, c["H"], c["d"])
        s["q_row"], s["q_col"] = ints(q_ids[0]), ints(q_ids[1])
    if c["kind"] == "step":
        s["freqs"], s["axes"] = _frequencies(c["d"]), _axis_of_pairs(c, c["d"] // 2)
        s["K"], s["V"] = (values(B, 1, c["Hkv"], c["d"]).transpose(1, 2) for _ in range(2))
        s["Q"] = values(B, 1, c["H"], c["d"]).transpose(1, 2)
        # (no new token where the last one's page is the table's: shared pages are not written)
        s["counts"] = ints([n > 0 for t in tails for n in t])
        s["new_row"], s["new_col"] = (ints(np.full((B, 1), _TEXT)) for _ in range(2))
        s["pos"] = ints(_positions(c, rng, B, 1))


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    s = state
    c = s["c"]
    if c["kind"] == "axes":
        Q, K = _own_axes(s) if own else _plain_axes(s)
        return {"Q": Q, "K": K}
    if c["kind"] == "step":
        Q = _own_step(s) if own else _plain_step(s)
        return {"Q": Q, "k": s["k"], "v": s["v"], "row_ids": s["row_ids"], "col_ids": s["col_ids"]}
    if c["kind"] == "groups":
        return {"groups": _own_groups(s) if own else _plain_groups(s)}
    O, LSE = _own_shared(s) if own else _plain_shared(s)
    return {"O": O, "LSE": LSE}


# ---- the library's calls

def _own_axes(s):
    import paper_2109_04312_b200 as mate
    c = s["c"]
    return mate.mate_rope_axes(s["Q"], s["pos"], s["freqs"], s["axes"], K=s["K"], interleaved=c["interleaved"], backward=c["backward"])


def _own_step(s):
    import paper_2109_04312_b200 as mate
    return mate.mate_cache_append_axes(s["cache"], s["K"], s["V"], s["freqs"], s["pos"], s["axes"], seqs=s["seqs"], counts=s["counts"],
                                       row_ids=s["new_row"], col_ids=s["new_col"], interleaved=s["c"]["interleaved"], Q=s["Q"])


def _own_groups(s):
    import paper_2109_04312_b200 as mate
    return mate.mate_cache_groups(s["cache"], s["seqs"], min_len=s["c"]["min_len"])


def _own_shared(s):
    import paper_2109_04312_b200 as mate
    return mate.mate_attn_decode_shared(s["cache"], s["Q"], s["q_row"], s["q_col"], s["groups"], seqs=s["seqs"],
                                        max_len=s["c"]["L"] + s["c"]["tail"])


# ---- plain forms

def _turn(x, pos, axes, freqs, interleaved, backward=False):
    """x [..., N, d], pos [A, ..., N] (broadcasting): the first 2 len(freqs) elements rotated, pair i by the positions of axis axes[i]."""
    r = 2 * len(freqs)
    angle = pos.double()[axes].movedim(0, -1) * freqs * (-1 if backward else 1)
    cos, sin = angle.cos().float(), angle.sin().float()
    y = x.float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if interleaved else (y[..., :r // 2], y[..., r // 2:r])
    u, w = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_axes(s):
    c = s["c"]
    pos = s["pos"] if c["layout"] == "packed" else s["pos"][:, :, None]
    return tuple(_turn(s[t], pos, s["axes"], s["freqs"], c["interleaved"], c["backward"]) for t in ("Q", "K"))


def _plain_step(s):
    c = s["c"]
    ps, seqs = c["page"], s["seqs"].long()
    pos = s["pos"][:, :, None]
    K = _turn(s["K"], pos, s["axes"], s["freqs"], c["interleaved"])
    b = torch.nonzero(s["counts"] > 0).view(-1)
    at = s["lens"][seqs[b]].long() - 1
    page, slot = s["table"][seqs[b], at // ps].long(), at % ps
    s["k"][0][page, :, slot], s["v"][0][page, :, slot] = K[b, :, 0], s["V"][b, :, 0]
    s["row_ids"][page, slot], s["col_ids"][page, slot] = s["new_row"][b, 0], s["new_col"][b, 0]
    return _turn(s["Q"], pos, s["axes"], s["freqs"], c["interleaved"]).contiguous()


def _plain_groups(s):
    c = s["c"]
    ps, seqs = c["page"], s["seqs"].long()
    rows, full = s["table"][seqs], s["lens"][seqs].long() // ps
    B, i = len(seqs), torch.arange(rows.shape[1], device="cuda")
    same = (rows[1:] == rows[:-1]) & (rows[1:] >= 0) & (i < torch.minimum(full[1:], full[:-1])[:, None])
    common = torch.cat([full.new_zeros(1), same.long().cumprod(1).sum(1)])
    begins = common < max(1, -(-c["min_len"] // ps))
    group = begins.long().cumsum(0) - 1
    count = full.new_zeros(B).index_add_(0, group, torch.ones_like(group))
    least = full.new_full((B,), 1 << 40).scatter_reduce_(0, group, torch.where(begins, 1 << 40, common), "amin")
    first = count.cumsum(0) - count
    return torch.stack([first[group], count[group], torch.where(count[group] > 1, least[group] * ps, 0)]).int()


def _plain_shared(s):
    c = s["c"]
    H, Hkv, d, ps = c["H"], c["Hkv"], c["d"], c["page"]
    G, view = H // Hkv, (torch.arange(H, device="cuda") >= c["n_row"]).long()
    out, lse = [], []

    def masks(r, col, valid, at, q_row, q_col, prefix):  # of keys [n or 1, j] for n new tokens: [n, Hkv, G, j]
        valid = valid & (r >= 0) & (q_row >= 0)
        always = (at < prefix) | (r == _TEXT) | (q_row == _TEXT)
        by = torch.stack([valid & (always | (r == q_row)), valid & (always | (col == q_col))], 1)
        return by[:, view].view(len(by), Hkv, G, -1)

    for first, n, shared, tail in s["host"]:
        seqs = s["seqs"][first:first + n].long()
        q_row, q_col, prefix = s["q_row"][first:first + n, None], s["q_col"][first:first + n, None], s["prefix"][seqs][:, None]
        q = s["Q"][first:first + n].float().view(n, Hkv, G, d)
        # the own tokens of every sequence
        where = (shared // ps + torch.arange(tail, device="cuda")).clamp(max=s["table"].shape[1] - 1)
        pages = s["table"][seqs][:, where].clamp(min=0).long()
        keys, vals = (s[t][0][pages].permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, d).float() for t in ("k", "v"))
        ids = [s[t][pages].view(n, -1) for t in ("row_ids", "col_ids")]
        at = shared + torch.arange(tail * ps, device="cuda")
        mask = masks(ids[0], ids[1], at < s["lens"][seqs][:, None], at, q_row, q_col, prefix)
        scores = [(torch.matmul(q, keys.transpose(2, 3)) / math.sqrt(d)).masked_fill(~mask, -math.inf)]
        if shared:  # those of the table
            pages = s["table"][seqs[0], :shared // ps].long()
            k0, v0 = (s[t][0][pages].transpose(0, 1).reshape(Hkv, shared, d).float() for t in ("k", "v"))
            ids = [s[t][pages].view(1, -1) for t in ("row_ids", "col_ids")]
            mask = masks(ids[0], ids[1], torch.ones_like(ids[0], dtype=torch.bool), torch.arange(shared, device="cuda"), q_row, q_col, prefix)
            rows = q.transpose(0, 1).reshape(Hkv, n * G, d)
            score = (torch.matmul(rows, k0.transpose(1, 2)) / math.sqrt(d)).view(Hkv, n, G, shared).transpose(0, 1)
            scores.append(score.masked_fill(~mask, -math.inf))
        top = torch.stack([x.amax(-1) for x in scores]).amax(0).clamp(min=torch.finfo(torch.float32).min)[..., None]
        p = [(x - top).exp() for x in scores]
        total = sum(x.sum(-1, keepdim=True) for x in p)
        O = torch.matmul(p[0], vals)
        if shared:
            O = O + torch.matmul(p[1].transpose(0, 1).reshape(Hkv, n * G, shared), v0).view(Hkv, n, G, d).transpose(0, 1)
        out.append((O / total.clamp(min=1e-30)).reshape(n, H, d))
        lse.append((top + total.log()).view(n, H))
    return torch.cat(out).to(s["Q"].dtype), torch.cat(lse)


# ---------------------------------------------------------------------------------------------- in 64 bits

def _exact_turn(c, x, pos, rot, backward=False):
    """Pairs as complex numbers, multiplied by exp(i t); pair after pair."""
    y, axes = x.double().clone(), _axis_of_pairs(c, rot // 2)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + rot // 2)
        t = pos[axes[i]].double() * math.exp(-math.log(10000.0) * 2 * i / rot)
        z = torch.complex(y[..., a], y[..., b]) * torch.complex(t.cos(), (-t if backward else t).sin())
        y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    if c["kind"] == "groups":  # whole numbers
        return None
    s = prepare(c, seed)
    if c["kind"] == "axes":
        pos = s["pos"] if c["layout"] == "packed" else s["pos"][:, :, None]
        return {t: _exact_turn(c, s[t], pos, c["rot"], c["backward"]) for t in ("Q", "K")}
    if c["kind"] == "step":
        k, v, lens, table = s["k"].double(), s["v"].double(), s["lens"].tolist(), s["table"].tolist()
        K = _exact_turn(c, s["K"], s["pos"][:, :, None], c["d"])
        for i, b in enumerate(s["seqs"].tolist()):
            if int(s["counts"][i]):
                page, slot = table[b][(lens[b] - 1) // c["page"]], (lens[b] - 1) % c["page"]
                k[0, page, :, slot], v[0, page, :, slot] = K[i, :, 0], s["V"][i, :, 0].double()
        return {"Q": _exact_turn(c, s["Q"], s["pos"][:, :, None], c["d"]), "k": k, "v": v, "row_ids": None, "col_ids": None}
    # sequence after sequence, each with all of its pages
    B, G = len(s["seqs"]), c["H"] // c["Hkv"]
    O = torch.zeros(B, c["H"], c["d"], dtype=torch.float64, device="cuda")
    LSE = torch.full((B, c["H"]), -math.inf, dtype=torch.float64, device="cuda")
    lens, prefix, q_ids = s["lens"].tolist(), s["prefix"].tolist(), list(zip(s["q_row"].tolist(), s["q_col"].tolist()))
    for i, b in enumerate(s["seqs"].tolist()):
        n = lens[b]
        pages = s["table"][b, :-(-n // c["page"])].long()
        key, val = (s[t][0, pages].transpose(0, 1).reshape(c["Hkv"], -1, c["d"])[:, :n].double() for t in ("k", "v"))
        ids = [s[t][pages].view(-1)[:n] for t in ("row_ids", "col_ids")]
        for view, (lo, hi) in enumerate(((0, c["n_row"]), (c["n_row"], c["H"]))):
            among = (torch.arange(n, device="cuda") < prefix[b]) | (ids[0] == _TEXT) | (ids[view] == q_ids[i][view])
            at = torch.nonzero(among | (q_ids[i][0] == _TEXT)).view(-1)
            for kv in range(c["Hkv"]):
                h0, h1 = max(lo, kv * G), min(hi, kv * G + G)
                if h1 <= h0 or len(at) == 0:
                    continue
                score = s["Q"][i, h0:h1].double() @ key[kv, at].T / math.sqrt(c["d"])
                LSE[i, h0:h1] = torch.logsumexp(score, -1)
                O[i, h0:h1] = torch.softmax(score, -1) @ val[kv, at]
    return {"O": O, "LSE": LSE}
