"""Reading a table one token at a time, as cases that can be timed: rotary positions, the paged key-value cache and the
attention of one new token over it (mate_rope, mate_cache_*, mate_attn_decode), in plain torch operations and through the
library's entry points.

A case's kind is one call, or the few that belong together, of a layer or of a step of a server's loop:
  "rope"     Q and K of a batch rotated, or their gradients turned back
  "append"   the new token of every running sequence: Q and K rotated, K, V and ids into the pages
  "admit"    tables leave and new ones come: their pages freed, handed out again, and filled
  "decode"   the new token of every sequence against what is cached
  "fork"     beams of the last step dropped, new ones made from their parents (all layers of the cache)
  "compact"  a fragmented cache moved together (all layers)
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
_TEXT = 0x7FFFFFFF  # id of text behind the table: attends, and is attended by, everything


def _rope(name, B, N, H, Hkv, d, rot, dtype="bf16", interleaved=False, backward=False, layout="padded", scaled=False):
    return {"name": name, "kind": "rope", "B": B, "N": N, "H": H, "Hkv": Hkv, "d": d, "rot": rot, "dtype": dtype,
            "interleaved": interleaved, "backward": backward, "layout": layout, "scaled": scaled}


def _cached(name, kind, B, L, H, Hkv, d, page, n_row, dtype="bf16", text=0.5, prefix=64, cols=8, ragged=True, layers=1, slots_first=False,
            interleaved=False):
    return {"name": name, "kind": kind, "B": B, "L": L, "H": H, "Hkv": Hkv, "d": d, "page": page, "n_row": n_row, "dtype": dtype,
            "text": text, "prefix": prefix, "cols": cols, "ragged": ragged, "layers": layers, "slots_first": slots_first,
            "interleaved": interleaved}


def listed():
    return [
        # one table in single precision with a head size that is no power of two and half of it rotated (a unit test, a
        # gradient check): nothing but latency
        _rope("rope_one_table_f32", 1, 512, 4, 4, 40, 20, dtype="f32"),
        # a training step on medium tables: Q and K as views of the fused projection's output, per-cell positions
        _rope("rope_train", 4, 2048, 12, 12, 64, 64, layout="fused"),
        # gradients of a packed batch of long documents, grouped heads, frequencies scaled for long contexts
        _rope("rope_long_backward", 1, 32768, 32, 8, 128, 128, interleaved=True, backward=True, layout="packed", scaled=True),
        # one step of a busy server, one layer: a token for each of 64 sequences
        _cached("append_step", "append", 64, 2048, 32, 8, 128, 16, 16),
        # eight tables leave, eight come (one layer's keys and values)
        _cached("admit_tables", "admit", 8, 2048, 12, 12, 64, 16, 6, prefix=128, cols=10),
        # one question about one table at a server: the smallest call
        _cached("decode_one_table", "decode", 1, 512, 12, 12, 64, 16, 6, text=1.0, ragged=False),
        # cells of long tables filled in: the new token attends its row or column and the prefix
        _cached("decode_cells", "decode", 16, 8192, 12, 12, 64, 16, 6, text=0.0, prefix=256),
        # answers written about tables of every length, grouped heads
        _cached("decode_text", "decode", 64, 4096, 32, 8, 128, 16, 16, text=1.0, prefix=128, slots_first=True),
        # one very long document, few heads: the length has to be split
        _cached("decode_long", "decode", 1, 131072, 16, 4, 128, 64, 8, text=1.0, prefix=256, ragged=False),
        # single precision, odd head size and pages, row and column heads in one group, cells and text in one batch
        _cached("decode_f32", "decode", 3, 1500, 6, 2, 48, 24, 2, dtype="f32", cols=5),
        # beam search over eight tables, eight beams each, twelve layers
        _cached("fork_beams", "fork", 8, 2048, 12, 12, 64, 16, 6, layers=12),
        # half of the sequences are gone and their pages lie between the others'
        _cached("compact", "compact", 32, 1024, 12, 12, 64, 16, 6, layers=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges of the listed ones: sizes over their logarithm, odd ones among them."""
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0), work(c)["bytes"])
    while True:
        kind = rng.choice(["rope", "rope", "append", "admit", "decode", "decode", "decode", "fork", "compact"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        Hkv = rng.choice([1, 2, 3, 4, 8, 12])
        H = Hkv * rng.choice([1, 1, 2, 3, 4, 8])
        if kind == "rope":
            d = rng.choice([16, 40, 64, 80, 96, 128])
            rot = rng.choice([d, d, d // 2 // 2 * 2, 8 * rng.randint(1, d // 8)])
            c = _rope("", rng.randint(1, 8), _log_int(rng, 1, 16384), H, Hkv, d, rot, dtype, rng.random() < 0.5, rng.random() < 0.5,
                      rng.choice(["padded", "fused", "packed"]), rng.random() < 0.5)
            if c["layout"] == "packed":
                c["B"] = 1
        else:
            L = _log_int(rng, 1, 65536 if kind == "decode" else 4096)
            c = _cached("", kind, _log_int(rng, 1, 64), L, H, Hkv, rng.choice([16, 48, 64, 64, 128, 128]), rng.choice([1, 8, 16, 16, 24, 64]),
                        rng.randint(0, H), dtype, rng.choice([0.0, 0.5, 1.0]), min(L, _log_int(rng, 1, 256)), rng.randint(2, 30), True,
                        rng.randint(2, 12) if kind in ("fork", "compact") else 1, rng.random() < 0.5, rng.random() < 0.5)
        if work(c)["bytes"] <= most[kind] and _pool_bytes(c) <= 4 << 30:
            del c["name"]
            return c


# ---------------------------------------------------------------------------------------------- sizes

def _lengths(c):
    """Cached tokens of every sequence: they belong to the case; one in ten is still empty."""
    if not c["ragged"]:
        return np.full(c["B"], c["L"], np.int64)
    rng = np.random.default_rng(c["L"] * 1000 + c["B"])
    n = np.exp(rng.uniform(np.log(max(1, c["L"] / 8)), np.log(c["L"] + 0.999), c["B"])).astype(np.int64)
    n[0] = c["L"]
    if c["kind"] in ("decode", "fork") and c["B"] > 1:
        n[1:][rng.random(c["B"] - 1) < 0.1] = 0
    return np.minimum(n, c["L"])


def _beams(c):
    return 8


def _ids(c, rng, n):
    """Row and column ids of the n tokens of a sequence: prefix, table row by row, a little text at the end."""
    P, answer = min(c["prefix"], n), min(n // 16, 32)
    cells = rng.geometric(0.45, size=n + 1).clip(max=16)
    cell = np.repeat(np.arange(len(cells)), cells)[:max(0, n - P - answer)]
    ids = np.full((2, n), _TEXT, np.int32)
    ids[:, :P] = 0
    ids[0, P:P + len(cell)], ids[1, P:P + len(cell)] = cell // c["cols"] + 1, cell % c["cols"] + 1
    return ids, P


def _pool_bytes(c):
    if c["kind"] == "rope":
        return 0
    pages = sum(-(-int(n) // c["page"]) for n in _lengths(c)) + _beams(c) * c["B"] + 8
    return 2 * c["layers"] * pages * c["page"] * c["Hkv"] * c["d"] * _SIZE[c["dtype"]]


def _new_ids(c, rng, ids):
    """The new token's ids: text, or those of a cell of the sequence that is being filled in."""
    table = np.flatnonzero(ids[0] != _TEXT)
    if rng.random() < c["text"] or not len(table):
        return np.full(2, _TEXT, np.int32)
    return ids[:, table[int(rng.integers(len(table)))]]


def _attended(c, ids, q, P):
    """(n,) truth values per view: the keys that the new token attends."""
    n = ids.shape[1]
    always = (np.arange(n) < P) | (ids[0] == _TEXT) | (q[0] == _TEXT)
    return [always | (ids[v] == q[v]) for v in (0, 1)]


def work(case):
    c = case
    size = _SIZE[c["dtype"]]
    if c["kind"] == "rope":
        values = c["B"] * c["N"] * (c["H"] + c["Hkv"]) * c["d"]
        return {"bytes": 2 * values * size + 4 * c["B"] * c["N"], "flops": 3 * values * c["rot"] // c["d"]}
    lens, row = _lengths(c), c["Hkv"] * c["d"] * size
    if c["kind"] == "append":
        return {"bytes": c["B"] * (2 * (c["H"] * c["d"] * size) + 4 * row + 16), "flops": 3 * c["B"] * (c["H"] + c["Hkv"]) * c["d"]}
    if c["kind"] == "admit":
        n = int(lens.sum())
        return {"bytes": n * (4 * row + 16), "flops": 3 * n * c["Hkv"] * c["d"]}
    if c["kind"] == "fork":
        slots = sum(int(n) % c["page"] for n in lens) * _beams(c)
        return {"bytes": slots * 2 * (2 * row * c["layers"] + 8) + 8 * _beams(c) * sum(-(-int(n) // c["page"]) for n in lens) + 64,
                "flops": 0}
    if c["kind"] == "compact":
        live = sum(-(-int(n) // c["page"]) for n in lens[::2])
        total = sum(-(-int(n) // c["page"]) for n in lens)
        moved = live - live * live // max(1, total)  # of the live pages, those that lie behind the first `live`
        return {"bytes": moved * c["page"] * 2 * (2 * row * c["layers"] + 8) + 8 * total, "flops": 0}
    rng = np.random.default_rng(0)
    G, rows, pairs, seen = c["H"] // c["Hkv"], 0, 0, 0
    for n in lens:
        ids, P = _ids(c, rng, int(n))
        q = _new_ids(c, rng, ids)
        by_row, by_col = _attended(c, ids, q, P)
        counts = [int(by_row.sum()), int(by_col.sum())]
        pairs += c["n_row"] * counts[0] + (c["H"] - c["n_row"]) * counts[1]
        for g in range(c["Hkv"]):
            first, last = g * G < c["n_row"], (g + 1) * G - 1 < c["n_row"]
            rows += counts[0] if last else counts[1] if not first else int((by_row | by_col).sum())
        seen += int(n) * (4 if q[0] == _TEXT else 8)
    return {"bytes": rows * 2 * c["d"] * size + seen + c["B"] * c["H"] * (2 * c["d"] * size + 4), "flops": 4 * c["d"] * pairs}


# ---------------------------------------------------------------------------------------------- inputs

def _frequencies(rot, scaled):
    """Radians per position of every pair.  Scaled: eight times the context, high frequencies kept, low ones stretched."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if scaled:
        turns = 8192 * f / (2 * math.pi)  # within the original context
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        f = f * keep + f / 8 * (1 - keep)
    return f


def _cell_positions(rng, n, P):
    """The prefix counts on; every cell of the table starts again."""
    cells = rng.geometric(0.45, size=n + 1).clip(max=16)
    starts = np.cumsum(cells) - cells
    within = np.arange(int(cells.sum())) - np.repeat(starts, cells)
    return np.concatenate([np.arange(min(P, n)), within[:max(0, n - P)]])[:n].astype(np.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = _DTYPES[c["dtype"]]

    def values(*shape):
        return torch.randn(shape, device="cuda", dtype=dt, generator=g) * 0.5

    s = {"c": c}
    if c["kind"] == "rope":
        B, N, H, Hkv, d = (c[k] for k in ("B", "N", "H", "Hkv", "d"))
        s["freqs"] = _frequencies(c["rot"], c["scaled"])
        if c["layout"] == "packed":  # documents, numbered through
            s["Q"], s["K"] = values(H, N, d), values(Hkv, N, d)
            s["pos"] = torch.arange(N, device="cuda", dtype=torch.int32) + int(rng.integers(1000))
            return s
        if c["layout"] == "fused":
            qkv = values(B, N, H + 2 * Hkv, d)
            s["Q"], s["K"] = qkv[:, :, :H].transpose(1, 2), qkv[:, :, H:H + Hkv].transpose(1, 2)
        else:
            s["Q"], s["K"] = values(B, H, N, d), values(B, Hkv, N, d)
        s["pos"] = torch.from_numpy(np.stack([_cell_positions(rng, N, 128) for _ in range(B)])).cuda()
        return s
    _cache(s, rng, values)
    if own:
        import paper_2109_04312_b200 as mate
        s["cache"] = mate.Cache(s["k"], s["v"], s["row_ids"], s["col_ids"], s["table"], s["lens"], s["prefix"], s["refs"],
                                [0] * c["n_row"] + [1] * (c["H"] - c["n_row"]))
    return s


def _cache(s, rng, values):
    """Pages, tables and ids of the sequences as a server has them, pages in no order; what the case's calls take."""
    c = s["c"]
    B, ps, lens = c["B"], c["page"], _lengths(c)
    need = -(-lens // ps)
    beams = _beams(c) if c["kind"] == "fork" else 0
    n_seqs, width = B * (1 + beams), max(1, int(need.max()))
    total = int(need.sum())
    n_pages = total + B * beams + 8
    shape = (c["layers"], n_pages, ps, c["Hkv"], c["d"]) if c["slots_first"] else (c["layers"], n_pages, c["Hkv"], ps, c["d"])
    s["k"], s["v"] = values(*shape), values(*shape)
    if c["slots_first"]:
        s["k"], s["v"] = s["k"].transpose(2, 3), s["v"].transpose(2, 3)
    order = rng.permutation(total if c["kind"] == "compact" else n_pages)[:total]
    table = np.full((n_seqs, width), -1, np.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    ids = np.zeros((2, n_pages * ps), np.int32)
    q_ids, tokens = np.zeros((B, 2), np.int32), []
    for b in range(B):
        n, pages = int(lens[b]), order[at[b]:at[b + 1]]
        table[b, :len(pages)] = pages
        t, _ = _ids(c, rng, n)
        tokens.append(t)
        slots = (pages[:, None].astype(np.int64) * ps + np.arange(ps)).reshape(-1)[:n]
        ids[:, slots] = t
        q_ids[b] = _new_ids(c, rng, t)
    all_lens = np.concatenate([lens, np.zeros(n_seqs - B, np.int64)])
    refs = np.zeros(n_pages, np.int64)
    refs[order] = 1
    if c["kind"] == "compact":  # every other sequence has left
        refs[table[1::2][table[1::2] >= 0]] = 0
        table[1::2], all_lens[1::2] = -1, 0
    prefix = np.minimum(c["prefix"], np.concatenate([lens] + [lens * 0] * beams)) if B else all_lens
    # one buffer, so that a server (and a pass below) can put the whole state back by one copy
    flat = torch.from_numpy(np.concatenate([table.reshape(-1), all_lens, prefix, refs]).astype(np.int32)).cuda()
    s["flat"], s["saved"] = flat, flat.clone()
    parts = torch.split(flat, [n_seqs * width, n_seqs, n_seqs, n_pages])
    s["table"], s["lens"], s["prefix"], s["refs"] = parts[0].view(n_seqs, width), parts[1], parts[2], parts[3]
    dev_ids = torch.from_numpy(ids).cuda()
    s["row_ids"], s["col_ids"] = dev_ids[0].view(n_pages, ps), dev_ids[1].view(n_pages, ps)
    s["seqs"] = torch.from_numpy(rng.permutation(B).astype(np.int32)).cuda()  # the batch's order is not the cache's
    order_b = s["seqs"].cpu().numpy()
    if c["kind"] == "decode":
        s["Q"] = values(B, c["H"], c["d"])
        s["q_row"], s["q_col"] = (torch.from_numpy(np.ascontiguousarray(q_ids[order_b, v])).cuda() for v in (0, 1))
    if c["kind"] in ("append", "admit"):
        n = 1 if c["kind"] == "append" else int(lens.max())
        s["freqs"] = _frequencies(c["d"], False)
        s["K"], s["V"] = (values(B, n, c["Hkv"], c["d"]).transpose(1, 2) for _ in range(2))
        counts = np.minimum(lens, n)[order_b]
        s["counts"] = torch.from_numpy(counts.astype(np.int32)).cuda()
        new = np.zeros((2, B, n), np.int32)
        pos = np.zeros((B, n), np.int32)
        for i, b in enumerate(order_b):
            k = int(counts[i])
            new[:, i, :k] = tokens[b][:, int(lens[b]) - k:]
            pos[i, :k] = _cell_positions(rng, k, c["prefix"]) if n > 1 else int(lens[b]) - 1
        s["new_row"], s["new_col"] = (torch.from_numpy(x).cuda() for x in new)
        s["pos"] = torch.from_numpy(pos).cuda()
        if c["kind"] == "append":
            s["Q"] = values(B, n, c["H"], c["d"]).transpose(1, 2)
    if c["kind"] == "fork":
        s["parents"] = s["seqs"].repeat_interleave(beams)
        s["children"] = torch.arange(B, B * (1 + beams), device="cuda", dtype=torch.int32)


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    s = state
    c = s["c"]
    if c["kind"] == "rope":
        Q, K = _own_rope(s) if own else _plain_rope(s)
        return {"Q": Q, "K": K}
    if c["kind"] == "append":
        Q = _own_append(s) if own else _plain_append(s)
        return {"Q": Q, "k": s["k"], "v": s["v"], "row_ids": s["row_ids"], "col_ids": s["col_ids"]}
    if c["kind"] == "admit":
        if own:
            _own_admit(s)
        else:
            _plain_free(s, s["seqs"])
            _plain_extend(s, s["seqs"], s["counts"])
            _plain_append(s)
        return {k: s[k] for k in ("k", "v", "row_ids", "col_ids", "table", "lens", "refs")}
    if c["kind"] == "decode":
        O, LSE = _own_decode(s) if own else _plain_decode(s)
        return {"O": O, "LSE": LSE}
    if c["kind"] == "fork":
        if own:
            _own_fork(s)
        else:
            _plain_free(s, s["children"])
            _plain_fork(s)
        return {k: s[k] for k in ("k", "v", "row_ids", "col_ids", "table", "lens", "prefix", "refs")}
    s["flat"].copy_(s["saved"])  # the fragmented state again
    n_live = _own_compact(s) if own else _plain_compact(s)
    return {"n_live": n_live, **{k: s[k] for k in ("k", "v", "row_ids", "col_ids", "table", "refs")}}


# ---- the library's calls

def _own_rope(s):
    import paper_2109_04312_b200 as mate
    c = s["c"]
    return mate.mate_rope(s["Q"], s["pos"], s["freqs"], K=s["K"], interleaved=c["interleaved"], backward=c["backward"])


def _own_append(s):
    import paper_2109_04312_b200 as mate
    return mate.mate_cache_append(s["cache"], s["K"], s["V"], s["seqs"], s["counts"], s["new_row"], s["new_col"], freqs=s["freqs"],
                                  positions=s["pos"], interleaved=s["c"]["interleaved"], Q=s.get("Q"))


def _own_admit(s):
    import paper_2109_04312_b200 as mate
    mate.mate_cache_free(s["cache"], s["seqs"])
    granted = mate.mate_cache_extend(s["cache"], s["seqs"], s["counts"])
    mate.mate_cache_append(s["cache"], s["K"], s["V"], s["seqs"], granted, s["new_row"], s["new_col"], freqs=s["freqs"],
                           positions=s["pos"], interleaved=s["c"]["interleaved"])


def _own_decode(s):
    import paper_2109_04312_b200 as mate
    return mate.mate_attn_decode(s["cache"], s["Q"], s["q_row"], s["q_col"], seqs=s["seqs"], max_len=s["c"]["L"])


def _own_fork(s):
    import paper_2109_04312_b200 as mate
    mate.mate_cache_free(s["cache"], s["children"])
    mate.mate_cache_fork(s["cache"], s["parents"], s["children"])


def _own_compact(s):
    import paper_2109_04312_b200 as mate
    return mate.mate_cache_compact(s["cache"])


# ---- plain forms

def _turn(x, pos, freqs, interleaved, backward=False):
    """x [..., N, d] with pos broadcasting to [..., N]: the first 2 len(freqs) elements rotated."""
    r = 2 * len(freqs)
    angle = pos.double()[..., None] * freqs * (-1 if backward else 1)
    cos, sin = angle.cos().float(), angle.sin().float()
    y = x.float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if interleaved else (y[..., :r // 2], y[..., r // 2:r])
    u, w = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_rope(s):
    c = s["c"]
    pos = s["pos"] if c["layout"] == "packed" else s["pos"][:, None]
    return tuple(_turn(s[t], pos, s["freqs"], c["interleaved"], c["backward"]) for t in ("Q", "K"))


def _plain_append(s):
    c = s["c"]
    ps, seqs, counts = c["page"], s["seqs"].long(), s["counts"].long()
    pos = s["pos"][:, None]
    K = _turn(s["K"], pos, s["freqs"], c["interleaved"])
    n = K.shape[2]
    i = torch.arange(n, device="cuda")
    at = (s["lens"][seqs].long() - counts)[:, None] + i
    b, i = torch.nonzero(i < counts[:, None], as_tuple=True)
    at = at[b, i]
    page, slot = s["table"][seqs[b], at // ps].long(), at % ps
    s["k"][0][page, :, slot], s["v"][0][page, :, slot] = K[b, :, i], s["V"][b, :, i]
    s["row_ids"][page, slot], s["col_ids"][page, slot] = s["new_row"][b, i], s["new_col"][b, i]
    return _turn(s["Q"], pos, s["freqs"], c["interleaved"]).contiguous() if "Q" in s else None


def _plain_free(s, seqs):
    seqs = seqs.long()
    pages = s["table"][seqs]
    i = torch.arange(pages.shape[1], device="cuda") * s["c"]["page"]
    held = (i < s["lens"][seqs][:, None]).int()
    s["refs"].index_add_(0, pages.clamp(min=0).view(-1).long(), -held.view(-1))
    s["table"][seqs] = -1
    s["lens"][seqs] = 0


def _plain_extend(s, seqs, counts):
    seqs, ps = seqs.long(), s["c"]["page"]
    before = s["lens"][seqs]
    after = before + counts
    first, last = (before + ps - 1) // ps, (after + ps - 1) // ps
    i = torch.arange(s["table"].shape[1], device="cuda")
    row, col = torch.nonzero((i >= first[:, None]) & (i < last[:, None]), as_tuple=True)
    pages = torch.nonzero(s["refs"] == 0).view(-1)[:len(row)]
    s["table"][seqs[row], col] = pages.int()
    s["refs"][pages] = 1
    s["lens"][seqs] = after


def _plain_fork(s):
    ps, p, ch = s["c"]["page"], s["parents"].long(), s["children"].long()
    lens = s["lens"][p]
    full, part = (lens // ps).long(), lens % ps
    rows = s["table"][p]
    which = torch.nonzero(part > 0).view(-1)
    free = torch.nonzero(s["refs"] == 0).view(-1)[:len(which)]
    src, fill = rows[which, full[which]].long(), part[which]
    i = torch.arange(rows.shape[1], device="cuda")
    shared = (i < full[:, None]).int()
    s["refs"].index_add_(0, rows.clamp(min=0).view(-1).long(), shared.view(-1))
    s["refs"][free] = 1
    rows[which, full[which]] = free.int()
    s["table"][ch], s["lens"][ch], s["prefix"][ch] = rows, lens, s["prefix"][p]
    w, slot = torch.nonzero(torch.arange(ps, device="cuda") < fill[:, None], as_tuple=True)
    s["k"][:, free[w], :, slot] = s["k"][:, src[w], :, slot]
    s["v"][:, free[w], :, slot] = s["v"][:, src[w], :, slot]
    s["row_ids"][free[w], slot] = s["row_ids"][src[w], slot]
    s["col_ids"][free[w], slot] = s["col_ids"][src[w], slot]


def _plain_compact(s):
    live = s["refs"] > 0
    n_live = live.sum()
    i = torch.arange(len(live), device="cuda")
    holes, movers = torch.nonzero(~live & (i < n_live)).view(-1), torch.nonzero(live & (i >= n_live)).view(-1)
    s["k"][:, holes], s["v"][:, holes] = s["k"][:, movers], s["v"][:, movers]
    s["row_ids"][holes], s["col_ids"][holes] = s["row_ids"][movers], s["col_ids"][movers]
    s["refs"][holes] = s["refs"][movers]
    s["refs"][movers] = 0
    to = i.int()
    to[movers] = holes.int()
    t = s["table"]
    t.copy_(torch.where(t >= 0, to[t.clamp(min=0).long()], t))
    return n_live.int()


def _plain_decode(s):
    c = s["c"]
    B, H, Hkv, d, ps = (c[k] for k in ("B", "H", "Hkv", "d", "page"))
    G, seqs = H // Hkv, s["seqs"].long()
    pages = s["table"][seqs].clamp(min=0).long()
    keys, vals = (s[t][0][pages].permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d).float() for t in ("k", "v"))
    ids = [s[t][pages].view(B, -1) for t in ("row_ids", "col_ids")]
    i = torch.arange(keys.shape[2], device="cuda")
    q_row, q_col = s["q_row"][:, None], s["q_col"][:, None]
    valid = (i < s["lens"][seqs][:, None]) & (ids[0] >= 0) & (q_row >= 0)
    always = (i < s["prefix"][seqs][:, None]) | (ids[0] == _TEXT) | (q_row == _TEXT)
    by_view = torch.stack([valid & (always | (ids[0] == q_row)), valid & (always | (ids[1] == q_col))], 1)
    view = (torch.arange(H, device="cuda") >= c["n_row"]).long()
    mask = by_view[:, view].view(B, Hkv, G, -1)
    score = torch.matmul(s["Q"].float().view(B, Hkv, G, d), keys.transpose(2, 3)) / math.sqrt(d)
    score = score.masked_fill(~mask, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = (score - top).exp()
    total = p.sum(-1, keepdim=True)
    O = torch.matmul(p, vals) / total.clamp(min=1e-30)
    return O.view(B, H, d).to(s["Q"].dtype), (top + total.log()).view(B, H)


# ---------------------------------------------------------------------------------------------- in 64 bits

def _exact_turn(c, x, pos, rot, scaled, backward):
    """Pairs as complex numbers, multiplied by exp(i t)."""
    j = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    f = torch.exp(-math.log(10000.0) * 2 * j / rot)
    if scaled:
        wave = 2 * math.pi / f
        mix = (8192 / wave - 1) / 3
        f = torch.where(wave < 2048, f, torch.where(wave > 8192, f / 8, (1 - mix) * f / 8 + mix * f))
    t = pos.double()[..., None] * f
    unit = torch.complex(t.cos(), (-t if backward else t).sin())
    y = x.double().clone()
    if c["interleaved"]:
        z = torch.complex(y[..., 0:rot:2], y[..., 1:rot:2]) * unit
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    else:
        z = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * unit
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def exact(case, seed):
    c = case
    if c["kind"] in ("fork", "compact"):  # nothing is computed but whole numbers and places
        return None
    s = prepare(c, seed)
    if c["kind"] == "rope":
        pos = s["pos"] if c["layout"] == "packed" else s["pos"][:, None]
        return {t: _exact_turn(c, s[t], pos, c["rot"], c["scaled"], c["backward"]) for t in ("Q", "K")}
    if c["kind"] == "append":
        k, v, lens, table = s["k"].double(), s["v"].double(), s["lens"].tolist(), s["table"].tolist()
        K = _exact_turn(c, s["K"], s["pos"][:, None], c["d"], False, False)
        for i, b in enumerate(s["seqs"].tolist()):
            if int(s["counts"][i]) == 0:
                continue
            at = lens[b] - 1
            page, slot = table[b][at // c["page"]], at % c["page"]
            k[0, page, :, slot], v[0, page, :, slot] = K[i, :, 0], s["V"][i, :, 0].double()
        return {"Q": _exact_turn(c, s["Q"], s["pos"][:, None], c["d"], False, False), "k": k, "v": v, "row_ids": None, "col_ids": None}
    if c["kind"] == "admit":  # free and hand out again: the lowest pages that the other sequences do not hold, in the batch's order
        k, v, counts = s["k"].double(), s["v"].double(), s["counts"].tolist()
        K = _exact_turn(c, s["K"], s["pos"][:, None], c["d"], False, False)
        held, page = set(), 0  # (all sequences are replaced: none is held by another)
        for i in range(c["B"]):
            for first in range(0, counts[i], c["page"]):
                while page in held:
                    page += 1
                n = min(c["page"], counts[i] - first)
                k[0, page, :, :n], v[0, page, :, :n] = K[i, :, first:first + n], s["V"][i, :, first:first + n].double()
                page += 1
        return {"k": k, "v": v, "row_ids": None, "col_ids": None, "table": None, "lens": None, "refs": None}
    O = torch.zeros(c["B"], c["H"], c["d"], dtype=torch.float64, device="cuda")
    LSE = torch.full((c["B"], c["H"]), -math.inf, dtype=torch.float64, device="cuda")
    G = c["H"] // c["Hkv"]
    lens, prefix, q_ids = s["lens"].tolist(), s["prefix"].tolist(), list(zip(s["q_row"].tolist(), s["q_col"].tolist()))
    for i, b in enumerate(s["seqs"].tolist()):
        n = lens[b]
        pages = s["table"][b, :-(-n // c["page"])].long()
        key, val = (s[t][0, pages].transpose(0, 1).reshape(c["Hkv"], -1, c["d"])[:, :n].double() for t in ("k", "v"))
        ids = [s[t][pages].view(-1)[:n] for t in ("row_ids", "col_ids")]
        for view, (lo, hi) in enumerate(((0, c["n_row"]), (c["n_row"], c["H"]))):
            among = (torch.arange(n, device="cuda") < prefix[b]) | (ids[0] == _TEXT) | (ids[view] == q_ids[i][view])
            at = torch.nonzero(among | (q_ids[i][0] == _TEXT)).view(-1)
            if hi == lo or len(at) == 0:
                continue
            kv = torch.arange(lo, hi, device="cuda") // G
            score = torch.einsum("hd,hjd->hj", s["Q"][i, lo:hi].double(), key[kv][:, at]) / math.sqrt(c["d"])
            LSE[i, lo:hi] = torch.logsumexp(score, -1)
            O[i, lo:hi] = torch.einsum("hj,hjd->hd", torch.softmax(score, -1), val[kv][:, at])
    return {"O": O, "LSE": LSE}
