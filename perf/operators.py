"""The operators around a ragged, paged batch, with inputs for them and their plain forms.

A serving program that runs decoder layers of its own on this library's caches makes four calls besides the matrix
products: once a step it turns the requests' lengths into block tables, slots and key ranges (map); in every layer it
normalises queries and keys head by head, rotates them and writes keys and values into their slots (norm), and attends
over the cache with capped or biased scores under a document or prefix mask (attention); and when an agent takes over
another's segment it moves the cached rows to their new slots and positions (move).

A case is a dict of plain numbers and texts; `listed` gives the fixed ones, `draw` others of the same ranges.  `run`
computes a case in plain torch operations, or, where `own` is set, with the library's kernels.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False


def _rc():
    from paper_2603_13289_amd import binding
    return binding


def _case(name, op, **kw):
    return dict({"name": name, "op": op, "lens": 1}, **kw)


# head layouts of the repository's workloads: queries, keys, head size
_HEADS = {"tiny": (4, 2, 64), "mistral7b": (32, 8, 128), "qwen32b": (40, 8, 128), "small": (8, 2, 128)}


def listed():
    return [
        # One token for each of 32 running sequences: the most requests one call of the library takes.
        _case("map_decode_32", "map", n_seq=32, new_lo=1, new_hi=1, cached_lo=64, cached_hi=9000, page=16, docs=0,
              prefix=False, spare=0.1),
        # Packed prompts of many documents, some with a two-way prefix: a large scoring batch.
        _case("map_packed_256", "map", n_seq=256, new_lo=200, new_hi=1900, cached_lo=0, cached_hi=300, page=16, docs=6,
              prefix=True, spare=0.0),
        # One token for each of 16 sequences: bf16 projections, interleaved pairs.
        _case("norm_decode_16", "norm", heads="mistral7b", dtype="bf16", qkv="bf16", rows=16, page=16, layout="interleaved",
              rotary=128, scaling="plain", gains=True, keep=False, far=9000),
        # The live rows of the dense layer of the 4k reuse: float projections, long-context frequencies.
        _case("norm_dense_5120", "norm", heads="mistral7b", dtype="bf16", qkv="f32", rows=5120, page=0, layout="half",
              rotary=128, scaling="turns", gains=True, keep=True, far=5120),
        # Rows of the float decoder, half of each head rotated.
        _case("norm_float_384", "norm", heads="tiny", dtype="f32", qkv="f32", rows=384, page=16, layout="half", rotary=32,
              scaling="linear", gains=True, keep=False, far=384),
        # A short hand-off of rotated keys between two agents' pages.
        _case("move_short_300", "move", heads="mistral7b", dtype="bf16", rows=300, page=16, layout="half", rotary=128,
              scaling="pairs", rotated=True, far=2000),
        # A 32k segment of keys stored before rotation, part of each head rotated.
        _case("move_long_32768", "move", heads="qwen32b", dtype="bf16", rows=32768, page=16, layout="interleaved", rotary=64,
              scaling="plain", rotated=False, far=36864),
        # One new token behind 5120 cached rows, scores capped.
        _case("attn_decode_one", "attention", heads="mistral7b", dtype="bf16", n_seq=1, new_lo=1, new_hi=1, cached_lo=5120,
              cached_hi=5120, page=16, cap=50.0, bias=False, docs=0, prefix=False, spread=False),
        # One new token for each of 16 ragged sequences, scores biased by distance.
        _case("attn_decode_16", "attention", heads="mistral7b", dtype="bf16", n_seq=16, new_lo=1, new_hi=1, cached_lo=1280,
              cached_hi=10240, page=16, cap=0.0, bias=True, docs=0, prefix=False, spread=False),
        # Packed prompts: documents that do not see each other, a two-way prefix in front.
        _case("attn_documents", "attention", heads="qwen32b", dtype="bf16", n_seq=4, new_lo=900, new_hi=2100, cached_lo=0,
              cached_hi=500, page=16, cap=30.0, bias=False, docs=3, prefix=True, spread=False),
        # The sparse layers of the 16k reuse: selected rows all over a long context, scores capped.
        _case("attn_selected_16k", "attention", heads="mistral7b", dtype="bf16", n_seq=1, new_lo=3687, new_hi=3687,
              cached_lo=14745, cached_hi=14745, page=0, cap=50.0, bias=False, docs=0, prefix=False, spread=True),
        # The float decoder's prompt, capped and biased.
        _case("attn_float_384", "attention", heads="tiny", dtype="f32", n_seq=1, new_lo=384, new_hi=384, cached_lo=0,
              cached_hi=0, page=16, cap=20.0, bias=True, docs=0, prefix=False, spread=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["op"]] = max(most.get(c["op"], 0.0), w["bytes"] / 4e12 + w["flops"] / 4e14)
    while True:
        op = rng.choice(["map", "norm", "move", "attention", "attention"])
        heads = rng.choice(["tiny", "small", "mistral7b", "mistral7b", "qwen32b"])
        dtype = "f32" if heads == "tiny" else "bf16"
        dh = _HEADS[heads][2]
        page = rng.choice([0, 16, 16, 24, 64])
        c = {"op": op, "lens": rng.randrange(1 << 20)}
        rot = dict(heads=heads, dtype=dtype, page=page, layout=rng.choice(["half", "interleaved"]),
                   rotary=rng.choice([dh, dh, dh // 2, dh // 4]), scaling=rng.choice(["plain", "linear", "turns", "pairs"]))
        if op == "map":
            new = rng.choice([1, _log_uniform(rng, 2, 1900)])
            cached = _log_uniform(rng, 1, 9000)
            c.update(n_seq=_log_uniform(rng, 1, 256), new_lo=1 if new == 1 else new // 9, new_hi=new,
                     cached_lo=cached // 7, cached_hi=cached, page=rng.choice([16, 16, 24, 64]), docs=rng.choice([0, 0, 3, 9]),
                     prefix=rng.random() < 0.4, spare=rng.choice([0.0, 0.1, 0.3]))
        elif op == "norm":
            n = _log_uniform(rng, 1, 5120)
            c.update(rot, rows=n, qkv=rng.choice(["f32", dtype]), gains=rng.random() < 0.8, keep=rng.random() < 0.4,
                     far=n + _log_uniform(rng, 1, 40000))
        elif op == "move":
            n = _log_uniform(rng, 1, 32768)
            c.update(rot, rows=n, rotated=rng.random() < 0.5, far=n + _log_uniform(rng, 1, 40000))
        else:
            if rng.random() < 0.5:
                top = 700 if dtype == "f32" else 10240
                cached = _log_uniform(rng, 1, top)
                c.update(n_seq=rng.choice([1, 1, 3, 8, 16, 32]), new_lo=1, new_hi=1, cached_lo=cached // 8, cached_hi=cached,
                         docs=0, prefix=False, spread=False)
            else:
                new = _log_uniform(rng, 2, 500 if dtype == "f32" else 3000)
                cached = rng.choice([0, _log_uniform(rng, 1, 700 if dtype == "f32" else 9000)])
                docs = rng.choice([0, 0, 2, 5])
                c.update(n_seq=rng.choice([1, 1, 2, 5]), new_lo=max(1, new // 4), new_hi=new, cached_lo=cached // 3,
                         cached_hi=cached, docs=docs, prefix=rng.random() < 0.3, spread=docs == 0 and rng.random() < 0.3)
            c.update(heads=heads, dtype=dtype, page=page, cap=rng.choice([0.0, 20.0, 50.0]), bias=rng.random() < 0.4)
        w = work(c)
        if w["bytes"] / 4e12 + w["flops"] / 4e14 <= most[op]:
            return c


# ------------------------------------------------------------------ sizes of a case
def _range_of(case, what, salt):
    rng = random.Random(case["lens"] * 8 + salt)
    return [rng.randint(case[what + "_lo"], case[what + "_hi"]) for _ in range(case["n_seq"])]


def _batch(case):
    """Per sequence: rows cached, new rows, prefix length (0: none), first positions of its documents ([]: one)."""
    rng = random.Random(case["lens"] * 8 + 3)
    out = []
    for c, n in zip(_range_of(case, "cached", 1), _range_of(case, "new", 2)):
        docs = sorted(rng.sample(range(1, c + n), min(case["docs"], c + n - 1))) if case["docs"] and c + n > 1 else []
        out.append((c, n, rng.randint(0, (c + n) // 2) if case["prefix"] else 0, [0] + docs if docs else []))
    return out


def _positions(case, c, n, salt):
    """Positions of a sequence's rows: the last n, or, spread, some of all c + n of them."""
    if not case.get("spread"):
        return list(range(c, c + n))
    return sorted(random.Random(case["lens"] * 64 + salt).sample(range(c + n), n))


def _ranges(case):
    """Per sequence: (length, [(position, first key, last key)] of its rows)."""
    out = []
    for s, (c, n, prefix, docs) in enumerate(_batch(case)):
        at = 0
        rows = []
        for p in _positions(case, c, n, s):
            while at + 1 < len(docs) and docs[at + 1] <= p:
                at += 1
            first = docs[at] if docs else 0
            end = docs[at + 1] if at + 1 < len(docs) else c + n
            rows.append((p, first, min(max(p, prefix - 1), end - 1)))
        out.append((c + n, rows))
    return out


def work(case):
    """Each input read once and each output written once; for attention every key row that some row of its sequence
    sees, and four operations for each element of a head and visible (query, key) pair."""
    op = case["op"]
    if op == "map":
        rows = sum(n for _, n, _, _ in _batch(case))
        blocks = sum(-(-(c + n) // case["page"]) - -(-c // case["page"]) for c, n, _, _ in _batch(case))
        return {"bytes": float(case["n_seq"] * 20 + rows * 20 + blocks * 8), "flops": float(rows * 8)}
    hq, hkv, dh = _HEADS[case["heads"]]
    es = 2 if case["dtype"] == "bf16" else 4
    if op == "norm":
        n = case["rows"]
        in_es = 2 if case["qkv"] == "bf16" else 4
        nbytes = n * dh * ((hq + 2 * hkv) * in_es + (hq + 2 * hkv + (hkv if case["keep"] else 0)) * es) + 8 * n
        return {"bytes": float(nbytes), "flops": float(n * (hq + hkv) * (4 * dh + 3 * case["rotary"]))}
    if op == "move":
        n = case["rows"]
        return {"bytes": float(n * hkv * dh * 4 * es + n * (16 if case["rotated"] else 12)),
                "flops": float(n * hkv * 3 * case["rotary"])}
    pairs, rows, keys = 0, 0, 0
    for length, r in _ranges(case):
        pairs += sum(hi - lo + 1 for _, lo, hi in r)
        rows += len(r)
        keys += max(hi for _, _, hi in r) - min(lo for _, lo, _ in r) + 1
    return {"bytes": float(2 * rows * hq * dh * es + 2 * keys * hkv * dh * es), "flops": 4.0 * dh * hq * pairs}


# ------------------------------------------------------------------ inputs
class _Inputs:
    def __init__(self, case, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.rng = random.Random(seed)
        self.td = torch.bfloat16 if case.get("dtype") == "bf16" else torch.float32
        self.case = case

    def normal(self, *size, dtype=None, mean=0.0, std=1.0):
        return torch.empty(size, dtype=dtype or self.td, device="cuda").normal_(mean, std, generator=self.g)

    def ints(self, values):
        return torch.tensor(list(values), dtype=torch.int32, device="cuda")

    def blocks(self, lens, page):
        """(block table as a list, number of blocks, block size): pages in random order."""
        if not page:
            return [[i] for i in range(len(lens))], len(lens), max(lens)
        need = [-(-n // page) for n in lens]
        ids = list(range(sum(need) + 3))
        self.rng.shuffle(ids)
        table, at = [], 0
        for n in need:
            table.append(ids[at:at + n] + [-1] * (max(need) - n))
            at += n
        return table, len(ids), page

    def pool(self, n_blocks, size, std=1.0):
        _, hkv, dh = _HEADS[self.case["heads"]]
        return self.normal(n_blocks, hkv, size, dh, std=std)


def _rotary_numbers(case):
    """What a program knows of its rotation: base, scaling factor, trained length, amplitude."""
    n = {"base": 5.0e5, "factor": 1.0, "trained": 8192, "slow": 1.0, "fast": 4.0, "amplitude": 1.0}
    if case["scaling"] == "linear":
        n.update(factor=4.0)
    elif case["scaling"] == "turns":
        n.update(factor=8.0)
    elif case["scaling"] == "pairs":
        n.update(factor=4.0, fast=32.0, amplitude=0.1 * math.log(4.0) + 1.0)
    return n


def _rotary_plan(case):
    rc = _rc()
    n = _rotary_numbers(case)
    layout = {"half": rc.RC_ROTARY_HALF, "interleaved": rc.RC_ROTARY_INTERLEAVED}[case["layout"]]
    scaling = {"plain": rc.RC_ROTARY_PLAIN, "linear": rc.RC_ROTARY_LINEAR, "turns": rc.RC_ROTARY_BY_TURNS,
               "pairs": rc.RC_ROTARY_BY_PAIR}[case["scaling"]]
    return rc.rc_rotary_init(layout, case["rotary"], n["base"], scaling=scaling, factor=n["factor"],
                             trained_len=n["trained"], slow_turns=n["slow"], fast_turns=n["fast"],
                             amplitude=n["amplitude"])


def _layer(s, k, v, size, table):
    rc = _rc()
    s.keep = getattr(s, "keep", [])
    kv = rc.PagedKV.from_pools([k], [v], table, rc.RC_BF16 if s.case["dtype"] == "bf16" else rc.RC_F32)
    s.keep.append(kv)
    return kv.layer(0)


def prepare(case, seed):
    s = {"map": _prepare_map, "norm": _prepare_norm, "move": _prepare_move, "attention": _prepare_attention}[case["op"]](case, seed)
    return s


def _prepare_map(case, seed):
    """Requests' lengths, the tables of what they hold already, and a shuffled list of free blocks."""
    i = _Inputs(case, seed)
    b = _batch(case)
    page = case["page"]
    have = [-(-c // page) for c, _, _, _ in b]
    need = [-(-(c + n) // page) for c, n, _, _ in b]
    spare = int(case["spare"] * sum(need)) + 3
    ids = list(range(sum(need) + spare))
    i.rng.shuffle(ids)
    width = max(need) + 2
    table, at = [], 0
    for h in have:
        table.append(ids[at:at + h] + [-1] * (width - h))
        at += h
    rows = sum(n for _, n, _, _ in b)
    s = SimpleNamespace(case=case, page=page, n_blocks=len(ids), rows=rows + 5, n_seq=len(b))
    s.n_cached, s.n_new = i.ints(c for c, _, _, _ in b), i.ints(n for _, n, _, _ in b)
    s.table = i.ints(x for r in table for x in r).view(len(b), width)
    s.free = i.ints(ids[at:])
    s.free_first = i.ints([0])
    s.prefix = i.ints(p for _, _, p, _ in b) if case["prefix"] else None
    s.doc_start = s.doc_first = None
    if case["docs"]:
        starts = [0]
        for _, _, _, d in b:
            starts.append(starts[-1] + len(d))
        s.doc_start, s.doc_first = i.ints(starts), i.ints([p for _, _, _, d in b for p in d] + [0])
    new = lambda n: torch.full((n,), -7, dtype=torch.int32, device="cuda")
    s.out = {"row_start": new(len(b) + 1), "row_seq": new(s.rows), "row_pos": new(s.rows), "row_slot": new(s.rows),
             "row_lo": new(s.rows), "row_hi": new(s.rows), "kv_len": new(len(b)), "counts": new(3)}
    if own:
        s.own_rows = _rc().BatchRows(**s.out)
    return s


def _slots(table, size, seqs, positions):
    return [table[q][p // size] * size + p % size for q, p in zip(seqs, positions)]


def _prepare_norm(case, seed):
    """A layer's projections of live rows anywhere in one sequence; gains near 1 as trained ones are."""
    i = _Inputs(case, seed)
    hq, hkv, dh = _HEADS[case["heads"]]
    n, far = case["rows"], case["far"]
    table, n_blocks, size = i.blocks([far], case["page"])
    pos = sorted(i.rng.sample(range(far), n))
    s = SimpleNamespace(case=case, n=n, size=size)
    s.qkv = i.normal(n, (hq + 2 * hkv) * dh, dtype=torch.float32 if case["qkv"] == "f32" else torch.bfloat16)
    s.g_q, s.g_k = (i.normal(dh, mean=1.0, std=0.1), i.normal(dh, mean=1.0, std=0.1)) if case["gains"] else (None, None)
    s.eps = 1e-5
    s.pos, s.slot = i.ints(pos), i.ints(_slots(table, size, [0] * n, pos))
    s.k, s.v = i.pool(n_blocks, size), i.pool(n_blocks, size)
    s.k_pre = i.pool(n_blocks, size) if case["keep"] else None
    s.q = torch.zeros((n, hq, dh), dtype=i.td, device="cuda")
    if own:
        s.rotary = _rotary_plan(case)
        s.layer = _layer(s, s.k, s.v, size, i.ints(x for r in table for x in r).view(len(table), -1))
    return s


def _prepare_move(case, seed):
    """A segment of one agent's cache and its place in another's."""
    i = _Inputs(case, seed)
    n, far = case["rows"], case["far"]
    old0, new0 = i.rng.randrange(far - n + 1), i.rng.randrange(far - n + 1)
    s = SimpleNamespace(case=case, n=n)
    t_src, b_src, size = i.blocks([far], case["page"])
    t_dst, b_dst, _ = i.blocks([far], case["page"])
    old, new = range(old0, old0 + n), range(new0, new0 + n)
    s.src_slot, s.dst_slot = i.ints(_slots(t_src, size, [0] * n, old)), i.ints(_slots(t_dst, size, [0] * n, new))
    s.old, s.new = i.ints(old) if case["rotated"] else None, i.ints(new)
    s.size = size
    s.k_src, s.v_src = i.pool(b_src, size), i.pool(b_src, size)
    s.k, s.v = i.pool(b_dst, size), i.pool(b_dst, size)
    if own:
        s.rotary = _rotary_plan(case)
        s.src = _layer(s, s.k_src, s.v_src, size, i.ints(x for r in t_src for x in r).view(1, -1))
        s.dst = _layer(s, s.k, s.v, size, i.ints(x for r in t_dst for x in r).view(1, -1))
    return s


def _prepare_attention(case, seed):
    """Queries and keys as norms leave them (scores of a few units), values N(0, 1); slopes a geometric series."""
    i = _Inputs(case, seed)
    hq, hkv, dh = _HEADS[case["heads"]]
    seqs = _ranges(case)
    table, n_blocks, size = i.blocks([length for length, _ in seqs], case["page"])
    rows = [r for _, rs in seqs for r in rs]
    starts = [0]
    for _, rs in seqs:
        starts.append(starts[-1] + len(rs))
    s = SimpleNamespace(case=case, size=size, lens=[length for length, _ in seqs], starts=starts)
    s.k, s.v = i.pool(n_blocks, size, std=1.5), i.pool(n_blocks, size)
    s.table = i.ints(x for r in table for x in r).view(len(table), -1)
    s.q = i.normal(len(rows), hq, dh, std=1.5)
    s.row_start = i.ints(starts)
    s.pos, s.lo, s.hi = (i.ints(r[j] for r in rows) for j in range(3))
    s.cap = case["cap"]
    s.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], device="cuda") if case["bias"] else None
    if own:
        rc = _rc()
        s.out = torch.zeros_like(s.q)
        s.layer = _layer(s, s.k, s.v, size, s.table)
        s.plan = rc.MaskedAttention(s.row_start, s.pos, n_rows=len(rows), max_rows_per_seq=max(len(r) for _, r in seqs),
                                    max_len=max(s.lens), row_lo=s.lo, row_hi=s.hi, cap=s.cap, slopes=s.slopes)
        s.ws = rc.alloc_workspace(rc.rc_masked_attention_workspace_bytes(s.plan, hq, s.layer))
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    return {"map": _run_map, "norm": _run_norm, "move": _run_move, "attention": _run_attention}[state.case["op"]](state)


def _run_map(s):
    if own:
        _rc().rc_batch_map(s.n_cached, s.n_new, s.table, s.page, s.n_blocks, s.free, s.own_rows, free_first=s.free_first,
                           prefix_len=s.prefix, doc_start=s.doc_start, doc_first=s.doc_first)
        return dict(s.out, table=s.table)
    page, o = s.page, s.out
    total = s.n_cached + s.n_new
    have, need = (s.n_cached + page - 1) // page, (total + page - 1) // page
    start = torch.zeros_like(o["row_start"])
    start[1:] = torch.cumsum(s.n_new, 0)
    taken = torch.cumsum(need - have, 0)
    block0 = taken - (need - have) + s.free_first            # a sequence's first entry of the free list
    col = torch.arange(s.table.shape[1], device="cuda")[None]
    fresh = (col >= have[:, None]) & (col < need[:, None])
    entry = (block0[:, None] + col - have[:, None]).clamp(0, s.free.numel() - 1)
    s.table.copy_(torch.where(fresh, s.free[entry.long()], s.table))
    r = torch.arange(s.rows, device="cuda")
    live = r < start[-1]
    seq = (r[:, None] >= start[None, 1:]).sum(1).clamp(max=s.n_seq - 1)
    pos = s.n_cached[seq] + r - start[seq]
    width = s.table.shape[1]
    slot = s.table[seq, (pos // page).clamp(max=width - 1)] * page + pos % page
    lo, end = torch.zeros_like(pos), total[seq].long()
    if s.doc_start is not None:
        first, last = s.doc_start[seq].long(), s.doc_start[seq + 1].long()
        for j in range(s.case["docs"] + 1):
            at = (first + j).clamp(max=s.doc_first.numel() - 1)
            p = s.doc_first[at].long()
            inside = first + j < last
            lo = torch.where(inside & (p <= pos), p, lo)
            end = torch.where(inside & (p > pos), torch.minimum(end, p), end)
    hi = pos if s.prefix is None else torch.maximum(pos, s.prefix[seq] - 1)
    hi = torch.minimum(hi, end - 1)
    for name, x in (("row_seq", seq), ("row_pos", pos), ("row_slot", slot), ("row_lo", lo), ("row_hi", hi)):
        o[name].copy_(torch.where(live, x.int(), o[name]))
    o["row_start"].copy_(start)
    o["kv_len"].copy_(total)
    o["counts"].copy_(torch.stack([start[-1], s.free_first[0] + taken[-1].int(), torch.zeros_like(start[-1])]))
    return dict(o, table=s.table)


def _frequencies(case):
    """Angle per position of each rotary pair, 64 bits."""
    n, r = _rotary_numbers(case), case["rotary"]
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    f = n["base"] ** (-2.0 * i / r)
    if case["scaling"] == "plain":
        return f
    if case["scaling"] == "linear":
        return f / n["factor"]
    if case["scaling"] == "turns":      # kept where a pair turns often over the trained length, slowed down where it does not
        keep = ((n["trained"] * f / (2 * math.pi) - n["slow"]) / (n["fast"] - n["slow"])).clamp(0, 1)
    else:
        pair = lambda turns: r * math.log(n["trained"] / (turns * 2 * math.pi)) / (2 * math.log(n["base"]))
        a, b = max(math.floor(pair(n["fast"])), 0), min(math.ceil(pair(n["slow"])), r // 2 - 1)
        keep = 1 - ((i - a) / max(b - a, 0.001)).clamp(0, 1)
    return f * keep + f / n["factor"] * (1 - keep)


def _pairs(case, x):
    """The two halves of every rotary pair, as views of x."""
    r = case["rotary"]
    return (x[..., :r // 2], x[..., r // 2:r]) if case["layout"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])


def _rotate(case, x, pos, amplitude):
    angle = pos.double()[:, None, None] * _frequencies(case)
    c, s = (amplitude * torch.cos(angle)).to(x.dtype), (amplitude * torch.sin(angle)).to(x.dtype)
    a, b = _pairs(case, x)
    y = x.clone()
    ya, yb = _pairs(case, y)
    ya.copy_(a * c - b * s)
    yb.copy_(b * c + a * s)
    return y


def _put(pool, size, slot, rows):
    pool[slot.long() // size, :, slot.long() % size] = rows.to(pool.dtype)


def _run_norm(s):
    case = s.case
    if own:
        _rc().rc_norm_rotary_rows(s.qkv, s.n, _HEADS[case["heads"]][0], s.rotary, s.pos, s.slot, s.layer, s.q, g_q=s.g_q,
                                  g_k=s.g_k, eps=s.eps, k_pre=s.k_pre)
        return {"q": s.q, "k": s.k, "v": s.v, "k_pre": s.k_pre}
    hq, hkv, dh = _HEADS[case["heads"]]
    x = s.qkv.float().view(s.n, hq + 2 * hkv, dh)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if case["gains"]:
        q = q / torch.sqrt((q * q).mean(-1, keepdim=True) + s.eps) * s.g_q.float()
        k = k / torch.sqrt((k * k).mean(-1, keepdim=True) + s.eps) * s.g_k.float()
    amplitude = _rotary_numbers(case)["amplitude"]
    s.q.copy_(_rotate(case, q, s.pos, amplitude))
    _put(s.k, s.size, s.slot, _rotate(case, k, s.pos, amplitude))
    _put(s.v, s.size, s.slot, v)
    if s.k_pre is not None:
        _put(s.k_pre, s.size, s.slot, k)
    return {"q": s.q, "k": s.k, "v": s.v, "k_pre": s.k_pre}


def _take(pool, size, slot):
    return pool[slot.long() // size, :, slot.long() % size]


def _run_move(s):
    case = s.case
    if own:
        _rc().rc_rotary_move(s.src, s.src_slot, s.dst, s.dst_slot, s.n, s.rotary, s.new, old_pos=s.old)
        return {"k": s.k, "v": s.v}
    k = _take(s.k_src, s.size, s.src_slot).float()
    if s.old is None:
        k = _rotate(case, k, s.new, _rotary_numbers(case)["amplitude"])
    else:
        k = _rotate(case, k, s.new - s.old, 1.0)
    _put(s.k, s.size, s.dst_slot, k)
    _put(s.v, s.size, s.dst_slot, _take(s.v_src, s.size, s.src_slot))
    return {"k": s.k, "v": s.v}


def _run_attention(s):
    hq, hkv, dh = _HEADS[s.case["heads"]]
    if own:
        rc = _rc()
        rc.rc_masked_attention(s.q, s.plan, hq, s.layer, s.out, s.ws)
        return s.out
    out = torch.zeros_like(s.q)
    for b, length in enumerate(s.lens):
        at = torch.arange(length, device="cuda")
        block, slot = s.table[b][at // s.size].long(), at % s.size
        k = s.k[block, :, slot].float().permute(1, 2, 0).contiguous()      # [heads][dh][keys]
        v = s.v[block, :, slot].float().transpose(0, 1).contiguous()       # [heads][keys][dh]
        step = max(1, (1 << 28) // (hq * length))
        for r0 in range(s.starts[b], s.starts[b + 1], step):
            r1 = min(r0 + step, s.starts[b + 1])
            q = s.q[r0:r1].float().view(r1 - r0, hkv, hq // hkv, dh).permute(1, 2, 0, 3).reshape(hkv, -1, dh)
            x = torch.matmul(q, k).view(hq, r1 - r0, length) / math.sqrt(dh)
            if s.cap:
                x = s.cap * torch.tanh(x / s.cap)
            if s.slopes is not None:
                x = x - s.slopes[:, None, None] * (s.pos[r0:r1, None] - at[None]).abs()
            seen = (at[None] >= s.lo[r0:r1, None]) & (at[None] <= s.hi[r0:r1, None])
            x = x.masked_fill(~seen, -math.inf)
            m = x.amax(-1, keepdim=True)
            p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
            l = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(hkv, -1, length), v).view(hq, r1 - r0, dh) / torch.where(l == 0, 1.0, l)
            out[r0:r1] = o.transpose(0, 1).to(out.dtype)
    return out


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    """What `run` returns, computed in float64 from the definitions, row by row or head by head; whole numbers have to
    be equal and need no such value."""
    if case["op"] == "map":
        return None
    s = prepare(case, seed)
    return {"norm": _exact_norm, "move": _exact_move, "attention": _exact_attention}[case["op"]](s)


def _turn(case, x, pos, amplitude):
    """x [rows][heads][dh] in float64: pair j of a head, as a complex number, times amplitude * exp(i * pos * w_j)."""
    n, r = _rotary_numbers(case), case["rotary"]
    w = []
    for j in range(r // 2):
        f = math.pow(n["base"], -2.0 * j / r)
        if case["scaling"] == "linear":
            f /= n["factor"]
        elif case["scaling"] == "turns":
            turns = n["trained"] * f / (2 * math.pi)
            keep = min(max((turns - n["slow"]) / (n["fast"] - n["slow"]), 0.0), 1.0)
            f = keep * f + (1 - keep) * f / n["factor"]
        elif case["scaling"] == "pairs":
            edge = [r * math.log(n["trained"] / (t * 2 * math.pi)) / (2 * math.log(n["base"])) for t in (n["fast"], n["slow"])]
            a, b = max(math.floor(edge[0]), 0), min(math.ceil(edge[1]), r // 2 - 1)
            slow = min(max((j - a) / max(b - a, 0.001), 0.0), 1.0)
            f = (1 - slow) * f + slow * f / n["factor"]
        w.append(f)
    turn = torch.polar(torch.full((len(pos), r // 2), amplitude, dtype=torch.float64, device="cuda"),
                       pos.double()[:, None] * torch.tensor(w, dtype=torch.float64, device="cuda")[None])
    body = x[..., :r]
    z = torch.complex(body[..., :r // 2].contiguous(), body[..., r // 2:].contiguous()) if case["layout"] == "half" \
        else torch.view_as_complex(body.reshape(*body.shape[:-1], r // 2, 2).contiguous())
    z = z * turn[:, None]
    back = torch.cat([z.real, z.imag], -1) if case["layout"] == "half" else torch.view_as_real(z).reshape(body.shape)
    return torch.cat([back, x[..., r:]], -1)


def _exact_norm(s):
    case = s.case
    hq, hkv, dh = _HEADS[case["heads"]]
    q, k, v = s.qkv.double().split([hq * dh, hkv * dh, hkv * dh], 1)
    q, k, v = q.view(-1, hq, dh), k.view(-1, hkv, dh), v.view(-1, hkv, dh)
    if case["gains"]:
        q, k = (x * (x.pow(2).sum(-1, keepdim=True) / dh + s.eps).rsqrt() * g.double() for x, g in ((q, s.g_q), (k, s.g_k)))
    a = _rotary_numbers(case)["amplitude"]
    out = {"q": _turn(case, q, s.pos, a), "k": s.k.double(), "v": s.v.double(), "k_pre": None if s.k_pre is None else s.k_pre.double()}
    block, at = s.slot.long() // s.size, s.slot.long() % s.size
    out["k"][block, :, at] = _turn(case, k, s.pos, a)
    out["v"][block, :, at] = v
    if s.k_pre is not None:
        out["k_pre"][block, :, at] = k
    return out


def _exact_move(s):
    n = _rotary_numbers(s.case)
    out = {"k": s.k.double(), "v": s.v.double()}
    fb, fa, tb, ta = s.src_slot.long() // s.size, s.src_slot.long() % s.size, s.dst_slot.long() // s.size, s.dst_slot.long() % s.size
    k = s.k_src[fb, :, fa].double()
    out["k"][tb, :, ta] = _turn(s.case, k, s.new, n["amplitude"]) if s.old is None else _turn(s.case, k, s.new.long() - s.old, 1.0)
    out["v"][tb, :, ta] = s.v_src[fb, :, fa].double()
    return out


def _exact_attention(s):
    hq, hkv, dh = _HEADS[s.case["heads"]]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(s.lens):
        at = torch.arange(length, device="cuda")
        where = s.table[b].long()[at // s.size]
        for h in range(hq):
            g = h // (hq // hkv)
            k, v = s.k[where, g, at % s.size].double(), s.v[where, g, at % s.size].double()
            for r0 in range(s.starts[b], s.starts[b + 1], 2048):
                r = slice(r0, min(r0 + 2048, s.starts[b + 1]))
                z = s.q[r, h].double() @ k.t() * dh ** -0.5
                if s.cap:
                    z = s.cap * (z / s.cap).tanh()
                if s.slopes is not None:
                    z = z - s.slopes[h].double() * (s.pos[r].double()[:, None] - at[None].double()).abs()
                hidden = (at[None] < s.lo[r, None]) | (at[None] > s.hi[r, None])
                z = torch.where(hidden, torch.full_like(z, -math.inf), z)
                w = torch.softmax(z, -1).nan_to_num(0.0)
                out[r, h] = w @ v
    return out
