"""rc_masked_attention against a plain 64-bit statement, row by row."""
import numpy as np
import pytest
import torch

from paper_2603_13289_amd import binding as rc
from tests import batch_reference as ref

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(np.asarray(values).tolist(), dtype=torch.int32, device="cuda")


class Batch:
    """Sequences of (cached, new) rows in shuffled pages (size 0: one block a sequence), queries for the new rows."""

    def __init__(self, dtype, hq, hkv, dh, seqs, size, seed=0, std=1.0):
        self.rng = np.random.default_rng(seed)
        self.code = rc.RC_BF16 if dtype == "bf16" else rc.RC_F32
        self.td, self.hq, self.dh, self.seqs = rc.torch_dtype(self.code), hq, dh, seqs
        self.lens = [c + n for c, n in seqs]
        size = size or max(max(self.lens), 1)
        width = max(-(-max(self.lens) // size), 1)
        ids = self.rng.permutation(len(seqs) * width + 2)
        table = ids[:len(seqs) * width].reshape(len(seqs), width)
        self.kv = rc.PagedKV(1, len(ids), size, hkv, dh, self.code, table.tolist())
        self.k, self.v = [], []
        for s, n in enumerate(self.lens):
            k, v = (torch.from_numpy(self.rng.standard_normal((n, hkv, dh)).astype(np.float32) * std).to(self.td) for _ in range(2))
            if n:
                self.kv.write("k", 0, s, k.cuda())
                self.kv.write("v", 0, s, v.cuda())
            self.k.append(k)
            self.v.append(v)
        self.starts = np.concatenate([[0], np.cumsum([n for _, n in seqs])])
        self.n = int(self.starts[-1])
        self.q = torch.from_numpy(self.rng.standard_normal((self.n, hq, dh)).astype(np.float32) * std).to(self.td)
        self.pos = np.concatenate([np.arange(c, c + n) for c, n in seqs]).astype(int)
        self.lo, self.hi = np.zeros(self.n, int), self.pos.copy()

    def slopes(self):
        return 2.0 ** (-8.0 * (np.arange(self.hq) + 1) / self.hq)

    def run(self, cap=0.0, bias=False, scale=0.0, split=True, ranges=True, slack=0, seq=None, stream=None, max_len=None):
        out = torch.full((self.n + slack, self.hq, self.dh), 5.0, dtype=self.td, device="cuda")
        q = torch.cat([self.q.cuda(), torch.full((slack, self.hq, self.dh), float("nan"), dtype=self.td, device="cuda")])
        pad = lambda x: ints(list(x) + [0] * slack)
        self.plan = rc.MaskedAttention(ints(self.starts), pad(self.pos), self.n + slack, max(max(n for _, n in self.seqs), 1) + slack,
                                       max_len or max(max(self.lens), 1), row_lo=pad(self.lo) if ranges else None,
                                       row_hi=pad(self.hi) if ranges else None, seq=None if seq is None else ints(seq),
                                       slopes=torch.tensor(self.slopes(), dtype=torch.float32, device="cuda") if bias else None,
                                       scale=scale, cap=cap)
        layer = self.kv.layer(0)
        ws = rc.alloc_workspace(rc.rc_masked_attention_workspace_bytes(self.plan, self.hq, layer)) if split else None
        if ws is not None:
            ws.fill_(0xff)                                      # NaN wherever a kernel reads what nobody wrote
        self.keep = (q, ws)
        rc.rc_masked_attention(q, self.plan, self.hq, layer, out, ws, stream=stream)
        return out

    def check(self, got, cap=0.0, bias=False, scale=0.0, rows=None):
        """Tolerance, from the arithmetic.  A score is a sum of dh products in 32 bits (at most dh + 2 roundings of its absolute sum), the capped
        score adds four roundings of the cap, the bias two of its own size; an error d of scores changes weights by 2d relative.
        Weights are rounded to the type for the second product (bf16: half a step) and added up as rounded, so each moves the quotient by half a step of
        its share of |v - out|, at most of mass + |out|; sums of at most 4096 terms per accumulator in 32 bits, the output once to the type."""
        g = got.double().cpu().numpy()
        assert np.isfinite(g[:self.n]).all()
        slopes = self.slopes() if bias else None
        for s, (c, n) in enumerate(self.seqs):
            pick = range(n) if rows is None else sorted({int(i * (n - 1) / max(rows - 1, 1)) for i in range(rows)} if n else [])
            if not len(pick):
                continue
            at = self.starts[s] + np.array(pick)
            f64 = lambda t: t.double().cpu().numpy()
            want, mass, size = ref.attention(f64(self.q)[at], f64(self.k[s]), f64(self.v[s]), self.pos[at], self.lo[at], self.hi[at],
                                             scale or self.dh ** -0.5, cap, slopes)
            u = 2.0 ** -24
            d = (self.dh + 2) * u * np.minimum(size, 1e30) + 4 * 2 * u * cap
            if bias:
                reach = np.maximum(np.abs(self.pos[at] - self.lo[at]), np.abs(self.hi[at] - self.pos[at]))
                d = d + 2 * u * (slopes.max() * reach)[:, None, None]
            half = ref.step_of(self.td)
            weights = half if self.code == rc.RC_BF16 else 0.0
            bound = (weights + 2 * d + 4096 * u) * mass * (1 + 2 ** -7) + (half + weights) * np.abs(want) * (1 + 2 ** -7) + 1e-30
            err = np.abs(g[at] - want)
            assert (err <= bound).all(), (s, float((err - bound).max()), float(err.max()))


HEADS = [("bf16", 32, 8, 128), ("bf16", 5, 1, 128), ("bf16", 2, 2, 128), ("bf16", 40, 8, 128), ("bf16", 71, 1, 128),
         ("f32", 4, 2, 64), ("f32", 3, 3, 128), ("f32", 33, 1, 64)]
SEQS = {"one": [(0, 1)], "single": [(70, 1)], "tokens": [(0, 1), (62, 1), (63, 1), (64, 1), (200, 1), (0, 0), (31, 1)],
        "few": [(5, 3), (0, 2), (190, 7), (64, 1)], "ragged": [(0, 65), (13, 64), (0, 0), (100, 31), (3, 1), (0, 130)]}


@pytest.mark.parametrize("dtype,hq,hkv,dh", HEADS)
@pytest.mark.parametrize("seqs", list(SEQS))
@pytest.mark.parametrize("size,cap,bias", [(16, 0.0, False), (0, 30.0, False), (24, 0.0, True), (5, 2.0, True), (208, 100.0, False), (24, 55.0, False)])
def test_causal(dtype, hq, hkv, dh, seqs, size, cap, bias):
    b = Batch(dtype, hq, hkv, dh, SEQS[seqs], size, seed=hq, std=1.5)
    got = b.run(cap, bias, ranges=size != 0, slack=3)
    b.check(got, cap, bias)
    assert bool((got[b.n:] == 5.0).all())                       # rows behind the last sequence are left as they were


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("kind", ["documents", "prefix", "window", "single_key", "whole", "random"])
@pytest.mark.parametrize("poison", [False, True])
def test_ranges(dtype, hq, hkv, dh, kind, poison):
    """Documents, prefixes, windows, rows that see nothing or one key.  poison: infinities and NaN in every place that no row of the
    batch sees, and in places that only the other documents' rows see."""
    seqs = [(0, 150), (40, 90), (128, 5), (300, 1)]
    b = Batch(dtype, hq, hkv, dh, seqs, 16, seed=3)
    for s, (c, n) in enumerate(seqs):
        r = slice(b.starts[s], b.starts[s + 1])
        p = b.pos[r]
        if kind == "documents":
            first = np.array([0, 37, 64, 101])
            b.lo[r] = [first[first <= x].max() for x in p]
        elif kind == "prefix":
            b.hi[r] = np.maximum(p, (c + n) // 2)
        elif kind == "window":
            b.lo[r] = np.maximum(p - 20, 0)
        elif kind == "single_key":
            b.lo[r] = b.hi[r] = b.rng.integers(0, c + n, n)
        elif kind == "whole":
            b.hi[r] = c + n - 1
        else:
            b.lo[r], b.hi[r] = b.rng.integers(-5, c + n, n), b.rng.integers(-5, c + n + 9, n)
    if kind == "random":
        b.hi = np.minimum(b.hi, np.repeat(b.lens, [n for _, n in seqs]) - 1)
    b.lo[::7], b.hi[::7] = 9, 8                                 # rows that see nothing
    if poison:
        for s in range(len(seqs)):
            r = slice(b.starts[s], b.starts[s + 1])
            for j in range(b.lens[s]):
                if not ((b.lo[r] <= j) & (j <= b.hi[r])).any():
                    bad = [float("nan"), float("inf"), -float("inf")][j % 3]
                    b.k[s][j], b.v[s][j] = bad, bad
            b.kv.write("k", 0, s, b.k[s].cuda())
            b.kv.write("v", 0, s, b.v[s].cuda())
    got = b.run(cap=10.0, bias=True)
    b.check(got, cap=10.0, bias=True)
    assert bool((got[::7] == 0).all())


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows", [40, 3])
def test_bad_rows_stay_in_their_document(dtype, hq, hkv, dh, bad, rows):
    """Rows of one document hold no finite numbers: the other documents' rows do not notice, and the document's own rows show it."""
    b = Batch(dtype, hq, hkv, dh, [(0, 120)] if rows == 40 else [(117, 3)], 16, seed=1)
    edges = [0, 37, 81] if rows == 40 else [0, 118, 119]
    b.lo = np.array([max(e for e in edges if e <= p) for p in b.pos])
    sick = range(edges[1], edges[2])
    for j in sick:
        b.v[0][j, :, 5] = bad
    b.kv.write("v", 0, 0, b.v[0].cuda())
    got = b.run().double().cpu().numpy()
    own = np.array([p in sick for p in b.pos])
    assert np.isfinite(got[~own]).all()
    rest = [d for d in range(dh) if d != 5]
    assert np.isfinite(got[own][:, :, rest]).all()
    x = got[own][:, :, 5]
    assert np.isnan(x).all() if np.isnan(bad) else (x == bad).all()
    for s in ("k", "v"):
        getattr(b, s)[0][list(sick)] = 0.0                       # the healthy rows against the statement
    b.pos, b.lo, b.hi, keep = b.pos[~own], b.lo[~own], b.hi[~own], b.q
    b.q, b.n = b.q[torch.from_numpy(~own)], int((~own).sum())
    b.seqs, b.starts = [(0, b.n)], np.array([0, b.n])
    b.check(torch.from_numpy(got[~own]))


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("seqs,size", [([(5000, 1)], 16), ([(4093, 1), (12, 1), (2600, 1)], 24), ([(3000, 40)], 0),
                                       ([(2500, 3), (0, 1), (900, 5)], 16)])
@pytest.mark.parametrize("split", [True, False])
def test_long_ranges(dtype, hq, hkv, dh, seqs, size, split):
    b = Batch(dtype, hq, hkv, dh, seqs, size, seed=2)
    b.lo[::2] = b.pos[::2] // 3
    b.lo[-1], b.hi[-1] = 7, 6
    b.check(b.run(cap=40.0, split=split), cap=40.0, rows=6)


@pytest.mark.parametrize("hq,hkv,rows", [(40, 8, 2000), (32, 8, 2100), (16, 16, 4096)])
@pytest.mark.parametrize("size,cap,bias", [(16, 50.0, False), (24, 0.0, True), (0, 100.0, False), (32, 0.0, False)])
def test_wide_tiles(hq, hkv, rows, size, cap, bias):
    """Enough long ranges for tiles of eight wavefronts: causal rows, windows, rows that see nothing, other documents' values that are no numbers."""
    b = Batch("bf16", hq, hkv, 128, [(4300 - rows // 2, rows // 2), (700, 7), (0, rows - rows // 2)], size, seed=rows)
    b.lo[1::3] = np.maximum(b.pos[1::3] - 300, 0)
    b.lo[5::50], b.hi[5::50] = 4, 3
    at = slice(b.starts[2], b.starts[3])
    b.lo[at] = np.where(b.pos[at] >= 90, np.maximum(b.lo[at], 90), b.lo[at])
    b.v[2][60:90, :, 3] = float("inf")
    b.lo[at] = np.where((b.pos[at] >= 60) & (b.pos[at] < 90), b.hi[at] + 1, b.lo[at])
    b.kv.write("v", 0, 2, b.v[2].cuda())
    got = b.run(cap=cap, bias=bias, max_len=4300)
    b.v[2][60:90, :, 3] = 0.0
    b.check(got, cap=cap, bias=bias, rows=9)
    assert bool((got[5::50] == 0).all())


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 4, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("std,scale,cap", [(40.0, 0.0, 0.0), (40.0, 0.0, 50.0), (1.0, 3.0, 1e-3), (1.0, 1e-4, 1e6), (12.0, 1.0, 5.0)])
def test_extreme_scores(dtype, hq, hkv, dh, std, scale, cap):
    """Scores of thousands, caps far below and far above the scores."""
    if dtype == "bf16":
        cap = min(cap, 4096.0)                                  # the largest that bf16 takes
    b = Batch(dtype, hq, hkv, dh, [(20, 70), (100, 1)], 16, seed=4, std=std)
    b.check(b.run(cap=cap, scale=scale), cap=cap, scale=scale)


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("bf16", 40, 1, 128), ("f32", 4, 2, 64)])
def test_a_batch_without_rows(dtype, hq, hkv, dh):
    """Bounds for rows that there are none of: nothing is written, split or not."""
    b = Batch(dtype, hq, hkv, dh, [(300, 1), (20, 2)], 16)
    b.run()
    q, ws = b.keep
    out = torch.full_like(q, 5.0)
    for most, n in ((1, 3), (3, 3), (60, 3)):
        plan = rc.MaskedAttention(ints([0, 0, 0]), ints([0] * 3), n, most, 301)
        ws = rc.alloc_workspace(rc.rc_masked_attention_workspace_bytes(plan, hq, b.kv.layer(0)))
        rc.rc_masked_attention(q, plan, hq, b.kv.layer(0), out, ws)
        rc.rc_masked_attention(q, plan, hq, b.kv.layer(0), out)
    assert bool((out == 5.0).all())


def test_two_streams_at_once():
    """Calls that overlap in time, each with a workspace of its own, give the bits of calls one after the other."""
    many = [Batch("bf16", 8, 2, 128, [(2000 + 100 * i, 1), (500, 2)], 16, seed=i) for i in range(4)]
    want = [b.run(cap=30.0) for b in many]
    streams = [torch.cuda.Stream() for _ in many]
    torch.cuda.synchronize()
    outs = [torch.zeros_like(w) for w in want]
    for _ in range(5):
        for b, o, st in zip(many, outs, streams):
            rc.rc_masked_attention(b.keep[0], b.plan, 8, b.kv.layer(0), o, b.keep[1], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(w, o) for w, o in zip(want, outs))


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 40, 1, 128), ("bf16", 2, 1, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("n_seq", [64, 65, 200, 4500])
def test_many_sequences(dtype, hq, hkv, dh, n_seq):
    """More sequences than lanes look for a row's one at a time; some without rows."""
    rng = np.random.default_rng(n_seq)
    seqs = [(int(c), int(n)) for c, n in zip(rng.integers(0, 20, n_seq), rng.integers(0, 4, n_seq))]
    b = Batch(dtype, hq, hkv, dh, seqs, 8, seed=n_seq)
    got = b.run(cap=30.0, split=n_seq < 100)
    some = sorted(set(rng.integers(0, n_seq, 60).tolist()) | {0, n_seq - 1})
    every, b.seqs = b.seqs, [q if s in some else (q[0], 0) for s, q in enumerate(b.seqs)]
    b.check(got, cap=30.0)
    assert bool((got != 5.0).any(2).all()) and sum(n for _, n in every) == got.shape[0]


def test_block_table_rows_and_other_streams():
    """seq names the block-table rows; the call on a stream of the caller's; rows of a table entry outside the pool are some row, not a fault."""
    b = Batch("bf16", 8, 2, 128, [(40, 9), (70, 1), (0, 20)], 16, seed=6)
    want = b.run(bias=True)
    order = [2, 0, 1]
    side = torch.cuda.Stream()
    moved = b.kv.block_table[order].contiguous()
    back = [order.index(s) for s in range(3)]
    b.kv.block_table.copy_(moved)
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    got = b.run(bias=True, seq=back, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("decode", [True, False])
def test_replays_with_other_lengths(dtype, hq, hkv, dh, decode):
    """A captured call replayed while positions, ranges and sequence starts change inside the bounds, against the eager call."""
    seqs = [(700, 1), (30, 1), (512, 1)] if decode else [(300, 40), (0, 60), (80, 30)]
    b = Batch(dtype, hq, hkv, dh, seqs, 16, seed=8)
    out = b.run(cap=20.0, slack=5)
    plan, (q, ws) = b.plan, b.keep
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rc.rc_masked_attention(q, plan, hq, b.kv.layer(0), out, ws)
    for i in range(4):
        if decode:
            plan.row_hi[:3].copy_(ints([600 - 150 * i, 5 * i, 511 - i]))
        else:
            plan.row_lo[:130].copy_(ints(np.minimum(b.pos, 13 * i)))
            plan.row_start.copy_(ints([0, 40 - i, 90, 130 - 7 * i]))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.full_like(out, 5.0)
        rc.rc_masked_attention(q, plan, hq, b.kv.layer(0), eager, ws)
        assert torch.equal(eager, out), i
        assert bool(torch.isfinite(out.float()).all())


def test_pools_behind_32_bits():
    """Blocks whose byte offsets pass 2^32 (and element offsets 2^31)."""
    hq, hkv, dh, size = 4, 2, 128, 4096
    n_blocks = 2100                                             # 2100 * 2 * 4096 * 128 elements = 4.4 GB a pool
    kv = rc.PagedKV(1, n_blocks, size, hkv, dh, rc.RC_BF16, [[2099, 2090]])
    b = Batch("bf16", hq, hkv, dh, [(4100, 1)], 0, seed=9)
    kv.write("k", 0, 0, b.k[0].cuda())
    kv.write("v", 0, 0, b.v[0].cuda())
    b.kv = kv
    b.check(b.run())
    b = Batch("bf16", hq, hkv, dh, [(4100, 70)], 0, seed=9)
    kv.write("k", 0, 0, b.k[0].cuda())
    kv.write("v", 0, 0, b.v[0].cuda())
    b.kv = kv
    b.check(b.run(), rows=5)


def test_garbage_on_the_device_stays_in_bounds():
    """Starts that do not ascend, sequences and blocks outside their tables, ranges beyond the cache: some numbers, no fault."""
    b = Batch("bf16", 8, 2, 128, [(40, 30), (70, 9), (0, 20)], 16, seed=6)
    b.starts = np.array([0, 500, -7, 59])
    b.lo[:], b.hi[:] = -1000, 1 << 30
    b.kv.block_table.fill_(1 << 30)
    b.run(seq=[5, -5, 1 << 30], cap=3.0, bias=True)
    torch.cuda.synchronize()
    b.seqs = [(40, 1), (70, 1), (0, 1)]
    b.run(seq=[5, -5, 1 << 30], cap=3.0, bias=True)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("seqs", [[(300, 1)], [(300, 2), (3000, 1)], [(0, 301)], [(0, 70), (2000, 60)]])
@pytest.mark.parametrize("cap", [0.0, 20.0, 100.0])
def test_a_key_without_a_number(dtype, hq, hkv, dh, seqs, cap):
    """One NaN among a row's keys makes its outputs NaN, wherever ranges are cut: also where it is all that a part of the range has.
    Rows that do not see it keep their outputs."""
    for key in (0, 32, 63, 64, 299):
        b = Batch(dtype, hq, hkv, dh, seqs, 16, seed=key)
        if key == 32:
            b.hi = np.minimum(b.hi, 32)                         # the only key of its block that rows see
        elif key == 64:
            b.lo[::2] = np.where(b.pos[::2] > 64, 65, b.lo[::2])
        for s, n in enumerate(b.lens):
            if key < n:
                b.k[s][key] = float("nan")
                b.kv.write("k", 0, s, b.k[s].cuda())
        got = b.run(cap=cap).float().cpu().numpy()
        sees = (b.lo <= key) & (key <= b.hi)
        assert np.isnan(got[sees]).all() and np.isfinite(got[~sees]).all(), key


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("seqs", [[(0, 90)], [(1500, 1)]])
@pytest.mark.parametrize("cap", [50.0, 55.0, 60.0, 0.0])
@pytest.mark.parametrize("sign,size", [(1.0, 2.0 ** 40), (-1.0, 2.0 ** -20)])
def test_scores_at_the_cap(dtype, hq, hkv, dh, seqs, cap, sign, size):
    """Every score at one end of what the cap lets through, large and small values: weights far from 1 leave the quotient as it is."""
    b = Batch(dtype, hq, hkv, dh, seqs, 16, seed=2)
    b.q = torch.full_like(b.q, 8.0)
    for s in range(len(seqs)):
        b.k[s] = torch.full_like(b.k[s], 8.0 * sign)
        b.v[s] = torch.sign(b.v[s]) * (1 + b.v[s].abs() / 8) * size
        b.kv.write("k", 0, s, b.k[s].cuda())
        b.kv.write("v", 0, s, b.v[s].cuda())
    b.check(b.run(cap=cap), cap=cap)


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("f32", 33, 1, 64)])
@pytest.mark.parametrize("seqs", [[(300, 1)], [(3000, 1), (12, 2)], [(9, 160), (0, 0), (1200, 70)]])
@pytest.mark.parametrize("split", [True, False])
def test_out_in_the_place_of_q(dtype, hq, hkv, dh, seqs, split):
    b = Batch(dtype, hq, hkv, dh, seqs, 16, seed=5)
    b.lo[::9], b.hi[::9] = 2, 1
    want = b.run(cap=30.0, split=split, slack=2)
    q, ws = b.keep
    before = q.clone()
    rc.rc_masked_attention(q, b.plan, hq, b.kv.layer(0), q, ws)
    assert torch.equal(q[:b.n], want[:b.n])
    assert torch.equal(q[b.n:].view(torch.uint8), before[b.n:].view(torch.uint8))


@pytest.mark.parametrize("hq,hkv,rows,longest", [(16, 8, 4300, 900), (40, 8, 1900, 500), (71, 1, 600, 300), (32, 8, 2400, 4200)])
@pytest.mark.parametrize("n_seq", [1, 9, 700])
def test_tiles_in_order_of_length(hq, hkv, rows, longest, n_seq):
    """More tiles than run at a time: a workspace changes their order and no bit, and every row is written; empty sequences, rows that see nothing."""
    rng = np.random.default_rng(n_seq)
    cuts = np.sort(rng.integers(0, rows + 1, n_seq - 1))
    new = np.diff(np.concatenate([[0], cuts, [rows]]))
    seqs = [(int(rng.integers(0, 60)), int(n)) for n in new]
    b = Batch("bf16", hq, hkv, 128, seqs, 16, seed=rows)
    b.lo = np.maximum(b.pos - rng.integers(0, longest, b.n), 0)
    b.lo[::3] = b.pos[::3] // 128 * 128
    b.lo[4::31], b.hi[4::31] = 9, 8
    most = max(max(b.lens), 4096 if longest > 4096 else 1)
    b.kv.block_table = torch.cat([b.kv.block_table, b.kv.block_table[:, :1].expand(-1, 4300 // 16)], 1).contiguous()
    b.kv.max_blocks = b.kv.block_table.shape[1]
    plain = b.run(cap=30.0, split=False, max_len=most)
    got = b.run(cap=30.0, max_len=most)
    assert b.keep[1].numel() >= 16
    assert torch.equal(plain, got)
    assert bool((got != 5.0).any(2).all()) and bool((got[4::31] == 0).all())
    keep, some = b.seqs, set(rng.integers(0, n_seq, 12).tolist()) | {0}
    b.seqs = [q if s in some else (q[0], 0) for s, q in enumerate(keep)]
    b.check(got, cap=30.0, rows=4)


def test_replays_in_order_of_length():
    """A captured call whose tiles are put in order on the device, replayed with other starts and ranges inside the bounds, against calls without an order."""
    b = Batch("bf16", 16, 8, 128, [(30, 1500), (0, 2000), (200, 800)], 16, seed=12)
    out = b.run(cap=20.0, slack=9)
    plan, (q, ws) = b.plan, b.keep
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rc.rc_masked_attention(q, plan, 16, b.kv.layer(0), out, ws)
    for i in range(4):
        plan.row_start.copy_(ints([0, 1500 - 400 * i, 3000 + 100 * i, 4300 - 77 * i]))
        plan.row_lo[:4300].copy_(ints(np.maximum(b.pos - 300 * i, 0)))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.full_like(out, 5.0)
        rc.rc_masked_attention(q, plan, 16, b.kv.layer(0), eager)
        assert torch.equal(eager, out), i


def test_garbage_stays_in_bounds_where_tiles_are_ordered():
    """Starts, ranges and table entries of any value: some numbers, no fault, and rows of the batch alone are written."""
    b = Batch("bf16", 16, 8, 128, [(30, 1500), (0, 2000), (200, 800)], 16, seed=13)
    b.starts = np.array([-7, 1 << 30, 900, -(1 << 31)])
    b.lo[:], b.hi[:] = -1000, 1 << 30
    b.kv.block_table.fill_(-(1 << 30))
    b.run(seq=[5, -5, 1 << 30], cap=3.0, bias=True)
    assert b.keep[1].numel() >= 16
    b.starts = np.array([4300, 100, 100, 4299])
    b.run(cap=3.0)
    torch.cuda.synchronize()
