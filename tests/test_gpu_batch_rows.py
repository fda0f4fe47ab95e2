"""rc_batch_map, rc_norm_rotary_rows and rc_rotary_move against plain 64-bit statements."""
import numpy as np
import pytest
import torch

from paper_2603_13289_amd import binding as rc
from tests import batch_reference as ref

pytestmark = pytest.mark.gpu

NAMES = ("row_seq", "row_pos", "row_slot", "row_lo", "row_hi")


def ints(values, device="cuda"):
    return torch.tensor(list(values), dtype=torch.int32, device=device)


# ------------------------------------------------------------------ batch map
def run_map(cached, new, table, size, n_blocks, free, first=None, prefix=None, docs=None, max_rows=None, stream=None):
    n = len(new)
    rows = max_rows if max_rows is not None else sum(max(x, 0) for x in new) + 3
    out = rc.BatchRows(*[torch.full((m,), -9, dtype=torch.int32, device="cuda") for m in (n + 1, rows, rows, rows, rows, rows, n, 3)])
    t = torch.tensor(table, dtype=torch.int32, device="cuda")
    starts = np.concatenate([[0], np.cumsum([len(d) for d in docs])]) if docs else None
    rc.rc_batch_map(ints(cached), ints(new), t, size, n_blocks, ints(free), out,
                    free_first=None if first is None else ints([first]), prefix_len=None if prefix is None else ints(prefix),
                    doc_start=ints(starts) if docs else None, doc_first=ints([p for d in docs for p in d]) if docs else None,
                    stream=stream)
    return out, t


def check_map(out, t, want, table):
    n = want["counts"][0]
    for name in NAMES:
        got = getattr(out, name).tolist()
        assert got[:n] == want[name], name
        assert all(x == -9 for x in got[n:]), name            # rows behind the last sequence are left as they were
    assert out.row_start.tolist() == want["row_start"]
    assert out.kv_len.tolist() == want["kv_len"]
    assert out.counts.tolist() == want["counts"]
    assert t.tolist() == table


@pytest.mark.parametrize("n_seq,size,longest", [(1, 16, 1), (1, 1, 40), (3, 16, 100), (7, 24, 300), (64, 16, 33), (256, 16, 40),
                                                (257, 5, 17), (1000, 16, 9), (3000, 64, 3), (65536, 4, 2)])
@pytest.mark.parametrize("extras", [False, True])
def test_batch_map(n_seq, size, longest, extras):
    rng = np.random.default_rng(n_seq * 100 + size)
    cached = rng.integers(0, longest * 2, n_seq).tolist()
    new = (rng.integers(0, longest + 1, n_seq) * (rng.random(n_seq) < 0.8)).tolist()
    width = -(-max(c + n for c, n in zip(cached, new)) // size) + 1
    n_blocks = n_seq * width + 9
    ids = rng.permutation(n_blocks).tolist()
    table, at = [], 0
    for c in cached:
        h = -(-c // size)
        table.append(ids[at:at + h] + [-1] * (width - h))
        at += h
    free = ids[at:]
    prefix = rng.integers(0, longest * 3, n_seq).tolist() if extras else None
    docs = [sorted(set(rng.integers(0, max(c + n, 1), 4).tolist())) if i % 3 else [] for i, (c, n) in enumerate(zip(cached, new))] if extras else None
    first = 4 if extras else None
    out, t = run_map(cached, new, table, size, n_blocks, free, first, prefix, docs)
    want = ref.batch_map(cached, new, table, size, n_blocks, free, first or 0, prefix, docs)
    check_map(out, t, want, table)


@pytest.mark.parametrize("free,max_rows", [(list(range(50, 53)), None), ([], None), (list(range(50, 90)), 30), (list(range(50, 90)), 0)])
def test_batch_map_refuses_whole_sequences(free, max_rows):
    """A free list or row arrays too short, a sequence longer than its table row, negative counts, blocks outside the pool."""
    cached = [5, 0, 60, 16, -4, 3]
    new = [3, 20, 9, 1, 2, -1]
    table = [[0, -1, -1, -1], [-1, -1, -1, -1], [1, 2, 3, 4], [5, -1, -1, -1], [-1, -1, -1, -1], [99, -1, -1, -1]]
    out, t = run_map(cached, new, table, 16, 64, free, max_rows=max_rows)
    want = ref.batch_map(cached, new, table, 16, 64, free, max_rows=max_rows)
    check_map(out, t, want, table)
    assert want["counts"][2] > 0


def test_batch_map_replayed_with_other_lengths():
    """A captured step, replayed with lengths that change between replays, against the eager statement every time."""
    size, n_blocks, n_seq = 16, 400, 5
    cached, new, first = ints([0] * n_seq), ints([0] * n_seq), ints([0])
    table = torch.full((n_seq, 40), -1, dtype=torch.int32, device="cuda")
    free = ints(np.random.default_rng(0).permutation(n_blocks))
    rows = rc.BatchRows.alloc(n_seq, 500)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rc.rc_batch_map(cached, new, table, size, n_blocks, free, rows, free_first=first)
    have, host = [0] * n_seq, table.tolist()
    at = 0
    for step, lengths in enumerate([[7, 0, 40, 1, 99], [1, 1, 1, 1, 1], [1, 16, 0, 1, 1], [30, 30, 30, 30, 30]]):
        cached.copy_(ints(have))
        new.copy_(ints(lengths))
        first.copy_(ints([at]))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.batch_map(have, lengths, host, size, n_blocks, free.tolist(), at)
        n = want["counts"][0]
        for name in NAMES:
            assert getattr(rows, name)[:n].tolist() == want[name], (step, name)
        assert rows.counts.tolist() == want["counts"] and table.tolist() == host
        have, at = want["kv_len"], want["counts"][1]


# ------------------------------------------------------------------ norm and rotation
SCALED = dict(plain={}, linear=dict(factor=4.0), turns=dict(factor=8.0, trained=8192, slow=1.0, fast=4.0),
              pairs=dict(factor=16.0, trained=4096, slow=1.0, fast=32.0))
CODES = dict(plain=rc.RC_ROTARY_PLAIN, linear=rc.RC_ROTARY_LINEAR, turns=rc.RC_ROTARY_BY_TURNS, pairs=rc.RC_ROTARY_BY_PAIR)


def rotation(layout, dim, scaling, amplitude=1.0, base=1e4):
    a = SCALED[scaling]
    plan = rc.rc_rotary_init(rc.RC_ROTARY_HALF if layout == "half" else rc.RC_ROTARY_INTERLEAVED, dim, base, scaling=CODES[scaling],
                             factor=a.get("factor", 1.0), trained_len=a.get("trained", 0), slow_turns=a.get("slow", 1.0),
                             fast_turns=a.get("fast", 32.0), amplitude=amplitude)
    return plan, ref.frequencies(dim, base, scaling, **a)


def pool_cache(dtype, n_blocks, hkv, size, dh, width=1):
    td = torch.bfloat16 if dtype == rc.RC_BF16 else torch.float32
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn((n_blocks, hkv, size, dh), generator=g).to(td).cuda() for _ in range(2))
    return rc.PagedKV.from_pools([k], [v], torch.zeros((1, width), dtype=torch.int32, device="cuda"), dtype)


def rows_of(pool, slot, size):
    s = torch.as_tensor(slot, device=pool.device).long()
    return pool[s // size, :, s % size].double().cpu().numpy()


def assert_close(got, want, size, out_dtype, what):
    """Norm and rotation in 32 bits: a sum of squares of 128 terms in runs of 8 and a tree (at most 12 roundings, halved by the root),
    division, two products; then two products, a sum and angles good to 2^-24: 16 steps of 2^-24 of the pair's size cover them.  One
    rounding to the type at the end."""
    bound = 16 * 2.0 ** -24 * size + ref.step_of(out_dtype) * np.abs(want) * (1 + 2.0 ** -8) + 1e-37
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, float(np.abs(got - want)[bad].max()), int(bad.sum()))


@pytest.mark.parametrize("dtype,qkv,hq,hkv,dh", [("bf16", "f32", 32, 8, 128), ("bf16", "bf16", 40, 8, 128), ("f32", "f32", 4, 2, 64),
                                                 ("f32", "bf16", 7, 7, 128), ("bf16", "bf16", 9, 1, 128), ("f32", "f32", 1, 1, 64),
                                                 ("bf16", "f32", 64, 64, 128), ("f32", "f32", 32, 16, 128)])
@pytest.mark.parametrize("n,size,layout,part,scaling", [(1, 16, "half", 1, "plain"), (5, 1, "interleaved", 2, "linear"),
                                                        (67, 24, "half", 4, "turns"), (130, 1000, "interleaved", 1, "pairs"),
                                                        (33, 16, "half", 8, "pairs")])
@pytest.mark.parametrize("gains", [True, False])
def test_norm_rotary_rows(dtype, qkv, hq, hkv, dh, n, size, layout, part, scaling, gains):
    rng = np.random.default_rng(n + hq)
    code = rc.RC_BF16 if dtype == "bf16" else rc.RC_F32
    td = rc.torch_dtype(code)
    n_blocks = -(-2 * n // size) + 2
    kv = pool_cache(code, n_blocks, hkv, size, dh)
    k_pre = torch.full_like(kv.k[0], 3.0)
    before = [kv.k[0].clone(), kv.v[0].clone(), k_pre.clone()]
    slot = rng.permutation(n_blocks * size)[:n]
    slot[n // 2:n // 2 + 1] = -1 if n > 1 else slot[0]         # a row that leaves the cache alone
    pos = rng.integers(0, 1 << (8 if n < 60 else 20), n)
    width = (hq + 2 * hkv) * dh
    x = torch.from_numpy(rng.standard_normal((n, width + 8)).astype(np.float32) * rng.choice([0.01, 1.0, 30.0], (n, 1)).astype(np.float32))
    x = x.to(torch.bfloat16 if qkv == "bf16" else torch.float32).cuda()[:, :width]    # rows further apart than they are long
    gq, gk = ((1 + 0.2 * torch.randn(dh)).to(td).cuda() for _ in range(2)) if gains else (None, None)
    plan, freq = rotation(layout, dh // part, scaling, amplitude=1.2 if scaling == "pairs" else 1.0)
    q = torch.full((n, hq, dh), 7.0, dtype=td, device="cuda")
    rc.rc_norm_rotary_rows(x, n, hq, plan, ints(pos), ints(slot), kv.layer(0), q, g_q=gq, g_k=gk, eps=1e-5, k_pre=k_pre)
    h = x.double().cpu().numpy().reshape(n, hq + 2 * hkv, dh)
    rq, rk, rv = h[:, :hq], h[:, hq:hq + hkv], h[:, hq + hkv:]
    if gains:
        rq, rk = ref.head_norm(rq, gq.double().cpu().numpy(), 1e-5), ref.head_norm(rk, gk.double().cpu().numpy(), 1e-5)
    wq, sq = ref.rotate(rq, pos, freq, layout, plan.amplitude)
    wk, sk = ref.rotate(rk, pos, freq, layout, plan.amplitude)
    assert_close(q.double().cpu().numpy(), wq, sq, td, "q")
    ok = slot >= 0
    for pool, old, want, room, what in ((kv.k[0], before[0], wk, sk, "k"), (kv.v[0], before[1], rv, np.abs(rv), "v"),
                                        (k_pre, before[2], rk, np.abs(rk), "k_pre")):
        assert_close(rows_of(pool, slot[ok], size), want[ok], room[ok], td, what)
        mine = torch.zeros((n_blocks, size), dtype=torch.bool)
        mine.view(-1)[torch.from_numpy(slot[ok])] = True
        rest = ~mine.cuda()[:, None, :, None].expand_as(pool)
        assert torch.equal(pool[rest], old[rest]), what       # nothing else of the cache is written


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("dim", [8, 24, 40, 56])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotated_parts_that_are_no_multiple_of_16(dtype, dh, dim, layout):
    code = rc.RC_BF16 if dtype == "bf16" else rc.RC_F32
    td = rc.torch_dtype(code)
    kv, plan, freq = pool_cache(code, 4, 2, 16, dh), *rotation(layout, dim, "plain", base=1e3)
    n, hq = 9, 6
    rng = np.random.default_rng(dim)
    x = torch.from_numpy(rng.standard_normal((n, (hq + 4) * dh)).astype(np.float32)).to(td).cuda()
    q = torch.zeros((n, hq, dh), dtype=td, device="cuda")
    pos, slot = rng.integers(0, 5000, n), rng.permutation(64)[:n]
    rc.rc_norm_rotary_rows(x, n, hq, plan, ints(pos), ints(slot), kv.layer(0), q)
    h = x.double().cpu().numpy().reshape(n, -1, dh)
    for got, part, what in ((q.double().cpu().numpy(), h[:, :hq], "q"), (rows_of(kv.k[0], slot, 16), h[:, hq:hq + 2], "k")):
        want, room = ref.rotate(part, pos, freq, layout)
        assert_close(got, want, room, td, what)
    moved = pool_cache(code, 4, 2, 16, dh)
    rc.rc_rotary_move(kv.layer(0), ints(slot), moved.layer(0), ints(slot[::-1].copy()), n, plan, ints(pos[::-1].copy()), ints(pos))
    want, room = ref.rotate(rows_of(kv.k[0], slot, 16), pos[::-1] - pos, freq, layout)
    assert_close(rows_of(moved.k[0], slot[::-1].copy(), 16), want, room, td, "moved")


def test_norm_rotary_rows_behind_the_live_ones_are_left():
    kv = pool_cache(rc.RC_BF16, 8, 2, 16, 128)
    before = kv.k[0].clone()
    plan, _ = rotation("half", 128, "plain")
    x = torch.randn((10, 8 * 128), device="cuda")
    q = torch.full((10, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    live = ints([4])
    rc.rc_norm_rotary_rows(x, 10, 4, plan, ints(range(10)), ints(range(10)), kv.layer(0), q, n_live=live)
    assert bool((q[4:] == 7.0).all()) and not bool((q[:4] == 7.0).all(2).any())
    assert torch.equal(kv.k[0][0, :, 4:], before[0, :, 4:]) and not torch.equal(kv.k[0][0, :, :4], before[0, :, :4])


def test_norm_of_zeros_and_infinities():
    """A head of zeros stays zeros (eps > 0); slots outside the pool on either side are skipped."""
    kv = pool_cache(rc.RC_F32, 2, 1, 16, 64)
    before = kv.k[0].clone()
    plan, _ = rotation("interleaved", 64, "plain")
    g = torch.ones(64, device="cuda")
    q = torch.empty((2, 1, 64), device="cuda")
    rc.rc_norm_rotary_rows(torch.zeros((2, 192), device="cuda"), 2, 1, plan, ints([3, 1 << 30]), ints([32, -2147483648]), kv.layer(0), q, g_q=g, g_k=g)
    assert bool((q == 0).all()) and torch.equal(kv.k[0], before)


# ------------------------------------------------------------------ moves
@pytest.mark.parametrize("dtype,hkv,dh", [("bf16", 8, 128), ("f32", 2, 64), ("f32", 3, 128), ("bf16", 1, 128)])
@pytest.mark.parametrize("n,ss,ds,layout,part,scaling", [(1, 16, 16, "half", 1, "plain"), (3, 1, 7, "interleaved", 2, "pairs"),
                                                         (100, 16, 24, "half", 2, "turns"), (257, 300, 16, "interleaved", 1, "linear")])
@pytest.mark.parametrize("rotated", [False, True])
def test_rotary_move(dtype, hkv, dh, n, ss, ds, layout, part, scaling, rotated):
    rng = np.random.default_rng(n + ss)
    code = rc.RC_BF16 if dtype == "bf16" else rc.RC_F32
    td = rc.torch_dtype(code)
    src, dst = pool_cache(code, -(-2 * n // ss) + 1, hkv, ss, dh), pool_cache(code, -(-2 * n // ds) + 1, hkv, ds, dh)
    before = [dst.k[0].clone(), dst.v[0].clone()]
    a = rng.permutation(src.n_blocks * ss)[:n]
    b = rng.permutation(dst.n_blocks * ds)[:n]
    if n > 2:
        a[1], b[2] = src.n_blocks * ss, -1                     # outside the pools: such rows are not moved
    old, new = rng.integers(0, 40000, n), rng.integers(0, 40000, n)
    plan, freq = rotation(layout, dh // part, scaling, amplitude=1.3)
    rc.rc_rotary_move(src.layer(0), ints(a), dst.layer(0), ints(b), n, plan, ints(new), ints(old) if rotated else None)
    ok = (a < src.n_blocks * ss) & (b >= 0)
    x = rows_of(src.k[0], a[ok], ss)
    want, room = ref.rotate(x, (new - old if rotated else new)[ok], freq, layout, 1.0 if rotated else 1.3)
    assert_close(rows_of(dst.k[0], b[ok], ds), want, room, td, "k")
    assert np.array_equal(rows_of(dst.v[0], b[ok], ds), rows_of(src.v[0], a[ok], ss))
    mine = torch.zeros((dst.n_blocks, ds), dtype=torch.bool)
    mine.view(-1)[torch.from_numpy(b[ok])] = True
    rest = ~mine.cuda()[:, None, :, None].expand_as(dst.k[0])
    assert torch.equal(dst.k[0][rest], before[0][rest]) and torch.equal(dst.v[0][rest], before[1][rest])


def test_rotary_move_in_place_and_live_rows():
    kv = pool_cache(rc.RC_F32, 4, 2, 16, 64)
    k0, v0 = kv.k[0].clone(), kv.v[0].clone()
    plan, freq = rotation("half", 64, "plain")
    slot = ints(range(20))
    rc.rc_rotary_move(kv.layer(0), slot, kv.layer(0), slot, 20, plan, ints([90] * 20), ints([50] * 20), n_live=ints([17]))
    want, room = ref.rotate(rows_of(k0, range(17), 16), [40] * 17, freq, "half")
    assert_close(rows_of(kv.k[0], range(17), 16), want, room, torch.float32, "k")
    assert torch.equal(kv.v[0], v0) and np.array_equal(rows_of(kv.k[0], range(17, 64), 16), rows_of(k0, range(17, 64), 16))


def test_rows_on_another_stream_and_in_a_graph():
    """The same bits from a stream of the caller's and from replays of a captured call, with other work between."""
    kv = pool_cache(rc.RC_BF16, 8, 2, 16, 128)
    plan, _ = rotation("half", 128, "plain")
    x = torch.randn((20, 8 * 128), device="cuda")
    q = [torch.empty((20, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    at = ints(range(20))
    rc.rc_norm_rotary_rows(x, 20, 4, plan, at, at, kv.layer(0), q[0])
    k0 = kv.k[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rc.rc_norm_rotary_rows(x, 20, 4, plan, at, at, kv.layer(0), q[1], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rc.rc_norm_rotary_rows(x, 20, 4, plan, at, at, kv.layer(0), q[2])
        rc.rc_rotary_move(kv.layer(0), at, kv.layer(0), at, 20, plan, at, at)
    for _ in range(3):
        q[2].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q[2], q[0]) and torch.equal(q[1], q[0]) and torch.equal(kv.k[0], k0)   # moved from where it was to where it was
