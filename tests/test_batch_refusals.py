"""The calls for ragged batches refuse what they cannot do on the host, before any launch (no GPU); the rotation's frequencies, which are
host work, against their definition."""
import math

import numpy as np
import pytest
import torch

from paper_2603_13289_amd import binding as rc
from tests import batch_reference as ref


def status(fn):
    with pytest.raises(rc.RcError) as e:
        fn()
    return e.value.status


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


@pytest.mark.parametrize("scaling,args", [("plain", {}), ("linear", dict(factor=4.0)),
                                          ("turns", dict(factor=8.0, trained=8192, slow=1.0, fast=4.0)),
                                          ("pairs", dict(factor=16.0, trained=4096, slow=1.0, fast=32.0)),
                                          ("pairs", dict(factor=2.0, trained=64, slow=20.0, fast=30.0))])
@pytest.mark.parametrize("dim,base", [(128, 1e4), (64, 5e5), (8, 1e6), (96, 1e4)])
def test_frequencies(scaling, args, dim, base):
    code = {"plain": rc.RC_ROTARY_PLAIN, "linear": rc.RC_ROTARY_LINEAR, "turns": rc.RC_ROTARY_BY_TURNS, "pairs": rc.RC_ROTARY_BY_PAIR}
    kw = dict(factor=args.get("factor", 1.0), trained_len=args.get("trained", 0), slow_turns=args.get("slow", 1.0),
              fast_turns=args.get("fast", 32.0))
    r = rc.rc_rotary_init(rc.RC_ROTARY_HALF, dim, base, scaling=code[scaling], amplitude=1.25, **kw)
    want = ref.frequencies(dim, base, scaling, **args)
    got = np.array(r.freq[:dim // 2])
    assert (r.rotary_dim, r.amplitude) == (dim, 1.25)
    # a power, a logarithm's quotient and a few products, each off by a step or two of 2^-53
    assert np.all(np.abs(got - want) <= 1e-14 * want)


def test_rotary_init_refusals():
    init = rc.rc_rotary_init
    assert status(lambda: init(2, 64, 1e4)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 0, 1e4)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 60, 1e4)) == rc.RC_E_UNSUPPORTED
    assert status(lambda: init(0, 136, 1e4)) == rc.RC_E_UNSUPPORTED
    assert status(lambda: init(0, 64, 0.0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 64, math.nan)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 64, 1e4, scaling=7)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 64, 1e4, amplitude=0.0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 64, 1e4, scaling=rc.RC_ROTARY_LINEAR, factor=0.0)) == rc.RC_E_INVALID_ARG
    by_turns = dict(scaling=rc.RC_ROTARY_BY_TURNS, factor=2.0)
    assert status(lambda: init(0, 64, 1e4, trained_len=0, **by_turns)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 64, 1e4, trained_len=100, slow_turns=4.0, fast_turns=4.0, **by_turns)) == rc.RC_E_INVALID_ARG
    assert status(lambda: init(0, 64, 1.0, trained_len=100, scaling=rc.RC_ROTARY_BY_PAIR, factor=2.0)) == rc.RC_E_INVALID_ARG


def test_batch_map_refusals():
    table = torch.zeros((2, 4), dtype=torch.int32)
    rows = rc.BatchRows.alloc(2, 8, device="cpu")

    def call(n_cached=ints(0, 0), n_new=ints(1, 1), size=16, n_blocks=8, rows=rows, **kw):
        rc.rc_batch_map(n_cached, n_new, table, size, n_blocks, ints(0, 1, 2), rows, **kw)

    assert status(lambda: call(size=0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(n_blocks=0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(n_blocks=1 << 28)) == rc.RC_E_CAPACITY
    assert status(lambda: call(n_new=rows.kv_len)) == rc.RC_E_INVALID_ARG                       # an output that is an input
    assert status(lambda: call(n_cached=rows.kv_len)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(free_first=rows.counts[1:])) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(prefix_len=rows.row_start[1:])) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(n_cached=rows.row_hi[5:7])) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(n_cached=table.view(-1)[2:4])) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(doc_first=ints(3))) == rc.RC_E_INVALID_ARG                       # documents without their starts
    with pytest.raises(ValueError):
        call(n_cached=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        call(n_new=ints(1, 1, 1))
    big = torch.zeros(65537, dtype=torch.int32)
    assert status(lambda: rc.rc_batch_map(big, big, torch.zeros((65537, 1), dtype=torch.int32), 16, 8, ints(0),
                                          rc.BatchRows.alloc(65537, 8, device="cpu"))) == rc.RC_E_CAPACITY


def test_norm_rotary_refusals():
    rot = rc.rc_rotary_init(rc.RC_ROTARY_HALF, 64, 1e4)
    kv = rc.PagedKV.contiguous(1, 1, 16, 2, 64, rc.RC_F32, device="cpu")
    q = torch.zeros((3, 4, 64))
    qkv = torch.zeros((3, 8 * 64 + 8))

    def call(qkv=qkv, n=3, hq=4, rot=rot, layer=kv.layer(0), q=q, pos=ints(0, 1, 2), **kw):
        rc.rc_norm_rotary_rows(qkv, n, hq, rot, pos, pos, layer, q, **kw)

    call(n=0)
    assert status(lambda: call(n=-1)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(hq=3)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(hq=8, q=torch.zeros((3, 8, 64)))) == rc.RC_E_INVALID_ARG                                    # rows shorter than the heads
    assert status(lambda: call(eps=-1.0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(qkv=torch.zeros((3, 8 * 64 + 6)))) == rc.RC_E_UNSUPPORTED        # stride
    assert status(lambda: call(qkv=torch.zeros(3 * 520 + 1)[1:].view(3, 520))) == rc.RC_E_UNSUPPORTED   # alignment
    assert status(lambda: call(rot=rc.rc_rotary_init(rc.RC_ROTARY_HALF, 128, 1e4))) == rc.RC_E_UNSUPPORTED
    bf = rc.PagedKV.contiguous(1, 1, 16, 2, 64, rc.RC_BF16, device="cpu")
    assert status(lambda: call(layer=bf.layer(0), q=q.bfloat16())) == rc.RC_E_UNSUPPORTED       # bf16 needs heads of 128
    with pytest.raises(ValueError):
        call(pos=ints(0, 1))
    with pytest.raises(ValueError):
        call(q=q[:2])
    with pytest.raises(ValueError):
        call(g_q=torch.ones(64, dtype=torch.bfloat16))
    both = torch.zeros(3 * 520 + 512)                                                           # queries over projections
    assert status(lambda: call(qkv=both[:3 * 520].view(3, 520), q=both[3 * 520 - 256:].view(3, 4, 64)[:3])) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(k_pre=kv.k[0])) == rc.RC_E_INVALID_ARG


def test_rotary_move_refusals():
    rot = rc.rc_rotary_init(rc.RC_ROTARY_INTERLEAVED, 32, 1e4)
    a = rc.PagedKV.contiguous(1, 1, 16, 2, 64, rc.RC_F32, device="cpu")
    b = rc.PagedKV.contiguous(1, 1, 16, 1, 64, rc.RC_F32, device="cpu")
    i = ints(0, 1)

    def call(src=a, dst=a, n=2, rot=rot):
        rc.rc_rotary_move(src.layer(0), i, dst.layer(0), i, n, rot, i)

    call(n=0)
    assert status(lambda: call(n=-1)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(dst=b)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(rot=rc.rc_rotary())) == rc.RC_E_INVALID_ARG
    with pytest.raises(ValueError):
        call(n=3)


def test_masked_attention_refusals():
    kv = rc.PagedKV(1, 8, 4, 1, 64, rc.RC_F32, [[0, 1], [2, 3]], device="cpu")
    starts, pos = ints(0, 2, 4), ints(0, 1, 0, 1)

    def call(hq=2, q=None, out=None, layer=kv.layer(0), ws=None, starts=starts, **kw):
        q = torch.zeros((4, max(hq, 1), 64)) if q is None else q
        out = torch.zeros_like(q) if out is None else out
        a = dict(n_rows=4, max_rows_per_seq=2, max_len=8)
        a.update(kw)
        rc.rc_masked_attention(q, rc.MaskedAttention(starts, pos, **a), hq, layer, out, ws)

    call(n_rows=0)
    assert status(lambda: call(hq=0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(max_len=0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(max_len=9)) == rc.RC_E_CAPACITY
    assert status(lambda: call(max_rows_per_seq=0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(n_rows=-1)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(cap=-1.0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(cap=math.inf)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(cap=math.nan)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(scale=-1.0)) == rc.RC_E_INVALID_ARG
    assert status(lambda: call(hq=129)) == rc.RC_E_UNSUPPORTED
    assert status(lambda: call(starts=ints(0, 1, 2, 4))) == rc.RC_E_CAPACITY                    # more sequences than the table has
    assert status(lambda: call(q=torch.zeros(4 * 128 + 1)[1:])) == rc.RC_E_UNSUPPORTED          # alignment
    bf = rc.PagedKV(1, 8, 4, 1, 128, rc.RC_BF16, [[0, 1], [2, 3]], device="cpu")
    q16 = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    assert status(lambda: call(q=q16, layer=bf.layer(0), cap=4097.0)) == rc.RC_E_UNSUPPORTED
    assert rc.lib.rc_masked_attention(None, None, 2, None, None, None, 0, None) == rc.RC_E_INVALID_ARG
    with pytest.raises(ValueError):
        call(q=torch.zeros((3, 2, 64)))
    with pytest.raises(ValueError):
        call(layer=bf.layer(0))
    with pytest.raises(ValueError):
        call(row_lo=ints(0))
    bad = torch.zeros(512, dtype=torch.uint8)
    off = (-bad.data_ptr()) % 256 + 16
    assert status(lambda: call(ws=bad[off:off + 128])) == rc.RC_E_WORKSPACE


def test_arrays_that_overlap_in_part():
    rot = rc.rc_rotary_init(rc.RC_ROTARY_HALF, 64, 1e4)
    kv = rc.PagedKV(1, 8, 4, 2, 64, rc.RC_F32, [[0, 1], [2, 3]], device="cpu")
    pos = ints(0, 1, 0, 1)
    for pool in (kv.k[0], kv.v[0]):
        assert status(lambda: rc.rc_norm_rotary_rows(torch.zeros((4, 512)), 4, 4, rot, pos, pos, kv.layer(0), torch.zeros((4, 4, 64)),
                                                     k_pre=pool.reshape(-1)[64:])) == rc.RC_E_INVALID_ARG
    both = torch.zeros(5, 4, 64)
    for q, out in ((both[1:], both[:4]), (both[:4], both[1:])):
        assert status(lambda: rc.rc_masked_attention(q, rc.MaskedAttention(ints(0, 2, 4), pos, 4, 2, 8), 4, kv.layer(0), out)) == rc.RC_E_INVALID_ARG
