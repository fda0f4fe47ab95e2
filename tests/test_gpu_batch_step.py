"""The calls for ragged batches one behind the other, as a program uses them: lengths to tables and slots, projections to queries and cache rows,
attention, decoding steps, and another agent's rows taken over from the un-rotated keys."""
import numpy as np
import pytest
import torch

from paper_2603_13289_amd import binding as rc
from tests import batch_reference as ref

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


class Program:
    """One layer's cache of up to n_seq sequences and what the program holds beside it: lengths, free blocks, the rows' projections (for the statement)."""

    def __init__(self, dtype, hq, hkv, dh, n_seq, size, width, layout, part, cap, bias):
        self.code = rc.RC_BF16 if dtype == "bf16" else rc.RC_F32
        self.td, self.hq, self.hkv, self.dh, self.size, self.n_seq, self.cap = rc.torch_dtype(self.code), hq, hkv, dh, size, n_seq, cap
        self.rng = np.random.default_rng(11)
        self.n_blocks = n_seq * width + 5
        self.free = ints(self.rng.permutation(self.n_blocks))
        self.first = ints([0])
        self.kv = rc.PagedKV(1, self.n_blocks, size, hkv, dh, self.code, np.full((n_seq, width), -1).tolist(), fill=float("nan"))
        self.k_pre = torch.full_like(self.kv.k[0], float("nan"))
        self.pre = rc.PagedKV.from_pools([self.k_pre], self.kv.v, self.kv.block_table, self.code)
        self.cached = ints([0] * n_seq)
        self.rotary = rc.rc_rotary_init(rc.RC_ROTARY_HALF if layout == "half" else rc.RC_ROTARY_INTERLEAVED, dh // part, 1e4,
                                        scaling=rc.RC_ROTARY_BY_TURNS, factor=8.0, trained_len=64, slow_turns=1.0, fast_turns=4.0)
        self.freq, self.layout = ref.frequencies(dh // part, 1e4, "turns", factor=8.0, trained=64, slow=1.0, fast=4.0), layout
        self.gq, self.gk = (torch.from_numpy(1 + 0.2 * self.rng.standard_normal(dh)).to(self.td) for _ in range(2))
        self.slope = 2.0 ** (-8.0 * (np.arange(hq) + 1) / hq) if bias else None
        self.slopes = torch.tensor(self.slope, dtype=torch.float32, device="cuda") if bias else None
        self.k_ref, self.v_ref = [[] for _ in range(n_seq)], [[] for _ in range(n_seq)]     # un-rotated keys, values
        self.slots = [[] for _ in range(n_seq)]

    def map(self, new, spare=0):
        rows = rc.BatchRows.alloc(self.n_seq, sum(new) + spare)
        rc.rc_batch_map(self.cached, ints(new), self.kv.block_table, self.size, self.n_blocks, self.free, rows, free_first=self.first)
        return rows

    def advance(self, rows, new):
        self.cached.copy_(rows.kv_len)
        self.first.copy_(rows.counts[1:2])
        assert rows.counts[2].item() == 0
        for s in range(self.n_seq):
            a, b = rows.row_start[s].item(), rows.row_start[s + 1].item()
            self.slots[s] += rows.row_slot[a:b].tolist()

    def project(self, rows, new, spare=0, from_row=None, to_row=None):
        """Random projections of the rows; queries and cache rows from them.  from_row, to_row: of which rows (all)."""
        n = sum(new)
        a, b = from_row or 0, n if to_row is None else to_row
        x = torch.from_numpy(self.rng.standard_normal((b - a + spare, (self.hq + 2 * self.hkv) * self.dh)).astype(np.float32))
        q = torch.full((b - a + spare, self.hq, self.dh), float("nan"), dtype=self.td, device="cuda")
        live = rows.row_start[self.n_seq:] if spare else None
        rc.rc_norm_rotary_rows(x.cuda(), b - a + spare, self.hq, self.rotary, rows.row_pos[a:], rows.row_slot[a:], self.kv.layer(0), q, g_q=self.gq.cuda(),
                               g_k=self.gk.cuda(), k_pre=self.k_pre, n_live=live)
        h = x[:b - a].double().numpy().reshape(b - a, -1, self.dh)
        seq = rows.row_seq[a:b].tolist()
        k = ref.head_norm(h[:, self.hq:self.hq + self.hkv], self.gk.double().numpy(), 1e-5)
        for i, s in enumerate(seq):
            self.k_ref[s].append(k[i])
            self.v_ref[s].append(h[i, self.hq + self.hkv:])
        qn = ref.head_norm(h[:, :self.hq], self.gq.double().numpy(), 1e-5)
        return q, ref.rotate(qn, rows.row_pos[a:b].tolist(), self.freq, self.layout)[0]

    def attend(self, rows, new, q, q_ref, spare=0, starts=None, a=0, most=None):
        """Attention of the rows from a on, against the statement on this program's own 64-bit rows."""
        n = q_ref.shape[0]
        out = torch.full_like(q, 3.0)
        plan = rc.MaskedAttention(rows.row_start if starts is None else starts, rows.row_pos[a:], n + spare, most or max(new), max(self.cached.tolist()),
                                  row_lo=rows.row_lo[a:], row_hi=rows.row_hi[a:], slopes=self.slopes, cap=self.cap)
        layer = self.kv.layer(0)
        ws = rc.alloc_workspace(rc.rc_masked_attention_workspace_bytes(plan, self.hq, layer))
        rc.rc_masked_attention(q, plan, self.hq, layer, out, ws)
        got = out.double().cpu().numpy()
        assert (got[n:] == 3.0).all()
        half = ref.step_of(self.td)
        u = 2.0 ** -24
        for i in range(n):
            s, p = rows.row_seq[a + i].item(), rows.row_pos[a + i].item()
            k = ref.rotate(np.array(self.k_ref[s]), np.arange(len(self.k_ref[s])), self.freq, self.layout)[0]
            want, mass, size = ref.attention(q_ref[i:i + 1], k, np.array(self.v_ref[s]), [p], [0], [p], self.dh ** -0.5, self.cap, self.slope)
            # a query, a key and (moved rows) its un-rotated form are rounded to the type, each worth half a step of the score's absolute sum; a key's rotation
            # adds up two elements (a factor of sqrt 2 of it); 32-bit steps of norm, rotation and sum: 200
            d = (4.5 * half + 200 * u) * size + 8 * u * self.cap + (2 * u * p if self.slope is not None else 0.0)
            bound = (2 * half + 2 * d + 4096 * u) * mass + 2 * half * np.abs(want) + 1e-30
            assert (np.abs(got[i:i + 1] - want) <= bound).all(), (s, p, float((np.abs(got[i:i + 1] - want) - bound).max()))


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("size,layout,part,cap,bias", [(16, "half", 1, 0.0, True), (24, "interleaved", 2, 20.0, False), (1, "half", 4, 5.0, True)])
def test_prompts_tokens_and_a_take_over(dtype, hq, hkv, dh, size, layout, part, cap, bias):
    g = Program(dtype, hq, hkv, dh, 4, size, -(-160 // size), layout, part, cap, bias)
    new = [70, 1, 33, 0]                                       # prompts; the fourth sequence comes later
    rows = g.map(new)
    q, q_ref = g.project(rows, new)
    g.advance(rows, new)
    g.attend(rows, new, q, q_ref)
    for step in range(3):                                      # a token each, arrays with room for more rows
        new = [1, 1, 1, 0]
        rows = g.map(new, spare=2)
        q, q_ref = g.project(rows, new, spare=2)
        g.advance(rows, new)
        g.attend(rows, new, q, q_ref, spare=2)
    # the fourth agent: rows 20 .. 59 of the first one's cache behind nothing, then eight rows of its own
    new = [0, 0, 0, 48]
    rows = g.map(new)
    taken = g.slots[0][20:60]
    rc.rc_rotary_move(g.pre.layer(0), ints(taken), g.kv.layer(0), rows.row_slot[:40], 40, g.rotary, rows.row_pos[:40])
    g.k_ref[3], g.v_ref[3] = g.k_ref[0][20:60], g.v_ref[0][20:60]
    q, q_ref = g.project(rows, new, from_row=40)
    g.advance(rows, new)
    g.attend(rows, new, q, q_ref, starts=ints([0, 0, 0, 0, 8]), a=40, most=8)
    # and the other way: its rotated keys to the positions that follow the second agent's rows
    new = [0, 11, 0, 0]
    rows = g.map(new)
    at = g.cached[1].item()
    rc.rc_rotary_move(g.kv.layer(0), ints(g.slots[3][37:47]), g.kv.layer(0), rows.row_slot[:10], 10, g.rotary, rows.row_pos[:10], old_pos=ints(range(37, 47)))
    g.k_ref[1] += g.k_ref[3][37:47]
    g.v_ref[1] += g.v_ref[3][37:47]
    q, q_ref = g.project(rows, new, from_row=10)
    g.advance(rows, new)
    assert g.cached.tolist() == [73, at + 11, 36, 48]
    g.attend(rows, new, q, q_ref, starts=ints([0, 0, 1, 1, 1]), a=10, most=1)
