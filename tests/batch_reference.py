"""Plain 64-bit statements of the calls for ragged batches, in loops over sequences and rows, on the CPU."""
import math

import numpy as np
import torch


def batch_map(cached, new, table, size, n_blocks, free, first=0, prefix=None, docs=None, max_rows=None):
    """docs: per sequence a list of first positions.  Returns the call's outputs as lists and changes `table` in place."""
    out = {n: [] for n in ("row_seq", "row_pos", "row_slot", "row_lo", "row_hi")}
    row_start, kv_len, at, taken, refused = [0], [], first, first, 0
    full = False
    for s, (c, n) in enumerate(zip(cached, new)):
        c, n = max(c, 0), max(n, 0)
        have, want = -(-c // size), -(-(c + n) // size)
        fits = c + n <= len(table[s]) * size
        need = want - have if fits else 0
        listed = need == 0 or at + need <= len(free)
        roomy = max_rows is None or row_start[-1] + n <= max_rows
        served = fits and listed and roomy and not (full and need)
        if served and need:
            for i in range(need):
                table[s][have + i] = free[at + i]
            taken = at + need
        full = full or (fits and need > 0 and not listed)
        at += need
        kv_len.append(c + n if served else c)
        refused += not served
        for i in range(n):
            if max_rows is not None and row_start[-1] + i >= max_rows:
                break
            p, slot, lo, hi = c + i, -1, 0, -1
            if served:
                b = table[s][p // size]
                slot = b * size + p % size if 0 <= b < n_blocks else -1
                marks = docs[s] if docs else []
                lo = max([d for d in marks if d <= p], default=0)
                end = min([d for d in marks if d > p], default=c + n)
                hi = min(max(p, (prefix[s] if prefix else 0) - 1), end - 1)
            for name, x in zip(out, (s, p, slot, lo, hi)):
                out[name].append(x)
        row_start.append(min(row_start[-1] + n, max_rows if max_rows is not None else 1 << 62))
    out.update(row_start=row_start, kv_len=kv_len, counts=[row_start[-1], taken, refused])
    return out


def frequencies(rotary_dim, base, scaling="plain", factor=1.0, trained=0, slow=1.0, fast=32.0):
    out = []
    for i in range(rotary_dim // 2):
        f = base ** (-2.0 * i / rotary_dim)
        keep = 1.0
        if scaling == "linear":
            keep = 0.0
        elif scaling == "turns":
            keep = min(max((trained * f / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0)
        elif scaling == "pairs":
            lo, hi = (rotary_dim * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (fast, slow))
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rotary_dim // 2 - 1)
            keep = 1 - min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
        out.append(f * keep + f / factor * (1 - keep))
    return np.array(out)


def rotate(x, pos, freq, layout, amplitude=1.0):
    """x [rows][heads][dh] float64 (numpy), pos [rows]; also the bound |a| + |b| of each element's pair."""
    y, size = x.copy(), np.abs(x)
    r = 2 * len(freq)
    ia, ib = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = (x[..., ia] + 1j * x[..., ib]) * (amplitude * np.exp(1j * np.asarray(pos, np.float64)[:, None] * freq))[:, None]
    y[..., ia], y[..., ib] = z.real, z.imag
    both = (np.abs(x[..., ia]) + np.abs(x[..., ib])) * max(amplitude, 1.0)
    size[..., ia], size[..., ib] = both, both
    return y, size


def head_norm(x, gain, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def attention(q, k, v, pos, lo, hi, scale, cap=0.0, slopes=None):
    """One sequence: q [rows][Hq][dh], k and v [keys][Hkv][dh], float64 numpy.  Returns (out, mass, size): mass is sum p |v| / sum p, size the
    largest sum of |q_d k_d| times scale over a row's keys (what rounding errors of scores are relative to)."""
    n, hq, dh = q.shape
    g = hq // k.shape[1]
    out, mass, size = np.zeros_like(q), np.zeros_like(q), np.zeros((n, hq, 1))
    for i in range(n):
        a, b = max(int(lo[i]), 0), min(int(hi[i]), len(k) - 1)
        if a > b:
            continue
        for h in range(hq):
            kk, vv = k[a:b + 1, h // g], v[a:b + 1, h // g]
            with np.errstate(invalid="ignore", over="ignore"):
                x = kk @ q[i, h] * scale
                size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * abs(scale)
                if cap:
                    x = cap * np.tanh(x / cap)
                if slopes is not None:
                    x = x - slopes[h] * np.abs(pos[i] - np.arange(a, b + 1))
                p = np.exp(x - x.max())
                out[i, h], mass[i, h] = p @ vv / p.sum(), p @ np.abs(vv) / p.sum()
    return out, mass, size


def step_of(dtype):
    """Half a rounding step of a type, relative to the value."""
    return torch.finfo(dtype).eps / 2
