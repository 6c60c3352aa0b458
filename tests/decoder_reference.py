"""Plain CPU forms of the decoder's attention operators: 64-bit arithmetic on the inputs' exact values, loops over
sequences and heads, nothing shared with the kernels."""
import math

import torch

LARGEST = {"i8": 127.0, "e4m3": 448.0}
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def bits8(t):
    return t.view(torch.int8)


def r32(x):
    """A 64-bit value rounded to binary32 (one operation on binary32 operands, done in 64 bits, rounds the same way)."""
    return x.to(torch.float32).to(torch.float64)


def to_eight(x, cache):
    """64-bit values to the nearest number of the 8-bit type, ties to even, saturated."""
    top = LARGEST[cache]
    if cache == "i8":
        return torch.round(x).clamp(-top, top).to(torch.int8)
    mag = x.abs().clamp(max=top)
    step = torch.exp2(torch.floor(torch.log2(mag.clamp(min=2.0 ** -6))) - 3)
    return torch.copysign(torch.round(mag / step) * step, x).to(torch.float8_e4m3fn)      # (a zero keeps its sign)


def append(k, v, ks, vs, table, new_k, new_v, start, count):
    """The cache after an append: new tensors.  new_k, new_v [batch, T, heads, d]; start, count: lists."""
    k, v, ks, vs = k.clone(), v.clone(), ks.clone(), vs.clone()
    cache = "i8" if k.dtype == torch.int8 else "e4m3"
    blocks, heads, bt, d = k.shape
    step = r32(torch.tensor(1.0 / LARGEST[cache], dtype=torch.float64))
    for b in range(table.shape[0]):
        s0 = max(0, start[b])
        n = min(max(0, count[b]), new_k.shape[1])
        for col in range(s0 // bt, min(table.shape[1], (s0 + n + bt - 1) // bt)):
            lo, hi = max(s0, col * bt), min(s0 + n, (col + 1) * bt)
            bid = int(table[b, col])
            if lo >= hi or not 0 <= bid < blocks:
                continue
            for pool, scale, new, transposed in ((k, ks, new_k, False), (v, vs, new_v, True)):
                x = torch.nan_to_num(new[b, lo - s0:hi - s0].to(torch.float32)).double().transpose(0, 1)          # [heads, tokens, d]
                held = lo - col * bt
                was = scale[bid].double() if held else torch.zeros(heads, dtype=torch.float64)
                now = torch.maximum(was, r32(x.abs().amax((1, 2)) * step).clamp(min=2.0 ** -64))
                inv = r32(1.0 / now)
                tile = pool[bid].transpose(1, 2) if transposed else pool[bid]                                     # [heads, bt, d]
                if held:
                    tile[:, :held] = to_eight(r32(tile[:, :held].double() * r32(was * inv)[:, None, None]), cache)
                tile[:, held:held + hi - lo] = to_eight(r32(x * inv[:, None, None]), cache)
                scale[bid] = now.float()
    return k, v, ks, vs


def softmax_rows(q, k, v, scale, allowed):
    """(o, T, lse, p) of one head's rows: row i sees the keys j with allowed[i, j]; T = sum_j p_j |v_j|.  A row that sees none: zeros, -inf."""
    w = q.double() @ k.double().T * scale
    w = torch.where(allowed, w, -math.inf)
    top = w.amax(1, keepdim=True) if k.shape[0] else torch.full((q.shape[0], 1), -math.inf, dtype=torch.float64)
    e = torch.where(allowed, torch.exp(w - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = e.sum(1, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    lse = (torch.where(top == -math.inf, 0.0, top) + torch.log(total)).squeeze(1)
    v = torch.where(allowed.any(0)[:, None], v.double(), 0.0)
    return p @ v, p @ v.abs(), lse, p


def cache_attention(q, k, v, ks, vs, table, lens, count, scale):
    """(o, T) [batch, T, Hq, d] in 64 bits, NaN in the rows that are left as they were."""
    batch, T, hq, d = q.shape
    blocks, heads, bt, _ = k.shape
    g = hq // heads
    o = torch.full((batch, T, hq, d), math.nan, dtype=torch.float64)
    tt = torch.zeros_like(o)
    cap = table.shape[1] * bt
    for b in range(batch):
        n = min(max(0, lens[b]), cap)
        c = min(max(0, count[b]), T)
        ids = [int(x) for x in table[b, :-(-n // bt)]]
        there = torch.tensor([0 <= i < blocks for i in ids], dtype=torch.bool).repeat_interleave(bt)[:n]
        ids = torch.tensor([i if 0 <= i < blocks else 0 for i in ids], dtype=torch.long)
        last = n - c + torch.arange(c)
        for h in range(heads):
            kk = (k[ids, h].double() * ks[ids, h].double()[:, None, None]).reshape(-1, d)[:n]
            vv = (v[ids, h].double() * vs[ids, h].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[:n]
            kk, vv = torch.where(there[:, None], kk, 0.0), torch.where(there[:, None], vv, 0.0)
            allowed = (torch.arange(n)[None, :] <= last[:, None]) & there[None, :]
            for j in range(h * g, (h + 1) * g):
                if c:
                    o[b, :c, j], tt[b, :c, j], _, _ = softmax_rows(q[b, :c, j], kk, vv, scale, allowed)
    return o, tt


def cross_attention(q, k, v, lens, scale, do=None):
    """o, T [batch, M, Hq, d] and lse [batch, Hq, M] in 64 bits; with do also dq, dk, dv and, for each, the sum of the magnitudes that its
    last product adds up."""
    batch, m, hq, d = q.shape
    n, heads = k.shape[1], k.shape[2]
    g = hq // heads
    f64 = dict(dtype=torch.float64)
    r = {"o": torch.zeros(q.shape, **f64), "T": torch.zeros(q.shape, **f64), "lse": torch.zeros((batch, hq, m), **f64)}
    if do is not None:
        r.update({x: torch.zeros(y.shape, **f64) for x, y in (("dq", q), ("dk", k), ("dv", v), ("dq_sum", q), ("dk_sum", k), ("dv_sum", v))})
    for b in range(batch):
        nb = n if lens is None else min(max(0, lens[b]), n)
        for j in range(hq):
            h = j // g
            qq, kk, vv = q[b, :, j].double(), k[b, :nb, h].double(), v[b, :nb, h].double()
            allowed = torch.ones((m, nb), dtype=torch.bool)
            r["o"][b, :, j], r["T"][b, :, j], r["lse"][b, j], p = softmax_rows(qq, kk, vv, scale, allowed)
            if do is not None:
                go = do[b, :, j].double()
                dp = go @ vv.T
                mean = (p * dp).sum(1, keepdim=True)
                ds = p * (dp - mean) * scale
                # magnitudes: what a rounding of p, dp or the mean is relative to
                mag = p * (go.abs() @ vv.abs().T + (p * (go.abs() @ vv.abs().T)).sum(1, keepdim=True)) * abs(scale)
                r["dq"][b, :, j] = ds @ kk
                r["dq_sum"][b, :, j] = mag @ kk.abs()
                r["dk"][b, :nb, h] += ds.T @ qq
                r["dk_sum"][b, :nb, h] += mag.T @ qq.abs()
                r["dv"][b, :nb, h] += p.T @ go
                r["dv_sum"][b, :nb, h] += p.T @ go.abs()
    return r
