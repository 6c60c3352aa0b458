"""The two attentions of a decoder layer, as a serving or training program calls them.

  append   tir_cache_append: new tokens' keys and values into a paged cache of 8-bit values with one scale per block of
           tokens and head
  cached   tir_cache_attention: the new tokens' queries over that cache, each up to its own position
  cross    tir_cross_attention: a decoder's queries over an encoder's states of another length
  grad     tir_cross_attention_backward: the gradients of that with respect to queries, keys and values

With `own` false, run() computes the operators from elementary torch operations in 32 bits; with `own` true it calls the
library.  The definitions are those of include/tir.h.
"""
import math

import torch

own = False

_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
_LARGEST = {"i8": 127.0, "e4m3": 448.0}
_MIN_SCALE = 2.0 ** -64
_workspaces = {}


# ------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoding step's new token of 32 sequences, 8 key heads: nothing but latency
        dict(name="append_token_i8", kind="append", batch=32, new=1, held=1500, heads=8, d=128, block=64, dtype="f16", cache="i8"),
        # prompts of eight sequences written into an empty cache, not one of them whole blocks long
        dict(name="append_prompt_e4m3", kind="append", batch=8, new=2039, held=0, heads=8, d=128, block=32, dtype="bf16", cache="e4m3"),
        # one token of one short conversation: the smallest call of a decoding loop
        dict(name="cached_token_short", kind="cached", batch=1, new=1, longest=777, shortest=777, heads=8, group=1, d=64, block=16, dtype="f16", cache="i8"),
        # decoding 64 sequences of 4 to 8 thousand tokens, four query heads per key head
        dict(name="cached_token_batch", kind="cached", batch=64, new=1, longest=8190, shortest=4001, heads=8, group=4, d=128, block=64, dtype="bf16", cache="i8"),
        # one token over one very long context: all of the chip on eight key heads
        dict(name="cached_token_long", kind="cached", batch=1, new=1, longest=200003, shortest=200003, heads=8, group=4, d=128, block=128, dtype="f16", cache="e4m3"),
        # the next piece of four prompts, 500-odd tokens behind 3500 that the cache holds
        dict(name="cached_piece_e4m3", kind="cached", batch=4, new=509, longest=4096, shortest=3301, heads=8, group=4, d=128, block=32, dtype="f16", cache="e4m3"),
        # one token of eight sequences over 1500 encoder states (a speech encoder's half minute)
        dict(name="cross_token_f16", kind="cross", batch=8, m=1, n=1500, heads=16, group=1, d=64, ragged=False, lse=False, dtype="f16"),
        # an image's 64 x 64 positions over 77 text states
        dict(name="cross_image_bf16", kind="cross", batch=4, m=4096, n=77, heads=8, group=1, d=64, ragged=False, lse=False, dtype="bf16"),
        # long targets over long sources of ragged lengths, shared key heads, kept for training
        dict(name="cross_long_bf16", kind="cross", batch=2, m=2047, n=4095, heads=4, group=4, d=128, ragged=True, lse=True, dtype="bf16"),
        # gradients of a translation batch: 12 heads of 64
        dict(name="grad_batch_f16", kind="grad", batch=16, m=250, n=333, heads=12, group=1, d=64, ragged=True, dtype="f16"),
        # gradients for an image's positions over 77 text states: few keys, many queries
        dict(name="grad_image_bf16", kind="grad", batch=4, m=4096, n=77, heads=8, group=1, d=64, ragged=False, dtype="bf16"),
        # gradients of the long case
        dict(name="grad_long_bf16", kind="grad", batch=2, m=2047, n=4095, heads=4, group=4, d=128, ragged=True, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw_once(rng):
    kind = rng.choice(["append", "cached", "cached", "cross", "cross", "grad", "grad"])
    dtype = rng.choice(["f16", "bf16"])
    d = rng.choice([64, 128])
    if kind == "append":
        return dict(kind=kind, batch=_log_int(rng, 1, 64), new=_log_int(rng, 1, 4096) if rng.random() < 0.6 else 1, held=rng.randint(0, 2000), heads=_log_int(rng, 1, 16), d=d,
                    block=rng.choice([16, 32, 64, 128]), dtype=dtype, cache=rng.choice(["i8", "e4m3"]))
    heads, group = _log_int(rng, 1, 16), rng.choice([1, 1, 2, 3, 4, 8])
    if kind == "cached":
        longest = _log_int(rng, 1, 200000)
        shortest = rng.randint(max(0, longest // 4), longest)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 1000)
        return dict(kind=kind, batch=_log_int(rng, 1, 64), new=min(new, max(1, shortest)), longest=longest, shortest=shortest, heads=heads, group=group, d=d,
                    block=rng.choice([16, 32, 64, 128]), dtype=dtype, cache=rng.choice(["i8", "e4m3"]))
    case = dict(kind=kind, batch=_log_int(rng, 1, 32), m=_log_int(rng, 1, 4096), n=_log_int(rng, 1, 4096), heads=heads, group=group, d=d, ragged=rng.random() < 0.5, dtype=dtype)
    if kind == "cross":
        case["lse"] = rng.random() < 0.5
    return case


def draw(rng):
    most = [work(c) for c in listed()]
    while True:
        case = _draw_once(rng)
        w = work(case)
        rows = case["batch"] * case["heads"] * case.get("group", 1)
        scores = rows * case["new"] * case["longest"] if case["kind"] == "cached" else rows * case["m"] * case["n"] if "m" in case else 0
        if w["bytes"] <= max(x["bytes"] for x in most) and w["flops"] <= max(x["flops"] for x in most) and scores <= 3e8:
            return case


def _spread(lo, hi, n):
    """n whole numbers evenly from hi down to lo."""
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _counts(case):
    """New tokens per sequence: ragged where there is more than one."""
    return _spread((case["new"] + 1) // 2, case["new"], case["batch"])


def _held(case):
    return _spread(case["held"] // 2, case["held"], case["batch"])


def _keys(case):
    """Encoder states per sequence; the shortest sequence of a ragged batch may be a third of the longest."""
    return _spread(case["n"] // 3, case["n"], case["batch"]) if case["ragged"] else [case["n"]] * case["batch"]


def work(case):
    d, heads, batch = case["d"], case["heads"], case["batch"]
    if case["kind"] == "append":
        new = sum(_counts(case)) * heads * d * 2
        blocks = sum((h + c - 1) // case["block"] - h // case["block"] + 1 for h, c in zip(_held(case), _counts(case)))
        return {"bytes": new * 3 + blocks * heads * 16 + batch * 8, "flops": new * 2}
    if case["kind"] == "cached":
        lens = _spread(case["shortest"], case["longest"], batch)
        pairs = sum(c * n - c * (c - 1) // 2 for c, n in zip(_counts(case), lens)) * heads * case["group"]
        kv = sum(lens) * heads * d * 2 + sum(-(-n // case["block"]) for n in lens) * (heads * 8 + 4)
        return {"bytes": kv + sum(_counts(case)) * heads * case["group"] * d * 4 + batch * 8, "flops": 4 * pairs * d}
    q = batch * case["m"] * heads * case["group"] * d * 2
    keys = sum(_keys(case))
    pairs = keys * case["m"] * heads * case["group"]
    kv = keys * heads * d * 4
    rows = batch * case["m"] * heads * case["group"] * 4
    if case["kind"] == "cross":
        return {"bytes": 2 * q + kv + (rows if case["lse"] else 0), "flops": 4 * pairs * d}
    return {"bytes": 4 * q + kv + batch * case["n"] * heads * d * 4 + rows, "flops": 10 * pairs * d}


# ------------------------------------------------------------------------------------------------- inputs
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)


def _randn(g, shape, dtype):
    return torch.randn(shape, device="cuda", generator=g).to(dtype)


def _pool(g, case, blocks):
    """A cache's pool with values as quantised ones are spread, and the blocks of each sequence in no order."""
    h, d, t = case["heads"], case["d"], case["block"]
    top = _LARGEST[case["cache"]]

    def eight(shape):
        out = torch.empty(shape, dtype=_TORCH[case["cache"]], device="cuda")
        for part in out.split(max(1, (1 << 27) // (h * d * t))):
            x = (torch.randn(part.shape, device="cuda", generator=g) * (top / 3.5)).clamp_(-top, top)
            part.copy_(x.round_() if case["cache"] == "i8" else x)
        return out

    def scales():
        return (torch.rand((blocks, h), device="cuda", generator=g) + 0.5) * (3.5 / top)

    return {"k": eight((blocks, h, t, d)), "v": eight((blocks, h, d, t)), "k_scale": scales(), "v_scale": scales()}


def _table(g, lens, block, cols):
    """int32 [batch, cols]: each sequence's blocks from a permutation of the pool, -1 behind them; and the pool's size."""
    need = [-(-n // block) for n in lens]
    perm = torch.randperm(sum(need) + 2, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), cols), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, sum(need) + 2


def _register_workspace():
    """The split-reduction workspace of the current stream, registered once as a program does when it starts."""
    from paper_2207_04296_amd import binding as B
    st = torch.cuda.current_stream()
    if st.cuda_stream not in _workspaces:
        _workspaces[st.cuda_stream] = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
        B.tir_set_workspace(_workspaces[st.cuda_stream], st)


def prepare(case, seed):
    g = _gen(seed)
    t = _TORCH[case["dtype"]]
    s = {"case": dict(case)}
    batch, heads, d = case["batch"], case["heads"], case["d"]
    if own:
        _register_workspace()
    if case["kind"] in ("append", "cached"):
        counts = _counts(case)
        if case["kind"] == "append":
            before = _held(case)
            lens = [h + c for h, c in zip(before, counts)]
            s["start"] = _ints(before)
        else:
            lens = _spread(case["shortest"], case["longest"], batch)
        s["table"], blocks = _table(g, lens, case["block"], -(-max(lens) // case["block"]) + 1)
        s.update(_pool(g, case, blocks))
        s["lens"] = _ints(lens)
        s["counts"] = _ints(counts) if case["new"] > 1 else None
    if case["kind"] == "append":
        # keys and values as one projection gives them
        kv = _randn(g, (batch, case["new"], 2, heads, d), t)
        s["new_k"], s["new_v"] = kv[:, :, 0], kv[:, :, 1]
    elif case["kind"] == "cached":
        s["q"] = _randn(g, (batch, case["new"], heads * case["group"], d), t)
        s["o"] = torch.zeros_like(s["q"])
    else:
        hq = heads * case["group"]
        s["q"] = _randn(g, (batch, case["m"], hq, d), t)
        kv = _randn(g, (batch, case["n"], 2, heads, d), t)
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        s["lens"] = _ints(_keys(case)) if case["ragged"] else None
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((batch, hq, case["m"]), dtype=torch.float32, device="cuda") if case.get("lse", True) else None
        if case["kind"] == "grad":
            # what the forward pass left, and the gradient that arrives
            s["o"], s["lse"] = _plain_cross(s, s["q"].dtype)
            s["do"] = _randn(g, s["q"].shape, t)
            s["dq"] = torch.empty_like(s["q"])
            s["dkv"] = torch.empty_like(kv)
            s["delta"] = torch.empty_like(s["lse"])
    if case["kind"] in ("append", "cached") and own:
        from paper_2207_04296_amd import binding as B
        s["cache"] = B.make_kv_cache(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"])
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _to_eight(x, inv, cache):
    """x * inv in the cache's 8 bits."""
    y = torch.nan_to_num(x) * inv
    top = _LARGEST[cache]
    return (torch.round(y).clamp(-top, top) if cache == "i8" else y.clamp(-top, top)).to(_TORCH[cache])


def _bytes_of(x):
    return x.view(torch.int8)


def _append_side(pool, scale, new, s, transposed):
    """One of keys and values: the touched blocks are read whole, changed and written back."""
    case = s["case"]
    t, cols = case["block"], s["table"].shape[1]
    start = s["start"].long()
    count = s["counts"].long() if s["counts"] is not None else torch.full_like(start, case["new"])
    touched = (case["new"] + t - 2) // t + 1
    col = (start // t)[:, None] + torch.arange(touched, device=start.device)                      # [batch, touched]
    written = col * t < (start + count)[:, None]
    written &= col < cols
    block = torch.gather(s["table"].long(), 1, col.clamp(max=cols - 1))
    spare = torch.gather(s["table"].long(), 1, (start // t)[:, None].clamp(max=cols - 1))
    block = torch.where(written, block, spare)
    pos = col[:, :, None] * t + torch.arange(t, device=start.device)                              # [batch, touched, t]
    tok = pos - start[:, None, None]
    fresh = (tok >= 0) & (tok < count[:, None, None]) & written[:, :, None]
    old = (tok < 0) & written[:, :, None]
    at = tok.clamp(0, case["new"] - 1)
    x = new.float()[torch.arange(new.shape[0], device=new.device)[:, None, None], at]             # [batch, touched, t, heads, d]
    x = torch.where(fresh[..., None, None], torch.nan_to_num(x), 0.0).permute(0, 1, 3, 2, 4)      # [batch, touched, heads, t, d]
    fresh, old = fresh[:, :, None, :, None], old[:, :, None, :, None]
    was = _bytes_of(pool)[block]
    was8 = was.view(_TORCH[case["cache"]])
    if transposed:
        x, fresh, old = x.transpose(3, 4), fresh.transpose(3, 4), old.transpose(3, 4)
    s_old = torch.where(old.flatten(2).any(2)[:, :, None], scale[block], 0.0)                     # [batch, touched, heads]
    # (a tensor by a number would be a division on some devices and a product with the reciprocal on others: the definition has the product)
    step = torch.tensor(1.0 / _LARGEST[case["cache"]], dtype=torch.float32, device=x.device)
    s_new = torch.maximum(s_old, (x.abs().amax((3, 4)) * step).clamp(min=_MIN_SCALE))
    inv = torch.ones_like(s_new) / s_new
    q_new = _bytes_of(_to_eight(x, inv[..., None, None], case["cache"]))
    q_old = _bytes_of(_to_eight(was8.float(), (s_old * inv)[..., None, None], case["cache"]))
    q = torch.where(fresh, q_new, torch.where(old, q_old, was))
    # a column that gets no token stands for the first one: write what that one gets
    first = torch.zeros_like(col)
    pick = torch.where(written, torch.arange(touched, device=col.device), first)
    rows = torch.arange(col.shape[0], device=col.device)[:, None]
    _bytes_of(pool)[block] = q[rows, pick]
    scale[block] = s_new[rows, pick]


def _plain_append(s):
    _append_side(s["k"], s["k_scale"], s["new_k"], s, False)
    _append_side(s["v"], s["v_scale"], s["new_v"], s, True)
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _softmax(scores, seen):
    """Softmax over the last axis of what is seen; rows that see nothing are zero.  And log(sum(exp))."""
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(scores - top)
    total = e.sum(-1, keepdim=True)
    return torch.where(total > 0, e / total, 0.0), (top + torch.log(total)).squeeze(-1)


def _plain_cached(s):
    case = s["case"]
    batch, new, h, g, d = case["batch"], case["new"], case["heads"], case["group"], case["d"]
    table = s["table"].long().clamp(min=0)
    k = (s["k"].float() * s["k_scale"][..., None, None])[table].transpose(1, 2).reshape(batch, h, -1, d)
    v = (s["v"].float() * s["v_scale"][..., None, None])[table].permute(0, 2, 1, 4, 3).reshape(batch, h, -1, d)
    lens = s["lens"].long()
    counts = s["counts"].long() if s["counts"] is not None else torch.full_like(lens, new)
    q = s["q"].float().view(batch, new, h, g, d).permute(0, 2, 3, 1, 4).reshape(batch, h, g * new, d)
    scores = (q @ k.transpose(2, 3)).view(batch, h, g, new, -1) * d ** -0.5
    last = (lens - counts)[:, None] + torch.arange(new, device=lens.device)                       # [batch, new]
    seen = torch.arange(k.shape[2], device=lens.device) <= last[:, None, None, :, None]
    # padded positions of a block may hold anything
    live = torch.arange(k.shape[2], device=lens.device) < lens[:, None]
    v = torch.where(live[:, None, :, None], v, 0.0)
    p, _ = _softmax(scores, seen)
    o = (p.view(batch, h, g * new, -1) @ v).view(batch, h, g, new, d).permute(0, 3, 1, 2, 4).reshape(batch, new, h * g, d)
    asked = torch.arange(new, device=lens.device) < counts[:, None]
    return torch.where(asked[:, :, None, None], o.to(s["o"].dtype), s["o"])


def _cross_parts(s):
    """q [batch, heads, group * m, d], k and v [batch, heads, n, d] in 32 bits, and what is seen."""
    case = s["case"]
    batch, m, h, g, d = case["batch"], case["m"], case["heads"], case["group"], case["d"]
    q = s["q"].float().view(batch, m, h, g, d).permute(0, 2, 3, 1, 4).reshape(batch, h, g * m, d)
    k, v = (x.float().transpose(1, 2).contiguous() for x in (s["k"], s["v"]))
    n = torch.arange(case["n"], device=q.device)
    seen = n < s["lens"].long()[:, None, None, None] if s["lens"] is not None else (n >= 0)[None, None, None]
    return q, k, v, seen


def _back(x, case):
    """[batch, heads, group * m, d] to [batch, m, query heads, d]."""
    return x.view(case["batch"], case["heads"], case["group"], case["m"], -1).permute(0, 3, 1, 2, 4).reshape(case["batch"], case["m"], case["heads"] * case["group"], -1)


def _plain_cross(s, dtype):
    case = s["case"]
    q, k, v, seen = _cross_parts(s)
    p, lse = _softmax((q @ k.transpose(2, 3)) * case["d"] ** -0.5, seen)
    return _back(p @ v, case).to(dtype), lse.view(case["batch"], case["heads"] * case["group"], case["m"])


def _plain_grad(s):
    case = s["case"]
    q, k, v, seen = _cross_parts(s)
    scale = case["d"] ** -0.5
    do = s["do"].float().view(case["batch"], case["m"], case["heads"], case["group"], case["d"]).permute(0, 2, 3, 1, 4).reshape(q.shape)
    p, _ = _softmax((q @ k.transpose(2, 3)) * scale, seen)
    dv = p.transpose(2, 3) @ do
    dp = do @ v.transpose(2, 3)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    t = s["q"].dtype
    return {"dq": _back(dq, case).to(t), "dk": dk.transpose(1, 2).to(t), "dv": dv.transpose(1, 2).to(t)}


# ------------------------------------------------------------------------------------------------- one pass
def _strides(x):
    return x.stride()[:3]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "append":
            return _plain_append(s)
        if kind == "cached":
            return {"o": _plain_cached(s)}
        if kind == "cross":
            o, lse = _plain_cross(s, s["q"].dtype)
            return {"o": o, "lse": lse} if case["lse"] else {"o": o}
        return _plain_grad(s)
    from paper_2207_04296_amd import binding as B
    dt, batch, heads, d = case["dtype"], case["batch"], case["heads"], case["d"]
    if kind == "append":
        B.tir_cache_append(s["cache"], s["new_k"], s["new_v"], s["start"], s["counts"], batch, case["new"], *_strides(s["new_k"]), *_strides(s["new_v"]), dt)
        return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    hq = heads * case["group"]
    if kind == "cached":
        B.tir_cache_attention(s["q"], s["cache"], s["o"], s["lens"], s["counts"], batch, case["new"], hq, *_strides(s["q"]), *_strides(s["o"]), d ** -0.5, dt, dt)
        return {"o": s["o"]}
    if kind == "cross":
        B.tir_cross_attention(s["q"], s["k"], s["v"], s["o"], s["lse"], s["lens"], batch, case["m"], case["n"], hq, heads, d,
                              *_strides(s["q"]), *_strides(s["k"]), *_strides(s["v"]), *_strides(s["o"]), d ** -0.5, dt, dt)
        return {"o": s["o"], "lse": s["lse"]} if case["lse"] else {"o": s["o"]}
    dk, dv = s["dkv"][:, :, 0], s["dkv"][:, :, 1]
    B.tir_cross_attention_backward(s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["lens"], s["dq"], dk, dv, s["delta"], batch, case["m"], case["n"], hq, heads, d,
                                   *_strides(s["q"]), *_strides(s["k"]), *_strides(s["v"]), *_strides(s["o"]), d ** -0.5, dt)
    return {"dq": s["dq"], "dk": dk, "dv": dv}


# ------------------------------------------------------------------------------------------------- in 64 bits
def _exact_eight(x, cache):
    if cache == "i8":
        return torch.round(x).clamp(-127, 127).to(torch.int8)
    # the nearest of the format's values, ties to the even one: steps of 2^-9 below 2^-6, of an eighth of the power of two above
    mag = x.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(mag.clamp(min=2.0 ** -6))) - 3)
    return (torch.sign(x) * torch.round(mag / step) * step).to(torch.float8_e4m3fn)


def _exact_append(s):
    """Sequence by sequence and block by block.  The definition's binary32 roundings (of scale, reciprocal, ratio and products) are made on 64-bit values."""
    case = s["case"]
    t, cache, cols = case["block"], case["cache"], s["table"].shape[1]
    r32 = lambda x: x.float().double()  # noqa: E731
    step = r32(torch.tensor(1.0 / _LARGEST[cache], dtype=torch.float64)).item()
    table, starts = s["table"].tolist(), s["start"].tolist()
    counts = s["counts"].tolist() if s["counts"] is not None else [case["new"]] * case["batch"]
    for b in range(case["batch"]):
        for col in range(starts[b] // t, min(cols, (starts[b] + counts[b] - 1) // t + 1)):
            lo, hi = max(starts[b], col * t), min(starts[b] + counts[b], (col + 1) * t)
            for pool, scale, new, axis in ((s["k"], s["k_scale"], s["new_k"], 1), (s["v"], s["v_scale"], s["new_v"], 2)):
                x = new[b, lo - starts[b]:hi - starts[b]].double().transpose(0, 1)               # [heads, tokens, d]
                blk = pool[table[b][col]]
                q = blk if axis == 1 else blk.transpose(1, 2)                                     # [heads, block, d]
                was = scale[table[b][col]].double() if lo > col * t else torch.zeros(case["heads"], dtype=torch.float64, device=x.device)
                now = torch.maximum(was, r32(x.abs().amax((1, 2)) * step).clamp(min=_MIN_SCALE))
                inv = r32(1.0 / now)
                held = lo - col * t
                if held:
                    q[:, :held] = _exact_eight(r32(q[:, :held].double() * r32(was * inv)[:, None, None]), cache)
                q[:, held:held + hi - lo] = _exact_eight(r32(x * inv[:, None, None]), cache)
                scale[table[b][col]] = now.float()
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double()}


def _exact_rows(q, k, v, scale, allowed):
    """Output and log-sum-exp of one head's queries over its keys; allowed: how many of the keys each query sees."""
    w = q.double() @ k.double().T * scale
    w = w.masked_fill(torch.arange(k.shape[0], device=q.device) >= allowed[:, None], -math.inf)
    lse = torch.logsumexp(w, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(w - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    return p, p @ v.double(), lse


def _exact_cached(s):
    case = s["case"]
    t, new, d = case["block"], case["new"], case["d"]
    out = s["o"].double()
    lens = s["lens"].tolist()
    counts = s["counts"].tolist() if s["counts"] is not None else [new] * case["batch"]
    for b in range(case["batch"]):
        ids = s["table"][b, :-(-lens[b] // t)].long()
        seen = (lens[b] - counts[b] + 1 + torch.arange(counts[b], device=out.device)).clamp(0, lens[b])
        for h in range(case["heads"]):
            k = (s["k"][ids, h].double() * s["k_scale"][ids, h].double()[:, None, None]).reshape(-1, d)[:lens[b]]
            v = (s["v"][ids, h].double() * s["v_scale"][ids, h].double()[:, None, None]).transpose(1, 2).reshape(-1, d)[:lens[b]]
            own_heads = slice(h * case["group"], (h + 1) * case["group"])
            q = s["q"][b, :counts[b], own_heads].reshape(-1, d)
            _, o, _ = _exact_rows(q, k, v, d ** -0.5, seen.repeat_interleave(case["group"]))
            out[b, :counts[b], own_heads] = o.view(counts[b], case["group"], d)
    return {"o": out}


def _exact_cross(s, grad):
    case = s["case"]
    g, d, scale = case["group"], case["d"], case["d"] ** -0.5
    f64 = dict(dtype=torch.float64, device=s["q"].device)
    o, lse = torch.zeros(s["q"].shape, **f64), torch.zeros((case["batch"], case["heads"] * g, case["m"]), **f64)
    dq, dk, dv = torch.zeros(s["q"].shape, **f64), torch.zeros(s["k"].shape, **f64), torch.zeros(s["v"].shape, **f64)
    lens = s["lens"].tolist() if s["lens"] is not None else [case["n"]] * case["batch"]
    for b in range(case["batch"]):
        for hq in range(case["heads"] * g):
            h, n = hq // g, lens[b]
            q, k, v = s["q"][b, :, hq], s["k"][b, :n, h], s["v"][b, :n, h]
            p, o[b, :, hq], lse[b, hq] = _exact_rows(q, k, v, scale, torch.full((case["m"],), n, device=q.device))
            if grad:
                go = s["do"][b, :, hq].double()
                w = go @ v.double().T
                w = scale * p * (w - (p * w).sum(1, keepdim=True))
                dq[b, :, hq] = w @ k.double()
                dk[b, :n, h] += w.T @ q.double()
                dv[b, :n, h] += p.T @ go
    if grad:
        return {"dq": dq, "dk": dk, "dv": dv}
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "cached":
        return _exact_cached(s)
    return _exact_cross(s, case["kind"] == "grad")
