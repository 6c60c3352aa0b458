"""Attention over another sequence's states and its gradients, against plain 64-bit forms.

Forward tolerances are those of tir.h: 2e-3 * T + 1e-5 (F16) and 6e-3 * T + 1e-5 (BF16) with T = sum_j p_j |v_j|, a 16-bit output's half
step of 2^-11 |o| or 2^-8 |o| on top; log-sum-exp to 1e-5 + 2^-22 * max|score|: the scores' fp32 products and sums, an exponential's and a logarithm's last bits."""
import sys

import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R

FAKE = 0x1000


def _say(msg):
    print(f"[case] {msg}", flush=True)
    sys.stdout.flush()


def _gen(seed):
    import torch
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------------------------------ refusals, on the host
def _forward(**over):
    a = dict(Q=FAKE, K=FAKE, V=FAKE, O=FAKE, lse=FAKE, lens=FAKE, batch=2, M=5, N=7, Hq=4, Hkv=2, d=64, q=(1280, 256, 64), k=(896, 128, 64), v=(896, 128, 64), o=(1280, 256, 64),
             scale=0.125, i="f16", out="f16")
    a.update(over)
    return B.tir_cross_attention_status(a["Q"], a["K"], a["V"], a["O"], a["lse"], a["lens"], a["batch"], a["M"], a["N"], a["Hq"], a["Hkv"], a["d"], *a["q"], *a["k"], *a["v"], *a["o"],
                                        a["scale"], a["i"], a["out"])


FAULTS = [
    (dict(Q=0), B.TIR_ERR_INVALID_ARG), (dict(K=0), B.TIR_ERR_INVALID_ARG), (dict(V=0), B.TIR_ERR_INVALID_ARG), (dict(O=0), B.TIR_ERR_INVALID_ARG),
    (dict(batch=-1), B.TIR_ERR_INVALID_ARG), (dict(M=-1), B.TIR_ERR_INVALID_ARG), (dict(N=-1), B.TIR_ERR_INVALID_ARG), (dict(Hkv=0), B.TIR_ERR_INVALID_ARG), (dict(Hkv=3), B.TIR_ERR_INVALID_ARG),
    (dict(scale=float("inf")), B.TIR_ERR_INVALID_ARG), (dict(i=17), B.TIR_ERR_INVALID_ARG), (dict(k=(896, -128, 64)), B.TIR_ERR_INVALID_ARG),
    (dict(d=80), B.TIR_ERR_UNSUPPORTED), (dict(i="i8"), B.TIR_ERR_UNSUPPORTED),
    (dict(M=2 ** 31), B.TIR_ERR_UNSUPPORTED), (dict(N=2 ** 31), B.TIR_ERR_UNSUPPORTED), (dict(M=2 ** 30, Hq=8, Hkv=1), B.TIR_ERR_UNSUPPORTED), (dict(batch=2 ** 30, M=200), B.TIR_ERR_UNSUPPORTED),
    (dict(k=(896, 2 ** 24, 64)), B.TIR_ERR_UNSUPPORTED),
    # more workgroups than a launch has room for: few rows, and many
    (dict(batch=2 ** 24, M=1, N=1), B.TIR_ERR_UNSUPPORTED), (dict(batch=2 ** 23, M=200, N=1), B.TIR_ERR_UNSUPPORTED),
    (dict(Q=FAKE + 8), B.TIR_ERR_ALIGNMENT), (dict(K=FAKE + 2), B.TIR_ERR_ALIGNMENT), (dict(v=(896, 132, 64)), B.TIR_ERR_ALIGNMENT), (dict(lens=FAKE + 2), B.TIR_ERR_ALIGNMENT), (dict(lse=FAKE + 1), B.TIR_ERR_ALIGNMENT),
]


@pytest.mark.parametrize("over,status", FAULTS + [
    (dict(o=(0, 256, 64)), B.TIR_ERR_INVALID_ARG), (dict(o=(1280, 0, 64)), B.TIR_ERR_INVALID_ARG), (dict(o=(1280, 256, 0)), B.TIR_ERR_INVALID_ARG), (dict(out="bf16"), B.TIR_ERR_UNSUPPORTED),
    (dict(out="i32"), B.TIR_ERR_UNSUPPORTED)])
def test_cross_attention_rejects_bad_arguments(over, status):
    assert _forward(**over) == status and B.last_error()


def test_nothing_to_do_needs_no_device():
    assert _forward(batch=0, Q=0) == B.TIR_OK and _forward(M=0) == B.TIR_OK and _forward(Hq=0) == B.TIR_OK


# ------------------------------------------------------------------------------------------------ on the device
MARK = 77.0


def _inputs(g, dtype, batch, m, n, heads, group, d, lens, poison=True):
    """q, and k and v as the slices of one projection; what lies behind a sequence's states is NaN and infinity."""
    import torch
    t = R.TORCH[dtype]
    q = torch.randn((batch, m, heads * group, d), generator=g).to(t)
    kv = torch.randn((batch, n, 2, heads, d), generator=g).to(t)
    if lens is not None and poison:
        for b, x in enumerate(lens):
            kv[b, min(max(0, x), n):, 0] = float("nan")
            kv[b, min(max(0, x), n):, 1] = float("inf")
    return q, kv


def _to_device(x):
    import torch
    return x.cuda() if 0 in x.stride() else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").copy_(x)


def _run(q, kv, lens, scale, dtype, out, want_lse=True, stream=None, o=None):
    import torch
    qd, kvd = _to_device(q), _to_device(kv)
    k, v = kvd[:, :, 0], kvd[:, :, 1]
    batch, m, hq, d = q.shape
    o = torch.full(q.shape, MARK, dtype=R.TORCH[out], device="cuda") if o is None else o
    lse = torch.full((batch, hq, m), MARK, device="cuda") if want_lse else None
    ld = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    B.tir_cross_attention(qd, k, v, o, lse, ld, batch, m, k.shape[1], hq, k.shape[2], d, *qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3], scale, dtype, out, stream)
    torch.cuda.synchronize()
    return o.cpu(), None if lse is None else lse.cpu()


def _tolerance(T, ref, dtype, out):
    return (2e-3 if dtype == "f16" else 6e-3) * T + 1e-5 + (0 if out == "f32" else (2.0 ** -11 if out == "f16" else 2.0 ** -8)) * ref.abs()


def _check(q, kv, lens, scale, dtype, out, what, **kw):
    import torch
    o, lse = _run(q, kv, lens, scale, dtype, out, **kw)
    ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], lens, scale)
    err = (o.double() - ref["o"]).abs()
    tol = _tolerance(ref["T"], ref["o"], dtype, out)
    assert torch.all(err <= tol), f"{what}: worst {float((err / tol).nan_to_num(nan=1e9).max()):.3g} of the tolerance"
    if lse is not None:
        none = ref["lse"] == -float("inf")
        assert torch.equal(lse == -float("inf"), none)
        big = 0.0 if none.all() else float(ref["lse"][~none].abs().max()) + 20.0        # (the largest score is within log N of the largest log-sum-exp)
        assert torch.all((lse.double() - ref["lse"])[~none].abs() <= 1e-5 + 2.0 ** -22 * big), what
    return o, lse


@pytest.fixture
def workspace():
    import torch
    ws = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
    B.tir_set_workspace(ws)
    yield ws
    torch.cuda.synchronize()
    B.tir_set_workspace(None)


# (batch, m, n, key heads, query heads per key head, lens)
SHAPES = [
    (2, 1, 1, 1, 1, None), (1, 1, 700, 2, 1, None), (3, 1, 333, 2, 4, [333, 0, 100]), (2, 33, 65, 1, 3, [65, 1]), (2, 130, 77, 2, 1, None), (4, 7, 200, 3, 2, [200, 64, 63, 65]),
    (1, 300, 129, 1, 1, [128]), (2, 64, 500, 1, 2, [-3, 10000]), (40, 50, 40, 4, 1, None), (1, 257, 1030, 1, 1, None),
    (2, 1, 90, 3, 2, None), (3, 3, 50, 2, 1, [50, 0, 17]), (2, 2, 31, 1, 2, [31, 1]), (2, 5, 40, 2, 1, None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_cross_attention_matches_the_plain_form(workspace, shape, dtype, out, d):
    batch, m, n, heads, group, lens = shape
    g = _gen(batch + m + n)
    what = f"cross attention {dtype}->{out} {shape} d={d}"
    _say(what)
    q, kv = _inputs(g, dtype, batch, m, n, heads, group, d, lens)
    _check(q, kv, lens, d ** -0.5, dtype, out, what)


# every kernel of the dispatch, for rows of key heads: (batch, m, n, key heads, query heads per key head, d)
KERNELS = [(150, 40, 64, 4, 1, 64), (9, 250, 70, 5, 7, 64), (15, 500, 300, 17, 1, 64), (6, 515, 300, 16, 8, 64), (3, 250, 300, 8, 65, 64), (4, 60, 900, 130, 2, 64),
           (150, 40, 64, 4, 1, 128), (9, 250, 170, 5, 7, 128), (3, 250, 600, 5, 67, 128), (4, 60, 900, 130, 2, 128), (2, 500, 300, 16, 8, 128), (5, 250, 600, 16, 2, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", KERNELS)
def test_every_kernel_of_the_dispatch(shape):
    """Calls large enough for the tiles of 128 and 256 rows, on repeated sequences that have to agree to the bit; the plain form of one of them."""
    import torch
    batch, m, n, heads, group, d = shape
    g = _gen(sum(shape))
    dtype = "bf16" if n % 4 else "f16"
    q, kv = _inputs(g, dtype, 1, m, n, 1, group, d, None)
    _say(f"cross attention {shape} {dtype}: {B.tir_debug_attention_kernel(batch * heads, m * group, n, d, dtype)}")
    qd = _to_device(q).expand(batch, -1, -1, -1).repeat(1, 1, heads, 1)
    kvd = _to_device(kv).expand(batch, -1, -1, -1, -1).repeat(1, 1, 1, heads, 1)
    k, v = kvd[:, :, 0], kvd[:, :, 1]
    o = torch.empty_like(qd)
    lse = torch.empty((batch, heads * group, m), device="cuda")
    B.tir_cross_attention(qd, k, v, o, lse, None, batch, m, n, heads * group, heads, d, *qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3], d ** -0.5, dtype, dtype)
    torch.cuda.synchronize()
    first = o[0, :, :group]
    assert torch.equal(o.view(batch, m, heads, group, d), first[None, :, None].expand(batch, m, heads, group, d))
    ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], None, d ** -0.5)
    assert torch.all((first.cpu().double() - ref["o"][0]).abs() <= _tolerance(ref["T"], ref["o"], dtype, dtype)[0])


def test_the_shapes_reach_every_kernel():
    reached = {(d, B.tir_debug_attention_kernel(b * h, m * g, n, d, "bf16" if n % 4 else "f16")) for b, m, n, h, g, d in KERNELS}
    reached |= {(d, B.tir_debug_attention_kernel(b * h, m * g, n, d, "f16")) for b, m, n, h, g, _ in SHAPES for d in (64, 128)}
    names = {(64, x) for x in ("t64_groups4", "t128_chunks32", "t128", "t128_sequential", "t256_sequential")} | {(128, x) for x in ("t64_groups4", "t128_chunks32", "t128", "t256")}
    assert names <= reached, names - reached


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_keys_and_values_beyond_the_memory_side_cache(d):
    """Heads of one tile whose keys and values are more than 256 MB, copied past the caches: one sequence's states for all by a batch stride of zero would not be; repeated ones are."""
    import torch
    batch, m, n, heads = 70, 9, 1000, 1024 // d
    q, kv = _inputs(_gen(5), "bf16", 1, m, n, 1, 1, d, None)
    kernel = B.tir_debug_attention_kernel(batch * heads, m, n, d, "bf16")
    _say(f"cross attention of {batch * heads} heads, d={d}: {kernel}")
    assert kernel == ("t128_sequential" if d == 64 else "t128_stream")
    qd = _to_device(q).repeat(batch, 1, heads, 1)
    kvd = _to_device(kv).repeat(batch, 1, 1, heads, 1)
    k, v = kvd[:, :, 0], kvd[:, :, 1]
    o = torch.empty(qd.shape, device="cuda")
    B.tir_cross_attention(qd, k, v, o, None, None, batch, m, n, heads, heads, d, *qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3], 0.125, "bf16", "f32")
    torch.cuda.synchronize()
    assert torch.equal(o, o[:1, :, :1].expand_as(o))
    ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], None, 0.125)
    assert torch.all((o[0, :, :1].cpu().double() - ref["o"][0]).abs() <= _tolerance(ref["T"], ref["o"], "bf16", "f32")[0])


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.125, 2.0, 40.0])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_scales(workspace, dtype, scale):
    """Scale zero (the mean of the values), a negative one, and scores of hundreds and thousands (where the largest is nearly all of the sum, and fp32's 2^-24 of a score
    of 2000 moves a probability by 2.4e-4 of itself, within the slack of either bound)."""
    q, kv = _inputs(_gen(7), dtype, 2, 40, 600, 2, 2, 64, [600, 17])
    _say(f"cross attention {dtype} scale={scale}")
    _check(q, kv, [600, 17], scale, dtype, "f32", f"scale {scale}")


@pytest.mark.gpu
def test_broadcast_inputs_strides_and_rows_behind(workspace):
    """One encoder's states for all sequences (batch stride 0), one query for all positions (row stride 0), outputs into a larger buffer."""
    import torch
    g = _gen(11)
    for d in (64, 128):
        _, kv = _inputs(g, "f16", 1, 1, 300, 2, 1, d, None)
        wide = torch.randn((3, 1, 4, d + 64), generator=g).to(torch.float16)
        q = wide[..., 32:32 + d].expand(3, 70, 4, d)
        kvd = _to_device(kv)
        k, v = kvd[:, :, 0].expand(3, -1, -1, -1), kvd[:, :, 1].expand(3, -1, -1, -1)
        wd = _to_device(wide)
        qd = wd[..., 32:32 + d].expand(3, 70, 4, d)
        assert qd.stride()[1] == 0 and k.stride()[0] == 0
        o = torch.full((3, 72, 5, d + 8), MARK, dtype=torch.float16, device="cuda")
        view = o[:, :70, :4, :d]
        _say(f"cross attention, broadcast inputs, d={d}")
        B.tir_cross_attention(qd, k, v, view, None, None, 3, 70, 300, 4, 2, d, *qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *view.stride()[:3], 0.1, "f16", "f16")
        torch.cuda.synchronize()
        ref = R.cross_attention(q, kv[:, :, 0].expand(3, -1, -1, -1), kv[:, :, 1].expand(3, -1, -1, -1), None, 0.1)
        assert torch.all((view.cpu().double() - ref["o"]).abs() <= _tolerance(ref["T"], ref["o"], "f16", "f16"))
        view.fill_(MARK)
        assert torch.all(o == MARK)


@pytest.mark.gpu
def test_outputs_with_far_strides():
    """Rows 2^21 elements apart, further than a tile is addressed with 31 bits, and heads 2^20 apart; nothing between them changes."""
    import torch
    q, kv = _inputs(_gen(23), "f16", 1, 40, 90, 2, 1, 64, None)
    qd, kvd = _to_device(q), _to_device(kv)
    k, v = kvd[:, :, 0], kvd[:, :, 1]
    flat = torch.full((40 << 21,), MARK, dtype=torch.float16, device="cuda")
    o = flat.as_strided((1, 40, 2, 64), (40 << 21, 1 << 21, 1 << 20, 1))
    _say("cross attention, far rows")
    B.tir_cross_attention(qd, k, v, o, None, None, 1, 40, 90, 2, 2, 64, *qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3], 0.125, "f16", "f16")
    torch.cuda.synchronize()
    ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], None, 0.125)
    assert torch.all((o.cpu().double() - ref["o"]).abs() <= _tolerance(ref["T"], ref["o"], "f16", "f16"))
    o.fill_(MARK)
    assert bool((flat == MARK).all())


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,group", [(1, 4), (1, 1), (3, 4)])
def test_keys_shared_among_workgroups(d, m, group):
    """Few rows over many keys, with and without a workspace: the slices did run, and the same call gives the same bits."""
    import torch
    lens = [7000, 0, 1, 5000]
    q, kv = _inputs(_gen(13), "bf16", 4, m, 7000, 2, group, d, lens)
    q = (q * 2).to(q.dtype)
    _say(f"cross attention in slices, m={m} group={group} d={d}")
    B.tir_set_workspace(None)
    alone, _ = _check(q, kv, lens, d ** -0.5, "bf16", "f32", "one workgroup")
    ws = torch.full((B.tir_workspace_bytes(),), 255, dtype=torch.uint8, device="cuda")
    B.tir_set_workspace(ws)
    try:
        shared = [_check(q, kv, lens, d ** -0.5, "bf16", "f32", "slices") for _ in range(3)]
    finally:
        torch.cuda.synchronize()
        B.tir_set_workspace(None)
    for o, lse in shared:
        assert torch.equal(o, shared[0][0]) and torch.equal(lse, shared[0][1])
    assert not torch.equal(alone, shared[0][0])
