"""Gradients of the attention over another sequence's states, against the formulas in 64 bits and against differences.

Tolerances.  With u the input type's half step (2^-11 F16, 2^-8 BF16, where the operators' contract says 'of T' with their own slack), per element:
  - P is rounded once for dV: u * sum_i P |dO|;
  - dS is rounded once for dQ and dK: u * sum |dS| |K|; D is taken from an O that was rounded to u of itself, which moves dS by u * P * sum_c |dO| |O| <= u * P * (P |dO| |V|),
    what decoder_reference's *_sum adds up, with the |dP| beside it: 2u * sum covers both, fp32 sums and exponents (scores below 100: 1.2e-5 of P) add less than u/8 each in F16;
  - the result is rounded to u of itself, and F16 subnormals to 2^-25.
So |error| <= 3u * sum + u * |ref| + 1e-6, where sum runs over magnitudes."""
import sys

import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R
from tests.test_cross_attention import FAKE, FAULTS, MARK, _gen, _inputs, _say, _to_device

U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _backward(**over):
    a = dict(Q=FAKE, K=FAKE, V=FAKE, O=FAKE, dO=FAKE, lse=FAKE, lens=FAKE, dQ=FAKE, dK=FAKE, dV=FAKE, delta=FAKE, batch=2, M=5, N=7, Hq=4, Hkv=2, d=64, q=(1280, 256, 64), k=(896, 128, 64),
             v=(896, 128, 64), o=(1280, 256, 64), go=(1280, 256, 64), scale=0.125, i="f16")
    a.update(over)
    return B.tir_cross_attention_backward_status(*[a[x] for x in ("Q", "K", "V", "O", "dO", "lse", "lens", "dQ", "dK", "dV", "delta", "batch", "M", "N", "Hq", "Hkv", "d")], *a["q"], *a["k"], *a["v"],
                                                 *a["o"], *a["go"], a["scale"], a["i"])


@pytest.mark.parametrize("over,status", FAULTS + [
    (dict(dO=0), B.TIR_ERR_INVALID_ARG), (dict(lse=0), B.TIR_ERR_INVALID_ARG), (dict(dQ=0), B.TIR_ERR_INVALID_ARG), (dict(dK=0), B.TIR_ERR_INVALID_ARG), (dict(dV=0), B.TIR_ERR_INVALID_ARG),
    (dict(delta=0), B.TIR_ERR_INVALID_ARG), (dict(q=(0, 256, 64)), B.TIR_ERR_INVALID_ARG), (dict(q=(1280, 0, 64)), B.TIR_ERR_INVALID_ARG), (dict(k=(0, 128, 64)), B.TIR_ERR_INVALID_ARG),
    (dict(v=(896, 0, 64)), B.TIR_ERR_INVALID_ARG), (dict(k=(896, 128, 0)), B.TIR_ERR_INVALID_ARG), (dict(go=(-8, 256, 64)), B.TIR_ERR_INVALID_ARG), (dict(go=(1280, 4, 64)), B.TIR_ERR_ALIGNMENT), (dict(dO=FAKE + 8), B.TIR_ERR_ALIGNMENT), (dict(dQ=FAKE + 8), B.TIR_ERR_ALIGNMENT),
    (dict(delta=FAKE + 2), B.TIR_ERR_ALIGNMENT), (dict(i="f32"), B.TIR_ERR_UNSUPPORTED)])
def test_backward_rejects_bad_arguments(over, status):
    assert _backward(**over) == status and B.last_error()


def test_nothing_to_do_needs_no_device():
    assert _backward(batch=0, Q=0) == B.TIR_OK and _backward(Hq=0) == B.TIR_OK


def _forward_and_backward(q, kv, do, lens, scale, dtype, stream=None):
    """The library's forward and backward pass; everything as CPU tensors.  Outputs are marked before, and gradients of k and v are slices of one tensor."""
    import torch
    batch, m, hq, d = q.shape
    n, heads = kv.shape[1], kv.shape[3]
    qd, kvd, dod = _to_device(q), _to_device(kv), _to_device(do)
    k, v = kvd[:, :, 0], kvd[:, :, 1]
    o, lse, delta = torch.empty_like(qd), torch.empty((batch, hq, m), device="cuda"), torch.empty((batch, hq, m), device="cuda")
    # (a gradient has the strides of what it is of, gaps included, which full_like would close)
    dq, dkv = torch.empty_strided(qd.shape, qd.stride(), dtype=qd.dtype, device="cuda").fill_(MARK), torch.full_like(kvd, MARK)
    dk, dv = dkv[:, :, 0], dkv[:, :, 1]
    ld = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    strides = (*qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3])
    torch.cuda.synchronize()
    B.tir_cross_attention(qd, k, v, o, lse, ld, batch, m, n, hq, heads, d, *strides, scale, dtype, dtype, stream)
    B.tir_cross_attention_backward(qd, k, v, o, dod, lse, ld, dq, dk, dv, delta, batch, m, n, hq, heads, d, *strides, *dod.stride()[:3], scale, dtype, stream)
    torch.cuda.synchronize()
    return dict(dq=dq.cpu(), dk=dk.cpu(), dv=dv.cpu(), delta=delta.cpu())


def _check(q, kv, do, lens, scale, dtype, what, stream=None):
    import torch
    got = _forward_and_backward(q, kv, do, lens, scale, dtype, stream)
    ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], lens, scale, do)
    u = U[dtype]
    worst = {}
    for x in ("dq", "dk", "dv"):
        err = (got[x].double() - ref[x]).abs()
        tol = 3 * u * ref[x + "_sum"] + u * ref[x].abs() + 1e-6
        worst[x] = float((err / tol).nan_to_num(nan=1e9).max()) if err.numel() else 0.0
    _say(f"{what}: worst of the tolerance {worst}")
    assert all(w <= 1 for w in worst.values()), (what, worst)
    if lens is not None:
        for b, x in enumerate(lens):
            assert torch.all(got["dk"][b, max(0, x):] == 0) and torch.all(got["dv"][b, max(0, x):] == 0)
            if x <= 0:
                assert torch.all(got["dq"][b] == 0)
    return got


@pytest.fixture
def workspace():
    import torch
    ws = torch.full((B.tir_workspace_bytes(),), 255, dtype=torch.uint8, device="cuda")
    B.tir_set_workspace(ws)
    yield ws
    torch.cuda.synchronize()
    B.tir_set_workspace(None)


# (batch, m, n, key heads, query heads per key head, lens)
SHAPES = [
    (1, 1, 1, 1, 1, None), (2, 1, 40, 1, 3, [40, 0]), (2, 33, 65, 2, 1, [65, 1]), (1, 64, 64, 1, 1, None), (3, 70, 129, 1, 2, [129, 64, 127]), (2, 200, 77, 2, 1, None),
    (2, 129, 300, 1, 4, [300, 31]), (1, 700, 20, 1, 2, None), (2, 5, 900, 1, 1, [900, 899]), (1, 257, 257, 3, 1, [256]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradients_match_the_formulas(workspace, shape, dtype, d):
    import torch
    batch, m, n, heads, group, lens = shape
    g = _gen(batch + m + n + d)
    q, kv = _inputs(g, dtype, batch, m, n, heads, group, d, lens)
    do = torch.randn(q.shape, generator=g).to(R.TORCH[dtype])
    _check(q, kv, do, lens, d ** -0.5, dtype, f"gradients {dtype} {shape} d={d}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,size", [("f16", 2.0 ** -12), ("f16", 300.0), ("bf16", 2.0 ** -60), ("bf16", 2.0 ** 60)])
def test_gradients_of_any_magnitude(workspace, dtype, size):
    """What arrives may be small or large: relative to it the results are as exact.  (The absolute 1e-6 of the tolerance goes along, down to F16's own subnormals.)"""
    import torch
    g = _gen(3)
    q, kv = _inputs(g, dtype, 2, 150, 200, 1, 2, 64, [200, 90])
    kv = (kv * 0.5).to(kv.dtype)
    do = (torch.randn(q.shape, generator=g) * size).to(R.TORCH[dtype])
    got = _forward_and_backward(q, kv, do, [200, 90], 0.125, dtype)
    ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], [200, 90], 0.125, do)
    u = U[dtype]
    for x in ("dq", "dk", "dv"):
        tol = 3 * u * ref[x + "_sum"] + u * ref[x].abs() + 1e-6 * size + (2.0 ** -25 if dtype == "f16" else 0)
        ratio = float(((got[x].double() - ref[x]).abs() / tol).nan_to_num(nan=1e9).max())
        _say(f"gradients {dtype} of size {size:.3g}: {x} {ratio:.3g} of the tolerance")
        assert ratio <= 1


@pytest.mark.gpu
def test_rows_of_very_different_magnitude(workspace):
    """F16: one query's gradient is 2^18 times the others', late and early: the factor that a key's sums are held times shrinks on the way, or is small from the start."""
    import torch
    for at in (3, 140):
        g = _gen(at)
        q, kv = _inputs(g, "f16", 1, 150, 70, 1, 1, 64, None)
        do = torch.randn(q.shape, generator=g) * 2.0 ** -9
        do[0, at] *= 2.0 ** 18
        _check(q, kv, do.to(torch.float16), None, 0.125, "f16", f"one large row at {at}")


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.5])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_gradients_with_other_scales(workspace, dtype, scale):
    import torch
    g = _gen(5)
    q, kv = _inputs(g, dtype, 2, 90, 130, 2, 1, 64, [130, 64])
    do = torch.randn(q.shape, generator=g).to(R.TORCH[dtype])
    _check(q, kv, do, [130, 64], scale, dtype, f"gradients {dtype}, scale {scale}")


@pytest.mark.gpu
def test_gradients_against_differences(workspace):
    """The directional derivative of sum(dO o O) along random directions, by 64-bit differences of the formula, and by the library's gradients."""
    import torch
    g = _gen(7)
    q, kv = _inputs(g, "f16", 2, 60, 100, 1, 2, 64, [100, 37], poison=False)
    kv[1, 37:] = 0
    do = torch.randn(q.shape, generator=g).to(torch.float16)
    got = _forward_and_backward(q, kv, do, [100, 37], 0.125, "f16")

    def value(q64, k64, v64):
        return float((R.cross_attention(q64, k64, v64, [100, 37], 0.125)["o"] * do.double()).sum())
    x = [q.double(), kv[:, :, 0].double(), kv[:, :, 1].double()]
    grads = [got["dq"].double(), got["dk"].double(), got["dv"].double()]
    for i, name in enumerate(("q", "k", "v")):
        way = torch.randn(x[i].shape, generator=g, dtype=torch.float64)
        step = 1e-5
        up, down = ([y + (s * step * way if j == i else 0) for j, y in enumerate(x)] for s in (1, -1))
        slope = (value(*up) - value(*down)) / (2 * step)
        # each gradient is within 3 * 2^-11 of its magnitudes' sum; over the direction these errors are as random as the terms
        size = float((grads[i] * way).square().sum().sqrt())
        _say(f"d/d{name}: differences {slope:.6g}, gradients {float((grads[i] * way).sum()):.6g}, of terms {size:.3g}")
        assert abs(float((grads[i] * way).sum()) - slope) <= 0.02 * size + 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", [(1, 1500, 77, 2, 1, None), (2, 8, 1500, 1, 2, [1500, 3])])
def test_sums_shared_among_workgroups(shape, d):
    """Few keys and many rows, few rows and many keys, with and without a workspace: within the tolerance both ways, to the bit each time."""
    import torch
    batch, m, n, heads, group, lens = shape
    g = _gen(9)
    q, kv = _inputs(g, "bf16", batch, m, n, heads, group, d, lens)
    do = torch.randn(q.shape, generator=g).to(torch.bfloat16)
    B.tir_set_workspace(None)
    alone = [_check(q, kv, do, lens, 0.1, "bf16", f"alone {shape} d={d}") for _ in range(2)]
    ws = torch.full((B.tir_workspace_bytes(),), 255, dtype=torch.uint8, device="cuda")
    B.tir_set_workspace(ws)
    try:
        shared = [_check(q, kv, do, lens, 0.1, "bf16", f"shared {shape} d={d}") for _ in range(2)]
    finally:
        torch.cuda.synchronize()
        B.tir_set_workspace(None)
    for pair in (alone, shared):
        assert all(torch.equal(pair[0][x], pair[1][x]) for x in ("dq", "dk", "dv"))


@pytest.mark.gpu
def test_many_sequences_agree_with_one(workspace):
    """Enough tiles that no sum is shared: repeated sequences agree to the bit, and with the plain form."""
    import torch
    g = _gen(11)
    for d, dtype in ((64, "f16"), (128, "bf16")):
        q, kv = _inputs(g, dtype, 1, 140, 150, 1, 2, d, None)
        do = torch.randn(q.shape, generator=g).to(R.TORCH[dtype])
        got = _forward_and_backward(q.repeat(150, 1, 1, 1), kv.repeat(150, 1, 1, 1, 1), do.repeat(150, 1, 1, 1), None, 0.1, dtype)
        ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], None, 0.1, do)
        for x in ("dq", "dk", "dv"):
            assert torch.equal(got[x], got[x][:1].expand_as(got[x]))
            tol = 3 * U[dtype] * ref[x + "_sum"] + U[dtype] * ref[x].abs() + 1e-6
            assert torch.all((got[x][:1].double() - ref[x]).abs() <= tol), (x, d)


@pytest.mark.gpu
def test_gradients_that_arrive_in_other_orders(workspace):
    """dO head by head, broadcast over the queries (the gradient of a sum), and as a slice; queries and keys as slices of wider tensors."""
    import torch
    for d in (64, 128):
        g = _gen(19)
        q, kv = _inputs(g, "f16", 2, 70, 90, 2, 2, d, [90, 31])
        q = torch.randn((2, 70, 4, d + 24), generator=g).to(torch.float16)[..., 8:8 + d]
        by_head = torch.randn((2, 4, 70, d), generator=g).to(torch.float16).transpose(1, 2)
        one = torch.randn((2, 1, 4, d), generator=g).to(torch.float16).expand(2, 70, 4, d)
        part = torch.randn((2, 70, 4, 2 * d), generator=g).to(torch.float16)[..., d:]
        for do in (by_head, one, part):
            _check(q, kv, do, [90, 31], 0.1, "f16", f"dO of strides {do.stride()}")


@pytest.mark.gpu
def test_gradients_with_far_strides():
    """Queries (and so their gradients) 2^21 elements apart, keys 2^19: nothing between the rows changes."""
    import torch
    m, n = 40, 90
    q, kv = _inputs(_gen(29), "f16", 1, m, n, 2, 1, 64, None)
    do = torch.randn(q.shape, generator=_gen(31)).to(torch.float16)
    ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], None, 0.125, do)
    far = {}
    for name, x, rs in (("q", q, 1 << 21), ("k", kv[:, :, 0], 1 << 19), ("v", kv[:, :, 1], 1 << 19), ("dq", None, 1 << 21), ("dk", None, 1 << 19), ("dv", None, 1 << 19)):
        rows = m if name in ("q", "dq") else n
        flat = torch.full((rows * rs,), MARK, dtype=torch.float16, device="cuda")
        view = flat.as_strided((1, rows, 2, 64), (rows * rs, rs, rs // 2, 1))
        if x is not None:
            view.copy_(x)
        far[name] = (flat, view)
    qd, k, v, dq, dk, dv = (far[x][1] for x in ("q", "k", "v", "dq", "dk", "dv"))
    dod = do.cuda()
    o, lse, delta = torch.empty_like(dod), torch.empty((1, 2, m), device="cuda"), torch.empty((1, 2, m), device="cuda")
    strides = (*qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3])
    _say("gradients, far rows")
    B.tir_cross_attention(qd, k, v, o, lse, None, 1, m, n, 2, 2, 64, *strides, 0.125, "f16", "f16")
    B.tir_cross_attention_backward(qd, k, v, o, dod, lse, None, dq, dk, dv, delta, 1, m, n, 2, 2, 64, *strides, *dod.stride()[:3], 0.125, "f16")
    torch.cuda.synchronize()
    for x in ("dq", "dk", "dv"):
        flat, view = far[x]
        tol = 3 * U["f16"] * ref[x + "_sum"] + U["f16"] * ref[x].abs() + 1e-6
        assert torch.all((view.cpu().double() - ref[x]).abs() <= tol), x
        view.fill_(MARK)
        assert bool((flat == MARK).all()), x


@pytest.mark.gpu
def test_no_queries_and_no_keys():
    import torch
    q, kv = _inputs(_gen(13), "f16", 2, 4, 6, 2, 1, 64, None)
    got = _forward_and_backward(q[:, :0], kv, q[:, :0], None, 0.1, "f16")
    assert torch.all(got["dk"] == 0) and torch.all(got["dv"] == 0)
    got = _forward_and_backward(q, kv[:, :0], q, None, 0.1, "f16")
    assert torch.all(got["dq"] == 0)


@pytest.mark.gpu
def test_a_training_step_in_a_graph():
    """Forward and backward captured on a stream of their own and replayed on new inputs, with eager work between the replays."""
    import torch
    batch, m, n, heads, group, d = 2, 40, 600, 1, 2, 64
    g = _gen(17)
    lens = [600, 450]
    q, kv = _inputs(g, "bf16", batch, m, n, heads, group, d, None)
    qd, kvd, dod = q.cuda(), kv.cuda(), torch.empty_like(q, device="cuda")
    k, v = kvd[:, :, 0], kvd[:, :, 1]
    o, lse, delta = torch.empty_like(qd), torch.empty((batch, heads * group, m), device="cuda"), torch.empty((batch, heads * group, m), device="cuda")
    dq, dkv = torch.empty_like(qd), torch.empty_like(kvd)
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    strides = (*qd.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st, capture_error_mode="global"):
        B.tir_set_workspace(ws, st)
        B.tir_cross_attention(qd, k, v, o, lse, ld, batch, m, n, heads * group, heads, d, *strides, 0.125, "bf16", "bf16", st)
        B.tir_cross_attention_backward(qd, k, v, o, dod, lse, ld, dq, dkv[:, :, 0], dkv[:, :, 1], delta, batch, m, n, heads * group, heads, d, *strides, *dod.stride()[:3], 0.125, "bf16", st)
    for i in range(4):
        q, kv = _inputs(g, "bf16", batch, m, n, heads, group, d, None)
        do = torch.randn(q.shape, generator=g).to(torch.bfloat16)
        qd.copy_(q), kvd.copy_(kv), dod.copy_(do)
        torch.cuda.synchronize()
        _say(f"replay {i}")
        graph.replay()
        torch.cuda.synchronize()
        ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], lens, 0.125, do)
        for x, got in (("dq", dq), ("dk", dkv[:, :, 0]), ("dv", dkv[:, :, 1])):
            tol = 3 * U["bf16"] * ref[x + "_sum"] + U["bf16"] * ref[x].abs() + 1e-6
            assert torch.all((got.cpu().double() - ref[x]).abs() <= tol), (i, x)
        assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())
    B.tir_set_workspace(None, st)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_strides_shorter_than_a_row(workspace, d):
    """On the device as they are: a dO whose rows are one row, or overlap; a single query and a single key whose row strides are 0.  What is behind the last row or key is that data again and must not count."""
    import torch
    for m, n, q_rs, k_rs, g_rs in ((70, 90, None, None, 0), (33, 40, None, None, 8), (1, 1, 0, 0, 0), (1, 75, 0, None, 0)):
        g = _gen(37)
        q, kv = _inputs(g, "f16", 2, m, n, 1, 1, d, None)
        flat = torch.randn((2, m * d + d), generator=g).to(torch.float16)
        do = flat.as_strided((2, m, 1, d), (m * d + d, g_rs, d, 1))
        dod = flat.cuda().as_strided(do.shape, do.stride())
        qd, kd, vd = q.cuda(), kv[:, :, 0].contiguous().cuda(), kv[:, :, 1].contiguous().cuda()
        o, lse, delta = torch.empty_like(qd), torch.empty((2, 1, m), device="cuda"), torch.empty((2, 1, m), device="cuda")
        dq, dk, dv = (torch.full_like(x, MARK) for x in (qd, kd, vd))
        rs = lambda x, r: (x.stride(0), x.stride(1) if r is None else r, x.stride(2))
        strides = (*rs(qd, q_rs), *rs(kd, k_rs), *rs(vd, k_rs), *o.stride()[:3])
        _say(f"short strides d={d}: {m} x {n}, {q_rs} {k_rs} {g_rs}")
        B.tir_cross_attention(qd, kd, vd, o, lse, None, 2, m, n, 1, 1, d, *strides, 0.1, "f16", "f16")
        B.tir_cross_attention_backward(qd, kd, vd, o, dod, lse, None, dq, dk, dv, delta, 2, m, n, 1, 1, d, *strides, *do.stride()[:3], 0.1, "f16")
        torch.cuda.synchronize()
        ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], None, 0.1, do)
        for x, got in (("dq", dq), ("dk", dk), ("dv", dv)):
            tol = 3 * U["f16"] * ref[x + "_sum"] + U["f16"] * ref[x].abs() + 1e-6
            assert torch.all((got.cpu().double() - ref[x]).abs() <= tol), (x, m, n, d)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f16", 64), ("f16", 128)])
def test_few_keys_with_nearly_the_same_values(workspace, dtype, d):
    """Values 8 and a tenth around it: dP - D is a hundredth of either, and an O that was rounded would be seen in D.  Per element: dS is rounded once, the result once, and dP and D are fp32 sums of d
    resp. n terms: 2^-24 * (d + 64 + 64) <= 2e-5 of sum_c |dO| |V| each, so |error| <= u * sum |dS| |K| * 1.01 + 4e-5 * sum P (|dO| |V|) |K| + u * |ref| (dK alike)."""
    import torch
    g = _gen(41)
    batch, m, n, scale, u = 3, 50, 60, 0.125, U[dtype]
    t = R.TORCH[dtype]
    lens = [60, 33, 5]
    q, k, do = (torch.randn((batch, x, 2, d), generator=g).to(t) for x in (m, n, m))
    v = (8 + 0.1 * torch.randn((batch, n, 2, d), generator=g)).to(t)
    got = _forward_and_backward(q, torch.stack((k, v), 2), do, lens, scale, dtype)
    worst = 0.0
    for b, length in enumerate(lens):
        Q, K, V, G = (x[b, :y].double().transpose(0, 1) for x, y in ((q, m), (k, length), (v, length), (do, m)))
        P = torch.softmax(scale * Q @ K.transpose(1, 2), -1)
        dP = G @ V.transpose(1, 2)
        dS = P * (dP - (P * dP).sum(-1, keepdim=True))
        fuzz = 4e-5 * P * (G.abs() @ V.abs().transpose(1, 2)) + 1.01 * u * dS.abs()
        for name, ref, mag, out in (("dq", dS @ K, fuzz @ K.abs(), got["dq"][b]), ("dk", dS.transpose(1, 2) @ Q, fuzz.transpose(1, 2) @ Q.abs(), got["dk"][b, :length])):
            ref, mag = scale * ref.transpose(0, 1), scale * mag.transpose(0, 1)
            worst = max(worst, float(((out.double() - ref).abs() / (mag + u * ref.abs() + 2.0 ** -25)).max()))
    _say(f"few keys, near values, {dtype} d={d}: {worst:.3g} of the tolerance")
    assert worst <= 1
