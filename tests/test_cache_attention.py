"""The paged 8-bit cache: appending to it, and attention over it, against plain 64-bit forms.

Appending is defined down to the last bit, so the cache is compared for equality.  Tolerances of the attention: those that
tir.h gives, 2e-3 * T + 1e-5 for F16 and 6e-3 * T + 1e-5 for BF16 with T = sum_j p_j |v_j|; a 16-bit output adds its own half step,
2^-11 |o| or 2^-8 |o|.  The kernel rounds weights once (2^-11 resp. 2^-8 of T) and sums n of them in fp32; scores of |t| <= 100
in fp32 move a probability by 100 * 2^-23 = 1.2e-5 of itself; that leaves a factor of 1.5 to 4."""
import ctypes
import sys

import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R

FAKE = 0x1000


def _say(msg):
    print(f"[case] {msg}", flush=True)
    sys.stdout.flush()


# ------------------------------------------------------------------------------------------------ refusals, on the host
def _fake_cache(**over):
    c = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, table=FAKE, blocks=4, heads=2, block_tokens=32, d=64, sequences=3, columns=3, dtype=B.TIR_I8)
    c.update(over)
    return B.KvCache(*[c[n] for n, _ in B.KvCache._fields_])


CACHE_FAULTS = [
    (dict(k=0), B.TIR_ERR_INVALID_ARG), (dict(table=0), B.TIR_ERR_INVALID_ARG), (dict(v_scale=0), B.TIR_ERR_INVALID_ARG),
    (dict(blocks=0), B.TIR_ERR_INVALID_ARG), (dict(heads=0), B.TIR_ERR_INVALID_ARG), (dict(columns=0), B.TIR_ERR_INVALID_ARG), (dict(blocks=-3), B.TIR_ERR_INVALID_ARG), (dict(sequences=1), B.TIR_ERR_INVALID_ARG),
    (dict(d=96), B.TIR_ERR_UNSUPPORTED), (dict(block_tokens=48), B.TIR_ERR_UNSUPPORTED), (dict(block_tokens=256), B.TIR_ERR_UNSUPPORTED), (dict(block_tokens=0), B.TIR_ERR_UNSUPPORTED),
    (dict(dtype=B.TIR_F16), B.TIR_ERR_UNSUPPORTED), (dict(columns=2 ** 31), B.TIR_ERR_UNSUPPORTED), (dict(columns=2 ** 26), B.TIR_ERR_UNSUPPORTED), (dict(columns=2 ** 26 - 2047), B.TIR_ERR_UNSUPPORTED), (dict(blocks=2 ** 31), B.TIR_ERR_UNSUPPORTED),
    (dict(k=FAKE + 8), B.TIR_ERR_ALIGNMENT), (dict(v=FAKE + 4), B.TIR_ERR_ALIGNMENT), (dict(k_scale=FAKE + 2), B.TIR_ERR_ALIGNMENT), (dict(table=FAKE + 1), B.TIR_ERR_ALIGNMENT),
]


def _append(cache="", **over):
    a = dict(K=FAKE, V=FAKE, start=FAKE, count=FAKE, batch=2, T=5, k=(640, 128, 64), v=(640, 128, 64), i="f16")
    a.update(over)
    return B.tir_cache_append_status(_fake_cache() if cache == "" else cache, a["K"], a["V"], a["start"], a["count"], a["batch"], a["T"], *a["k"], *a["v"], a["i"])


def _attend(cache="", **over):
    a = dict(Q=FAKE, O=FAKE, lens=FAKE, count=FAKE, batch=2, T=5, Hq=4, q=(1280, 256, 64), o=(1280, 256, 64), scale=0.125, i="f16", out="f16")
    a.update(over)
    return B.tir_cache_attention_status(a["Q"], _fake_cache() if cache == "" else cache, a["O"], a["lens"], a["count"], a["batch"], a["T"], a["Hq"], *a["q"], *a["o"], a["scale"], a["i"], a["out"])


@pytest.mark.parametrize("over,status", CACHE_FAULTS)
def test_both_entry_points_reject_a_bad_cache(over, status):
    assert _append(_fake_cache(**over)) == status and B.last_error()
    assert _attend(_fake_cache(**over)) == status and B.last_error()


@pytest.mark.parametrize("over,status", [
    (dict(cache=None), B.TIR_ERR_INVALID_ARG), (dict(K=0), B.TIR_ERR_INVALID_ARG), (dict(V=0), B.TIR_ERR_INVALID_ARG), (dict(start=0), B.TIR_ERR_INVALID_ARG),
    (dict(batch=-1), B.TIR_ERR_INVALID_ARG), (dict(T=-1), B.TIR_ERR_INVALID_ARG), (dict(i=9), B.TIR_ERR_INVALID_ARG), (dict(k=(-640, 128, 64)), B.TIR_ERR_INVALID_ARG),
    (dict(i="f32"), B.TIR_ERR_UNSUPPORTED), (dict(i="e4m3"), B.TIR_ERR_UNSUPPORTED), (dict(T=2 ** 31), B.TIR_ERR_UNSUPPORTED), (dict(batch=2 ** 31), B.TIR_ERR_INVALID_ARG),
    (dict(v=(2 ** 41, 128, 64)), B.TIR_ERR_UNSUPPORTED), (dict(batch=2 ** 23, cache=_fake_cache(sequences=2 ** 23)), B.TIR_ERR_UNSUPPORTED),
    (dict(K=FAKE + 2), B.TIR_ERR_ALIGNMENT), (dict(v=(640, 128, 60)), B.TIR_ERR_ALIGNMENT), (dict(start=FAKE + 2), B.TIR_ERR_ALIGNMENT), (dict(count=FAKE + 1), B.TIR_ERR_ALIGNMENT),
])
def test_append_rejects_bad_arguments(over, status):
    assert _append(**over) == status and B.last_error()


@pytest.mark.parametrize("over,status", [
    (dict(cache=None), B.TIR_ERR_INVALID_ARG), (dict(Q=0), B.TIR_ERR_INVALID_ARG), (dict(O=0), B.TIR_ERR_INVALID_ARG), (dict(lens=0), B.TIR_ERR_INVALID_ARG),
    (dict(batch=-1), B.TIR_ERR_INVALID_ARG), (dict(T=-1), B.TIR_ERR_INVALID_ARG), (dict(Hq=-4), B.TIR_ERR_INVALID_ARG), (dict(Hq=5), B.TIR_ERR_INVALID_ARG),
    (dict(scale=float("nan")), B.TIR_ERR_INVALID_ARG), (dict(scale=float("-inf")), B.TIR_ERR_INVALID_ARG), (dict(i=-1), B.TIR_ERR_INVALID_ARG),
    (dict(o=(0, 256, 64)), B.TIR_ERR_INVALID_ARG), (dict(o=(1280, 0, 64)), B.TIR_ERR_INVALID_ARG), (dict(o=(1280, 256, 0)), B.TIR_ERR_INVALID_ARG), (dict(q=(1280, 256, -64)), B.TIR_ERR_INVALID_ARG),
    (dict(out="bf16"), B.TIR_ERR_UNSUPPORTED), (dict(i="i8", out="i32"), B.TIR_ERR_UNSUPPORTED), (dict(T=2 ** 31), B.TIR_ERR_UNSUPPORTED), (dict(T=2 ** 30, Hq=8), B.TIR_ERR_UNSUPPORTED),
    (dict(batch=4), B.TIR_ERR_INVALID_ARG), (dict(batch=2 ** 24, cache=_fake_cache(sequences=2 ** 24)), B.TIR_ERR_UNSUPPORTED),
    (dict(Q=FAKE + 8), B.TIR_ERR_ALIGNMENT), (dict(O=FAKE + 8), B.TIR_ERR_ALIGNMENT), (dict(o=(1280, 256, 68)), B.TIR_ERR_ALIGNMENT), (dict(lens=FAKE + 2), B.TIR_ERR_ALIGNMENT),
])
def test_cache_attention_rejects_bad_arguments(over, status):
    assert _attend(**over) == status and B.last_error()


def test_nothing_to_do_needs_no_device():
    assert _append(batch=0, K=0) == B.TIR_OK and _append(T=0) == B.TIR_OK
    assert _attend(batch=0, Q=0) == B.TIR_OK and _attend(T=0) == B.TIR_OK and _attend(Hq=0) == B.TIR_OK


def test_make_kv_cache_checks_its_tensors():
    import torch
    k, v = torch.zeros((4, 2, 32, 64), dtype=torch.int8), torch.zeros((4, 2, 64, 32), dtype=torch.int8)
    s, t = torch.zeros((4, 2)), torch.zeros((3, 5), dtype=torch.int32)
    c = B.make_kv_cache(k, v, s, s.clone(), t)
    assert (c.blocks, c.heads, c.block_tokens, c.d, c.sequences, c.columns, c.dtype) == (4, 2, 32, 64, 3, 5, B.TIR_I8)
    assert ctypes.sizeof(B.KvCache) == 96
    for bad in (dict(v=k), dict(ks=s.double()), dict(vs=s[:, :1]), dict(t=t.long()), dict(t=t[:, ::2]), dict(k=k.to(torch.uint8), v=v.to(torch.uint8)), dict(k=k.half(), v=v.half())):
        a = dict(k=k, v=v, ks=s, vs=s, t=t)
        a.update(bad)
        with pytest.raises(ValueError):
            B.make_kv_cache(a["k"], a["v"], a["ks"], a["vs"], a["t"])
    with pytest.raises((TypeError, RuntimeError)):
        (B._native or B._load_native()).tir_cache_append(s, None, None, None, None, 0, 0, 0, 0, 0, 0, 0, 0, "f16", 0)


# ------------------------------------------------------------------------------------------------ on the device
def _gen(seed):
    import torch
    return torch.Generator().manual_seed(seed)


def _pool(g, cache, blocks, heads, bt, d):
    """CPU tensors of a pool whose every byte is set: normal numbers, and NaN bytes among the e4m3 ones are put in by the tests that want them."""
    import torch
    top = R.LARGEST[cache]

    def eight(shape):
        x = (torch.randn(shape, generator=g) * top / 3).clamp(-top, top)
        return (x.round() if cache == "i8" else x).to(R.TORCH[cache])
    scale = lambda: (torch.rand((blocks, heads), generator=g) * 1.5 + 0.5) * 3 / top  # noqa: E731
    return eight((blocks, heads, bt, d)), eight((blocks, heads, d, bt)), scale(), scale()


def _equal8(a, b):
    import torch
    return torch.equal(R.bits8(a.cpu()), R.bits8(b.cpu()))


def _run_append(pool, table, new_k, new_v, start, count, dtype):
    """The cache on the device after the call, as CPU tensors.  new_k, new_v: [batch, T, heads, d], any strides."""
    import torch
    dev = [x.cuda() for x in pool]
    t = table.cuda()
    cache = B.make_kv_cache(*dev, t)
    kd, vd = (torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").copy_(x) for x in (new_k, new_v))
    sd = torch.tensor(start, dtype=torch.int32, device="cuda")
    cd = None if count is None else torch.tensor(count, dtype=torch.int32, device="cuda")
    B.tir_cache_append(cache, kd, vd, sd, cd, new_k.shape[0], new_k.shape[1], *kd.stride()[:3], *vd.stride()[:3], dtype)
    torch.cuda.synchronize()
    return [x.cpu() for x in dev]


def _check_append(pool, table, new_k, new_v, start, count, dtype):
    import torch
    got = _run_append(pool, table, new_k, new_v, start, count, dtype)
    want = R.append(*pool, table, new_k, new_v, start, [new_k.shape[1]] * len(start) if count is None else count)
    for name, a, b in zip(("k_scale", "v_scale"), got[2:], want[2:]):
        assert torch.equal(a, b), name
    for name, a, b in zip(("k", "v"), got, want):
        assert _equal8(a, b), (name, int((R.bits8(a) != R.bits8(b)).sum()))
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bt,d,heads", [(16, 64, 1), (16, 128, 3), (32, 64, 2), (32, 128, 1), (64, 64, 3), (64, 128, 2), (128, 64, 1), (128, 128, 2)])
def test_append_is_the_definition(cache, dtype, bt, d, heads):
    """Single tokens at every kind of place in a block, and prompts that begin and end inside one; keys and values as slices of one projection."""
    import torch
    for T, start, count in [(1, [0, 1, bt - 1, bt, 2 * bt + 3], None), (1, [5, bt + 7, 0, 2, 3], [1, 0, 1, 1, 0]),
                            (2 * bt + 5, [0, 1, bt - 1, bt, 3], [2 * bt + 5, 2 * bt, 2, bt, 1]), (3, [bt - 1, bt - 2, bt - 3, 0, 2], None)]:
        g = _gen(bt * 7 + d + heads + T)
        batch, cols = len(start), 4
        pool = _pool(g, cache, batch * cols + 2, heads, bt, d)
        table = torch.randperm(batch * cols + 2, generator=g)[:batch * cols].to(torch.int32).view(batch, cols)
        kv = (torch.randn((batch, T, 2, heads, d), generator=g) * torch.rand((batch, T, 1, 1, 1), generator=g) * 4).to(R.TORCH[dtype])
        _say(f"append {cache} {dtype} bt={bt} d={d} heads={heads} T={T} start={start} count={count}")
        _check_append(pool, table, kv[:, :, 0], kv[:, :, 1], start, count, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["i8", "e4m3"])
@pytest.mark.parametrize("bt", [16, 32, 64, 128])
def test_append_rescales_held_tokens_when_the_scale_grows(cache, bt):
    """Token after token into one block, each larger than all before, then smaller ones: held values are rounded again, or kept to the bit."""
    import torch
    g = _gen(bt)
    heads, d = 2, 64
    pool = _pool(g, cache, 2, heads, bt, d)
    table = torch.tensor([[1]], dtype=torch.int32)
    for i in range(min(bt, 20)):
        size = 1.5 ** i if i < 12 else 0.01
        new = (torch.randn((1, 1, heads, d), generator=g) * size).to(torch.bfloat16)
        _say(f"append {cache} bt={bt} token {i} of size {size:.3g}")
        pool = _check_append(pool, table, new, new * 0.5, [i], None, "bf16")
    # the same token again at the same place: nothing changes
    again = _check_append(pool, table, new, new * 0.5, [min(bt, 20) - 1], None, "bf16")
    assert all(torch.equal(R.bits8(a) if a.dtype != torch.float32 else a, R.bits8(b) if b.dtype != torch.float32 else b) for a, b in zip(again, pool))


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["i8", "e4m3"])
def test_append_of_zeros_subnormals_infinities_and_nan(cache):
    import torch
    g = _gen(3)
    heads, d, bt = 4, 128, 16
    pool = _pool(g, cache, 3, heads, bt, d)
    table = torch.tensor([[2, 0]], dtype=torch.int32)
    new = torch.randn((1, 20, heads, d), generator=g).to(torch.bfloat16)
    new[0, :, 0] = 0
    new[0, :, 1] = 1e-39                                     # below every scale there is
    new[0, 3, 2, 5], new[0, 7, 2, 9], new[0, 8, 2, 1] = float("nan"), float("nan"), -float("nan")
    new[0, 2, 3, 0], new[0, 5, 3, 1] = float("inf"), -float("inf")
    _say(f"append {cache}, values that are not finite")
    got = _check_append(pool, table, new, new.flip(1), [0], None, "bf16")
    assert all(torch.isfinite(x.float()).all() for x in (got[2], got[3], got[0][2].float()))
    _check_append(pool, table, new.to(torch.float16), new.flip(1).to(torch.float16), [3], [13], "f16")


@pytest.mark.gpu
def test_append_drops_what_has_no_place():
    """Blocks outside the pool, positions behind the table, negative and too large starts and counts: everything else is written."""
    import torch
    g = _gen(4)
    heads, d, bt = 2, 64, 32
    pool = _pool(g, "i8", 12, heads, bt, d)
    table = torch.tensor([[0, -1, 1], [2, 12, 3], [4, 5, 6], [7, 8, 9], [10, 2 ** 31 - 1, -2 ** 31], [11, -1, -1]], dtype=torch.int32)
    new = torch.randn((6, 70, heads, d), generator=g).to(torch.float16)
    start, count = [10, 0, 90, -5, 2 ** 31 - 1, 2 ** 31 - 65], [70, 70, 70, 1000, 70, 2 ** 31 - 1]
    _say("append with no place for some")
    _check_append(pool, table, new, new * 2, start, count, "f16")
    _check_append(pool, table, new, new * 2, [3] * 6, [-1, 0, -2 ** 31, 1, 2, 2 ** 31 - 1], "f16")
    # and a table of one column, from which nearly everything falls
    _check_append(pool, table[:, :1].contiguous(), new, new * 2, [31, 30, 0, 5, 32, 1], None, "f16")


def _attention_case(g, cache, dtype, batch, T, heads, group, d, bt, lens, spare=3):
    """Pool, table, queries of a call; what no sequence holds is set to bytes that must not be used (NaN in e4m3)."""
    import torch
    cols = max(1, -(-max(lens) // bt)) + 1
    need = [-(-max(0, n) // bt) for n in lens]
    blocks = sum(need) + spare
    k, v, ks, vs = _pool(g, cache, blocks, heads, bt, d)
    perm = torch.randperm(blocks, generator=g).to(torch.int32)
    table = torch.full((batch, cols), -7, dtype=torch.int32)
    at = 0
    bad = 127 if cache == "e4m3" else -128
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
        if lens[b] % bt and n:                               # the rest of a sequence's last block
            last = int(table[b, n - 1])
            R.bits8(k)[last, :, lens[b] % bt:] = bad
            R.bits8(v)[last, :, :, lens[b] % bt:] = bad
        table[b, n:] = torch.tensor([blocks + 5, -1, 2 ** 31 - 1, int(perm[-1])], dtype=torch.int32).repeat(cols)[:cols - n]
    for unused in perm[at:].tolist():
        R.bits8(k)[unused], R.bits8(v)[unused], ks[unused], vs[unused] = bad, bad, float("nan"), float("nan")
    q = torch.randn((batch, T, heads * group, d), generator=g).to(R.TORCH[dtype])
    return (k, v, ks, vs), table, q


MARK = 77.0


def _run_attention(pool, table, q, lens, count, scale, dtype, out, stream=None, o_shape=None):
    import torch
    dev = [x.cuda() for x in pool]
    cache = B.make_kv_cache(*dev, table.cuda())
    qd = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device="cuda").copy_(q)
    o = torch.full(o_shape or q.shape, MARK, dtype=R.TORCH[out], device="cuda")
    view = o[:, :q.shape[1], :q.shape[2], :q.shape[3]]
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cd = None if count is None else torch.tensor(count, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    B.tir_cache_attention(qd, cache, view, ld, cd, q.shape[0], q.shape[1], q.shape[2], *qd.stride()[:3], *view.stride()[:3], scale, dtype, out, stream)
    torch.cuda.synchronize()
    return o.cpu(), view.cpu()


def _tolerance(T, ref, dtype, out):
    tol = (2e-3 if dtype == "f16" else 6e-3) * T + 1e-5
    return tol + (0 if out == "f32" else (2.0 ** -11 if out == "f16" else 2.0 ** -8)) * ref.abs()


def _check_attention(pool, table, q, lens, count, scale, dtype, out, what, **kw):
    import torch
    _, got = _run_attention(pool, table, q, lens, count, scale, dtype, out, **kw)
    ref, T = R.cache_attention(q, *pool, table, lens, [q.shape[1]] * q.shape[0] if count is None else count, scale)
    left = torch.isnan(ref)
    assert torch.all(got.double()[left] == MARK), f"{what}: rows that were not asked for changed"
    err = torch.where(left, 0.0, (got.double() - ref).abs())
    tol = _tolerance(T, torch.where(left, 0.0, ref), dtype, out)
    assert torch.all(err <= tol), f"{what}: worst {float((err / tol).nan_to_num(nan=1e9).max()):.3g} of the tolerance"      # (false for NaN)
    return got


@pytest.fixture
def workspace():
    """A registered workspace for the current stream, gone again afterwards."""
    import torch
    ws = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
    B.tir_set_workspace(ws)
    yield ws
    torch.cuda.synchronize()
    B.tir_set_workspace(None)


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("heads,group,d,bt,T,lens,count", [
    (2, 1, 64, 16, 1, [1, 15, 16, 17, 0, 33, 300], None),
    (1, 4, 128, 16, 1, [1, 31, 32, 129, 0, 1000], [1, 1, 0, 1, 1, 1]),
    (2, 3, 64, 32, 3, [3, 1, 100, 64, 0], [3, 3, 2, 1, 3]),            # more queries than tokens: the first see nothing
    (1, 8, 128, 32, 5, [5, 260, 97], None),
    (2, 2, 64, 64, 8, [8, 200, 63, 3], [8, 5, 1, 7]),                  # sixteen rows, some of which see nothing
    (1, 16, 128, 128, 1, [129, 1, 0, 640], None), (3, 5, 128, 16, 3, [3, 64, 65, 1000], [3, 3, 2, 3]),
    (3, 1, 128, 64, 40, [40, 333, 65, 17], [40, 40, 1, 17]),
    (1, 2, 64, 64, 150, [150, 700], [150, 133]),
    (2, 5, 64, 128, 31, [31, 129, 500], None),
    (1, 1, 128, 128, 257, [257, 600, 256], [257, 200, 129]),
])
def test_cache_attention_matches_the_plain_form(workspace, cache, dtype, out, heads, group, d, bt, T, lens, count):
    g = _gen(heads + group * 3 + d + bt + T)
    pool, table, q = _attention_case(g, cache, dtype, len(lens), T, heads, group, d, bt, lens)
    what = f"cache attention {cache} {dtype}->{out} heads={heads}x{group} d={d} bt={bt} T={T} lens={lens} count={count}"
    _say(what)
    _check_attention(pool, table, q, lens, count, d ** -0.5, dtype, out, what)


# calls that take the tiles of 256 rows: many heads, and few over many keys, shared among workgroups
TALL = [
    (2, 32, 5, 64, 32, 131, [400, 131], [131, 120], "rows256/z1"),      # (batch, key heads, query heads per key head, d, block, T, lens, count, kernel)
    (1, 64, 3, 128, 16, 180, [300], None, "rows256/z1"),
    (2, 32, 4, 64, 128, 140, [130, 400], None, "rows256/z1"),           # the first sequence is shorter than its queries
    (1, 4, 4, 64, 64, 130, [5001], None, "rows256/z20"),
    (2, 2, 8, 128, 32, 70, [4500, 63], [70, 70], "rows256/z17"),
    (3, 2, 8, 64, 16, 64, [4300, 4096, 200], [64, 1, 33], "rows256/z16"),
]


def test_the_tall_calls_take_the_tall_tiles():
    for batch, heads, group, d, bt, T, lens, count, kernel in TALL:
        assert B.tir_debug_cache_kernel(batch, T, heads * group, heads, d, bt, -(-max(lens) // bt) + 1) == kernel
    assert B.tir_debug_cache_kernel(64, 1, 32, 8, 128, 64, 128) == "rows16/z1"
    assert B.tir_debug_cache_kernel(1, 1, 32, 8, 128, 128, 1563) == "rows16/z32"
    assert B.tir_debug_cache_kernel(2, 5, 16, 4, 64, 16, 100) == "rows32/z7" and B.tir_debug_cache_kernel(2, 4, 16, 4, 64, 16, 100) == "rows16/z4"
    for beyond in ((2 ** 32, 1, 8, 8, 64, 16, 5), (1, 2 ** 31, 8, 8, 64, 16, 5), (1, 1, 2 ** 33, 2 ** 32, 64, 16, 5), (1, 1, 8, 8, 64, 16, 2 ** 32), (2 ** 30, 2 ** 20, 8, 8, 64, 16, 5)):
        assert B.tir_debug_cache_kernel(*beyond) == ""


@pytest.mark.gpu
@pytest.mark.parametrize("cache,dtype,out", [("i8", "f16", "f16"), ("e4m3", "f16", "f32"), ("i8", "bf16", "f32"), ("e4m3", "bf16", "bf16")])
@pytest.mark.parametrize("shape", TALL)
def test_cache_attention_of_many_rows(workspace, shape, cache, dtype, out):
    import torch
    batch, heads, group, d, bt, T, lens, count, kernel = shape
    g = _gen(heads + T)
    pool, table, q = _attention_case(g, cache, dtype, batch, T, heads, group, d, bt, lens)
    what = f"cache attention {cache} {dtype}->{out} {shape}"
    _say(what)
    first = _check_attention(pool, table, q, lens, count, d ** -0.5, dtype, out, what)
    again = _check_attention(pool, table, q, lens, count, d ** -0.5, dtype, out, what)
    assert torch.equal(first, again)
    table[0, 1] = -1                                         # a block that is not there, in the first chunk or the second
    _check_attention(pool, table, q, lens, count, -0.3, dtype, out, what + ", a block missing, negative scale")


@pytest.mark.gpu
@pytest.mark.parametrize("cache,dtype", [("i8", "f16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("scale", [0.0, 3.0, 100.0])
def test_many_rows_with_other_scales(workspace, cache, dtype, scale):
    """Scale zero, scores of hundreds, and of thousands, where exponent and reference are rounded apart.  A score s = scale * q.k is a sum of 64 products in fp32, off by up to
    16 * 2^-24 of their magnitudes' sum (the products' own order of summation: at most 16 additions deep), a probability by as much of itself, a row by twice that of T."""
    import torch
    batch, heads, group, d, bt, T, lens = 2, 32, 5, 64, 32, 131, [400, 131]
    g = _gen(61)
    pool, table, q = _attention_case(g, cache, dtype, batch, T, heads, group, d, bt, lens)
    pool = list(pool)
    pool[3] = pool[3] * torch.exp2(torch.randint(-12, 13, pool[3].shape, generator=g).float())
    _say(f"many rows, {cache} {dtype}, scale {scale}")
    _, got = _run_attention(pool, table, q, lens, None, scale, dtype, "f32")
    ref, tt = R.cache_attention(q, *pool, table, lens, [T] * 2, scale)
    largest = float((pool[0].float() * pool[2][..., None, None]).nan_to_num(0).abs().amax()) * float(q.float().abs().sum(-1).max())
    tol = _tolerance(tt, ref, dtype, "f32") + 2 * scale * largest * 2.0 ** -20 * tt
    assert torch.all((got.double() - ref).abs() <= tol)


@pytest.mark.gpu
@pytest.mark.parametrize("cache,dtype", [("i8", "f16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_cache_attention_scales(workspace, cache, dtype, scale):
    """Scale zero (the mean of the values), a negative one, and scores of hundreds; the keys' and values' scales of the blocks differ by up to 2^24."""
    import torch
    g = _gen(17)
    lens = [1, 40, 700]
    pool, table, q = _attention_case(g, cache, dtype, 3, 2, 2, 2, 64, 32, lens)
    pool = list(pool)
    pool[3] = pool[3] * torch.exp2(torch.randint(-12, 13, pool[3].shape, generator=g).float())
    _say(f"cache attention {cache} {dtype} scale={scale}")
    what = f"scale {scale}"
    # scores of |t| = 700 in fp32 move a probability by 700 * 2^-23 = 8e-5 of itself: within the tolerance's slack
    _check_attention(pool, table, q, lens, None, scale, dtype, "f32", what)


@pytest.mark.gpu
@pytest.mark.parametrize("cache,dtype", [("i8", "bf16"), ("e4m3", "f16")])
def test_cache_attention_without_some_blocks(workspace, cache, dtype):
    """Blocks that are not there are not seen, whatever block they fall into: first, middle, last, all."""
    import torch
    for bt in (16, 64):
        lens = [5 * bt + 3] * 5
        pool, table, q = _attention_case(_gen(bt), cache, dtype, 5, 2, 1, 4, 64, bt, lens)
        table[0, 0] = -1
        table[1, 2] = pool[0].shape[0]
        table[2, 5] = 2 ** 31 - 1
        table[3, :] = -2 ** 31
        table[4, 1::2] = -1
        _say(f"cache attention {cache} {dtype} bt={bt}, blocks missing")
        got = _check_attention(pool, table, q, lens, None, 0.2, dtype, "f32", f"missing blocks of {bt}")
        assert torch.all(got[3] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 70])
def test_cache_attention_strides_and_rows_behind(workspace, T):
    """Queries as a slice of a wider projection, outputs into a larger buffer: nothing outside the asked rows changes."""
    import torch
    g = _gen(23)
    lens, count = [70, 0, 400], [T, T, (T + 1) // 2]
    pool, table, q = _attention_case(g, "i8", "f16", 3, T, 2, 2, 64, 32, lens)
    wide = torch.randn((3, T, 4, 128 + 64), generator=g).to(torch.float16)
    q = wide[..., 64:128]
    _say(f"cache attention strided, T={T}")
    whole, view = _run_attention(pool, table, q, lens, count, 0.125, "f16", "f16", o_shape=(3, T + 2, 5, 80))
    ref, tt = R.cache_attention(q, *pool, table, lens, count, 0.125)
    asked = ~torch.isnan(ref)
    assert torch.all(((view.double() - ref).abs() <= _tolerance(tt, ref, "f16", "f16"))[asked])
    whole[:, :T, :4, :64][asked] = MARK
    assert torch.all(whole == MARK)


@pytest.mark.gpu
@pytest.mark.parametrize("cache,dtype", [("i8", "f16"), ("e4m3", "bf16")])
def test_cache_attention_of_clamped_lengths(workspace, cache, dtype):
    """Lengths and counts outside their ranges count as the nearest inside."""
    import torch
    bt, cap = 32, 4 * 32
    pool, table, q = _attention_case(_gen(29), cache, dtype, 4, 3, 1, 2, 64, bt, [cap - bt] * 4, spare=8)
    table[:, -1] = table[:, 0]
    _say("cache attention, lengths outside their range")
    _check_attention(pool, table, q, [2 ** 31 - 1, -5, cap + 1, cap], [3, 3, 2 ** 31 - 1, -2 ** 31], 0.1, dtype, "f32", "clamped")


@pytest.mark.gpu
@pytest.mark.parametrize("cache,dtype,d,bt", [("i8", "f16", 128, 64), ("e4m3", "bf16", 64, 16), ("i8", "bf16", 128, 128)])
@pytest.mark.parametrize("T", [1, 6])
def test_cache_attention_shared_among_workgroups(cache, dtype, d, bt, T):
    """Few queries over many keys with and without a workspace, and the same call again: the same bits again, within the tolerance of each other."""
    import torch
    lens = [9001, 130, 5003, 0, 1]
    pool, table, q = _attention_case(_gen(31), cache, dtype, 5, T, 2, 4, d, bt, lens)
    # ... with the weight of the softmax at one end, which most slices are far from
    q = q * 3
    q = q.to(R.TORCH[dtype])
    _say(f"cache attention {cache} {dtype} d={d} bt={bt} T={T} in slices")
    B.tir_set_workspace(None)
    alone = _check_attention(pool, table, q, lens, None, d ** -0.5, dtype, "f32", "one workgroup")
    ws = torch.full((B.tir_workspace_bytes(),), 255, dtype=torch.uint8, device="cuda")
    B.tir_set_workspace(ws)
    try:
        shared = [_check_attention(pool, table, q, lens, None, d ** -0.5, dtype, "f32", "slices") for _ in range(3)]
    finally:
        torch.cuda.synchronize()
        B.tir_set_workspace(None)
    assert all(torch.equal(x, shared[0]) for x in shared)
    assert not torch.equal(alone, shared[0])                 # (the sums are grouped differently: the slices did run)


@pytest.mark.gpu
def test_a_cache_of_more_than_4_gib():
    """Blocks whose bytes lie beyond 2^32: appended to and read."""
    import torch
    heads, d, bt = 8, 128, 128
    blocks = (1 << 32) // (heads * d * bt) + 40
    g = _gen(37)
    _say(f"cache of {blocks} blocks, {blocks * heads * d * bt / 2 ** 30:.1f} GiB twice")
    k = torch.zeros((blocks, heads, bt, d), dtype=torch.int8, device="cuda")
    v = torch.zeros((blocks, heads, d, bt), dtype=torch.int8, device="cuda")
    ks, vs = torch.zeros((blocks, heads), device="cuda"), torch.zeros((blocks, heads), device="cuda")
    ids = torch.tensor([[blocks - 1, blocks - 7, 3], [blocks - 3, 0, blocks - 20]], dtype=torch.int32)
    cache = B.make_kv_cache(k, v, ks, vs, ids.cuda())
    T = 300
    kv = torch.randn((2, T, 2, heads, d), generator=g).to(torch.float16)
    kd = kv.cuda()
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    B.tir_cache_append(cache, kd[:, :, 0], kd[:, :, 1], zero, None, 2, T, *kd[:, :, 0].stride()[:3], *kd[:, :, 1].stride()[:3], "f16")
    q = torch.randn((2, 2, heads, d), generator=g).to(torch.float16)
    o = torch.empty((2, 2, heads, d), device="cuda")
    qd, lens = q.cuda(), torch.full((2,), T, dtype=torch.int32, device="cuda")
    B.tir_cache_attention(qd, cache, o, lens, None, 2, 2, heads, *qd.stride()[:3], *o.stride()[:3], 0.09, "f16", "f32")
    torch.cuda.synchronize()
    # the same with the blocks moved together
    flat = ids.flatten().long()
    small = [x.new_zeros((6,) + x.shape[1:]).cpu() for x in (k, v, ks, vs)]
    tab = torch.arange(6, dtype=torch.int32).view(2, 3)
    want = R.append(*small, tab, kv[:, :, 0], kv[:, :, 1], [0, 0], [T, T])
    for a, b in zip((k, v, ks, vs), want):
        assert torch.equal(a[flat.cuda()].cpu(), b)
    ref, tt = R.cache_attention(q, *want, tab, [T, T], [2, 2], 0.09)
    assert torch.all((o.cpu().double() - ref).abs() <= _tolerance(tt, ref, "f16", "f32"))


@pytest.mark.gpu
@pytest.mark.parametrize("other_stream", [False, True])
def test_decoding_steps_in_a_graph(other_stream):
    """Append and attend captured once and replayed token after token, with the lengths advanced on the device and eager work between the replays:
    every step against the plain form of the whole sequence."""
    import torch
    heads, group, d, bt, batch, steps = 2, 4, 64, 16, 3, 6
    g = _gen(41)
    first = [0, 14, 300]
    cols = 22
    pool = [x.cuda() for x in _pool(g, "i8", batch * cols, heads, bt, d)]
    table = torch.randperm(batch * cols, generator=g).to(torch.int32).view(batch, cols)
    cache = B.make_kv_cache(*pool, table.cuda())
    kv_all = torch.randn((steps, batch, 1, 2, heads, d), generator=g).to(torch.bfloat16)
    q_all = torch.randn((steps, batch, 1, heads * group, d), generator=g).to(torch.bfloat16)
    kv, q = kv_all[0].cuda(), q_all[0].cuda()
    o = torch.zeros((batch, 1, heads * group, d), dtype=torch.float32, device="cuda")
    start, lens = (torch.tensor(first, dtype=torch.int32, device="cuda") for _ in range(2))
    one = torch.ones_like(start)
    ws = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream() if other_stream else torch.cuda.current_stream()
    cap = torch.cuda.Stream()

    def step(stream):
        B.tir_cache_append(cache, kv[:, :, 0], kv[:, :, 1], start, None, batch, 1, *kv[:, :, 0].stride()[:3], *kv[:, :, 1].stride()[:3], "bf16", stream)
        B.tir_cache_attention(q, cache, o, lens, None, batch, 1, heads * group, *q.stride()[:3], *o.stride()[:3], 0.125, "bf16", "f32", stream)

    lens.add_(one)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=cap, capture_error_mode="global"):
        B.tir_set_workspace(ws, cap)
        step(cap)
    want = [x.cpu() for x in pool]
    held = list(first)
    for i in range(steps):
        kv.copy_(kv_all[i])
        q.copy_(q_all[i])
        torch.cuda.synchronize()
        _say(f"decoding step {i}")
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        want = R.append(*want, table, kv_all[i][:, :, 0], kv_all[i][:, :, 1], held, [1] * batch)
        held = [x + 1 for x in held]
        for a, b in zip(pool, want):
            assert torch.equal(a.cpu(), b)
        ref, tt = R.cache_attention(q_all[i], *want, table, held, [1] * batch, 0.125)
        assert torch.all((o.cpu().double() - ref).abs() <= _tolerance(tt, ref, "bf16", "f32"))
        eager = torch.randn(1 << 16, device="cuda").sum()    # the program's own work between the replays
        start.add_(one)
        lens.add_(one)
        assert torch.isfinite(eager)
    B.tir_set_workspace(None, cap)


@pytest.mark.gpu
def test_two_streams_with_workspaces_of_their_own():
    import torch
    lens = [5000, 3000]
    cases = [_attention_case(_gen(43 + i), "e4m3", "f16", 2, 1, 2, 2, 128, 32, lens) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    wss = [torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = []
    keep = []
    torch.cuda.synchronize()
    for (pool, table, q), st, ws in zip(cases, streams, wss):
        dev = [x.cuda() for x in pool]
        cache = B.make_kv_cache(*dev, table.cuda())
        qd, o, ld = q.cuda(), torch.zeros(q.shape, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
        keep.append((cache, qd, ld))
        outs.append(o)
    torch.cuda.synchronize()
    _say("two streams")
    for st, ws in zip(streams, wss):
        B.tir_set_workspace(ws, st)
    for _ in range(10):
        for (cache, qd, ld), o, st in zip(keep, outs, streams):
            B.tir_cache_attention(qd, cache, o, ld, None, 2, 1, 4, *qd.stride()[:3], *o.stride()[:3], 0.1, "f16", "f32", st)
    torch.cuda.synchronize()
    for (pool, table, q), o, st in zip(cases, outs, streams):
        ref, tt = R.cache_attention(q, *pool, table, lens, [1, 1], 0.1)
        assert torch.all((o.cpu().double() - ref).abs() <= _tolerance(tt, ref, "f16", "f32"))
        B.tir_set_workspace(None, st)
