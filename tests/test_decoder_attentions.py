"""The plain forms themselves, against torch's own derivatives; and the operators together, as a decoder layer calls them."""
import math

import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R


def test_the_plain_gradients_are_the_derivatives():
    """decoder_reference's o, lse and gradients against torch's autograd of the definition in 64 bits, with shared key heads, a short and an empty sequence."""
    import torch
    g = torch.Generator().manual_seed(1)
    batch, m, n, heads, group, d, lens, scale = 3, 7, 11, 2, 3, 8, [11, 4, 0], 0.3
    q, k, v, do = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((batch, m, heads * group, d), (batch, n, heads, d), (batch, n, heads, d), (batch, m, heads * group, d)))
    want = R.cross_attention(q, k, v, lens, scale, do)
    q, k, v = (x.requires_grad_() for x in (q, k, v))
    kk, vv = k.repeat_interleave(group, 2), v.repeat_interleave(group, 2)
    total = 0
    for b in range(2):
        s = torch.einsum("ihc,jhc->hij", q[b], kk[b, :lens[b]]) * scale
        o = torch.einsum("hij,jhc->ihc", torch.softmax(s, -1), vv[b, :lens[b]])
        assert torch.allclose(o, want["o"][b], rtol=1e-12, atol=1e-12)
        assert torch.allclose(torch.logsumexp(s, -1), want["lse"][b], rtol=1e-12, atol=1e-12)
        total = total + (o * do[b]).sum()
    assert torch.all(want["o"][2] == 0) and torch.all(want["lse"][2] == -math.inf)
    for x, name in zip(torch.autograd.grad(total, (q, k, v)), ("dq", "dk", "dv")):
        assert torch.allclose(x, want[name], rtol=1e-11, atol=1e-11), name


@pytest.mark.parametrize("cache", ["i8", "e4m3"])
def test_the_plain_append_in_one_go_and_token_by_token(cache):
    """Values that never grow: quantising a prompt at once and token by token are then the same, and the error is half a step."""
    import torch
    g = torch.Generator().manual_seed(2)
    heads, d, bt, T = 2, 16, 8, 21
    new = torch.rand((1, T, heads, d), generator=g) * 2 - 1
    new[:, ::8, :, 0] = 1.5                                   # the first token of each block has its largest value
    new = new.to(torch.bfloat16)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    dt = R.TORCH[cache]
    empty = [torch.zeros((3, heads, bt, d), dtype=dt), torch.zeros((3, heads, d, bt), dtype=dt), torch.zeros((3, heads)), torch.zeros((3, heads))]
    once = R.append(*empty, table, new, new, [0], [T])
    steps = empty
    for t in range(T):
        steps = R.append(*steps, table, new[:, t:t + 1], new[:, t:t + 1], [t], [1])
    for a, b in zip(once, steps):
        assert torch.equal(a.float(), b.float())
    back = (once[0].float() * once[2][..., None, None])[table[0].long()].transpose(1, 2).reshape(-1, heads, d)[:T]
    half = 1.5 / 127 / 2 if cache == "i8" else 1.5 * 2.0 ** -4
    assert float((back - new[0].float()).abs().max()) <= half * (1 + 1e-6)
    assert torch.equal(once[1].transpose(2, 3).float(), once[0].float())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cache,group", [("bf16", "i8", 4), ("f16", "e4m3", 1)])
def test_a_decoder_layer_serves_prompts_and_tokens(dtype, cache, group):
    """Two attentions of a layer over ragged prompts and then token by token: projections by the library's products, keys and values appended, self attention over the
    cache, its output as the queries of the attention over an encoder's states.  Every step against the plain forms on the same inputs."""
    import torch
    g = torch.Generator().manual_seed(3)
    t = R.TORCH[dtype]
    batch, heads, d, bt, width, n = 3, 2, 64, 16, 96, 75
    hq = heads * group
    enc_lens, prompts = [75, 20, 50], [37, 1, 20]
    wq, wkv = (torch.randn((width, x), generator=g) * width ** -0.5 for x in (hq * d, 2 * heads * d))
    wq, wkv = wq.to(t), wkv.to(t)
    enc = torch.randn((batch, n, 2, heads, d), generator=g).to(t)
    cols = 5
    pool = [torch.zeros((batch * cols, heads, bt, d), dtype=R.TORCH[cache]), torch.zeros((batch * cols, heads, d, bt), dtype=R.TORCH[cache])]
    pool += [torch.zeros((batch * cols, heads)) for _ in range(2)]
    table = torch.randperm(batch * cols, generator=g).to(torch.int32).view(batch, cols)
    dev = [x.cuda() for x in pool]
    kvc = B.make_kv_cache(*dev, table.cuda())
    wqd, wkvd, encd = wq.cuda(), wkv.cuda(), enc.cuda()
    eld = torch.tensor(enc_lens, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
    B.tir_set_workspace(ws)
    held = [0] * batch
    try:
        for step, T in enumerate([37, 1, 1, 3]):
            counts = prompts if step == 0 else [T] * batch
            x = torch.randn((batch, T, width), generator=g).to(t)
            xd = x.cuda()
            q = torch.empty((batch, T, hq, d), dtype=t, device="cuda")
            kv = torch.empty((batch, T, 2, heads, d), dtype=t, device="cuda")
            for w, out in ((wqd, q), (wkvd, kv)):
                B.tir_gemm(xd, w, out, batch * T, w.shape[1], width, width, 1, w.shape[1], 1, w.shape[1], 1, dtype, dtype)
            start, cnt = (torch.tensor(y, dtype=torch.int32, device="cuda") for y in (held, counts))
            k, v = kv[:, :, 0], kv[:, :, 1]
            B.tir_cache_append(kvc, k, v, start, cnt, batch, T, *k.stride()[:3], *v.stride()[:3], dtype)
            lens = start + cnt
            a = torch.zeros((batch, T, hq, d), dtype=t, device="cuda")
            B.tir_cache_attention(q, kvc, a, lens, cnt, batch, T, hq, *q.stride()[:3], *a.stride()[:3], d ** -0.5, dtype, dtype)
            o = torch.empty_like(a)
            ek, ev = encd[:, :, 0], encd[:, :, 1]
            B.tir_cross_attention(a, ek, ev, o, None, eld, batch, T, n, hq, heads, d, *a.stride()[:3], *ek.stride()[:3], *ev.stride()[:3], *o.stride()[:3], d ** -0.5, dtype, dtype)
            torch.cuda.synchronize()
            print(f"[case] layer {dtype} {cache} step {step}: {T} tokens, {held} held", flush=True)
            # each operator on what it was given
            qc, kvc_, ac = q.cpu(), kv.cpu(), a.cpu()
            pool = R.append(*pool, table, kvc_[:, :, 0], kvc_[:, :, 1], held, counts)
            for got, want in zip(dev, pool):
                assert torch.equal(got.cpu().float(), want.float())
            held = [h + c for h, c in zip(held, counts)]
            ref, mag = R.cache_attention(qc, *pool, table, held, counts, d ** -0.5)
            u, half = (2e-3, 2.0 ** -11) if dtype == "f16" else (6e-3, 2.0 ** -8)
            asked = ~torch.isnan(ref)
            assert torch.all(((ac.double() - ref).abs() <= u * mag + 1e-5 + half * ref.abs())[asked])
            assert torch.all(ac[~asked] == 0)
            cross = R.cross_attention(ac, enc[:, :, 0], enc[:, :, 1], enc_lens, d ** -0.5)
            assert torch.all((o.cpu().double() - cross["o"]).abs() <= u * cross["T"] + 1e-5 + half * cross["o"].abs())
    finally:
        torch.cuda.synchronize()
        B.tir_set_workspace(None)


@pytest.mark.gpu
def test_threads_that_call_on_one_stream_take_turns():
    """Gradients and an attention whose partial results pass from one launch to the next, and a product with a split reduction, called by three threads on one stream: as when called alone, to the bit."""
    import threading

    import torch
    g = torch.Generator().manual_seed(5)
    m, n, d = 1500, 77, 64
    q, k, v, do = (torch.randn((1, x, 2, d), generator=g).to(torch.bfloat16).cuda() for x in (m, n, n, m))
    o, lse = torch.empty_like(q), torch.empty((1, 2, m), device="cuda")
    a, b = (torch.randn((64, 8192), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    heads, bt, length, T = 4, 64, 5001, 130                       # (256-row tiles, sliced)
    cols = -(-length // bt)
    pool = [torch.randint(-100, 100, s, generator=g).to(torch.int8).cuda() for s in ((cols, heads, bt, d), (cols, heads, d, bt))]
    cache = B.make_kv_cache(*pool, *(torch.full((cols, heads), 0.01, device="cuda") for _ in range(2)), torch.arange(cols, dtype=torch.int32, device="cuda")[None])
    cq = torch.randn((1, T, 4 * heads, d), generator=g).to(torch.bfloat16).cuda()
    lens = torch.tensor([length], dtype=torch.int32, device="cuda")
    st = torch.cuda.Stream()
    ws = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
    strides = (*q.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3])
    assert B.tir_debug_cache_kernel(1, T, 4 * heads, heads, d, bt, cols) == "rows256/z19"
    assert "/z" in B.tir_gemm_variant(1, 64, 64, 8192, 8192, 1, 1, 8192, 64, 1, "bf16", "f32")

    def backward():
        dq, dk, dv = (torch.empty_like(x) for x in (q, k, v))
        delta = torch.empty_like(lse)
        B.tir_cross_attention_backward(q, k, v, o, do, lse, None, dq, dk, dv, delta, 1, m, n, 2, 2, d, *strides, *do.stride()[:3], 0.1, "bf16", st)
        return dq, dk, dv

    def attend():
        out = torch.empty_like(cq)
        B.tir_cache_attention(cq, cache, out, lens, None, 1, T, 4 * heads, *cq.stride()[:3], *out.stride()[:3], 0.1, "bf16", "bf16", st)
        return (out,)

    def product():
        c = torch.empty((64, 64), device="cuda")
        B.tir_gemm(a, b, c, 64, 64, 8192, 8192, 1, 1, 8192, 64, 1, "bf16", "f32", st)
        return (c,)
    torch.cuda.synchronize()
    B.tir_set_workspace(ws, st)
    try:
        B.tir_cross_attention(q, k, v, o, lse, None, 1, m, n, 2, 2, d, *strides, 0.1, "bf16", "bf16", st)
        calls = (backward, attend, product)
        alone = [f() for f in calls]
        torch.cuda.synchronize()
        results = [[] for _ in calls]

        def work(i):
            with torch.cuda.stream(st):
                for _ in range(40):
                    results[i].append(calls[i]())
        threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
        for t in threads:
            t.start()
        for t in threads:
            t.join(60)
        torch.cuda.synchronize()
        print("[case] three threads on one stream", flush=True)
        for want, got in zip(alone, results):
            assert len(got) == 40 and all(torch.equal(x, y) for r in got for x, y in zip(want, r))
    finally:
        torch.cuda.synchronize()
        B.tir_set_workspace(None, st)


def test_the_binding_wants_lengths_and_statistics_as_they_are_read():
    """int64 (torch's default), host, or strided arrays of lengths, and other statistics than fp32 ones, are refused before anything is launched."""
    import torch
    assert B._load_native()
    x, wrong = 4096, [torch.tensor([1, 2]), torch.tensor([1, 2], dtype=torch.int32), torch.zeros(4, dtype=torch.int32)[::2]]
    cache = B.KvCache(x, x, x, x, x, 4, 2, 32, 64, 2, 3, B.TIR_I8)
    s = (640, 128, 64)
    for bad in wrong:
        for start, count in ((bad, None), (x, bad)):
            with pytest.raises(TypeError, match="int32"):
                B.tir_cache_append(cache, x, x, start, count, 2, 1, *s, *s, "f16", 0)
            with pytest.raises(TypeError, match="int32"):
                B.tir_cache_attention(x, cache, x, start, count, 2, 1, 2, *s, *s, 0.1, "f16", "f16", 0)
        with pytest.raises(TypeError, match="int32"):
            B.tir_cross_attention(x, x, x, x, None, bad, 2, 1, 3, 2, 2, 64, *s, *s, *s, *s, 0.1, "f16", "f16", 0)
    for bad in (torch.zeros(2, 2, 1), torch.zeros(2, 2, 1, dtype=torch.float64)):
        with pytest.raises(TypeError, match="float32"):
            B.tir_cross_attention(x, x, x, x, bad, None, 2, 1, 3, 2, 2, 64, *s, *s, *s, *s, 0.1, "f16", "f16", 0)
        for lse, delta in ((bad, x), (x, bad)):
            with pytest.raises(TypeError, match="float32"):
                B.tir_cross_attention_backward(x, x, x, x, x, lse, None, x, x, x, delta, 2, 1, 3, 2, 2, 64, *s, *s, *s, *s, *s, 0.1, "f16", 0)
