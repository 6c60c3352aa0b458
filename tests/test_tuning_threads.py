"""Tuning on a stream that another thread uses."""
import pytest

from paper_2207_04296_amd import binding as B


@pytest.mark.gpu
def test_tuning_and_operators_share_a_stream_and_its_workspace():
    """Gradients whose partial sums pass from one launch to the next, and a product with a split reduction, while another thread tunes such products on the same stream: as when called alone, to the bit."""
    import threading

    import torch
    g = torch.Generator().manual_seed(6)
    m, n, d, depth = 1500, 77, 64, 8192
    q, k, v, do = (torch.randn((1, x, 2, d), generator=g).to(torch.bfloat16).cuda() for x in (m, n, n, m))
    a, b = (torch.randn((64, depth), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    o, lse = torch.empty_like(q), torch.empty((1, 2, m), device="cuda")
    strides = (*q.stride()[:3], *k.stride()[:3], *v.stride()[:3], *o.stride()[:3])
    st = torch.cuda.Stream()
    ws = torch.empty(B.tir_workspace_bytes(), dtype=torch.uint8, device="cuda")
    problem = (64, 64, depth, 0, depth, 1, 0, 1, depth, 0, 64, 1, "bf16", "f32")

    def backward():
        dq, dk, dv = (torch.empty_like(x) for x in (q, k, v))
        delta = torch.empty_like(lse)
        B.tir_cross_attention_backward(q, k, v, o, do, lse, None, dq, dk, dv, delta, 1, m, n, 2, 2, d, *strides, *do.stride()[:3], 0.1, "bf16", st)
        return dq, dk, dv, delta

    def product(out=None):
        c = torch.empty((64, 64), device="cuda") if out is None else out
        B.tir_gemm(a, b, c, 64, 64, depth, depth, 1, 1, depth, 64, 1, "bf16", "f32", st)
        return (c,)
    torch.cuda.synchronize()
    B.tir_tune_clear()
    B.tir_set_workspace(ws, st)
    try:
        B.tir_cross_attention(q, k, v, o, lse, None, 1, m, n, 2, 2, d, *strides, 0.1, "bf16", "bf16", st)
        assert "/z" in B.tir_gemm_variant(1, 64, 64, depth, depth, 1, 1, depth, 64, 1, "bf16", "f32")
        alone = backward()
        want = (a.double() @ b.double().t()).cpu()
        torch.cuda.synchronize()
        tuned, times, done = torch.empty((64, 64), device="cuda"), [], threading.Event()

        def tune():
            try:
                times.append(B.tir_tune_batch_matmul(a, b, tuned, 1, *problem, reps=2, stream=st))
            finally:
                done.set()
        other = threading.Thread(target=tune)
        results = []
        with torch.cuda.stream(st):
            other.start()
            while not done.is_set() and len(results) < 4000:
                results.append((backward(), product()))
                if len(results) % 100 == 0:
                    st.synchronize()
                    assert all(torch.equal(x, y) for r, _ in results[-100:] for x, y in zip(alone, r))
                    results[-100:] = [results[-1]] + [None] * 99
        other.join(100)
        torch.cuda.synchronize()
        print(f"[case] {len(results)} calls beside a tuning of {times} us", flush=True)
        assert times and times[0] > 0 and len(results) > 5 and B.tir_tune_count() == 1
        # sums of 8192 products of normal numbers in fp32, in any order: far below 2^-24 * 8192 * 8192 ** 0.5
        bound = 2.0 ** -24 * depth * depth ** 0.5
        for r in results:
            if r is not None:
                assert all(torch.equal(x, y) for x, y in zip(alone, r[0]))
                assert float((r[1][0].cpu().double() - want).abs().max()) <= bound
        assert float((tuned.cpu().double() - want).abs().max()) <= bound
    finally:
        torch.cuda.synchronize()
        B.tir_set_workspace(None, st)
        B.tir_tune_clear()
