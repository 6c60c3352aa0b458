"""The gradients' two forms of call: with the strides of the gradient that arrives, and without them, where they are that tensor's own."""
import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R

FAKE = 0x1000
STRIDES = (1280, 256, 64, 896, 128, 64, 896, 128, 64, 1280, 256, 64)      # of Q, K, V, O


class Tensor:
    """What the binding asks of a tensor; its address is no address."""
    def __init__(self, shape, strides, address=FAKE):
        self.shape, self.strides, self.address = shape, strides, address

    def stride(self):
        return self.strides

    def data_ptr(self):
        return self.address


def _call(*rest, dO=FAKE, **named):
    return B.tir_cross_attention_backward_status(FAKE, FAKE, FAKE, FAKE, dO, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 2, 5, 7, 4, 2, 64, *STRIDES, *rest, **named)


def test_strides_left_out_are_those_of_the_tensor():
    """Refusals tell which strides were taken: of dO 4 is no multiple of 8, and -8 is negative."""
    odd, negative = Tensor((2, 5, 4, 64), (1280, 4, 64, 1)), Tensor((2, 5, 4, 64), (-8, 256, 64, 1))
    for rest, named in (((0.125, "f16"), {}), ((0.125, "f16", 0), {}), ((0.125, "f16"), {"stream": 0}), ((), {"scale": 0.125, "in_dtype": "f16"})):
        assert _call(*rest, dO=odd, **named) == B.TIR_ERR_ALIGNMENT and "strides of dO" in B.last_error()
        assert _call(*rest, dO=negative, **named) == B.TIR_ERR_INVALID_ARG and "stride of dO" in B.last_error()
    # given ones count, whatever the tensor's are
    good = Tensor((2, 5, 4, 64), (1280, 256, 64, 1))
    assert _call(1280, 4, 64, 0.125, "f16", dO=good) == B.TIR_ERR_ALIGNMENT
    assert _call(1280, 256, 64, 0.125, "f16", 0, dO=Tensor((2, 5, 4, 64), (1280, 4, 64, 1), FAKE + 8)) == B.TIR_ERR_ALIGNMENT and "16-byte" in B.last_error()
    # an address has O's
    assert _call(0.125, "f16", dO=FAKE + 8) == B.TIR_ERR_ALIGNMENT and "16-byte" in B.last_error()


@pytest.mark.parametrize("rest,named", [((), {}), ((0.125,), {}), ((1280, 256), {"scale": 0.125, "in_dtype": "f16"}), ((1280, 256, 64, 0.125), {}), ((0.125,), {"in_dtype": "f16"}),
                                        ((0.125, "f16"), {"scale": 0.125}), ((), {"in_dtype": "f16"})])
def test_half_of_the_strides_or_no_scale_is_refused(rest, named):
    with pytest.raises(TypeError, match="scale and in_dtype"):
        _call(*rest, **named)


def test_a_gradient_of_another_shape_needs_its_strides():
    by_head = Tensor((2, 4, 5, 64), (1280, 320, 64, 1))
    with pytest.raises(ValueError, match="left out"):
        _call(0.125, "f16", dO=by_head)
    assert _call(1280, 64, 320, 0.125, "f16", dO=Tensor((2, 4, 5, 64), (1280, 320, 64, 1), FAKE + 8)) == B.TIR_ERR_ALIGNMENT


@pytest.mark.gpu
def test_both_forms_give_the_same_gradients():
    """dO token by token while O is head by head, and a dO broadcast over the queries: the two forms agree to the bit, and with the formulas
    (tolerance: 3u * the sum of magnitudes + u * |ref| + 1e-6, u = 2^-11, as for the other gradient tests)."""
    import torch
    batch, m, n, heads, d = 2, 70, 90, 2, 64
    g = torch.Generator().manual_seed(43)
    q, k, v, do = (torch.randn((batch, x, heads, d), generator=g).to(torch.float16) for x in (m, n, n, m))
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    o = torch.empty((batch, heads, m, d), dtype=torch.float16, device="cuda").transpose(1, 2)
    lse, delta = torch.empty((batch, heads, m), device="cuda"), torch.empty((batch, heads, m), device="cuda")
    strides = (*qd.stride()[:3], *kd.stride()[:3], *vd.stride()[:3], *o.stride()[:3])
    B.tir_cross_attention(qd, kd, vd, o, lse, None, batch, m, n, heads, heads, d, *strides, 0.125, "f16", "f16")
    for dod in (do.cuda(), do.cuda()[:, :1].expand(-1, m, -1, -1)):
        results = []
        for rest in ((0.125, "f16"), (*dod.stride()[:3], 0.125, "f16")):
            grads = [torch.full_like(x, 77.0) for x in (qd, kd, vd)]
            B.tir_cross_attention_backward(qd, kd, vd, o, dod, lse, None, *grads, delta, batch, m, n, heads, heads, d, *strides, *rest)
            results.append(grads)
        torch.cuda.synchronize()
        print(f"[case] gradients with and without the strides of dO {dod.stride()}", flush=True)
        ref = R.cross_attention(q, k, v, None, 0.125, dod.cpu())
        for a, b, name in zip(*results, ("dq", "dk", "dv")):
            assert torch.equal(a, b), name
            tol = 3 * 2.0 ** -11 * ref[name + "_sum"] + 2.0 ** -11 * ref[name].abs() + 1e-6
            assert torch.all((a.cpu().double() - ref[name]).abs() <= tol), name
