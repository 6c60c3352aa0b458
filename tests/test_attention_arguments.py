"""What the binding of the decoder's attentions refuses before anything is launched: caches of host tensors, arrays with fewer elements than the kernels read."""
import pytest

from paper_2207_04296_amd import binding as B

X = 4096
S = (640, 128, 64)
FORMS = ["", "_status"]


class Array:
    """A device array as the binding sees one that is too short: no kernel may get its address."""
    def __init__(self, *shape):
        self.shape = shape

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def data_ptr(self):
        raise AssertionError("the array's address was taken")


def _cache(sequences=3):
    return B.KvCache(X, X, X, X, X, 4, 2, 32, 64, sequences, 3, B.TIR_I8)


@pytest.mark.parametrize("form", FORMS)
def test_a_cache_on_the_host_is_refused(form):
    import torch
    k, v = torch.zeros((4, 2, 32, 64), dtype=torch.int8), torch.zeros((4, 2, 64, 32), dtype=torch.int8)
    cache = B.make_kv_cache(k, v, torch.zeros((4, 2)), torch.zeros((4, 2)), torch.zeros((3, 5), dtype=torch.int32))
    append, attend = (getattr(B, x + form) for x in ("tir_cache_append", "tir_cache_attention"))
    with pytest.raises(ValueError, match="on the host"):
        append(cache, X, X, X, None, 2, 1, *S, *S, "f16", 0)
    with pytest.raises(ValueError, match="on the host"):
        attend(X, cache, X, X, None, 2, 1, 2, *S, *S, 0.1, "f16", "f16", 0)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("short", [Array(2), Array(1, 2), Array(0)])
def test_an_element_per_sequence_is_needed(form, short):
    append, attend, cross, grad = (getattr(B, x + form) for x in ("tir_cache_append", "tir_cache_attention", "tir_cross_attention", "tir_cross_attention_backward"))
    for first, count in ((short, None), (X, short)):
        with pytest.raises(ValueError, match="at least 3 elements"):
            append(_cache(), X, X, first, count, 3, 1, *S, *S, "f16", 0)
        with pytest.raises(ValueError, match="at least 3 elements"):
            attend(X, _cache(), X, first, count, 3, 1, 2, *S, *S, 0.1, "f16", "f16", 0)
    with pytest.raises(ValueError, match="lens: at least 3 elements"):
        cross(X, X, X, X, None, short, 3, 1, 3, 2, 2, 64, *S, *S, *S, *S, 0.1, "f16", "f16", 0)
    with pytest.raises(ValueError, match="lens: at least 3 elements"):
        grad(X, X, X, X, X, X, short, X, X, X, X, 3, 1, 3, 2, 2, 64, *S, *S, *S, *S, *S, 0.1, "f16", 0)


@pytest.mark.parametrize("form", FORMS)
def test_statistics_have_an_element_per_row(form):
    cross, grad = (getattr(B, x + form) for x in ("tir_cross_attention", "tir_cross_attention_backward"))
    short = Array(3, 2, 4)                       # of [3, 2, 5]
    with pytest.raises(ValueError, match="lse: at least 30 elements"):
        cross(X, X, X, X, short, None, 3, 5, 3, 2, 2, 64, *S, *S, *S, *S, 0.1, "f16", "f16", 0)
    for lse, delta, name in ((short, X, "lse"), (X, short, "delta")):
        with pytest.raises(ValueError, match=name + ": at least 30 elements"):
            grad(X, X, X, X, X, lse, None, X, X, X, delta, 3, 5, 3, 2, 2, 64, *S, *S, *S, *S, *S, 0.1, "f16", 0)


def test_arrays_that_are_long_enough_pass():
    """Refused for another reason, then: a K that is not aligned."""
    class Long(Array):
        def data_ptr(self):
            return X
    for n in (2, 3, 70):
        assert B.tir_cache_append_status(_cache(), X + 2, X, Long(n), Long(n), 2, 1, *S, *S, "f16") == B.TIR_ERR_ALIGNMENT
        assert B.tir_cross_attention_status(X, X + 2, X, X, Long(2, 2, n), Long(n), 2, 2, 3, 2, 2, 64, *S, *S, *S, *S, 0.1, "f16", "f16") == B.TIR_ERR_ALIGNMENT


@pytest.mark.parametrize("scale", [2.0 ** 127 * (1 + 2.0 ** -20), 2.5e38, -2.5e38])
def test_a_scale_whose_exponent_overflows_is_refused(scale):
    """scale * log2(e) would be infinite, and a score of zero NaN; 2^127 itself passes (and is refused for what is not aligned)."""
    for s, status in ((scale, B.TIR_ERR_INVALID_ARG), (2.0 ** 127, B.TIR_ERR_ALIGNMENT), (-2.0 ** 127, B.TIR_ERR_ALIGNMENT)):
        assert B.tir_cache_attention_status(X + 2, _cache(), X, X, X, 2, 1, 2, *S, *S, s, "f16", "f16") == status and B.last_error()
        assert B.tir_cross_attention_status(X + 2, X, X, X, X, X, 2, 1, 3, 2, 2, 64, *S, *S, *S, *S, s, "f16", "f16") == status
        assert B.tir_cross_attention_backward_status(X + 2, X, X, X, X, X, X, X, X, X, X, 2, 1, 3, 2, 2, 64, *S, *S, *S, *S, *S, s, "f16") == status
