"""Values that are not finite: the sums that hold one are infinite or NaN, all others are as exact as ever."""
import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R
from tests.test_cross_attention import _run, _tolerance, workspace  # noqa: F401  (a fixture)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,group", [(1, 1), (2, 1), (1, 3), (2, 2), (5, 1), (40, 2)])
@pytest.mark.parametrize("shared", [True, False])
def test_infinite_values_of_the_last_key(request, shared, m, group, dtype, d):
    """The last key of a sequence, which lanes behind it may read again, has an infinity of either sign and a NaN among its values; lengths that end inside a chunk and with it."""
    import torch
    if shared:
        request.getfixturevalue("workspace")
    else:
        B.tir_set_workspace(None)
    for lens in ([1, 3, 5], [31, 32, 33], [100, 64, 17], [1500, 1025, 2]):
        g = torch.Generator().manual_seed(lens[0] + m + d)
        t, n = R.TORCH[dtype], max(lens)
        q = torch.randn((3, m, 2 * group, d), generator=g).to(t)
        kv = torch.randn((3, n, 2, 2, d), generator=g).to(t)
        for b, x in enumerate(lens):
            kv[b, x - 1, 1, :, 5], kv[b, x - 1, 1, :, 9], kv[b, x - 1, 1, 1, d - 1] = float("inf"), -float("inf"), float("nan")
        out = "f32" if m == 1 else dtype
        print(f"[case] infinite values, {dtype}->{out} m={m} group={group} d={d} lens={lens} shared={shared}", flush=True)
        o, _ = _run(q, kv, lens, 0.125, dtype, out)
        ref = R.cross_attention(q, kv[:, :, 0], kv[:, :, 1], lens, 0.125)
        want, o = ref["o"], o.double()
        assert torch.equal(torch.isnan(o), torch.isnan(want))
        off = ~torch.isfinite(want)
        assert torch.equal(o[off].nan_to_num(nan=0.0), want[off].nan_to_num(nan=0.0))
        assert torch.all((o - want).abs()[~off] <= _tolerance(ref["T"], want, dtype, out)[~off])
