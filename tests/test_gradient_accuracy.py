"""Gradients where D_i = sum_j P_ij dP_ij is large beside what dP - D leaves: values far from zero, peaked probabilities, keys with a mean.

Tolerances, per element, with u the input type's half step, a_ij = sum_c |dO_ic| |V_jc| and its mean A_i = sum_j P_ij a_ij:
  - the estimate of D from the forward pass's output is off by E_i <= 2u A_i (probabilities and output rounded once each), and taken back to fp32 sums: of d terms in dP, of n in D, each at most
    128 * 2^-24 < 8e-6 of their magnitudes when they add up without cancelling, so D is within 2e-5 A_i and dP within 2e-5 a_ij;
  - dQ: dS' = P (dP - D') is rounded once, u (|dS| + P E); the P that goes with the correction once, u P E; so u |dS| + 4u^2 P A + 2e-5 P (a + A), times |K|, times scale;
  - dK: u |dS| + 2e-5 P (a + A), times |Q|, times scale;
  - the result is rounded to u of itself, F16 subnormals to 2^-25.  (1.01 for u^2 and the exponentials' last bits.)"""
import pytest

from paper_2207_04296_amd import binding as B
from tests import decoder_reference as R
from tests.test_cross_attention_gradients import U, _forward_and_backward, workspace  # noqa: F401  (a fixture)

HEADS, M = 2, 50
# values: (mean, spread), size of the queries, mean of the keys
DATA = [((8.0, 0.1), 1.0, 0.0), ((2.0, 1.0), 1.0, 0.0), ((0.0, 1.0), 4.0, 0.0), ((8.0, 0.1), 1.0, 3.0), ((-100.0, 1.0), 1.0, 0.0)]
LENS = [[65], [77], [128], [129, 64, 5, 65], [333, 64, 128], [1500, 300]]


def _inputs(dtype, d, lens, data):
    import torch
    (mean, spread), size, shift = data
    g, t = torch.Generator().manual_seed(len(lens) + lens[0] + d), R.TORCH[dtype]
    n = max(lens)
    q = (torch.randn((len(lens), M, HEADS, d), generator=g) * size).to(t)
    k = (torch.randn((len(lens), n, HEADS, d), generator=g) + shift).to(t)
    v = (mean + spread * torch.randn((len(lens), n, HEADS, d), generator=g)).to(t)
    return q, k, v, torch.randn(q.shape, generator=g).to(t)


def _worst(dtype, lens, scale, q, k, v, do, got):
    """The largest share of its tolerance that an element of dq, dk and delta takes."""
    import torch
    u = U[dtype]
    worst = {"dq": 0.0, "dk": 0.0, "delta": 0.0}
    for b, length in enumerate(lens):
        Q, K, V, G = (x[b, :y].double().transpose(0, 1) for x, y in ((q, M), (k, length), (v, length), (do, M)))
        P = torch.softmax(scale * Q @ K.transpose(1, 2), -1)
        dP, a = G @ V.transpose(1, 2), G.abs() @ V.abs().transpose(1, 2)
        D, A = (P * dP).sum(-1, keepdim=True), (P * a).sum(-1, keepdim=True)
        dS = P * (dP - D)
        sums = 1.01 * u * dS.abs() + 2e-5 * P * (a + A)
        for name, ref, mag, out in (("dq", dS @ K, (sums + 4 * u * u * P * A) @ K.abs(), got["dq"][b]), ("dk", dS.transpose(1, 2) @ Q, sums.transpose(1, 2) @ Q.abs(), got["dk"][b, :length])):
            ref, mag = scale * ref.transpose(0, 1), scale * mag.transpose(0, 1)
            worst[name] = max(worst[name], float(((out.double() - ref).abs() / (mag + u * ref.abs() + 2.0 ** -25)).nan_to_num(nan=1e9).max()))
        worst["delta"] = max(worst["delta"], float(((got["delta"][b].double() - D.squeeze(-1)).abs() / (2e-5 * A.squeeze(-1))).nan_to_num(nan=1e9).max()))
    return worst


def _emulated(dtype, lens, scale, q, k, v, do, corrected):
    """The gradients' arithmetic in fp32 with its roundings; not corrected: D from the rounded output alone."""
    import torch
    t = R.TORCH[dtype]
    r = lambda x: x.to(t).float()  # noqa: E731
    out = {"dq": torch.zeros(q.shape), "dk": torch.zeros(k.shape), "delta": torch.zeros((len(lens), HEADS, M))}
    for b, length in enumerate(lens):
        Q, K, V, G = (x[b, :y].float().transpose(0, 1) for x, y in ((q, M), (k, length), (v, length), (do, M)))
        P = torch.softmax(scale * Q @ K.transpose(1, 2), -1)
        dP = G @ V.transpose(1, 2)
        D = (G * r(P @ V)).sum(-1, keepdim=True)
        dS = P * (dP - D)
        dq = r(dS) @ K
        if corrected:
            e = dS.sum(-1, keepdim=True)
            dq, D = dq - e * (r(P) @ K), D + e
            dS = P * (dP - D)
        out["dq"][b] = r(scale * dq).transpose(0, 1)
        out["dk"][b, :length] = r(scale * r(dS).transpose(1, 2) @ Q).transpose(0, 1)
        out["delta"][b] = D.squeeze(-1)
    return out


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_the_tolerances_tell_a_rounded_output_from_a_corrected_one(dtype):
    for lens in LENS[:4]:
        args = (dtype, lens, 0.125, *_inputs(dtype, 64, lens, DATA[0]))
        plain, corrected = (_worst(*args, _emulated(*args, c)) for c in (False, True))
        assert max(corrected.values()) <= 1 < min(plain["dq"], plain["delta"]), (lens, plain, corrected)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("shared", [True, False])
def test_gradients_do_not_lose_what_the_output_rounds_away(request, shared, lens, dtype, d):
    """One length and ragged ones on both sides of a chunk's and a tile's end, keys shared among workgroups and not."""
    import torch
    if shared:
        request.getfixturevalue("workspace")
    else:
        B.tir_set_workspace(None)
    for data in DATA:
        q, k, v, do = _inputs(dtype, d, lens, data)
        kv = torch.stack((k, v), 2)
        for b, n in enumerate(lens):
            kv[b, n:] = float("nan")
        got = _forward_and_backward(q, kv, do, lens, 0.125, dtype)
        worst = _worst(dtype, lens, 0.125, q, k, v, do, got)
        print(f"[case] {dtype} d={d} lens={lens} shared={shared} data={data}: worst of the tolerance {worst}", flush=True)
        assert max(worst.values()) <= 1, worst
        for b, n in enumerate(lens):
            assert torch.all(got["dk"][b, n:] == 0) and torch.all(got["dv"][b, n:] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens", [[1], [1, 1, 1], [1, 40, 1], [70, 1, 0], [1, 300]])
def test_a_single_key_has_no_gradient(workspace, lens, dtype, d):  # noqa: F811
    """The probability of a single key is 1 whatever the query: dQ and dK of such a sequence are zero exactly, and dV is the sum of dO (rounded once: u of itself; a P within 1e-5 of 1
    rounds to 1, and fp32 sums of up to 50 terms are within 1e-5 of their magnitudes)."""
    import torch
    q, k, v, do = _inputs(dtype, d, lens, DATA[1])
    got = _forward_and_backward(q, torch.stack((k, v), 2), do, lens, 0.3, dtype)
    print(f"[case] single keys, {dtype} d={d} lens={lens}", flush=True)
    for b, n in enumerate(lens):
        if n == 1:
            assert torch.all(got["dq"][b] == 0) and torch.all(got["dk"][b] == 0)
            want, mag = do[b].double().sum(0), do[b].double().abs().sum(0)
            assert torch.all((got["dv"][b, 0].double() - want).abs() <= U[dtype] * want.abs() + 1e-5 * mag)


# (batch, m, n, key heads, query heads per key head, lens): few probabilities, or up to 16384 of them
SMALL = [(1, 2, 110, 8, 1, None), (2, 27, 2, 3, 1, [2, 1]), (1, 1, 3, 1, 1, None), (3, 5, 64, 1, 2, [64, 1, 0]), (1, 32, 32, 8, 2, None), (2, 1, 1024, 4, 2, [1024, 300]), (1, 128, 128, 1, 1, None),
         (16, 1, 64, 16, 1, None), (1, 3, 700, 2, 1, [651]), (1, 1024, 16, 1, 1, None), (1, 1, 500, 1, 8, None)]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", SMALL)
def test_small_calls_round_in_two_parts(workspace, shape, dtype, d):  # noqa: F811
    """P and dS as operands in two parts leave u^2 of themselves (F16: and 2^-38 of the largest of a row or key); P is within 1e-5 of itself (fp32 scores of up to ten), and D, dP as above:
    |error| <= u |ref| + |scale| sum (u^2 (|dS| + 4 P A) + 2^-36 max|dS| + 2e-5 P (a + A)) |K|, dK alike, dV: u |ref| + (u^2 + 1e-5) sum P |dO|.  In norm that is the result's own rounding: at most
    u / sqrt(3) of it if all were just above a power of two, and 1.02 for the rest."""
    import torch
    batch, m, n, heads, group, lens = shape
    g, t, u = torch.Generator().manual_seed(sum(shape[:5]) + d), R.TORCH[dtype], U[dtype]
    q, do = (torch.randn((batch, m, heads * group, d), generator=g).to(t) for _ in range(2))
    k, v = (torch.randn((batch, n, heads, d), generator=g).to(t) for _ in range(2))
    got = _forward_and_backward(q, torch.stack((k, v), 2), do, lens, d ** -0.5, dtype)
    ref = {x: torch.zeros(y.shape, dtype=torch.float64) for x, y in (("dq", q), ("dk", k), ("dv", v))}
    tol = {x: torch.zeros_like(y) for x, y in ref.items()}
    for b in range(batch):
        length = n if lens is None else lens[b]
        for j in range(heads * group):
            h = j // group
            Q, K, V, G = q[b, :, j].double(), k[b, :length, h].double(), v[b, :length, h].double(), do[b, :, j].double()
            P = torch.softmax(d ** -0.5 * Q @ K.T, 1) if length else torch.zeros((m, 0), dtype=torch.float64)
            dP, a = G @ V.T, G.abs() @ V.abs().T
            A = (P * a).sum(1, keepdim=True)
            dS = P * (dP - (P * dP).sum(1, keepdim=True))
            most = float(dS.abs().max()) if length else 0.0
            fuzz = u * u * (dS.abs() + 4 * P * A) + 2.0 ** -36 * most + 2e-5 * P * (a + A)
            ref["dq"][b, :, j] = d ** -0.5 * dS @ K
            tol["dq"][b, :, j] = d ** -0.5 * fuzz @ K.abs()
            ref["dk"][b, :length, h] += d ** -0.5 * dS.T @ Q
            tol["dk"][b, :length, h] += d ** -0.5 * fuzz.T @ Q.abs()
            ref["dv"][b, :length, h] += P.T @ G
            tol["dv"][b, :length, h] += (u * u + 1e-5) * P.T @ G.abs()
    worst, norms = {}, {}
    for x, want in ref.items():
        err = (got[x].double() - want).abs()
        worst[x] = float((err / (tol[x] + u * want.abs() + 2.0 ** -25)).max())
        norms[x] = float(err.norm() / (u * want.norm() + 1e-9 * want.numel() ** 0.5))
    print(f"[case] small call {shape} {dtype} d={d}: worst of the tolerance {worst}, norms in u {norms}", flush=True)
    assert max(worst.values()) <= 1, worst
    assert max(norms.values()) <= 1.02 * 3 ** -0.5, norms
