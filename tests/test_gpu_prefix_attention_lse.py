"""The log of the sum in fp32 attention, at scores where the scale's own rounding shows.

Products are exact here (one nonzero column, few bits). A score in log2 units is the product times
scale log2(e), whose rounding to fp32 is as large as it gets at the scale below: 2^-24.003 of it, 1.8e-6 nats
at a score of 31 where it is left out. With it made good, what remains is half a step of the result (2^-20 from 16
to 32), an exponential of about 1 (ex2.approx 2^-22), a logarithm of up to log 70 and the sum before the last
one (2^-23 and 2^-22): below 2^-20 + 2^-21 + 2^-23."""
import pytest
import torch

from test_gpu_prefix_attention import _ll

pytestmark = pytest.mark.gpu

SCALE = 0.08664359897375107                                # an fp32 number
TOL = 2.0 ** -20 + 2.0 ** -21 + 2.0 ** -23


@pytest.mark.parametrize("d", [64, 96])
@pytest.mark.parametrize("keys", ["own", "prefix", "both"])
def test_lse_of_scores_up_to_31(keys, d):
    ll = _ll()
    N, H, P, S = 600, 2, 70, 3
    s = (190.0 + torch.arange(N * H, device="cuda") * (112.0 / (N * H))).mul(64).round().div(64).view(N, H)
    q = torch.zeros((N, 1, H, d), device="cuda")
    q[:, 0, :, 5] = s
    pk, k = torch.zeros((1, P, H, d), device="cuda"), torch.zeros((N, S, H, d), device="cuda")
    pk[..., 5] = 1.0
    k[..., 5] = 1.0
    plen = torch.tensor([0 if keys == "own" else P], dtype=torch.int32, device="cuda")
    slen = torch.full((N,), 0 if keys == "prefix" else 1, dtype=torch.int32, device="cuda")
    out, lse = ll.prefix_attention(q, pk, pk + 1, k, k + 1, plen, slen, scale=SCALE)
    count = {"own": 1.0, "prefix": 70.0, "both": 71.0}[keys]
    want = s.double() * SCALE + torch.log(torch.tensor(count, dtype=torch.float64, device="cuda"))
    assert float(want.min()) > 16 and float(want.max()) < 32
    err = (lse[:, 0].double() - want).abs()
    assert float(err.max()) <= TOL, float(err.max())
    # means of equal values: up to 71 sums in turn, each off by 2^-24 of what is there so far (36 2^-24 of the
    # last in all), the normaliser's 8 and the join's and division's 6 such steps: below 2^-18 of the value
    assert bool((out[..., 5] - 2.0).abs().max() <= 2.0 ** -17) and bool((out[..., 0] - 1.0).abs().max() <= 2.0 ** -18)
