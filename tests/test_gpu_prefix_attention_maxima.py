"""Shared prefixes whose scores keep growing: the running maximum moves in either half of a tile, or
in both, of one row or of different rows, after a stream already has sums to rescale.

Queries and keys are whole numbers that bf16 holds, and the scale is log 2, so that a score in log2 units is their
product, exact in fp32: 32 more with each tile. What lies a tile back weighs 2^-32 or less of the newest, and
a sum that missed its rescaling would stand beside the right one at full size. Tolerances are those of
``test_gpu_prefix_attention`` (a score's error there covers log2(e) log 2 = 1 + 2.7e-8 here: the scores of
the keys that count differ by at most 64, so 2e-6 of a term, below 2^-15)."""
import math

import pytest
import torch

from test_gpu_prefix_attention import _check, _ll, path  # noqa: F401  (path: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W", [6, 150])                    # one row tile and two
@pytest.mark.parametrize("tiles", [99, 100])
def test_maxima_that_move_in_both_halves_of_a_tile(W, d, tiles, path):  # noqa: F811
    ll = _ll()
    H, P, S = 8, 128 * tiles, 8                            # six tiles a CTA: three of each stream, or six
    g = torch.Generator(device="cuda").manual_seed(d + W)
    k = torch.zeros((1, P, H, d), device="cuda")
    level = 32.0 * torch.arange(1, tiles + 1, device="cuda")[:, None]
    tile = k.view(tiles, 128, H, d)
    tile[:, 20, :, 0] = level                              # rows of the first kind move in the first half,
    tile[:, 90, :, 1] = level                              # of the second kind in the second half,
    tile[:, 20, :, 2] = level                              # of the third kind in both: by 32, then by 9,
    tile[:, 90, :, 2] = level
    tile[:, 90, :, 3] = 9.0
    tile[::2, 64:124, :, 2] = level[::2, :, None]          # to sums of one key or of sixty
    tile[::2, 64:124, :, 3] = 9.0
    v = 1.0 + torch.randn((1, P, H, d), generator=g, device="cuda")
    q = torch.zeros((W, 1, H, d), device="cuda")
    q[0::3, ..., 0] = 1.0
    q[1::3, ..., 1] = 1.0
    q[2::3, ..., 2:4] = 1.0
    own = torch.zeros((W, S, H, d), device="cuda")
    lens = (torch.tensor([P], dtype=torch.int32, device="cuda"),
            (torch.arange(W, device="cuda") % (S + 1)).int())
    x = [t.to(torch.bfloat16) for t in (q, k, v, own, own + 1.0)] + list(lens)
    assert torch.equal(x[1].float(), k)
    scale = float(torch.tensor(math.log(2.0)))             # as the call takes it, in fp32
    _check(ll.prefix_attention(*x, scale=scale), x, "bf16", scale=scale)
