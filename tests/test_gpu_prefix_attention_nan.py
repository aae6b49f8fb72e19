"""NaN in a query: its row is NaN in out and lse, whichever kernels take the call, and no other row
notices; absent sequences' queries may hold anything."""
import math

import pytest
import torch

from test_gpu_prefix_attention import _check, _inputs, _ll, path  # noqa: F401  (path: a fixture)

pytestmark = pytest.mark.gpu

SHAPES = [(1, 4, 1, 8, 2, 64, 200, 24), (2, 3, 1, 4, 4, 128, 65, 64), (2, 4, 16, 4, 2, 64, 129, 17),
          (1, 130, 1, 4, 2, 128, 700, 65), (1, 9, 3, 10, 1, 48, 1500, 129), (3, 2, 4, 8, 1, 64, 0, 530),
          (2, 3, 2, 8, 2, 64, 300, 0), (1, 40, 3, 8, 2, 128, 512, 7)]


def _run(shape, dtype, bad):
    ll = _ll()
    G, W, T, Hq = shape[:4]
    P, S = shape[6:]
    N = G * W
    x = _inputs(*shape, dtype, sum(shape), [P] * G, [-1 if n % 5 == 3 else S for n in range(N)])
    clean = x[0].clone()
    gone = x[6] < 0
    rows = torch.zeros((N, T, Hq), dtype=torch.bool, device="cuda")
    rows.view(-1)[::7] = True
    rows[gone] = True
    x[0][rows, 3] = bad
    x[0][gone] = bad
    out, lse = torch.full_like(x[0], 7.0), torch.full((N, T, Hq), 9.0, device="cuda")
    ll.prefix_attention(*x, out=out, lse=lse)
    assert bool((out[gone] == 7.0).all()) and bool((lse[gone] == 9.0).all())
    hit = rows & ~gone[:, None, None]
    assert bool(hit.any())
    assert bool(torch.isnan(out[hit]).all()) and bool(torch.isnan(lse[hit]).all())      # (every row sees a key)
    # the others, beside what the call gives without it (the kernels move maxima for 32 rows together, so that
    # a neighbour's roundings may differ: the usual bounds)
    y = [clean] + x[1:]
    want, wlse = ll.prefix_attention(*y)
    _check((torch.where(rows[..., None], want, out), torch.where(rows, wlse, lse)), y, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_query_that_is_not_finite(shape, dtype, bad):
    _run(shape, dtype, bad)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("shape", SHAPES)
def test_on_both_paths(shape, bad, path):  # noqa: F811
    _run(shape, "bf16", bad)
