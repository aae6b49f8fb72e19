"""beam_reorder of states of several layouts: moved together, or not at all."""
import pytest
import torch

from test_gpu_beam import _ll, _moved

pytestmark = pytest.mark.gpu


def _states(seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((2, 4, 6, 3, 8), generator=g).cuda(), torch.randn((2, 4, 6, 3, 8), generator=g).cuda(),
            torch.randn((2, 4, 9, 16), generator=g).cuda(),
            torch.randint(0, 255, (2, 4, 5, 7), generator=g, dtype=torch.uint8).cuda()]


PARENTS = [[1, 2, 3, 0], [3, 3, 0, 0]]


def test_layouts_move_together():
    ll = _ll()
    states, p = _states(1), torch.tensor(PARENTS, dtype=torch.int32)
    lengths = torch.tensor([4, 7], dtype=torch.int32)
    want = [_moved(s.cpu(), p, lengths) for s in states]
    assert ll.beam_reorder(states, p.cuda(), lengths.cuda()) is states
    assert all(torch.equal(s.cpu(), w) for s, w in zip(states, want))
    assert ll.beam_reorder([], p.cuda()) == []


@pytest.mark.parametrize("bad", ["shape", "tail", "overlap", "long"])
@pytest.mark.parametrize("at", [0, 2, 4])
def test_a_refused_state_leaves_the_others(bad, at):
    """Wherever the refused state stands, no other is moved, and the call without it moves each once."""
    ll = _ll()
    states, p = _states(2), torch.tensor(PARENTS, dtype=torch.int32)
    keep = [s.clone() for s in states]
    x = {"shape": torch.zeros((2, 3, 5), device="cuda"),
         "tail": torch.zeros((2, 4, 5, 4, 6), device="cuda").transpose(3, 4),
         "overlap": torch.zeros((2, 1, 5, 6), device="cuda").expand(2, 4, 5, 6),
         "long": torch.empty(1, dtype=torch.uint8, device="cuda").expand(2, 4, 1 << 33, 1)}[bad]
    with pytest.raises((ValueError, ll.LilicorrError)):
        ll.beam_reorder(states[:at] + [x] + states[at:], p.cuda())
    torch.cuda.synchronize()
    assert all(torch.equal(s, k) for s, k in zip(states, keep))
    ll.beam_reorder(states, p.cuda())
    assert all(torch.equal(s.cpu(), _moved(k.cpu(), p, None)) for s, k in zip(states, keep))


def test_layouts_that_share_memory_are_refused():
    """Views of one cache: of overlapping positions, refused and not moved; side by side, moved."""
    ll = _ll()
    p = torch.tensor(PARENTS, dtype=torch.int32)
    x = torch.arange(2 * 4 * 100 * 24, dtype=torch.float32, device="cuda").view(2, 4, 100, 24)
    keep = x.clone()
    for bad in ([x[:, :, :64], x[:, :, 32:]], [x[:, :, :, :16], x[:, :, 10:, 15:]],
                [x[:, :, 3:], x.view(torch.int32)[:, :, :50]]):
        with pytest.raises(ll.LilicorrError):
            ll.beam_reorder(bad, p.cuda())
        assert torch.equal(x, keep)
    ll.beam_reorder([x[:, :, :64, :16], x[:, :, 64:, :16], x[:, :, :, 16:]], p.cuda())
    assert torch.equal(x.cpu(), _moved(keep.cpu(), p, None))
