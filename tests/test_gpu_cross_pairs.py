"""Cross attention by pairs of CTAs: row sums that are very different from tile to tile, ragged ends of keys."""
import pytest
import torch

from test_gpu_cross import Case, Device, check, heart, same  # noqa: F401  (heart: a fixture)

pytestmark = pytest.mark.gpu


def stepped(c, every):
    """The queries of every `every` rows a factor of their own: row sums and references are no other tile's."""
    factor = torch.tensor([(0.05, 3.0, 0.6, 4.0, 0.2)[i // every % 5] for i in range(c.T)])
    c.Q = (c.Q.float() * factor[:, None, None]).to(torch.bfloat16)
    return c


# Whole tiles of one step and of some (32 heads x 19100 tokens over 32 tiles a CTA), and tiles that several pairs share (more than 64 MB of keys and values).
CASES = {
    "one step": dict(q=[19100], k=[33], Hq=32, Hkv=32),
    "two steps": dict(q=[9500, 9500], k=[140, 250], Hq=32, Hkv=32),
    "shared tiles": dict(q=[300], k=[4000], Hq=2, Hkv=2, pad_k=70000),
    "shared and ragged": dict(q=[700, 260, 130], k=[3001, 5007, 100], Hq=4, Hkv=2, pad_k=70000, layout="shuffled"),
}


@pytest.mark.parametrize("name", CASES)
def test_every_tile_has_its_own_row_sums(heart, name):
    c = stepped(Case(**CASES[name], seed=3, gain=1.0), 128)
    d = Device(heart, c)
    O, lse = d.attention()
    assert heart.heart_get_status(d.ws) == 0
    check(c, O, lse)
    for _ in range(20):
        P, M = d.attention()
        assert same(O, P) and same(lse, M)
    assert heart.heart_get_status(d.ws) == 0
