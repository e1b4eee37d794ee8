"""What the arrays of a paged cache's calls hold is checked on the device, however many sequences there are."""
import pytest
import torch

from cache_cases import Case, Device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def heart():
    from paper_2605_14513_b200 import heart as h

    return h


WRONG = {
    "a start behind the next": lambda w, c: w[1].__setitem__(17, int(w[1][18]) + 1),
    "starts that fall back": lambda w, c: w[1].__setitem__(20, 0),
    "a negative start": lambda w, c: w[1].__setitem__(0, -1),
    "an end behind the rows": lambda w, c: w[1].__setitem__(c.S, c.T + 1),
    "a length of a sequence with new tokens": lambda w, c: w[2].__setitem__(2, c.width * c.page + 1),
    "a length of one without": lambda w, c: w[2].__setitem__(9, c.width * c.page + 1),
    "a negative length": lambda w, c: w[2].__setitem__(9, -1),
    "the last length": lambda w, c: w[2].__setitem__(c.S - 1, 1 << 30),
}


@pytest.mark.parametrize("S", [33, 40, 300])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("what", WRONG)
def test_every_entry_is_checked(heart, what, kind, S):
    c = Case([20 + s % 5 for s in range(S)], [0 if s in (9, S - 1) else 1 + s % 3 for s in range(S)], Hq=2, Hkv=2, page=16, kind=kind, garbage=False, pad=5)
    d = Device(heart, c)
    d.where[0].clamp_(min=0)  # (lengths that are too long are taken as the longest: entries of tokens that were none are looked at)

    def calls():
        heart.heart_cache_write(d.cfg, d.K, d.V, d.cache, *d.where, d.ws)
        yield "write"
        heart.heart_cache_read(d.cfg, d.cache, *d.where, torch.zeros_like(d.K), torch.zeros_like(d.V), d.ws)
        yield "read"
        for max_new in (1, 0):
            d.cfg.max_new = max_new
            d.attention()
            yield f"attention, max_new {max_new}"

    for _ in calls():
        assert heart.heart_get_status(d.ws) == 0
    WRONG[what](d.where, c)
    for name in calls():
        assert heart.heart_get_status(d.ws) == heart.ERR_DEVICE_CHECK, name
