"""CPU: the binding takes the cache's lists as int32 on the GPU and nothing else; what it
refuses never reaches the library."""
import pytest
import torch

import paper_2607_21599_amd as daf
from test_cache_checks import BIG, FAKE, ROWS, _cache


class OnGpu:
    """Stands for a tensor on the GPU."""
    device = "cuda:0"
    is_cuda = True

    def __init__(self, x):
        self.x, self.dtype = x, x.dtype

    def __getattr__(self, name):
        return getattr(self.x, name)


GOOD = OnGpu(torch.zeros(4, dtype=torch.int32))
BAD = [OnGpu(torch.zeros(4, dtype=torch.int64)), OnGpu(torch.zeros(4)), OnGpu(torch.zeros(1, dtype=torch.int32)),
       OnGpu(torch.zeros(8, dtype=torch.int32)[::2]), torch.zeros(4, dtype=torch.int32)]
ONE = [BAD[0], BAD[1], OnGpu(torch.zeros(0, dtype=torch.int32)), BAD[4]]  # of one element


@pytest.mark.parametrize("bad", BAD)
def test_lists_of_rows(bad):
    for seq, pos in ((bad, None), (None, bad)):
        with pytest.raises(ValueError):
            daf.CacheRows([0, 1, 2, 4], seq, pos)


@pytest.mark.parametrize("bad", BAD)
def test_lists_of_page_calls(bad):
    c = _cache()
    for call in (lambda: daf.daf_pages_extend(c, 4, bad, FAKE, FAKE, 0),
                 lambda: daf.daf_pages_extend(c, 4, None, bad, FAKE, 0),
                 lambda: daf.daf_pages_fork(c, 4, bad, FAKE, FAKE, FAKE, BIG, 0),
                 lambda: daf.daf_pages_fork(c, 4, FAKE, bad, FAKE, FAKE, BIG, 0),
                 lambda: daf.daf_pages_free(c, 4, bad, 0),
                 lambda: daf.daf_pages_copy(c, 4, bad, FAKE, 0),
                 lambda: daf.daf_pages_copy(c, 4, FAKE, bad, 0)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("bad", ONE)
def test_single_numbers(bad):
    c = _cache()
    for call in (lambda: daf.daf_pages_extend(c, 1, FAKE, FAKE, bad, 0),
                 lambda: daf.daf_pages_fork(c, 1, FAKE, FAKE, bad, FAKE, BIG, 0),
                 lambda: daf.daf_pages_unshare(c, ROWS, bad, FAKE, BIG, 0),
                 lambda: daf.daf_pages_compact(c, bad, FAKE, BIG, 0)):
        with pytest.raises(ValueError):
            call()


def test_what_is_taken():
    r = daf.CacheRows([0, 1, 2, 4], GOOD, GOOD)
    assert r.seq == r.pos == GOOD.data_ptr()
    assert daf.CacheRows([0, 2], None, None).seq is None
