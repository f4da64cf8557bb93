"""Reading a cache that is bookkeeping only is refused by status, whatever the ranges (CPU)."""
import pytest

from paper_2605_13319_amd import inputs as I
from paper_2605_13319_amd import nav


@pytest.mark.parametrize("cache", [nav.PageCache, nav.KV4Cache])
@pytest.mark.parametrize("count,status", [(5, nav.ESTATE), (0, nav.ESTATE), (6, nav.ESTATE), (-1, nav.EINVAL)])
def test_reading_without_a_pool_is_refused(cache, count, status):
    c = cache(I.ModelShape("host", 2, 512, 4, 2, 64, 512, 512), 2, 10, on_device=False)
    c.extend([0], [5])
    with pytest.raises(nav.PipesdError) as e:
        c.read([0], [0], [count])
    assert e.value.status == status
