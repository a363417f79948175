"""Every variant of the eviction's selection kernel against the definition, with each CTA's run of keys in shared memory and beyond it."""
import pytest
import torch

from tests import host_rules
from tests import serving_util as su
from tests.test_gpu_paged_cache import check_evict

pytestmark = pytest.mark.gpu
CACHED = 24 * 1024   # keys of its run that a CTA of 1024 threads holds in shared memory


@pytest.mark.parametrize("batch,heads_kv,length,ranks,threads", [
    (2, 1, 900, 1, 256), (3, 1, 2000, 1, 1024), (40, 1, 25700, 1, 1024), (5, 5, 4200, 2, 1024), (3, 7, 50500, 2, 1024),
    (2, 8, 20000, 4, 1024), (1, 9, 8300, 4, 1024), (1, 9, 100001, 4, 1024), (4, 2, 16700, 8, 1024), (1, 1, 200003, 8, 1024)])
@pytest.mark.parametrize("weights", ["distinct", "ties", "zeros"])
def test_against_the_definition(batch, heads_kv, length, ranks, threads, weights):
    page, recent, keep = 256, 77, length // 3
    room = -(-length // page) * page
    for field, value in (("ranks", ranks), ("threads", threads)):
        assert host_rules.evaluate("cache_choice.h", f"sparsed::choose_evict_variant(rows, static_cast<int>(room)).{field}", "rows room",
                                   [(batch * heads_kv, room)]) == [value]
    gen = su.generator(length)
    k, v, table = su.paged_pool([length] * batch, page, heads_kv, torch.float16, gen)
    mass = torch.rand(batch, heads_kv, room, generator=gen, device="cuda")
    if weights == "ties":
        mass = (mass * 7).floor()
        mass[:, 0, 1::5] = float("nan")
        mass[:, -1, ::3] = float("inf")
    elif weights == "zeros":   # fewer keys with a weight than stay
        mass[mass < 0.8] = 0.0
        mass[:, :, ::11] *= -1.0
    lens = [length - 3 * i for i in range(batch)]
    lens[-1] = min(lens[-1], keep + 1) if batch > 2 else lens[-1]   # (a row that loses one key only)
    check_evict(k, v, table, lens, mass, keep, recent)


def test_runs_beyond_shared_memory_are_among_the_cases():
    for rows_ctas, length in ((1, 25700), (2, 50500), (4, 100001), (8, 200003)):
        assert (length - 77) // rows_ctas > CACHED
