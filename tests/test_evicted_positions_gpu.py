"""A bias goes by row numbers, which an eviction changes: behind one, steps and weights with slopes are refused."""
import pytest
import torch

from paper_2605_12471_b200 import binding
from tests.test_scored_gpu import BASE, chunk, make, slopes_of
from tests.test_scored_storage_gpu import inputs, paged

pytestmark = pytest.mark.gpu


def evicted(heads=(8, 2, 128), dtype="bf16", rows=500, budget=200, sinks=4, recent=50):
    src, gen = make(heads, dtype, 700, 64, prefix=rows)
    dst, _ = make(heads, dtype, 700, 64)
    src.evict(dst, torch.rand((heads[1], rows), generator=gen, device="cuda"), budget, n_sink=sinks, n_recent=recent)
    return src, dst, gen


def refused(cache, f):
    rows, count = len(cache), cache.launch_count()
    with pytest.raises(binding.KvfError) as e:
        f()
    assert e.value.code == binding.KVF_ERR_UNSUPPORTED and len(cache) == rows and cache.launch_count() == count


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "f32"), ((8, 2, 128), "f32")])
@pytest.mark.parametrize("n", [1, 40])
def test_slopes_behind_an_eviction_are_refused(heads, dtype, n):
    src, dst, gen = evicted(heads, dtype)
    q, k, v = chunk(dst, gen, n)
    lse, s = torch.zeros((n, heads[0]), device="cuda"), slopes_of(heads[0])
    for kw in (dict(slopes=s), dict(slopes=s, softcap=9.0)):
        refused(dst, lambda: dst.fold_step(q, k, v, pos0=500, **kw))
        refused(dst, lambda: dst.attend(q, pos0=500, **kw))
        refused(dst, lambda: dst.mass(q, lse, pos0=500, **kw))
    # everything else goes on, and so does the cache whose rows stand where they stood
    dst.mass(q, lse, softcap=9.0)
    dst.fold_step(q, k, v, pos0=500, softcap=9.0)
    refused(dst, lambda: dst.fold_step(q, k, v, pos0=500 + n, slopes=s))
    src.mass(q, lse, slopes=s)
    src.fold_step(q, k, v, slopes=s)


def test_rows_that_stand_at_their_own_numbers_take_slopes():
    s = slopes_of(8)
    src, dst, gen = evicted(budget=500)                       # nothing left out
    q, k, v = chunk(dst, gen, 3)
    dst.fold_step(q, k, v, slopes=s)
    src, dst, gen = evicted()
    refused(dst, lambda: dst.attend(q, slopes=s))
    dst.set_len(4)                                            # the rows that always stay are the first ones
    dst.attend(q, slopes=s)
    dst.fold_step(q, k, v, slopes=s)
    src, dst, gen = evicted()
    dst.reset()
    dst.fold_step(q, k, v, slopes=s)
    src, dst, gen = evicted(budget=4, recent=0)               # no row out of place yet, but the next one would be
    refused(dst, lambda: dst.fold_step(q, k, v, pos0=500, slopes=s))


def test_an_eviction_of_an_evicted_cache_does_not_bring_the_numbers_back():
    src, dst, gen = evicted()
    third, _ = make((8, 2, 128), "bf16", 700, 64)
    dst.evict(third, torch.rand((2, 200), generator=gen, device="cuda"), 200, n_sink=190)
    q = chunk(third, gen, 3)[0]
    refused(third, lambda: third.attend(q, slopes=slopes_of(8)))
    # a cache that is filled anew by one that has all its rows is as good as new
    src.evict(third, torch.rand((2, 500), generator=gen, device="cuda"), 500)
    third.attend(q, slopes=slopes_of(8))


def test_batches_with_an_evicted_member_refuse_slopes():
    gen = torch.Generator(device="cuda").manual_seed(1)
    cfg = binding.make_config(32, 8, 128, "bf16", 512, 256, rope_base=BASE)
    a, b, c = paged(cfg, gen, 3)
    for cache in (a, c):
        cache.fold_step(*inputs(gen, 200))
    c.evict(b, torch.rand((8, 200), generator=gen, device="cuda"), 150, n_sink=4)
    batch, x = binding.Batch([a, b]), inputs(gen, 2, 5)
    before = batch.launch_count()
    for call in (lambda **kw: batch.fold_step(*x, ragged=True, **kw), lambda **kw: batch.fold_step_varlen(*x, [5, 3], **kw)):
        with pytest.raises(binding.KvfError) as e:
            call(slopes=slopes_of(32))
        assert e.value.code == binding.KVF_ERR_UNSUPPORTED and (len(a), len(b)) == (200, 150) and batch.launch_count() == before
    batch.fold_step_varlen(*x, [5, 0], slopes=slopes_of(32))                  # (it sits the step out)
    batch.fold_step(*x, pos0=[205, 200], ragged=True, softcap=5.0)
