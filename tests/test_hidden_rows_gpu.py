"""Rows that no token of a warp sees choose none of its arithmetic: whatever finite numbers they hold, the bits are the same."""
import pytest
import torch

from paper_2605_12471_b200 import binding
from tests.test_mass_evict_gpu import paged_pair
from tests.test_scored_gpu import chunk, make, slopes_of
from tests.test_scored_storage_gpu import inputs

pytestmark = pytest.mark.gpu

PREFIX, FIRST = 600, 390                  # (both inside a key tile)
HEADS = [((8, 2, 128), "bf16"), ((28, 4, 128), "bf16"), ((4, 1, 64), "f32"), ((8, 2, 128), "f32")]


def plant(rows, size):
    """Rows of either sign, larger than any that is seen."""
    sign = torch.where(torch.arange(rows.shape[1], device="cuda") % 2 == 0, 1.0, -1.0)
    rows[:] = (size * sign)[None, :, None].to(rows.dtype)


def kinds(heads):
    return [dict(softcap=10.0), dict(softcap=1e5), dict(softcap=10.0, slopes=slopes_of(heads[0])), dict(softcap=1e5, slopes=slopes_of(heads[0]))]


@pytest.mark.parametrize("n", [1, 17, 40, 200])
@pytest.mark.parametrize("heads,dtype", HEADS)
@pytest.mark.parametrize("size", [1e4, 1e30])
def test_large_keys_in_the_hidden_prefix_and_behind_the_end_change_no_bit(heads, dtype, n, size):
    for kw in kinds(heads):
        got = []
        for large in (False, True):
            cache, gen = make(heads, dtype, 1024, n, prefix=PREFIX, seed=n)
            q, k, v = chunk(cache, gen, n)
            first = torch.full((n,), FIRST, dtype=torch.int32, device="cuda")
            if large:
                plant(cache.k_plane()[:, :FIRST], size)
                plant(cache.k_plane()[:, PREFIX + n:], size)
            lse = torch.empty((n, heads[0]), device="cuda")
            got.append((cache.fold_step(q, k, v, lse=lse, first=first, **kw), lse))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]), kw


@pytest.mark.parametrize("heads,dtype", HEADS)
def test_a_step_asked_again_on_a_cache_that_held_other_rows_gives_the_same_bits(heads, dtype):
    """No range at all: what lies behind the end is what an earlier use of the cache left there."""
    n = 37                                # (ends inside a key tile)
    for kw in kinds(heads):
        got = []
        for used in (False, True):
            cache, gen = make(heads, dtype, 1024, 200, prefix=PREFIX, seed=3)
            q, k, v = chunk(cache, gen, n)
            if used:
                cache.fold_step(*(x * 1e4 for x in chunk(cache, gen, 200)))
                cache.set_len(PREFIX)
            got.append(cache.fold_step(q, k, v, **kw))
            got.append(cache.attend(q, **kw))
        assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3]), kw


@pytest.mark.parametrize("n", [20, 40])
def test_large_keys_of_later_tokens_change_no_bit_of_the_warps_before(n):
    """A warp has 32 query rows, eight tokens here: the last token's key is seen by the last warp alone."""
    for kw in kinds((8, 2, 128)):
        got = []
        for large in (False, True):
            cache, gen = make((8, 2, 128), "bf16", 1024, n, prefix=PREFIX, seed=5)
            q, k, v = chunk(cache, gen, n)
            if large:
                k[-1] = 1e4
            got.append(cache.fold_step(q, k, v, **kw)[:(n - 1) // 8 * 8])
        assert torch.equal(*got), kw


@pytest.mark.parametrize("n", [17, 40, 200])
def test_a_recycled_page_gives_the_bits_of_a_fresh_one(n):
    rows = 1100
    for kw in kinds((8, 2, 128)):
        got = []
        for size in (0.0, 1e4, 1e30):
            _, cache, gen = paged_pair(rows, n, seed=n)
            pages = cache.page_rows(0)[cache.page_table.long()]                    # [pages, Hkv, 128, d], a copy
            pages[-1, :, (rows + n) % 128:] = size
            cache.page_rows(0)[cache.page_table.long()] = pages
            q, k, v = chunk(cache, gen, n)
            got.append(cache.fold_step(q, k, v, **kw))
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2]), kw


@pytest.mark.parametrize("flag", [binding.KVF_CACHE_INT8, binding.KVF_CACHE_INT4])
@pytest.mark.parametrize("n", [33, 128])
def test_large_scales_of_hidden_codes_change_no_bit(flag, n):
    for kw in kinds((32, 8, 128)):
        got = []
        for size in (1.0, 1e5):
            gen = torch.Generator(device="cuda").manual_seed(n)
            cache = binding.Cache(binding.make_config(32, 8, 128, "bf16", 1024, 1024, rope_base=10000.0, flags=flag))
            cache.storage.zero_()
            cache.fold_step(*inputs(gen, PREFIX))
            cache.scales(0)[:, :FIRST] *= size
            cache.scales(0)[:, PREFIX + n:] = size
            first = torch.full((n,), FIRST, dtype=torch.int32, device="cuda")
            got.append(cache.fold_step(*inputs(gen, n), first=first, **kw))
        assert torch.equal(*got), kw
