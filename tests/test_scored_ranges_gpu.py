"""Magnitudes beyond fp16 on fp32 caches whose plain steps compute on fp16 halves, whichever kind of step brings them in."""
import pytest
import torch

from paper_2605_12471_b200 import binding
from tests.test_scored_gpu import check, chunk, make, slopes_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 40, 300])
@pytest.mark.parametrize("kw", [dict(softcap=20.0), dict(first=True), dict(slopes=True)])
@pytest.mark.parametrize("which", ["k", "v"])
def test_rows_that_a_scored_step_appends_are_reported_as_a_plain_steps(n, kw, which):
    cache, gen = make((8, 2, 128), "f32", 1000, n, prefix=500, seed=1)
    q, k, v = chunk(cache, gen, n)
    (k if which == "k" else v)[0, 1, 3] = 1e5
    kw = {name: torch.zeros(n, dtype=torch.int32, device="cuda") if name == "first" else slopes_of(8) if name == "slopes" else x for name, x in kw.items()}
    out = cache.fold_step(q, k, v, **kw)
    assert cache.status() == binding.KVF_ERR_RANGE and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("heads,flags", [((8, 2, 128), 0), ((8, 2, 128), binding.KVF_FORCE_SIMT), ((4, 1, 64), 0)])
@pytest.mark.parametrize("n", [1, 40])
def test_queries_of_scored_steps_have_no_limit_and_rows_none_where_plain_steps_have_none(heads, flags, n):
    cache, gen = make(heads, "f32", 1000, n, prefix=500, seed=2, flags=flags)
    q, k, v = chunk(cache, gen, n, scale=1e5)
    if flags or heads[2] == 64:
        v = v * 1e5
    lse = torch.empty((n, heads[0]), device="cuda")
    out = cache.fold_step(q, k, v, lse=lse, softcap=20.0)
    check(cache, q, k, v, n, True, lse, out, 500, softcap=20.0)
    out = cache.attend(q, pos0=500 + n, lse=lse, softcap=20.0)
    check(cache, q, None, None, n, False, lse, out, 500 + n, softcap=20.0)


@pytest.mark.parametrize("flags", [0, binding.KVF_FORCE_SIMT])
@pytest.mark.parametrize("which", ["k", "v"])
def test_rows_that_an_eviction_brings_in_are_reported_where_they_matter(flags, which):
    """From a cache without limits, or one that has told of them itself, into one whose plain steps have them."""
    src, gen = make((8, 2, 128), "f32", 1000, 64, prefix=900, seed=3, flags=flags)
    plane = src.k_plane() if which == "k" else src.v_plane()
    plane[1, 700, 77] = -1e5
    mass = torch.rand((2, 900), generator=gen, device="cuda")
    for kept, to_flags in ((True, 0), (False, 0), (True, binding.KVF_FORCE_SIMT)):
        mass[1, 700] = 9.0 if kept else -1.0
        dst, _ = make((8, 2, 128), "f32", 1000, 64, flags=to_flags)
        src.evict(dst, mass, 400, n_sink=4, n_recent=50)
        assert dst.status() == (binding.KVF_ERR_RANGE if kept and not to_flags else binding.KVF_OK)
        assert src.status() == binding.KVF_OK
