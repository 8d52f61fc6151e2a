"""Scored steps, weights and evictions as calls: launches counted, tensors checked, views, merges left open, forms few callers use."""
import math

import pytest
import torch

from paper_2605_12471_b200 import binding
from tests import scored
from tests.test_scored_gpu import BASE, HEADS, check, chunk, make, slopes_of
from tests.test_scored_storage_gpu import H, KV, held, inputs, paged

pytestmark = pytest.mark.gpu


def test_launches_of_the_weight_are_counted():
    for heads, rows, n, kernels in (((16, 2, 128), 2900, 2900, 2), ((16, 2, 128), 2900, 1, 1), ((8, 2, 64), 300, 40, 1)):
        cache, gen = make(heads, "bf16", 3000, 2900, prefix=rows, seed=2)
        q = chunk(cache, gen, n)[0]
        lse = torch.zeros((n, heads[0]), device="cuda") + 8
        before = cache.launch_count()
        cache.mass(q, lse)
        assert cache.launch_count() - before == kernels, (heads, n)


def test_weights_in_splits_behind_open_merges():
    """Sums of splits lie where a step's partial results do: eight steps, whose merges alternate between two sets of them."""
    n, prefix, heads = 512, 1500, (16, 2, 128)
    got, kept = [], []
    for flags in (0, binding.KVF_COMBINE_BEHIND):
        cache, gen = make(heads, "bf16", 1500 + 8 * n, n, flags=flags, prefix=prefix, seed=6)
        for t in range(8):
            assert cache.plan(n)[3] == 3                                 # (the step leaves a merge)
            q, k, v = chunk(cache, gen, n)
            lse = torch.full((n, heads[0]), math.nan, device="cuda")
            q_rot = cache.rotate(q, pos0=len(cache))
            out = cache.fold_step(q, k, v, lse=lse)
            count = cache.launch_count()
            mass = cache.mass(q_rot, lse)
            assert t > 0 or cache.launch_count() - count == 2            # (and the weight is added up in splits)
            kept.append((out, lse))
            got.append((out, lse, mass))
        cache.flush()
        torch.cuda.synchronize()
    for a, b in zip(got[:8], got[8:]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert all(bool(torch.isfinite(m).all()) for _, _, m in got)


def test_plane_views_are_the_callers_own():
    cache, _ = make((8, 2, 128), "bf16", 300, 8)
    for plane in (cache.k_plane, cache.v_plane):
        view = plane()
        view.unsqueeze_(0)
        view.transpose_(1, 2)
        assert plane().shape == (2, 300, 128) and plane().stride() == (300 * 128, 128, 1)
        assert plane().data_ptr() == view.data_ptr()


def test_unpacked_codes_are_not_kept():
    cache = binding.Cache(binding.make_config(8, 2, 128, "bf16", 1 << 16, 8, flags=binding.KVF_CACHE_INT4))
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    cache.k_plane()
    cache.v_plane()
    assert torch.cuda.memory_allocated() == before


def test_tensors_of_other_shapes_and_devices_are_refused_before_any_launch():
    cache, gen = make((8, 2, 128), "bf16", 700, 64, prefix=500)
    q, k, v = chunk(cache, gen, 20)
    lse, wide = torch.zeros((20, 8), device="cuda"), torch.zeros((20, 8, 128), device="cuda")
    few, short, apart = q[:, :4].contiguous(), q[..., :64].contiguous(), torch.cat([q, q], -1)[..., :128]
    rows, count = len(cache), cache.launch_count()
    bad = []
    for x in (few, short, apart, q.cpu()):
        bad += [lambda x=x: cache.rotate(x), lambda x=x: cache.mass(x, lse), lambda x=x: cache.fold_step(x, k, v, softcap=5.0), lambda x=x: cache.attend(x, softcap=5.0)]
    bad += [lambda: cache.rotate(q, out=few), lambda: cache.rotate(q, out=torch.empty(q.shape, dtype=q.dtype)), lambda: cache.rotate(q, out=wide),
            lambda: cache.mass(q, lse[:10]), lambda: cache.mass(q, lse.cpu()),
            lambda: cache.fold_step(q, k[:10].contiguous(), v, softcap=5.0), lambda: cache.fold_step(q, k, v[:, :1].contiguous(), softcap=5.0),
            lambda: cache.fold_step(q, k, v, out=few, softcap=5.0), lambda: cache.fold_step(q, k, v, out=wide, softcap=5.0),
            lambda: cache.fold_step(q, k, v, lse=lse[:10], softcap=5.0), lambda: cache.fold_step(q, k, v, lse=lse.half(), softcap=5.0),
            lambda: cache.attend(q, out=few, softcap=5.0), lambda: cache.attend(q, lse=lse[:10], softcap=5.0)]
    for f in bad:
        with pytest.raises(AssertionError):
            f()
    cfg = binding.make_config(H, KV, 128, "bf16", 512, 256, rope_base=BASE)
    batch, x = binding.Batch(paged(cfg, gen, 2)), inputs(gen, 2, 5)
    lse2 = torch.zeros((2, 5, H), device="cuda")
    for f in (lambda: batch.fold_step(x[0][:, :, :4].contiguous(), *x[1:], softcap=5.0), lambda: batch.fold_step(x[0], x[1][:, :4].contiguous(), x[2], softcap=5.0),
              lambda: batch.fold_step(*x, out=x[0][:, :4].contiguous(), softcap=5.0), lambda: batch.fold_step(*x, lse=lse2[:1], softcap=5.0),
              lambda: batch.fold_step_varlen(x[0], x[1], x[2][:1], [5, 5], softcap=5.0), lambda: batch.fold_step_varlen(*x, [5, 5], lse=lse2.double(), softcap=5.0)):
        with pytest.raises(AssertionError):
            f()
    torch.cuda.synchronize()
    assert len(cache) == rows and cache.launch_count() == count and batch.launch_count() == 0


@pytest.mark.parametrize("heads,dtype", HEADS[4:])
@pytest.mark.parametrize("n", [1, 40, 300])
@pytest.mark.parametrize("pos0", [0, 250, 10000])
def test_biases_on_the_cuda_cores_of_tokens_before_among_and_behind_the_rows(heads, dtype, n, pos0):
    prefix, h = 500, heads[0]
    for kw in (dict(slopes=slopes_of(h)), dict(slopes=-slopes_of(h) / 16, softcap=8.0), dict(slopes=slopes_of(h) * 40)):
        cache, gen = make(heads, dtype, 900, n, prefix=prefix, seed=12)
        q, k, v = chunk(cache, gen, n)
        lse = torch.empty((n, h), device="cuda")
        out = cache.fold_step(q, k, v, pos0=pos0, lse=lse, **kw)
        check(cache, q, k, v, n, True, lse, out, pos0, **kw)
        out = cache.attend(q, pos0=pos0, lse=lse, **kw)
        check(cache, q, None, None, n, False, lse, out, pos0, **kw)


@pytest.mark.parametrize("flag", [binding.KVF_CACHE_INT8, binding.KVF_CACHE_INT4])
@pytest.mark.parametrize("is_paged", [False, True])
@pytest.mark.parametrize("n", [1, 4, 33, 128])
def test_queries_alone_on_quantised_rows(flag, is_paged, n):
    rows = 901
    for k in range(3):
        gen = torch.Generator(device="cuda").manual_seed(3 * n + k)
        cfg = binding.make_config(H, KV, 128, "bf16", 1024, 1024, rope_base=BASE, flags=flag)
        cache = paged(cfg, gen, 1)[0] if is_paged else binding.Cache(cfg)
        cache.fold_step(*inputs(gen, rows))
        q = inputs(gen, n)[0]
        first = torch.randint(-50, rows + 60, (n,), generator=gen, device="cuda", dtype=torch.int32)
        end = torch.randint(-50, rows + 60, (n,), generator=gen, device="cuda", dtype=torch.int32)
        kw = [dict(softcap=4.0), dict(first=first, end=end), dict(softcap=6.0, slopes=slopes_of(H), end=end)][k]
        lse = torch.empty((n, H), device="cuda")
        out = cache.attend(q, pos0=rows + 3, lse=lse, **kw)
        assert len(cache) == rows
        seen = scored.ranges(n, rows, rows, False, kw.get("first"), kw.get("end"))
        want, want_lse, bound, lse_bound = scored.attend(scored.turned(q, rows + 3, BASE), held(cache, 0, n), held(cache, 1, n), seen, 1 / math.sqrt(128),
                                                         rows + 3, kw.get("softcap", 0.0), kw.get("slopes"))
        assert bool(((out.double() - want).abs() <= bound).all())
        some = want_lse > -math.inf
        assert bool((lse[~some] == -math.inf).all()) and bool((out[~some] == 0).all())
        assert bool(((lse.double() - want_lse).abs() <= lse_bound)[some].all())
        assert cache.status() == binding.KVF_OK


@pytest.mark.parametrize("heads,dtype", HEADS)
@pytest.mark.parametrize("rows", [1, 5, 127, 129])
@pytest.mark.parametrize("n", [2, 40, 300])
def test_many_queries_alone_on_few_rows(heads, dtype, rows, n):
    cache, gen = make(heads, dtype, 400, n, prefix=rows, seed=rows)
    q = chunk(cache, gen, n)[0]
    h, scale = heads[0], 1 / math.sqrt(heads[2])
    first = torch.randint(0, rows + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
    for kw in (dict(softcap=3.0), dict(first=first, slopes=slopes_of(h)), dict(end=first, softcap=8.0)):
        lse = torch.empty((n, h), device="cuda")
        out = cache.attend(q, pos0=rows, lse=lse, **kw)
        check(cache, q, None, None, n, False, lse, out, rows, **kw)
        got = cache.mass(q, lse, appended=False, **kw)
        seen = scored.ranges(n, rows, rows, False, kw.get("first"), kw.get("end"))
        want, bound = scored.mass(q, cache.k_plane()[:, :rows], lse, seen, scale, rows, kw.get("softcap", 0.0), kw.get("slopes"),
                                  tensor_cores=dtype == "bf16" and heads[2] == 128)
        assert bool(((got.double() - want).abs() <= bound).all()), kw
