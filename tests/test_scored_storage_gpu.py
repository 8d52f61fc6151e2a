"""Scored steps on quantised rows and in batches of paged caches."""
import math

import pytest
import torch

from paper_2605_12471_b200 import binding
from tests import scored
from tests.test_mass_evict_gpu import rows_of
from tests.test_scored_gpu import BASE, slopes_of

pytestmark = pytest.mark.gpu

H, KV = 32, 8


def paged(cfg, gen, caches):
    pages = (cfg.capacity + 127) // 128
    pool = torch.zeros(binding.paged_pool_bytes(cfg, caches * pages), dtype=torch.uint8, device="cuda")
    tables = torch.randperm(caches * pages, generator=gen, device="cuda").to(torch.int32).view(caches, pages)
    return [binding.PagedCache(cfg, pool, caches * pages, tables[i]) for i in range(caches)]


def inputs(gen, *lead):
    return [torch.randn((*lead, heads, 128), generator=gen, device="cuda").bfloat16() for heads in (H, KV, KV)]


def held(cache, kv, n):
    """The rows a step reads, as it reads them: quantised steps of more than 16 query rows see them rounded to bf16."""
    rows, scale = rows_of(cache, kv)
    rows = rows[:, :len(cache)]
    if scale is None:
        return rows.double()
    x = rows.double() * scale[:, :len(cache), None].double()
    return x if n * (H // KV) <= 16 else (rows.float() * scale[:, :len(cache), None]).bfloat16().double()


def check(cache, q, out, lse, n, pos0, longest=None, **kw):
    rows = len(cache)
    seen = scored.ranges(n, rows, rows - n, True, kw.get("first"), kw.get("end"))
    want, want_lse, bound, lse_bound = scored.attend(scored.turned(q, pos0, BASE), held(cache, 0, longest or n), held(cache, 1, longest or n), seen,
                                                     1 / math.sqrt(128), pos0, kw.get("softcap", 0.0), kw.get("slopes"))
    off = (out.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
    some = want_lse > -math.inf
    assert bool((lse[~some] == -math.inf).all()) and bool((out[~some] == 0).all())
    assert bool(((lse.double() - want_lse).abs() <= lse_bound)[some].all())


# (128 tokens of 32 / 8 heads are 512 query rows: pairs of CTAs)
@pytest.mark.parametrize("n", [1, 4, 33, 128, 300])
@pytest.mark.parametrize("is_paged", [False, True])
@pytest.mark.parametrize("flag", [binding.KVF_CACHE_INT8, binding.KVF_CACHE_INT4])
def test_scored_steps_on_quantised_rows(flag, is_paged, n):
    prefix = 700
    for k in range(4):
        gen = torch.Generator(device="cuda").manual_seed(17 * n + k)
        cfg = binding.make_config(H, KV, 128, "bf16", 1024, 1024, rope_base=BASE, flags=flag)
        cache = paged(cfg, gen, 1)[0] if is_paged else binding.Cache(cfg)
        cache.fold_step(*inputs(gen, prefix))
        q, k_new, v_new = inputs(gen, n)
        kw = [dict(softcap=4.0), dict(slopes=slopes_of(H)),
              dict(first=torch.randint(0, prefix, (n,), generator=gen, device="cuda", dtype=torch.int32)),
              dict(softcap=6.0, slopes=slopes_of(H), first=torch.randint(0, prefix + n, (n,), generator=gen, device="cuda", dtype=torch.int32),
                   end=torch.randint(0, prefix + n, (n,), generator=gen, device="cuda", dtype=torch.int32))][k]
        lse = torch.empty((n, H), device="cuda")
        out = cache.fold_step(q, k_new, v_new, lse=lse, **kw)
        check(cache, q, out, lse, n, prefix, **kw)
        assert cache.status() == binding.KVF_OK


@pytest.mark.parametrize("flag", [0, binding.KVF_CACHE_INT8])
@pytest.mark.parametrize("n", [1, 40, 150])
@pytest.mark.parametrize("alike", [True, False])
def test_scored_batches(alike, n, flag):
    gen = torch.Generator(device="cuda").manual_seed(n + alike)
    cfg = binding.make_config(H, KV, 128, "bf16", 1024, 512, rope_base=BASE, flags=flag)
    caches = paged(cfg, gen, 4)
    lens = [300] * 4 if alike else [5, 400, 129, 333]
    for cache, rows in zip(caches, lens):
        cache.fold_step(*inputs(gen, rows))
    batch = binding.Batch(caches)
    for k in range(3):
        q, k_new, v_new = inputs(gen, 4, n)
        rows = torch.tensor([len(c) for c in caches], device="cuda")[:, None]
        first = (torch.rand((4, n), generator=gen, device="cuda") * (rows + n)).to(torch.int32)
        end = (rows + 1 + torch.arange(n, device="cuda")).clamp(min=int(rows[0]) // 2).to(torch.int32).contiguous()
        kw = [dict(softcap=5.0), dict(slopes=slopes_of(H), first=first), dict(softcap=7.0, end=end)][k]
        ns = [n, n, 0, max(1, n // 2)] if not alike and k == 2 else [n] * 4
        lse = torch.empty((4, n, H), device="cuda")
        before = [len(c) for c in caches]
        if ns[2] == 0:
            out = batch.fold_step_varlen(q, k_new, v_new, ns, lse=lse, **kw)
        else:
            out = batch.fold_step(q, k_new, v_new, lse=lse, ragged=not alike, **kw)
        for i, cache in enumerate(caches):
            assert len(cache) == before[i] + ns[i]
            if ns[i]:
                own = {key: (v[i, :ns[i]] if key in ("first", "end") else v) for key, v in kw.items()}
                check(cache, q[i, :ns[i]], out[i, :ns[i]], lse[i, :ns[i]], ns[i], before[i], longest=n, **own)
    assert batch.status_word() == 0


def test_plain_steps_of_a_batch_stay_plain_behind_scored_ones():
    gen = torch.Generator(device="cuda").manual_seed(3)
    cfg = binding.make_config(H, KV, 128, "bf16", 512, 256, rope_base=BASE)
    outs = []
    for scored_first in (False, True):
        gen.manual_seed(3)
        caches = paged(cfg, gen, 2)
        for cache in caches:
            cache.fold_step(*inputs(gen, 200))
        batch = binding.Batch(caches)
        x = inputs(gen, 2, 20)
        if scored_first:
            batch.fold_step(*x, softcap=3.0)
            for cache in caches:
                cache.set_len(200)
        outs.append(batch.fold_step(*x))
    assert torch.equal(*outs)
