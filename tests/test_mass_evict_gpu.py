"""The attention weight of a chunk and the eviction by it, against their plain statements."""
import math

import pytest
import torch

from paper_2605_12471_b200 import binding
from tests import scored
from tests.test_scored_gpu import BASE, HEADS, chunk, documents, make, slopes_of

pytestmark = pytest.mark.gpu


def lse_of(q, keys, seen, scale, pos0, **kw):
    s, _ = scored.scores(q, keys, scale, pos0, kw.get("softcap", 0.0), kw.get("slopes"))
    row = torch.arange(keys.shape[1], device=q.device)
    hidden = ~((row >= seen[0][:, None]) & (row < seen[1][:, None]))
    return torch.logsumexp(s.masked_fill(hidden[:, None], -math.inf), -1).float().contiguous()


@pytest.mark.parametrize("n,prefix", [(1, 0), (1, 1), (1, 1000), (3, 129), (6, 5000), (33, 515), (64, 0), (129, 127), (300, 1111), (1000, 40)])
@pytest.mark.parametrize("heads,dtype", HEADS)
def test_mass_matches_its_statement(heads, dtype, n, prefix):
    rows = prefix + n
    for seed, name in enumerate(["plain", "cap", "all", "attend"]):
        cache, gen = make(heads, dtype, rows + 9, n, prefix=rows, seed=seed)
        q = chunk(cache, gen, n, scale=2.0)[0]
        kw = {}
        if name in ("cap", "all"):
            kw["softcap"] = 5.0
        if name == "all":
            kw["slopes"] = slopes_of(heads[0])
            kw["first"], kw["end"] = documents(n, prefix, gen)
        appended = name != "attend"
        seen = scored.ranges(n, rows, prefix if appended else rows, appended, kw.get("first"), kw.get("end"))
        scale, pos0 = 1 / math.sqrt(heads[2]), prefix if appended else rows
        keys = cache.k_plane()[:, :rows]
        lse = lse_of(q.double(), keys, seen, scale, pos0, **kw)
        before = torch.rand((heads[1], rows + 9), generator=gen, device="cuda")
        if appended:
            before[:, prefix:] = math.nan                # (the step's own rows start from zero)
        decay = [1.0, 0.5, 0.0, 1.0][seed]
        out = torch.full((heads[1], rows + 4), -7.0, device="cuda")
        cache.mass(q, lse, mass=before, decay=decay, out=out, appended=appended, **kw)
        want, bound = scored.mass(q, keys, lse, seen, scale, pos0, kw.get("softcap", 0.0), kw.get("slopes"), before, decay,
                                  prefix if appended else rows, dtype == "bf16" and heads[2] == 128)
        off = (out[:, :rows].double() - want).abs()
        assert bool((off <= bound).all()), (name, float((off / bound).max()))
        assert bool((out[:, rows:] == -7.0).all())       # nothing behind the last row
        assert cache.status() == binding.KVF_OK


def test_mass_in_place_and_without_a_start():
    cache, gen = make((32, 8, 128), "bf16", 2000, 256, prefix=1500, seed=1)
    q = chunk(cache, gen, 100)[0]
    lse = torch.randn((100, 32), generator=gen, device="cuda") + 8
    fresh = cache.mass(q, lse)
    assert fresh.shape == (8, 1500)
    held = torch.rand((8, 2000), generator=gen, device="cuda")
    want = torch.where(torch.arange(2000, device="cuda") < 1400, held * 0.25, 0.0)[:, :1500] + fresh
    cache.mass(q, lse, mass=held, decay=0.25, out=held)
    assert float(((held[:, :1500] - want).abs() / (want + 1e-6)).max()) <= 2.0 ** -22
    # bit for bit the same again
    assert torch.equal(cache.mass(q, lse), fresh)


def test_mass_of_a_step_adds_up_to_its_tokens():
    """fold, rotate, mass: the weights of a step sum to one for every token and query head."""
    for heads, dtype in HEADS:
        n, prefix = 60, 700
        cache, gen = make(heads, dtype, 800, n, prefix=prefix, seed=2)
        q, k, v = chunk(cache, gen, n)
        lse = torch.empty((n, heads[0]), device="cuda")
        cache.fold_step(q, k, v, lse=lse, softcap=10.0)
        mass = cache.mass(cache.rotate(q), lse, softcap=10.0)
        want = n * heads[0] / heads[1]
        # (scores of fold and mass come from the same rounded queries; the denominators are fp32)
        assert float((mass.double().sum(1) - want).abs().max()) <= 1e-4 * want


def test_rotated_queries_are_the_rotation():
    for heads, dtype in HEADS:
        cache, gen = make(heads, dtype, 4000, 50, prefix=3000, seed=3)
        q = chunk(cache, gen, 50)[0]
        want = scored.turned(q, 2950, BASE)
        u = scored.U[cache.torch_dtype]
        size = scored.turned(q.abs(), 0, BASE).abs().amax() * 4
        got = cache.rotate(q)
        assert float((got.double() - want).abs().max()) <= u * float(want.abs().max()) + 2.0 ** -22 * float(size)
        inplace = q.clone()
        assert torch.equal(cache.rotate(inplace, out=inplace), got)


SHAPES = [(1, 1, 0, 0), (5, 3, 0, 0), (130, 130, 4, 20), (130, 24, 4, 20), (1000, 1, 0, 0), (1000, 999, 3, 0), (4097, 2000, 4, 700), (33000, 8193, 1, 256),
          (70001, 35000, 0, 1), (460001, 1234, 4, 1000)]


def rows_of(cache, kv):
    if isinstance(cache, binding.PagedCache):
        table = cache.page_table.long()
        if cache.cfg.flags & (binding.KVF_CACHE_INT8 | binding.KVF_CACHE_INT4):
            codes = cache.page_codes(kv)[table].permute(1, 0, 2, 3).reshape(cache.cfg.n_kv_heads, -1, cache.cfg.head_dim)
            scale = cache.page_scales(kv)[table].permute(1, 0, 2).reshape(cache.cfg.n_kv_heads, -1)
            return codes, scale
        return cache.page_rows(kv)[table].permute(1, 0, 2, 3).reshape(cache.cfg.n_kv_heads, -1, cache.cfg.head_dim), None
    plane = cache.v_plane() if kv else cache.k_plane()
    return plane, cache.scales(kv) if cache.cfg.flags & (binding.KVF_CACHE_INT8 | binding.KVF_CACHE_INT4) else None


def same_rows(src, dst, kept):
    head = torch.arange(kept.shape[0], device="cuda")[:, None]
    for kv in (0, 1):
        (a, sa), (b, sb) = rows_of(src, kv), rows_of(dst, kv)
        assert torch.equal(a[head, kept.long()], b[:, :kept.shape[1]])
        if sa is not None:
            assert torch.equal(sa[head, kept.long()], sb[:, :kept.shape[1]])


@pytest.mark.parametrize("rows,budget,sinks,recent", SHAPES)
@pytest.mark.parametrize("heads,dtype", [((4, 2, 128), "bf16"), ((3, 3, 64), "f32")])
def test_eviction_keeps_what_counts_most(heads, dtype, rows, budget, sinks, recent):
    src, gen = make(heads, dtype, rows, 1, prefix=rows, seed=rows)
    dst, _ = make(heads, dtype, budget + 3, 1)
    dst.storage.fill_(0xFF)                                        # NaN everywhere
    mass = (torch.randn((heads[1], rows + 1), generator=gen, device="cuda") * 3).exp().mul_(8).round_().div_(8)     # many alike
    out = torch.full((heads[1], budget + 2), -1.0, device="cuda")
    kept = src.evict(dst, mass, budget, n_sink=sinks, n_recent=recent, mass_out=out)
    assert len(dst) == budget and len(src) == rows
    assert torch.equal(kept.cpu(), scored.kept_rows(mass, rows, sinks, recent, budget))
    same_rows(src, dst, kept)
    head = torch.arange(heads[1], device="cuda")[:, None]
    assert torch.equal(out[:, :budget], mass[head, kept.long()]) and bool((out[:, budget:] == -1).all())
    # value rows behind the last one are zeros up to the tile's end, as after an append
    end = min((budget + 127) // 128 * 128, budget + 3)
    assert bool((dst.v_plane()[:, budget:end] == 0).all())


def test_eviction_of_odd_weights():
    """Ties, signs, infinities and NaN: a total order, the lower row first."""
    rows, budget = 700, 300
    for k, fill in enumerate([lambda m: m.zero_(), lambda m: m.fill_(math.nan), lambda m: m.neg_(),
                              lambda m: m.masked_fill_(torch.rand_like(m) < 0.6, math.nan),
                              lambda m: m.masked_fill_(torch.rand_like(m) < 0.2, math.inf).masked_fill_(torch.rand_like(m) < 0.7, -math.inf),
                              lambda m: m.mul_(0).copysign_(torch.randn_like(m)), lambda m: m.mul_(1e-42)]):
        src, gen = make((4, 2, 128), "bf16", rows, 1, prefix=rows, seed=k)
        dst, _ = make((4, 2, 128), "bf16", rows, 1)
        mass = torch.randn((2, rows), generator=gen, device="cuda")
        fill(mass)
        kept = src.evict(dst, mass, budget, n_sink=2, n_recent=10)
        assert torch.equal(kept.cpu(), scored.kept_rows(mass, rows, 2, 10, budget)), k
        same_rows(src, dst, kept)


@pytest.mark.parametrize("flag", [0, binding.KVF_CACHE_INT8, binding.KVF_CACHE_INT4])
@pytest.mark.parametrize("paged", [(False, False), (True, True), (False, True), (True, False)])
def test_eviction_of_every_storage(flag, paged):
    rows, budget, h, kv = 517, 260, 8, 2
    gen = torch.Generator(device="cuda").manual_seed(11)
    cfg = binding.make_config(h, kv, 128, "bf16", 640, 640, rope_base=BASE, flags=flag)
    pool = torch.zeros(binding.paged_pool_bytes(cfg, 12), dtype=torch.uint8, device="cuda")
    tables = torch.randperm(12, generator=gen, device="cuda").to(torch.int32)

    def one(is_paged, which):
        return binding.PagedCache(cfg, pool, 12, tables[5 * which:5 * which + 5]) if is_paged else binding.Cache(cfg)

    src, dst = one(paged[0], 0), one(paged[1], 1)
    q, k, v = (torch.randn((rows, heads, 128), generator=gen, device="cuda").bfloat16() for heads in (h, kv, kv))
    src.fold_step(q, k, v)
    held = lambda: [x[:, :rows].clone() for x in rows_of(src, 0) + rows_of(src, 1) if x is not None]      # (rows behind hold anything)
    before = held()
    mass = torch.rand((kv, rows), generator=gen, device="cuda")
    kept = src.evict(dst, mass, budget, n_sink=3, n_recent=50)
    assert torch.equal(kept.cpu(), scored.kept_rows(mass, rows, 3, 50, budget))
    same_rows(src, dst, kept)
    assert all(torch.equal(a, b) for a, b in zip(before, held()))
    # the next step on the smaller cache attends to the kept rows (and is told its position)
    q, k, v = (torch.randn((3, heads, 128), generator=gen, device="cuda").bfloat16() for heads in (h, kv, kv))
    out = dst.fold_step(q, k, v, pos0=rows)
    assert len(dst) == budget + 3 and bool(torch.isfinite(out.float()).all()) and dst.status() == binding.KVF_OK
    if not flag and not paged[1]:
        seen = scored.ranges(3, budget + 3, budget, True)
        want, _, bound, _ = scored.attend(scored.turned(q, rows, BASE), dst.k_plane()[:, :budget + 3], dst.v_plane()[:, :budget + 3], seen, 1 / math.sqrt(128), rows)
        assert bool(((out.double() - want).abs() <= bound).all())


def test_a_bounded_fold():
    """The loop the operators are for: fold a chunk, add up its weights, cut back to the budget, go on."""
    h, kv, budget, n = 8, 2, 300, 64
    caches = [make((h, kv, 128), "bf16", budget + n, n)[0] for _ in range(2)]
    gen = torch.Generator(device="cuda").manual_seed(5)
    mass = torch.zeros((kv, budget + n), device="cuda")
    spare = torch.zeros_like(mass)
    pos = 0
    for step in range(9):
        here, there = caches
        q, k, v = chunk(here, gen, n)
        lse = torch.empty((n, h), device="cuda")
        out = here.fold_step(q, k, v, pos0=pos, lse=lse, softcap=30.0)
        prefix = len(here) - n
        seen = scored.ranges(n, len(here), prefix, True)
        keys, values = here.k_plane()[:, :len(here)], here.v_plane()[:, :len(here)]
        want, _, bound, _ = scored.attend(scored.turned(q, pos, BASE), keys, values, seen, 1 / math.sqrt(128), pos, 30.0)
        assert bool(((out.double() - want).abs() <= bound).all())
        q_rot = here.rotate(q, pos0=pos)
        before = mass.clone()
        here.mass(q_rot, lse, mass=mass, decay=0.9, out=mass, softcap=30.0)
        sums, off = scored.mass(q_rot, keys, lse, seen, 1 / math.sqrt(128), pos, 30.0, mass_in=before, decay=0.9, held=prefix)
        assert bool(((mass[:, :len(here)].double() - sums).abs() <= off).all())
        pos += n
        if len(here) > budget:
            kept = here.evict(there, mass, budget, n_sink=4, n_recent=n, mass_out=spare)
            assert torch.equal(kept.cpu(), scored.kept_rows(mass, len(here), 4, n, budget))
            caches, mass, spare = caches[::-1], spare, mass
    assert all(c.status() == binding.KVF_OK for c in caches)


def paged_pair(rows, n, seed=0, h=8, kv=2):
    """A contiguous and a paged cache (pages in no order) that hold the same rows."""
    cfg = binding.make_config(h, kv, 128, "bf16", rows + n, max(n, 1), rope_base=BASE)
    pages = (rows + n + 127) // 128
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pool = torch.zeros(binding.paged_pool_bytes(cfg, pages + 3), dtype=torch.uint8, device="cuda")
    table = torch.randperm(pages + 3, generator=gen, device="cuda")[:pages].to(torch.int32)
    flat, paged = binding.Cache(cfg), binding.PagedCache(cfg, pool, pages + 3, table)
    flat.storage.zero_()
    for kvi, plane in enumerate((flat.k_plane(), flat.v_plane())):
        plane[:, :rows] = torch.randn((kv, rows, 128), generator=gen, device="cuda")
        padded = torch.zeros((kv, pages * 128, 128), dtype=torch.bfloat16, device="cuda")
        padded[:, :rows] = plane[:, :rows]
        paged.page_rows(kvi)[table.long()] = padded.view(kv, pages, 128, 128).transpose(0, 1)
    flat.set_len(rows)
    paged.set_len(rows)
    return flat, paged, gen


@pytest.mark.parametrize("n", [1, 40, 200])
def test_paged_caches_give_the_bits_of_contiguous_ones(n):
    rows = 1500
    flat, paged, gen = paged_pair(rows, n)
    q, k, v = chunk(flat, gen, n)
    kw = dict(softcap=12.0, first=torch.randint(0, rows, (n,), generator=gen, device="cuda", dtype=torch.int32), slopes=slopes_of(8))
    got = []
    for cache in (flat, paged):
        lse = torch.empty((n, 8), device="cuda")
        out = cache.fold_step(q, k, v, lse=lse, **kw)
        got.append((out, lse, cache.mass(cache.rotate(q), lse, **kw)))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("heads,dtype", [((32, 8, 128), "bf16"), ((28, 4, 128), "bf16"), ((8, 2, 128), "f32")])
@pytest.mark.parametrize("n", [1, 300])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_mass_of_rows_that_nobody_sees_is_nothing_whatever_they_hold(heads, dtype, n, bad):
    rows = 700
    cache, gen = make(heads, dtype, 800, 300, prefix=rows, seed=4)
    q = chunk(cache, gen, n)[0]
    lse = torch.randn((n, heads[0]), generator=gen, device="cuda") + 7
    first = torch.full((n,), 290, dtype=torch.int32, device="cuda")
    clean = cache.mass(q, lse, first=first)
    cache.k_plane()[:, 100:290] = bad
    dirty = cache.mass(q, lse, first=first)
    assert torch.equal(clean, dirty) and bool((clean[:, :290] == 0).all())


def test_operators_side_by_side_on_two_streams():
    """Two caches with workspaces of their own, a bounded fold on each, at the same time and one after the other: the same bits."""
    def run(stream, seed):
        a, gen = make((8, 2, 128), "bf16", 1300, 200, prefix=1000, seed=seed)
        b, _ = make((8, 2, 128), "bf16", 1300, 200)
        stream.wait_stream(torch.cuda.current_stream())
        got = []
        with torch.cuda.stream(stream):
            mass = torch.rand((2, 1300), generator=gen, device="cuda")
            for _ in range(4):
                q, k, v = chunk(a, gen, 150)
                lse = torch.empty((150, 8), device="cuda")
                got.append(a.fold_step(q, k, v, lse=lse, softcap=9.0))
                a.mass(a.rotate(q), lse, mass=mass, out=mass, softcap=9.0)
                left = torch.zeros_like(mass)
                got.append(a.evict(b, mass, 1000, n_sink=2, n_recent=100, mass_out=left))
                a, b, mass = b, a, left
            got.append(mass)
        return got
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    both = run(one, 1), run(two, 2)
    torch.cuda.synchronize()
    alone = []
    for seed in (1, 2):
        alone.append(run(torch.cuda.current_stream(), seed))
        torch.cuda.synchronize()
    for x, y in zip(both, alone):
        assert all(torch.equal(p, q) for p, q in zip(x, y))


def test_captured_mass_and_eviction_replay_on_new_weights():
    src, gen = make((8, 2, 128), "bf16", 900, 64, prefix=900, seed=3)
    dst, _ = make((8, 2, 128), "bf16", 500, 1)
    q = chunk(src, gen, 64)[0]
    lse = torch.randn((64, 8), generator=gen, device="cuda") + 7
    mass, out, left = torch.zeros((2, 900), device="cuda"), torch.zeros((2, 900), device="cuda"), torch.zeros((2, 500), device="cuda")
    kept = torch.zeros((2, 500), dtype=torch.int32, device="cuda")

    def steps():
        src.mass(q, lse, mass=mass, out=out)
        src.evict(dst, out, 500, n_sink=4, n_recent=64, mass_out=left, kept=kept)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        steps()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            steps()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        mass.copy_(torch.rand(mass.shape, generator=gen, device="cuda"))
        q.copy_(chunk(src, gen, 64)[0])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, src.mass(q, lse, mass=mass))
        assert torch.equal(kept.cpu(), scored.kept_rows(out, 900, 4, 64, 500))
        same_rows(src, dst, kept)


def test_a_denominator_that_is_nan_reaches_the_rows_its_token_sees_and_no_others():
    for heads, dtype in (((32, 8, 128), "bf16"), ((8, 2, 64), "f32")):
        for n in (1, 200):
            cache, gen = make(heads, dtype, 600, n, prefix=600, seed=1)
            q = chunk(cache, gen, n)[0]
            lse = torch.randn((n, heads[0]), generator=gen, device="cuda") + 7
            lse[0, 0] = math.nan
            first = torch.zeros(n, dtype=torch.int32, device="cuda")
            first[0] = 150
            mass = cache.mass(q, lse, first=first)
            seen = torch.arange(600, device="cuda")
            assert torch.equal(torch.isnan(mass[0]), (seen >= 150) & (seen <= 600 - n))
            assert not bool(torch.isnan(mass[1:]).any())


def test_mass_of_a_whole_large_chunk_in_many_splits():
    """Few keys and many queries: the query tiles are split over CTAs, whose sums are added in order."""
    cache, gen = make((16, 2, 128), "bf16", 3000, 2900, prefix=2900, seed=2)
    q = chunk(cache, gen, 2900)[0]
    keys = cache.k_plane()[:, :2900]
    seen = scored.ranges(2900, 2900, 0, True)
    lse = torch.cat([lse_of(q[a:a + 500].double(), keys, (seen[0][a:a + 500], seen[1][a:a + 500]), 1 / math.sqrt(128), a) for a in range(0, 2900, 500)])
    got = cache.mass(q, lse)
    want, off = 0, 0
    for a in range(0, 2900, 500):
        w, o = scored.mass(q[a:a + 500], keys, lse[a:a + 500], (seen[0][a:a + 500], seen[1][a:a + 500]), 1 / math.sqrt(128), a)
        want, off = want + w, off + o
    assert bool(((got.double() - want).abs() <= off + 2900 * 8 * 2.0 ** -24 * want).all())
    assert torch.equal(got, cache.mass(q, lse))


def test_weights_behind_a_step_whose_merge_is_open():
    n, prefix = 256, 20000
    got, held = [], []
    for flags in (0, binding.KVF_COMBINE_BEHIND):
        cache, gen = make((32, 8, 128), "bf16", 24000, n, flags=flags, prefix=prefix, seed=6)
        for _ in range(8):
            q, k, v = chunk(cache, gen, n)
            lse = torch.full((n, 32), math.nan, device="cuda")       # (what is read before the merge has written it stays NaN)
            q_rot = cache.rotate(q, pos0=len(cache))
            held.append((cache.fold_step(q, k, v, lse=lse), lse))    # (results belong to the library while their merge is open)
            got.append(cache.mass(q_rot, lse))
        cache.flush()
        torch.cuda.synchronize()
    for a, b in zip(got[:8], got[8:]):
        assert torch.equal(a, b)
    # a merge left open outside a capture is not joined inside it
    q, k, v = chunk(cache, gen, n)
    q_rot, out = cache.rotate(q, pos0=len(cache)), torch.empty((8, 24000), device="cuda")
    held.append(cache.fold_step(q, k, v, lse=lse))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    count = cache.launch_count()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(binding.KvfError) as e:
            cache.mass(q_rot, lse, out=out)
    assert e.value.code == binding.KVF_ERR_INVALID_ARG and cache.launch_count() == count
    cache.flush()
    torch.cuda.synchronize()


def test_refusals():
    src, gen = make((8, 2, 128), "bf16", 700, 64, prefix=500)
    dst, _ = make((8, 2, 128), "bf16", 300, 1)
    q = chunk(src, gen, 20)[0]
    lse = torch.zeros((20, 8), device="cuda")
    mass = torch.zeros((2, 700), device="cuda")

    def refused(code, f):
        with pytest.raises(binding.KvfError) as e:
            f()
        assert e.value.code == code and len(src) == 500 and len(dst) == 0

    invalid, cap, unsupported = binding.KVF_ERR_INVALID_ARG, binding.KVF_ERR_CAPACITY, binding.KVF_ERR_UNSUPPORTED
    refused(invalid, lambda: src.evict(src, mass, 100))
    refused(invalid, lambda: src.evict(dst, mass, 501))                        # more than there are
    refused(cap, lambda: src.evict(dst, mass, 301))                            # more than there is room for
    refused(invalid, lambda: src.evict(dst, mass, 100, n_sink=60, n_recent=41))
    refused(invalid, lambda: src.evict(dst, mass, 100, n_sink=-1))
    refused(invalid, lambda: src.evict(dst, mass, 100, mass_out=mass))         # over what is read
    refused(invalid, lambda: src.evict(dst, mass, 100, kept=mass.view(torch.int32).view(-1)[:200].view(2, 100)))
    for other in (make((8, 2, 64), "bf16", 300, 1)[0], make((8, 2, 128), "f32", 300, 1)[0], make((8, 4, 128), "bf16", 300, 1)[0],
                  binding.Cache(binding.make_config(8, 2, 128, "bf16", 300, 1, flags=binding.KVF_CACHE_INT8))):
        refused(invalid, lambda: src.evict(other, mass, 100))
    refused(invalid, lambda: src.mass(q, lse, mass=mass[:, 1:], out=mass))     # shifted in place
    for decay in (math.nan, math.inf):
        refused(invalid, lambda: src.mass(q, lse, mass=mass, decay=decay))
    refused(invalid, lambda: src.mass(chunk(src, gen, 65)[0], torch.zeros((65, 8), device="cuda")))       # chunks of 64
    refused(invalid, lambda: src.mass(q, lse, softcap=-2.0))
    refused(invalid, lambda: src.rotate(q, pos0=-1))
    src.set_window(4, 100)
    refused(unsupported, lambda: src.mass(q, lse))
    src.set_window(0, 0)
    coded = binding.Cache(binding.make_config(8, 2, 128, "bf16", 300, 64, flags=binding.KVF_CACHE_INT8))
    coded.set_len(100)
    refused(unsupported, lambda: coded.mass(q, lse))
    with pytest.raises(AssertionError):
        src.mass(q, lse, mass=mass[:, :499])
    with pytest.raises(AssertionError):
        src.evict(dst, mass.double(), 100)
    short, _ = make((8, 2, 128), "bf16", 700, 64, prefix=10)
    with pytest.raises(binding.KvfError):
        short.mass(q, lse)                                                     # 20 tokens appended to 10 rows
