"""Scored steps (softcap, slopes, ranges of rows per token) against their plain statement in 64 bits, element by element."""
import math

import pytest
import torch

from paper_2605_12471_b200 import binding
from tests import scored

pytestmark = pytest.mark.gpu

BASE = 10000.0


def make(heads, dtype, capacity, chunk, flags=0, prefix=0, seed=0, scale=1.0):
    h, kv, d = heads
    cfg = binding.make_config(h, kv, d, dtype, capacity, chunk, rope_base=BASE, flags=flags)
    cache = binding.Cache(cfg)
    cache.storage.zero_()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for plane in (cache.k_plane(), cache.v_plane()):
        plane[:, :prefix] = torch.randn((kv, prefix, d), generator=gen, device="cuda")
    cache.set_len(prefix)
    return cache, gen


def chunk(cache, gen, n, scale=1.0):
    c = cache.cfg
    return [(torch.randn((n, heads, c.head_dim), generator=gen, device="cuda") * s).to(cache.torch_dtype)
            for heads, s in ((c.n_q_heads, scale), (c.n_kv_heads, 1.0), (c.n_kv_heads, 1.0))]


def slopes_of(h):
    return torch.exp2(-8.0 * (torch.arange(h, device="cuda", dtype=torch.float32) + 1) / h)


def documents(n, prefix, gen, padded=True):
    """first, end of documents of random lengths packed into a chunk, the first of them going on from the prefix."""
    first, end = torch.zeros(n, dtype=torch.int32), torch.arange(prefix + 1, prefix + n + 1, dtype=torch.int32)
    cuts = sorted(set(torch.randint(0, n, (max(1, n // 40),), generator=gen, device="cuda").tolist()))
    for c in cuts:
        first[c:] = prefix + c
    if padded and n > 3:
        end[-2:] = 0                      # padding: sees nothing
        first[1] = prefix + n             # sees nothing either: begins behind its own row
    return first.cuda(), end.cuda()


def check(cache, q, k, v, n, appended, lse, out, pos0, **kw):
    rows = len(cache)
    prefix = rows - n if appended else rows
    seen = scored.ranges(n, rows, prefix, appended, kw.get("first"), kw.get("end"))
    d = cache.cfg.head_dim
    tc = cache.torch_dtype == torch.bfloat16 and d == 128
    want, want_lse, bound, lse_bound = scored.attend(
        scored.turned(q, pos0, BASE), cache.k_plane()[:, :rows], cache.v_plane()[:, :rows], seen, 1 / math.sqrt(d), pos0,
        kw.get("softcap", 0.0), kw.get("slopes"), cache.torch_dtype, cache.out_dtype, tc)
    off = (out.double() - want).abs()
    assert bool(torch.isfinite(out.float()).all())
    assert bool((off <= bound).all()), float((off / bound).max())
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert bool((out[empty] == 0).all())
    assert bool(((lse.double() - want_lse).abs() <= lse_bound)[~empty].all())
    assert cache.status() == binding.KVF_OK


HEADS = [((32, 8, 128), "bf16"), ((28, 4, 128), "bf16"), ((4, 4, 128), "bf16"), ((16, 1, 128), "bf16"),
         ((4, 1, 64), "f32"), ((8, 2, 64), "bf16"), ((8, 2, 128), "f32")]
MODS = ["cap", "slopes", "cap+slopes", "docs", "prefix", "all"]


def mods_of(name, h, n, prefix, gen):
    kw = {}
    if "cap" in name or name == "all":
        kw["softcap"] = 5.0                # (scores of either side of it)
    if "slopes" in name or name in ("prefix", "all"):
        kw["slopes"] = slopes_of(h)
    if name in ("docs", "all"):
        kw["first"], kw["end"] = documents(n, prefix, gen)
    if name == "prefix":
        kw["end"] = torch.arange(prefix + 1, prefix + n + 1, dtype=torch.int32, device="cuda").clamp(min=prefix + (n + 1) // 2)
    return kw


@pytest.mark.parametrize("n,prefix", [(1, 0), (1, 1), (1, 700), (3, 129), (5, 1000), (33, 515), (64, 0), (129, 127), (300, 1111)])
@pytest.mark.parametrize("heads,dtype", HEADS)
def test_scored_steps_match_their_statement(heads, dtype, n, prefix):
    for seed, name in enumerate(MODS):
        cache, gen = make(heads, dtype, prefix + n + 5, n, prefix=prefix, seed=seed)
        q, k, v = chunk(cache, gen, n, scale=2.0)
        kw = mods_of(name, heads[0], n, prefix, gen)
        lse = torch.empty((n, heads[0]), device="cuda")
        out = cache.fold_step(q, k, v, lse=lse, **kw)
        assert len(cache) == prefix + n
        check(cache, q, k, v, n, True, lse, out, prefix, **kw)


@pytest.mark.parametrize("n", [1, 7, 200])
@pytest.mark.parametrize("heads,dtype", HEADS[:2] + HEADS[4:])
def test_queries_alone_see_the_rows_their_ranges_name(heads, dtype, n):
    rows = 901
    cache, gen = make(heads, dtype, 1024, n, prefix=rows, seed=5)
    q = chunk(cache, gen, n)[0]
    first = torch.randint(-50, rows + 60, (n,), generator=gen, device="cuda", dtype=torch.int32)
    end = torch.randint(-50, rows + 60, (n,), generator=gen, device="cuda", dtype=torch.int32)
    for kw in (dict(softcap=3.0), dict(first=first), dict(end=end, slopes=slopes_of(heads[0])), dict(first=first, end=end, softcap=8.0)):
        lse = torch.empty((n, heads[0]), device="cuda")
        out = cache.attend(q, pos0=rows + 3, lse=lse, **kw)
        assert len(cache) == rows
        check(cache, q, None, None, n, False, lse, out, rows + 3, **kw)


def test_a_step_with_no_cap_and_no_mask_to_speak_of_is_the_plain_step():
    n, prefix = 100, 333
    outs = []
    for kw in ({}, dict(first=torch.zeros(n, dtype=torch.int32, device="cuda")), dict(slopes=torch.zeros(32, device="cuda"))):
        cache, gen = make((32, 8, 128), "bf16", 512, n, prefix=prefix, seed=3)
        q, k, v = chunk(cache, gen, n)
        outs.append(cache.fold_step(q, k, v, **kw).float())
    for o in outs[1:]:
        assert float((o - outs[0]).abs().max()) <= 2 * 2.0 ** -8 * float(outs[0].abs().max())


@pytest.mark.parametrize("heads,dtype", [((32, 8, 128), "bf16"), ((4, 1, 64), "f32")])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_keys_that_nobody_sees_change_nothing(heads, dtype, bad):
    n, prefix = 40, 400
    got = []
    for plant in (False, True):
        cache, gen = make(heads, dtype, 512, n, prefix=prefix, seed=9)
        q, k, v = chunk(cache, gen, n)
        first = torch.full((n,), 290, dtype=torch.int32, device="cuda")
        if plant:
            cache.k_plane()[:, 5:290] = bad
        lse = torch.empty((n, heads[0]), device="cuda")
        got.append((cache.fold_step(q, k, v, lse=lse, first=first, softcap=10.0), lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_scores_far_beyond_the_cap_stay_at_it():
    n, prefix = 70, 600
    cache, gen = make((8, 2, 128), "bf16", 1024, n, prefix=prefix, seed=4)
    q, k, v = chunk(cache, gen, n, scale=200.0)
    lse = torch.empty((n, 8), device="cuda")
    out = cache.fold_step(q, k, v, lse=lse, softcap=2.0)
    check(cache, q, k, v, n, True, lse, out, prefix, softcap=2.0)


def test_a_captured_step_reads_its_ranges_at_replay():
    n, prefix = 32, 500
    cache, gen = make((32, 8, 128), "bf16", 600, n, prefix=prefix, seed=6)
    q, k, v = chunk(cache, gen, n)
    first = torch.zeros(n, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((n, 32), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.fold_step(q, k, v, out=out, lse=lse, first=first, softcap=20.0)
        cache.set_len(prefix)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            cache.fold_step(q, k, v, out=out, lse=lse, first=first, softcap=20.0)
    torch.cuda.current_stream().wait_stream(side)
    for f in (0, 130, 511):
        first.fill_(f)
        graph.replay()
        torch.cuda.synchronize()
        check(cache, q, k, v, n, True, lse, out, prefix, first=first, softcap=20.0)


def test_a_step_split_many_ways_is_the_step():
    n, prefix = 20, 3000
    for splits in (1, 3, 7, 20):
        cache, gen = make((32, 8, 128), "bf16", 3100, n, prefix=prefix, seed=8)
        cache.set_splits(splits)
        q, k, v = chunk(cache, gen, n)
        first = torch.randint(0, prefix, (n,), generator=gen, device="cuda", dtype=torch.int32)
        lse = torch.empty((n, 32), device="cuda")
        kw = dict(first=first, softcap=6.0, slopes=slopes_of(32))
        out = cache.fold_step(q, k, v, lse=lse, **kw)
        check(cache, q, k, v, n, True, lse, out, prefix, **kw)


def test_repeated_steps_give_the_same_bits():
    n, prefix = 256, 5000
    got = []
    for _ in range(3):
        cache, gen = make((32, 8, 128), "bf16", 6000, n, prefix=prefix, seed=2)
        q, k, v = chunk(cache, gen, n)
        got.append(cache.fold_step(q, k, v, softcap=15.0, slopes=slopes_of(32)))
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("softcap", [1e-3, 0.5, 300.0, 1e5, 1e9])
@pytest.mark.parametrize("n", [1, 5, 40, 200])
def test_caps_of_every_size(softcap, n):
    prefix = 300
    cache, gen = make((32, 8, 128), "bf16", 600, n, prefix=prefix, seed=21)
    q, k, v = chunk(cache, gen, n, scale=2.0)
    lse = torch.empty((n, 32), device="cuda")
    out = cache.fold_step(q, k, v, lse=lse, softcap=softcap)
    # (a cap far above the scores leaves them as they are but for the polynomial's 2^-20 of the score itself)
    want, want_lse, bound, lse_bound = scored.attend(
        scored.turned(q, prefix, BASE), cache.k_plane()[:, :prefix + n], cache.v_plane()[:, :prefix + n], scored.ranges(n, prefix + n, prefix, True),
        1 / math.sqrt(128), prefix, softcap)
    plain = scored.attend(scored.turned(q, prefix, BASE), cache.k_plane()[:, :prefix + n], cache.v_plane()[:, :prefix + n],
                          scored.ranges(n, prefix + n, prefix, True), 1 / math.sqrt(128), prefix)
    if softcap >= 1e5:
        bound = plain[2] + 2.0 ** -18 * 20 * plain[0].abs() + 2.0 ** -14       # (scores reach 20 here: 2^-20 * 20 * log2(e) each)
    assert bool(((out.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("softcap", [1e-25, 1e-12, 1e-8, 1e20])
@pytest.mark.parametrize("n", [1, 40, 200])
@pytest.mark.parametrize("size", [0.0, 1.0])
def test_caps_whose_powers_leave_the_range_of_fp32(softcap, n, size):
    prefix = 700
    cache, gen = make((32, 8, 128), "bf16", 1000, n, prefix=prefix, seed=14)
    q, k, v = chunk(cache, gen, n)
    q = q * size                                   # (no query at all: every score is zero)
    lse = torch.empty((n, 32), device="cuda")
    out = cache.fold_step(q, k, v, lse=lse, softcap=softcap)
    # a cap far above the scores leaves them, one far below makes all rows alike
    check(cache, q, k, v, n, True, lse, out, prefix, softcap=0.0 if softcap > 1.0 else softcap)
    mass = cache.mass(cache.rotate(q), lse, softcap=softcap)
    assert float((mass.double().sum(1) - 4 * n).abs().max()) <= 1e-4 * 4 * n


def test_caps_beyond_the_range_of_fp32_are_refused():
    cache, gen = make((32, 8, 128), "bf16", 600, 64, prefix=300)
    q, k, v = chunk(cache, gen, 4)
    lse = torch.zeros((4, 32), device="cuda")
    for softcap in (1e-300, 1e-40, 1e31, 1e300):
        for f in (lambda: cache.fold_step(q, k, v, softcap=softcap), lambda: cache.attend(q, softcap=softcap), lambda: cache.mass(q, lse, softcap=softcap)):
            with pytest.raises(binding.KvfError) as e:
                f()
            assert e.value.code == binding.KVF_ERR_INVALID_ARG and len(cache) == 300


@pytest.mark.parametrize("n", [1, 3, 40, 300])
@pytest.mark.parametrize("pos0", [0, 250, 10000])
def test_biases_of_tokens_before_among_and_behind_the_rows(n, pos0):
    prefix = 500
    for kw in (dict(slopes=slopes_of(32)), dict(slopes=-slopes_of(32) / 16, softcap=8.0), dict(slopes=slopes_of(32) * 40)):
        cache, gen = make((32, 8, 128), "bf16", 900, n, prefix=prefix, seed=12)
        q, k, v = chunk(cache, gen, n)
        lse = torch.empty((n, 32), device="cuda")
        out = cache.fold_step(q, k, v, pos0=pos0, lse=lse, **kw)
        check(cache, q, k, v, n, True, lse, out, pos0, **kw)


@pytest.mark.parametrize("heads", [(64, 1, 128), (12, 2, 128), (5, 5, 128), (6, 1, 64)])
def test_groups_of_every_size(heads):
    for n in (1, 2, 37, 130):
        cache, gen = make(heads, "bf16", 700, n, prefix=400, seed=n)
        q, k, v = chunk(cache, gen, n)
        kw = mods_of("all", heads[0], n, 400, gen)
        lse = torch.empty((n, heads[0]), device="cuda")
        out = cache.fold_step(q, k, v, lse=lse, **kw)
        check(cache, q, k, v, n, True, lse, out, 400, **kw)


def test_scored_steps_with_the_merge_behind_them():
    n, prefix = 64, 2000
    cache, gen = make((32, 8, 128), "bf16", 3000, n, flags=binding.KVF_COMBINE_BEHIND, prefix=prefix, seed=5)
    steps = []
    for t in range(5):
        q, k, v = chunk(cache, gen, n)
        lse = torch.empty((n, 32), device="cuda")
        out = cache.fold_step(q, k, v, lse=lse, softcap=9.0, slopes=slopes_of(32))
        if t == 2:                              # the weights are added up beside an open merge: it reads partial results of its own
            cache.mass(cache.rotate(q), torch.zeros((n, 32), device="cuda") + 9, softcap=9.0)
        steps.append((q, out, lse, len(cache)))
    cache.flush()
    for q, out, lse, rows in steps:
        cache.set_len(rows)
        check(cache, q, None, None, n, True, lse, out, rows - n, softcap=9.0, slopes=slopes_of(32))


def test_refusals():
    cache, gen = make((32, 8, 128), "bf16", 600, 64, prefix=300)
    q, k, v = chunk(cache, gen, 40)

    def refused(code, f):
        rows, count = len(cache), cache.launch_count()
        with pytest.raises(binding.KvfError) as e:
            f()
        assert e.value.code == code and len(cache) == rows and cache.launch_count() == count

    invalid = binding.KVF_ERR_INVALID_ARG
    for cap in (-1.0, math.nan, math.inf):
        refused(invalid, lambda: cache.fold_step(q, k, v, softcap=cap))
        refused(invalid, lambda: cache.attend(q, softcap=cap))
    refused(invalid, lambda: cache.fold_step(q, k, v, softcap=1.0, pos0=-1))
    refused(invalid, lambda: cache.attend(torch.cat([q, q]), softcap=1.0))                       # 80 tokens, chunks of 64
    cache.set_len(580)
    refused(binding.KVF_ERR_CAPACITY, lambda: cache.fold_step(q, k, v, softcap=1.0))
    cache.set_len(0)
    refused(invalid, lambda: cache.attend(q, softcap=1.0))
    cache.set_len(300)
    cache.set_window(4, 100)
    refused(binding.KVF_ERR_UNSUPPORTED, lambda: cache.fold_step(q, k, v, softcap=1.0))
    refused(binding.KVF_ERR_UNSUPPORTED, lambda: cache.attend(q, softcap=1.0))
    cache.set_window(0, 0)
    with pytest.raises(AssertionError):
        cache.fold_step(q, k, v, first=torch.zeros(39, dtype=torch.int32, device="cuda"))
    with pytest.raises(AssertionError):
        cache.fold_step(q, k, v, slopes=torch.zeros(32, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(AssertionError):
        cache.fold_step(q, k, v, slopes=torch.zeros(32))
    assert cache.status() == binding.KVF_OK
