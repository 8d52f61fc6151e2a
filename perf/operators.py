"""The operators beside the plain fold step, as cases that can be timed and compared.

Three kinds of case, each on one layer's cache (`prefix` rows held, `tokens` new ones):
  fold   one fold step whose scores are capped by a tanh and / or biased by the distance, and whose tokens see what a
         mask of one range of rows per token leaves them (documents packed one after the other, a prefix that sees itself both ways)
  mass   the attention weight that a chunk's queries gave every row of the cache, added to what the rows had
  evict  the rows with the most weight, the first and the latest ones, moved in order into a smaller cache

Fields: q_heads, kv_heads, head_dim; dtype "bf16" / "f32"; prefix, tokens; scale (of the queries: how spread out the scores are);
softcap (0 = none), slopes (a bias that falls with the distance, another slope for each query head), mask "causal" / "docs" (with
`docs`, their mean length, and a few tokens of padding that see nothing) / "prefix" (the first `both` rows of the cache are seen by all
tokens); decay (of the weight held so far); evict: rows, budget, sinks, recent.  Inputs are Gaussian, as everywhere in this repository.
"""
import math
import random

import torch

own = False

_BASE = dict(op="fold", q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", prefix=0, tokens=1, scale=1.0, softcap=0.0, slopes=False,
             mask="causal", docs=0, both=0, decay=1.0, rows=0, budget=0, sinks=0, recent=0)
_HEADS = [(32, 8), (32, 8), (28, 4), (16, 16), (12, 2)]


def _case(**kw):
    return dict(_BASE, **kw)


def listed():
    return [
        # one decoded token of a model that caps its scores, behind a short prompt: latency
        _case(name="cap_decode_4k", prefix=4095, softcap=50.0, scale=2.0),
        # one decoded token of a model without rotary distances to go by, behind a long folded context: the bytes of the cache
        _case(name="slopes_decode_129k", prefix=129024, slopes=True),
        # a question of 33 tokens, capped, behind a context of no round length
        _case(name="cap_question_50k", prefix=50021, tokens=33, softcap=30.0),
        # a chunk of the deep chain with capped scores
        _case(name="cap_fold_31k_c256", prefix=31003, tokens=256, softcap=50.0, scale=2.0),
        # documents packed into one long chunk (training-like prefill): each token sees its own document
        _case(name="docs_8k", tokens=8192, mask="docs", docs=900),
        # a prompt that sees itself both ways, groups of 7, a bias by distance and a cap
        _case(name="prefix_slopes_2k", q_heads=28, kv_heads=4, prefix=6013, tokens=2048, mask="prefix", both=7500, slopes=True, softcap=50.0),
        # the toy model of the tests, fp32, all of it at once: launches
        _case(name="tiny_f32", q_heads=4, kv_heads=1, head_dim=64, dtype="f32", prefix=448, tokens=64, softcap=20.0, slopes=True),
        # the weight that one decoded token gives a long context's rows
        _case(name="mass_decode_129k", op="mass", prefix=129024, decay=0.99),
        # the weight of one chunk's queries on a folded context, scores capped
        _case(name="mass_31k_c256", op="mass", prefix=31003, tokens=256, softcap=50.0, scale=4.0),
        # the weight of a whole large chunk, groups of 7
        _case(name="mass_14k_c2048", op="mass", q_heads=28, kv_heads=4, prefix=14336, tokens=2048),
        # a budget of 1 K rows kept over a chunk of 256: the step that follows every chunk of a bounded fold
        _case(name="evict_1k", op="evict", rows=1280, budget=1024, sinks=4, recent=256),
        # a folded haystack cut down to a quarter
        _case(name="evict_128k_to_32k", op="evict", rows=131072, budget=32768, sinks=4, recent=1020),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    top = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= top:
            return case


def _cost(case):
    w = work(case)
    # (in the order of what a pass takes: fp32 on CUDA cores; scores computed, seen or not, where they are written out)
    pairs = case["q_heads"] * case["tokens"] * (case["prefix"] + case["tokens"]) if case["op"] != "evict" else 0
    return max(w["bytes"] / 6e12, w["flops"] * (8 if case["dtype"] == "f32" else 1) / 1e15, pairs * 4e-12)


def _draw(rng):
    kind = rng.choice(["decode", "decode", "fold", "fold", "docs", "prefix", "f32", "mass", "mass", "mass", "evict", "evict"])
    q, kv = rng.choice(_HEADS)
    shape = dict(q_heads=q, kv_heads=kv)
    score = dict(softcap=rng.choice([0.0, 20.0, 30.0, 50.0]), slopes=rng.random() < 0.4, scale=rng.choice([1.0, 1.5, 2.0]))
    if not score["softcap"]:
        score["slopes"] = True
    if kind == "decode":
        return _case(**shape, **score, prefix=_log(rng, 1, 130000), tokens=rng.choice([1, 1, 2, 3]))
    if kind == "fold":
        return _case(**shape, **score, prefix=rng.choice([0, _log(rng, 100, 60000)]), tokens=_log(rng, 5, 4096))
    if kind == "docs":
        tokens = _log(rng, 100, 8192)
        return _case(**shape, tokens=tokens, prefix=rng.choice([0, _log(rng, 100, 8000)]), mask="docs", docs=_log(rng, 20, 2000))
    if kind == "prefix":
        prefix, tokens = rng.choice([0, _log(rng, 100, 8000)]), _log(rng, 30, 4096)
        return _case(**shape, **score, prefix=prefix, tokens=tokens, mask="prefix", both=rng.randint(1, prefix + tokens))
    if kind == "f32":
        q, kv, d = rng.choice([(4, 1, 64), (8, 2, 64), (2, 2, 64), (8, 2, 128)])
        return _case(**score, q_heads=q, kv_heads=kv, head_dim=d, dtype="f32", prefix=rng.choice([0, _log(rng, 10, 4000)]), tokens=_log(rng, 1, 300))
    if kind == "mass":
        tokens = rng.choice([1, _log(rng, 1, 2048)])
        return _case(**shape, op="mass", prefix=_log(rng, 1, 130000), tokens=tokens, softcap=score["softcap"], scale=rng.choice([1.0, 2.0, 4.0]),
                     decay=rng.choice([0.0, 1.0, 0.95]))
    rows = _log(rng, 50, 131072)
    sinks, recent = rng.choice([(0, 0), (4, rows // 20), (1, rows // 5)])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    return _case(**shape, op="evict", dtype=dtype, rows=rows, sinks=sinks, recent=recent, budget=rng.randint(sinks + recent + 1, rows))


def _documents(case):
    """Lengths of the packed documents; the last tokens of the chunk (one in 64) are padding."""
    n = case["tokens"] - case["tokens"] // 64
    rng, lengths = random.Random(case["docs"] * 100003 + n), []
    while sum(lengths) < n:
        lengths.append(min(n - sum(lengths), max(1, int(rng.expovariate(1.0 / case["docs"])))))
    return lengths


def _ranges(case):
    """(first row, end) that each token of a step sees."""
    p, n = case["prefix"], case["tokens"]
    first, end = [0] * n, [p + i + 1 for i in range(n)]
    if case["mask"] == "prefix":
        end = [max(e, case["both"]) for e in end]
    if case["mask"] == "docs":
        first, at = [], p
        for length in _documents(case):
            # (the first document goes on from the rows held)
            first += [at if first else 0] * length
            at += length
        end = end[:len(first)] + [0] * (n - len(first))
        first += [0] * (n - len(first))
    return first, end


def work(case):
    h, kv, d, eb = case["q_heads"], case["kv_heads"], case["head_dim"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "evict":
        return {"bytes": 4 * kv * case["rows"] + case["budget"] * kv * (2 * 2 * d * eb + 8), "flops": 0}
    n = case["tokens"]
    first, end = _ranges(case)
    pairs = sum(max(0, e - f) for f, e in zip(first, end))
    rows = case["prefix"] + n
    if case["op"] == "mass":
        return {"bytes": kv * rows * (d * eb + 8) + n * h * (d * eb + 4), "flops": 2 * h * d * pairs}
    return {"bytes": 2 * kv * rows * d * eb + n * (2 * h + 2 * kv) * d * eb, "flops": 4 * h * d * pairs}


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _base(case):
    return 10000.0 if case["head_dim"] == 64 else 500000.0


def _inputs(case, seed):
    """What a case is made of, by name; the same for every side."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h, kv, d, n, t = case["q_heads"], case["kv_heads"], case["head_dim"], case["tokens"], _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=t)

    if case["op"] == "evict":
        # weights over several powers of ten, many of them alike
        mass = (torch.randn((kv, case["rows"]), generator=gen, device="cuda") * 2).exp().mul_(64).round_().div_(64)
        return {"planes": [normal(kv, case["rows"], d) for _ in range(2)], "mass": mass}
    rows = case["prefix"] + (n if case["op"] == "mass" else 0)
    got = {"planes": [normal(kv, rows, d) for _ in range(2)], "q": normal(n, h, d).mul_(case["scale"])}
    if case["op"] == "mass":
        got["mass"] = torch.rand((kv, rows), generator=gen, device="cuda")
        got["lse"] = _lse(case, got["q"], got["planes"][0])
        return got
    got["k"], got["v"] = normal(n, kv, d), normal(n, kv, d)
    if case["slopes"]:
        got["slopes"] = torch.exp2(-8.0 * (torch.arange(h, device="cuda", dtype=torch.float32) + 1) / h)
    first, end = _ranges(case)
    if case["mask"] == "docs":
        got["first"] = torch.tensor(first, dtype=torch.int32, device="cuda")
    if case["mask"] != "causal":
        got["end"] = torch.tensor(end, dtype=torch.int32, device="cuda")
    return got


def _lse(case, q, keys):
    """Denominators of the chunk's softmaxes, as the fold step before has left them: [tokens, q_heads] fp32."""
    n, kv, d, rows = case["tokens"], case["kv_heads"], case["head_dim"], keys.shape[1]
    group = case["q_heads"] // kv
    got = torch.empty((n, kv, group), device="cuda")
    some = max(1, (1 << 28) // (group * rows))
    for g in range(kv):
        for a in range(0, n, some):
            x = q[a:a + some].view(-1, kv, group, d)[:, g].float()
            s = (x.reshape(-1, d) @ keys[g].float().T).div_(math.sqrt(d))
            if case["softcap"]:
                s = s.div_(case["softcap"]).tanh_().mul_(case["softcap"])
            last = torch.arange(a, a + x.shape[0], device="cuda").repeat_interleave(group) + case["prefix"]
            s.masked_fill_(torch.arange(rows, device="cuda") > last[:, None], -math.inf)
            got[a:a + some, g] = s.logsumexp(-1).view(-1, group)
    return got.view(n, kv * group)


def prepare(case, seed):
    from paper_2605_12471_b200 import binding

    got = _inputs(case, seed)
    capacity = case["rows"] or case["prefix"] + case["tokens"]

    def cache(rows):
        cfg = binding.make_config(case["q_heads"], case["kv_heads"], case["head_dim"], case["dtype"], rows, max(1, min(case["tokens"], rows)), rope_base=_base(case))
        c = binding.Cache(cfg)
        c.storage.zero_()
        return c

    state = dict(got, case=case, cache=cache(capacity))
    held = got["planes"][0].shape[1]
    for plane, rows in zip((state["cache"].k_plane(), state["cache"].v_plane()), got["planes"]):
        plane[:, :held] = rows
    del state["planes"]
    state["cache"].set_len(held)
    if case["op"] == "evict":
        state["into"] = cache(case["budget"])
        state["kept"] = torch.empty((case["kv_heads"], case["budget"]), dtype=torch.int32, device="cuda")
    if case["op"] == "fold":
        state["out"] = torch.empty((case["tokens"], case["q_heads"], case["head_dim"]), dtype=_dtype(case), device="cuda")
    else:
        state["left"] = torch.empty((case["kv_heads"], case["budget"] or held), dtype=torch.float32, device="cuda")
    return state


def run(state):
    case, cache = state["case"], state["cache"]
    if case["op"] == "fold":
        new = slice(case["prefix"], case["prefix"] + case["tokens"])
        if own:
            cache.set_len(case["prefix"])
            cache.fold_step(state["q"], state["k"], state["v"], out=state["out"], softcap=case["softcap"], slopes=state.get("slopes"),
                            first=state.get("first"), end=state.get("end"))
        else:
            state["out"].copy_(_fold(state, cache.k_plane(), cache.v_plane()))
        return {"out": state["out"], "k": cache.k_plane()[:, new], "v": cache.v_plane()[:, new]}
    if case["op"] == "mass":
        if own:
            cache.mass(state["q"], state["lse"], softcap=case["softcap"], mass=state["mass"], decay=case["decay"], out=state["left"])
        else:
            state["left"].copy_(_mass(state, cache.k_plane()))
        return {"mass": state["left"]}
    into = state["into"]
    if own:
        cache.evict(into, state["mass"], case["budget"], n_sink=case["sinks"], n_recent=case["recent"], mass_out=state["left"], kept=state["kept"])
    else:
        _evict(state)
    return {"kept": state["kept"], "mass": state["left"], "k": into.k_plane(), "v": into.v_plane()}


def _turned(case, x):
    """x [n, heads, d] rotated at its positions: angles in 64 bits, products in 32."""
    d = case["head_dim"]
    inv = _base(case) ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
    angle = (case["prefix"] + torch.arange(x.shape[0], device="cuda", dtype=torch.float64))[:, None, None] * inv
    cos, sin = angle.cos().float(), angle.sin().float()
    a, b = x.float().split(d // 2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _scores(case, q, keys):
    """[kv_heads, tokens, group, rows] in 32 bits, capped."""
    kv, d, n = case["kv_heads"], case["head_dim"], q.shape[0]
    q = q.float().view(n, kv, -1, d).permute(1, 0, 2, 3).reshape(kv, -1, d)
    s = (q @ keys.float().transpose(1, 2)).mul_(1.0 / math.sqrt(d))
    if case["softcap"]:
        s = s.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    return s.view(kv, n, -1, keys.shape[1])


def _fold(state, k_plane, v_plane):
    case = state["case"]
    n, kv, d, p = case["tokens"], case["kv_heads"], case["head_dim"], case["prefix"]
    rows = p + n
    k_plane[:, p:rows] = _turned(case, state["k"]).transpose(0, 1)
    v_plane[:, p:rows] = state["v"].transpose(0, 1)
    s = _scores(case, _turned(case, state["q"]), k_plane[:, :rows])
    at, key = torch.arange(p, rows, device="cuda"), torch.arange(rows, device="cuda")
    if case["slopes"]:
        far = (at[:, None] - key).abs().float()
        s -= state["slopes"].view(kv, 1, -1, 1) * far[:, None, :]
    end = state["end"] if "end" in state else at + 1
    hidden = key >= end[:, None]
    if "first" in state:
        hidden |= key < state["first"][:, None]
    s.masked_fill_(hidden[:, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    s = s.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    den = s.sum(-1, keepdim=True)
    out = (s.reshape(kv, -1, rows) @ v_plane[:, :rows].float()).view(kv, n, -1, d)
    return (out / den.masked_fill(den == 0, 1.0)).permute(1, 0, 2, 3).reshape(n, -1, d)


def _mass(state, keys):
    case = state["case"]
    n, kv, rows = case["tokens"], case["kv_heads"], keys.shape[1]
    s = _scores(case, state["q"], keys)
    s -= state["lse"].view(n, kv, -1).permute(1, 0, 2)[..., None]
    s.exp_().masked_fill_((torch.arange(rows, device="cuda") > torch.arange(rows - n, rows, device="cuda")[:, None])[:, None, :], 0.0)
    # (the step's own rows start from nothing)
    held = state["mass"] * case["decay"]
    held[:, rows - n:] = 0
    return held + s.sum((1, 2))


def _evict(state):
    case = state["case"]
    rows, lo, hi = case["rows"], case["sinks"], case["rows"] - case["recent"]
    kv, some = case["kv_heads"], case["budget"] - case["sinks"] - case["recent"]
    best = torch.sort(state["mass"][:, lo:hi], dim=1, descending=True, stable=True)[1][:, :some] + lo
    fixed = torch.cat([torch.arange(lo, device="cuda"), torch.arange(hi, rows, device="cuda")]).expand(kv, -1)
    kept = torch.sort(torch.cat([best, fixed], dim=1), dim=1)[0]
    state["kept"].copy_(kept)
    state["left"].copy_(state["mass"].gather(1, kept))
    index = kept[..., None].expand(-1, -1, case["head_dim"])
    torch.gather(state["cache"].k_plane(), 1, index, out=state["into"].k_plane())
    torch.gather(state["cache"].v_plane(), 1, index, out=state["into"].v_plane())


def exact(case, seed):
    """The outputs of run in 64 bits, one KV head after the other, from what the operators are defined to be."""
    got = _inputs(case, seed)
    kv, d, n, p = case["kv_heads"], case["head_dim"], case["tokens"], case["prefix"]
    if case["op"] == "evict":
        rows, lo, hi = case["rows"], case["sinks"], case["rows"] - case["recent"]
        kept = []
        for weights in got["mass"].cpu().tolist():
            order = sorted(range(lo, hi), key=lambda r: (-weights[r], r))
            kept.append(sorted(order[:case["budget"] - lo - case["recent"]] + list(range(lo)) + list(range(hi, rows))))
        kept = torch.tensor(kept, device="cuda")
        head = torch.arange(kv, device="cuda")[:, None]
        return {"kept": kept.int(), "mass": got["mass"].double()[head, kept], "k": got["planes"][0][head, kept].double(), "v": got["planes"][1][head, kept].double()}
    group = case["q_heads"] // kv
    rows = p + n

    def turned(x):
        z = torch.complex(*x.double().split(d // 2, dim=-1))
        angle = torch.outer(torch.arange(p, rows, device="cuda", dtype=torch.float64), torch.exp(torch.arange(0, d, 2, device="cuda", dtype=torch.float64) * (-math.log(_base(case)) / d)))
        z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
        return torch.cat([z.real, z.imag], dim=-1)

    def score(q, keys):
        s = torch.einsum("tgd,rd->tgr", q, keys) / math.sqrt(d)
        return case["softcap"] * torch.tanh(s / case["softcap"]) if case["softcap"] else s

    first, end = (torch.tensor(x, device="cuda") for x in _ranges(case))
    key = torch.arange(rows, device="cuda")
    some = max(1, (1 << 27) // (group * rows))
    if case["op"] == "mass":
        mass = got["mass"].double() * case["decay"]
        mass[:, p:] = 0
        for g in range(kv):
            for a in range(0, n, some):
                b = min(n, a + some)
                s = score(got["q"][a:b, g * group:(g + 1) * group].double(), got["planes"][0][g].double())
                s = torch.exp(s - got["lse"][a:b, g * group:(g + 1) * group, None].double())
                mass[g] += torch.where(key <= torch.arange(p + a, p + b, device="cuda")[:, None, None], s, 0.0).sum((0, 1))
        return {"mass": mass}
    q, k, v = turned(got["q"]), turned(got["k"]), got["v"].double()
    out = torch.zeros((n, case["q_heads"], d), dtype=torch.float64, device="cuda")
    for g in range(kv):
        keys = torch.cat([got["planes"][0][g].double(), k[:, g].to(_dtype(case)).double()])
        values = torch.cat([got["planes"][1][g].double(), v[:, g]])
        for a in range(0, n, some):
            b = min(n, a + some)
            s = score(q[a:b, g * group:(g + 1) * group], keys)
            if case["slopes"]:
                s = s - got["slopes"][g * group:(g + 1) * group].double()[:, None] * (torch.arange(p + a, p + b, device="cuda")[:, None, None] - key).abs()
            seen = (key >= first[a:b, None]) & (key < end[a:b, None])
            s = torch.where(seen[:, None], s, -math.inf)
            out[a:b, g * group:(g + 1) * group] = torch.nan_to_num(torch.softmax(s, -1)) @ values
    return {"out": out, "k": k.transpose(0, 1), "v": v.transpose(0, 1)}
