"""The README's loop over a bounded cache, run as it stands there."""
import os
import re
import types

import pytest
import torch

from paper_2605_12471_b200 import binding
from tests import scored
from tests.test_scored_gpu import BASE

pytestmark = pytest.mark.gpu


def test_the_loop_over_a_bounded_cache_goes_on_at_the_right_positions(monkeypatch):
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    loop, = [b for b in blocks if ".evict(" in b]
    assert loop.count("8192") == 1 and loop.count("n_recent=256") == 1
    loop = loop.replace("8192", "600")                       # (a smaller budget; chunks of 200)
    gen = torch.Generator(device="cuda").manual_seed(1)
    chunks = [types.SimpleNamespace(**{name: torch.randn((200, heads, 128), generator=gen, device="cuda").bfloat16()
                                       for name, heads in (("q", 32), ("k", 8), ("v", 8))}) for _ in range(7)]
    rotations, folds, weights = [], [], []
    fold, rotate, weigh = binding.Cache.fold_step, binding.Cache.rotate, binding.Cache.mass

    def folded(self, q, k, v, **kw):
        before = len(self)
        out = fold(self, q, k, v, **kw)
        folds.append((q, k, self.k_plane()[:, before:before + 200].clone()))
        return out

    def rotated(self, q, **kw):
        rotations.append((q, rotate(self, q, **kw)))
        return rotations[-1][1]

    def weighed(self, *args, **kw):
        got = weigh(self, *args, **kw)
        weights.append(got[:, len(self) - 200:len(self)].clone())
        return got

    monkeypatch.setattr(binding.Cache, "fold_step", folded)
    monkeypatch.setattr(binding.Cache, "rotate", rotated)
    monkeypatch.setattr(binding.Cache, "mass", weighed)
    exec(loop, dict(torch=torch, binding=binding, chunks=chunks))
    assert len(folds) == len(rotations) == len(weights) == 7
    for step, ((q, k, rows), (asked, turned)) in enumerate(zip(folds, rotations)):
        want = scored.turned(k, 200 * step, BASE).transpose(0, 1)
        assert float((rows.double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 2.0 ** -18
        want = scored.turned(q, 200 * step, BASE)
        assert asked is q and float((turned.double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 2.0 ** -18
    assert all(bool((w >= 0).all()) and bool(torch.isfinite(w).all()) for w in weights)
