"""Scored steps, attention weight and eviction: what needs no GPU - layouts, refusals ahead of any CUDA call, the rules of the
kernels' barriers that show in their text, the polynomials."""
import ctypes
import os
import re

import pytest

from paper_2605_12471_b200 import build as kbuild

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_12471_b200", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


@pytest.fixture(scope="module")
def binding():
    kbuild.build_library()
    from paper_2605_12471_b200 import binding as b
    b.load()
    return b


def test_scores_layout(binding):
    c = binding.kvf_scores
    assert ctypes.sizeof(c) == 32
    assert (c.softcap.offset, c.slopes.offset, c.first.offset, c.end.offset) == (0, 8, 16, 24)


def test_null_handles_are_refused(binding):
    lib = binding.load()
    sc = binding.kvf_scores(1.0, None, None, None)
    bad = binding.KVF_ERR_INVALID_ARG
    p = 4096
    assert lib.kvf_fold_step_scored(None, p, p, p, 1, 0, ctypes.byref(sc), p, None, None) == bad
    assert lib.kvf_attend_scored(None, p, 1, 0, ctypes.byref(sc), p, None, None) == bad
    assert lib.kvf_batch_fold_step_scored(None, p, p, p, None, 1, None, ctypes.byref(sc), p, None, None) == bad
    assert lib.kvf_rotate_queries(None, p, 1, 0, p, None) == bad
    assert lib.kvf_cache_mass(None, p, 1, 1, 0, None, p, None, 0, 1.0, p, 16, None) == bad
    assert lib.kvf_cache_evict(None, None, p, 16, 0, 0, 1, None, 0, p, None) == bad


def test_keywords_that_ask_for_nothing_make_a_plain_step(binding):
    assert binding._scores(0.0, None, None, None, 32, 4, None) is None
    assert binding._scores(0, None, None, None, 32, 4, None) is None


def test_wrong_tensors_are_refused_by_the_binding(binding):
    import torch
    cpu = torch.device("cpu")
    with pytest.raises(AssertionError):
        binding._scores(0.0, torch.zeros(31), None, None, 32, 4, cpu)
    with pytest.raises(AssertionError):
        binding._scores(0.0, torch.zeros(32, dtype=torch.float64), None, None, 32, 4, cpu)
    with pytest.raises(AssertionError):
        binding._scores(0.0, None, torch.zeros(4, dtype=torch.int64), None, 32, 4, cpu)
    with pytest.raises(AssertionError):
        binding._scores(0.0, None, None, torch.zeros(8, dtype=torch.int32)[::2], 32, 4, cpu)


# The cap's polynomials, in fp32 as the kernels evaluate them: least relative error over their ranges as the comment says.
def test_polynomials_of_the_cap_and_of_two_to_the_x():
    import numpy as np
    text = source("scores.cuh")

    def coefficients(name):
        return [np.float32(x) for x in re.search(name + r"\[\d\] = \{([^}]*)\}", text).group(1).split(",")]

    for name, top, err in (("kSmallTanh", 0.5, 5.5e-7), ("kMiddleTanh", 0.75, 5.7e-7)):
        x = np.linspace(-top, top, 200001).astype(np.float32)
        x = x[x != 0]
        u = (x * x).astype(np.float32)
        y = np.zeros_like(x)
        for c in coefficients(name)[::-1]:
            y = (y * u + c).astype(np.float32)
        off = np.abs(x.astype(np.float64) * y / np.tanh(x.astype(np.float64)) - 1).max()
        # six roundings of half a step each on top of the polynomial's own error
        assert off <= err + 6 * 2.0 ** -24, (name, off)
    mass = source("attn_mass.cu")
    body = mass[mass.index("float2 exp2_fma"):mass.index("// What the roles have to agree on.")]
    c = [float(v) for v in re.findall(r"both\((\d\.\d{9,})f\)", body)]
    assert len(c) == 5
    f = np.linspace(-0.5, 0.5, 100001).astype(np.float32)
    y = np.full_like(f, np.float32(c[0]))
    for v in c[1:] + [1.0]:
        y = (y.astype(np.float64) * f + np.float64(np.float32(v))).astype(np.float32)
    assert np.abs(y / 2.0 ** f.astype(np.float64) - 1).max() <= 2.0 ** -22


# As for the other kernels: an issuing warp's waits end in a vote, and .aligned instructions stand behind a reconvergence.
def test_waits_of_the_issuing_warp_end_in_a_vote():
    text = source("attn_mass.cu")
    start = text.index("leader = elect_one()")
    lines = text[start:text.index("columns of the jobs, up to eight jobs ahead", start)].splitlines()
    waits = [line for line in lines if re.search(r"\bmbar_wait\w*\(", line) and "mbar_wait_drain(" not in line]
    assert waits and all(re.search(r"\bmbar_wait4?_warp\(", line) for line in waits)


@pytest.mark.parametrize("name", ["attn_mass.cu", "evict.cu"])
def test_aligned_instructions_stand_behind_a_reconvergence(name):
    apart = None
    for number, line in enumerate(source(name).splitlines(), 1):
        code = line.split("//")[0]
        if "// -----" in line or "tcgen05.alloc" in code or code.startswith(("__global__", "}")) or code.strip() == "continue;":
            apart = None
        if re.search(r"KVF_TMEM_(LD|ST)\d+\(|\.aligned;|cluster_sync_all\(\)|cluster_wait\(\)|cluster_arrive", code) and "auto meet" not in code:
            assert apart is None or "cluster_sync_all();" in code, f"{name}:{number}: behind the branch in line {apart}"
        if re.search(r"\b(if|for) \(.*\b(lane == 0|tid == 0|threadIdx\.x == 0|key >= L\)|i = tid;)", code):
            apart = number
        if re.search(r"__syncwarp|__syncthreads|_sync\(0xffffffffu|mbar_wait4?_warp\(", code):
            apart = None


def test_barriers_of_the_mass_kernel_keep_their_waiters_within_a_phase():
    """Producer, issuer, columns, exponentials as programs of waits and arrivals, every interleaving of a few jobs explored."""
    from tests.test_barrier_rules_cpu import _explore
    jobs, sets = 6, 2
    issuer, exps = [], []
    for j in range(jobs):
        s = j % sets
        if j >= sets:
            issuer.append(("wait", "empty%d" % s, j // sets - 1))
        issuer.append(("arrive", "full%d" % s, 1))
    for t in range(2):                           # the pairs of groups that take the jobs in turn
        mine = []
        for j in range(t, jobs, 2):
            mine += [("wait", "cols%d" % (j % 4), j // 4), ("wait", "full%d" % (j % sets), j // sets), ("arrive", "empty%d" % (j % sets), 1),
                     ("arrive", "free%d" % (j % 4), 1)]
        exps.append(mine)
    columns = []
    for t in range(2):                           # (four column slots here, eight in the kernel)
        mine = []
        for j in range(t, jobs, 2):
            if j >= 4:
                mine.append(("wait", "free%d" % (j % 4), j // 4 - 1))
            mine.append(("arrive", "cols%d" % (j % 4), 1))
        columns.append(mine)
    _explore([issuer] + exps + columns, {"full": 1, "empty": 1, "cols": 1, "free": 1})
