"""The waits between the warps of the dense attention's tensor-core kernels, on the CPU: a model of their mbarriers run
under random schedules, and what the sources must hold for the model to be theirs.

An mbarrier counts the phases it has completed; a wait for use u of it passes while that number's parity differs from
u's.  A run is stuck if no actor can go on and not all are done.
"""
import os
import random
import re

import pytest

from conftest import ROOT

CSRC = os.path.join(ROOT, "paper_2609_06712_gb300", "csrc")
KERNELS = ["attention_tc.cu", "attention_dq_tc.cu", "attention_dkdv_tc.cu"]


class Bar:
    def __init__(self, count=1):
        self.count, self.left, self.phases = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.phases = self.count, self.phases + 1

    def passed(self, use):
        return (self.phases & 1) != (use & 1)


def run(actors, rng):
    """Actors yield conditions.  Runs them in a random order with random pauses; True if all came to their end."""
    waiting = [(a, next(a, None)) for a in actors]
    waiting = [(a, c) for a, c in waiting if c is not None]
    weight = [rng.choice([1, 1, 4, 30]) for _ in actors]         # some actors far slower than others
    while waiting:
        ready = [i for i, (_, c) in enumerate(waiting) if c()]
        if not ready:
            return False
        i = rng.choices(ready, [1 / weight[j % len(weight)] for j in ready])[0]
        a, _ = waiting[i]
        c = next(a, None)
        if c is None:
            waiting.pop(i)
        else:
            waiting[i] = (a, c)
    return True


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//.*", "", f.read())


# ---------------------------------------------------------------- a wait that gives up

def leaves(barrier, rng):
    """Four warps through stages of (meet the others, wait for a product), while waits give up from some moment on:
    a wait whose phase is complete passes all the same.  barrier: they meet at a barrier of the CTA, which has no
    limit; else at an mbarrier whose wait is one like the others."""
    stages = 4
    meet, product, abort, arrived = Bar(4), [Bar() for _ in range(stages)], [], [0]

    def issuer():
        for k in range(stages):
            if k == 2:
                abort.append(1)              # what comes now is late: some waits have given up, some see it complete
            yield lambda: True
            product[k].arrive()

    def warp():
        for k in range(stages):
            if barrier:
                arrived[0] += 1
                yield lambda k=k: arrived[0] >= 4 * (k + 1)
            else:
                meet.arrive()
                yield lambda k=k: meet.passed(k) or abort
                if not meet.passed(k):
                    return
            yield lambda k=k: product[k].passed(0) or abort
            if not product[k].passed(0):
                return
    return run([issuer()] + [warp() for _ in range(4)], rng)


def test_a_warp_that_gives_up_leaves_no_other_behind():
    assert all(leaves(False, random.Random(i)) for i in range(400))
    assert not all(leaves(True, random.Random(i)) for i in range(400)), "the model does not show the fault"


@pytest.mark.parametrize("name", KERNELS)
def test_warps_meet_at_mbarriers_only(name):
    text = source(name)
    assert not re.findall(r"\b(bar_sync|bar_red_or|__syncthreads_\w+)\s*\(", text)
    # before the roles part and after they have ended
    assert text.count("__syncthreads()") == 2


# ---------------------------------------------------------------- the dq kernel's products and element-wise work

def dq_pipeline(pair, rng, stages=12):
    """The dq kernel's loop over stages, its tiles loaded: S and dP by one actor, dQ by another, two warps between
    them.  pair: dS is announced on a barrier for each of the two S buffers; else on one for all stages."""
    S, dP, read, done = [Bar(), Bar()], Bar(), Bar(2), [Bar(), Bar()]
    ds = [Bar(2), Bar(2)] if pair else [Bar(2)]
    holds = [None, None]                             # the stage whose S, then dS, is in each buffer

    def ds_of(n):
        return (ds[n & 1], n >> 1) if pair else (ds[0], n)

    def s_thread():
        for n in range(stages):
            if n >= 2:
                yield lambda n=n: done[n & 1].passed((n >> 1) - 1)
            assert holds[n & 1] is None, "S over a buffer that dQ has not read"
            holds[n & 1] = n
            S[n & 1].arrive()
            yield lambda: True
            if n >= 1:
                yield lambda n=n: read.passed(n - 1)
            dP.arrive()
            yield lambda: True

    def warp():
        for n in range(stages):
            yield lambda n=n: S[n & 1].passed(n >> 1)
            assert holds[n & 1] == n
            yield lambda n=n: dP.passed(n)
            read.arrive()
            yield lambda: True
            ds_of(n)[0].arrive()
            yield lambda: True

    def dq_thread():
        for n in range(stages):
            b, use = ds_of(n)
            yield lambda b=b, use=use: b.passed(use)
            assert holds[n & 1] == n
            holds[n & 1] = None
            done[n & 1].arrive()
            yield lambda: True                       # the next item's sizes, a commit: any time
    return run([s_thread(), warp(), warp(), dq_thread()], rng)


def test_dq_stages_follow_one_another_whatever_the_pace():
    assert all(dq_pipeline(True, random.Random(i)) for i in range(600))
    assert not all(dq_pipeline(False, random.Random(i)) for i in range(600)), "the model does not show the fault"


def test_dq_announces_ds_per_buffer():
    text = source("attention_dq_tc.cu")
    assert re.findall(r"wait\(DS_FULL[^;]*;", text) == ["wait(DS_FULL + (n & 1), n >> 1);"]
    assert re.findall(r"arrive\(DS_FULL[^;]*;", text) == ["arrive(DS_FULL + b);"] and "const int b = n & 1;" in text
    assert re.search(r"DS_FULL, DONE = DS_FULL \+ 2", text)


# ---------------------------------------------------------------- lanes of a warp

@pytest.mark.parametrize("name,role", [
    ("attention_tc.cu", "softmax + epilogue"), ("attention_dq_tc.cu", "element-wise work + epilogue"),
    ("attention_dkdv_tc.cu", "element-wise work + epilogue"), ("ffn_tc.cu", "-- epilogue"),
    ("ffn_few.cu", "this CTA's part of the sums")])
def test_warps_that_read_tensor_memory_give_up_as_a_whole(name, role):
    """Reading TMEM takes the whole warp, so its lanes must agree on how a wait ended (mbar_wait_warp votes); the wait
    for a warp's own last copies at its end, by one lane, may be a plain one."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert text.count(role) == 1
    role_text = re.sub(r"//.*", "", text[text.index(role):text.index("fence_before_sync();\n    ", text.index(role))])
    waits = [w for w in re.findall(r"\b(?:mbar_wait\w*|(?:warp_)?wait)\([^;]*;", role_text) if "&never" not in w]
    assert waits and all(w.startswith(("mbar_wait_warp(", "warp_wait(")) for w in waits), waits
    with open(os.path.join(CSRC, "tcgen05.cuh")) as f:
        assert re.search(r"bool mbar_wait_warp[^}]*__all_sync\(0xffffffffu, mbar_wait\(", f.read())


# ---------------------------------------------------------------- the dk / dv kernel's tiles

def dkdv_pipeline(waits_for_dO, rng, stages=10, slots=4):
    """The dk / dv kernel's loop over stages: Q and dO of each in a ring of slots, filled in their own time; S and dP
    by a thread of each of two groups, dV and dK by a third.  True if no product read a slot without its tile."""
    full, empty = [Bar() for _ in range(slots)], [Bar(2) for _ in range(slots)]
    S, dP, P, dS, V, K = ([Bar(), Bar()] for _ in range(6))
    tile, good = [None] * slots, [True]

    def read(use):
        good[0] &= tile[use % slots] == use

    issued = [0]

    def copies():
        for use in range(2 * stages):
            yield lambda: use < slots or empty[use % slots].passed(use // slots - 1)
            tile[use % slots] = None
            issued[0] += 1

    def landings(slot):                              # each whenever it likes
        for use in range(slot, 2 * stages, slots):
            yield lambda: issued[0] > use
            tile[slot] = use
            full[slot].arrive()

    def s_thread(g):
        for n in range(g, stages, 2):
            k = n >> 1
            for use, out, before in ((2 * n, S, V), (2 * n + 1, dP, K)):
                yield lambda: full[use % slots].passed(use // slots)
                yield lambda: k < 1 or before[g].passed(k - 1)
                read(use)
                out[g].arrive()
                empty[use % slots].arrive()

    def warp(g):
        for n in range(g, stages, 2):
            k = n >> 1
            yield lambda: S[g].passed(k)
            P[g].arrive()
            yield lambda: dP[g].passed(k)
            dS[g].arrive()

    def grad_thread():
        for n in range(stages):
            g, k, u0, u1 = n & 1, n >> 1, 2 * n, 2 * n + 1
            yield lambda: P[g].passed(k)
            if waits_for_dO:
                yield lambda: full[u1 % slots].passed(u1 // slots)
            read(u1)
            V[g].arrive()
            empty[u1 % slots].arrive()
            yield lambda: dS[g].passed(k)
            read(u0)
            K[g].arrive()
            empty[u0 % slots].arrive()
    ended = run([copies()] + [landings(i) for i in range(slots)] + [s_thread(0), s_thread(1), warp(0), warp(1), grad_thread()], rng)
    assert ended, "stuck"
    return good[0]


def test_dkdv_products_read_tiles_that_are_there():
    assert all(dkdv_pipeline(True, random.Random(i)) for i in range(300))
    assert not all(dkdv_pipeline(False, random.Random(i)) for i in range(300)), "the model does not show the fault"


def test_dv_waits_for_its_tile():
    text = source("attention_dkdv_tc.cu")
    grad = text[text.index("wait(P_FULL + g, k);"):text.index("gradient(tmem + kTmemV")]
    assert "wait(B_FULL + u1 % kSlots, u1 / kSlots);" in grad
