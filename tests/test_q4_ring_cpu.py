"""A model of the 4-bit product's pipeline, stepped in random orders: loads that arrive in any order, warpgroups that take the stages in
turns and wait by parity, MMAs, sums.  Whoever reads a place of the ring has to find the stage there that it came for.
"""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count = self.left = count
        self.phase = 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.phase, self.left = self.phase + 1, self.count

    def over(self, parity):
        """As the hardware answers: whether the phase of this parity that came last is over."""
        return (self.phase & 1) != parity


def run(stages, NA, ND, groups, n_it, rng):
    """The number of reads that found another stage; -1 if nothing could go on."""
    full, empty = [Barrier(1) for _ in range(stages)], [Barrier(2) for _ in range(stages)]
    a_full, a_empty = [Barrier(1) for _ in range(NA)], [Barrier(1) for _ in range(NA)]
    d_full, d_empty = [Barrier(1) for _ in range(ND)], [Barrier(1) for _ in range(ND)]
    ring, weights, flying, wrong = [None] * stages, [None] * NA, [], [0]

    def see(found, wanted):
        wrong[0] += found != wanted

    def wait(b, use):
        while not b.over(use & 1):
            yield

    def loads():
        for it in range(n_it):
            if it >= stages:
                yield from wait(empty[it % stages], it // stages - 1)
            flying.append(it)
            yield

    def arrivals():
        while True:
            if flying and rng.random() < 0.2:
                it = flying.pop(rng.randrange(len(flying)))
                ring[it % stages] = it
                full[it % stages].arrive()
            yield

    def dequant(g):
        for it in range(g, n_it, groups):
            yield from wait(full[it % stages], it // stages)
            see(ring[it % stages], it)
            held = ring[it % stages]
            empty[it % stages].arrive()
            yield
            if it >= NA:
                yield from wait(d_full[it % NA] if NA == ND else a_empty[it % NA], it // NA - 1)
            weights[it % NA] = held
            a_full[it % NA].arrive()
            yield

    def mmas():
        for it in range(n_it):
            yield from wait(full[it % stages], it // stages)
            if it >= ND:
                yield from wait(d_empty[it % ND], it // ND - 1)
            yield from wait(a_full[it % NA], it // NA)
            see(ring[it % stages], it)
            see(weights[it % NA], it)
            yield
            empty[it % stages].arrive()
            a_empty[it % NA].arrive()
            d_full[it % ND].arrive()
            yield

    def sums():
        for it in range(n_it):
            yield from wait(d_full[it % ND], it // ND)
            d_empty[it % ND].arrive()
            yield

    roles = [loads(), mmas(), sums()] + [dequant(g) for g in range(groups)]
    air, idle = arrivals(), 0
    while roles:
        next(air)
        r = rng.choice(roles)
        for _ in range(rng.choice((1, 1, 4, 30))):           # (a role that runs ahead, others that stand)
            try:
                next(r)
            except StopIteration:
                roles.remove(r)
                break
        idle += 1
        if idle > 400 * n_it:
            return -1
    return wrong[0]


def ring_stages(n, NA, groups):
    """As in csrc/q4.cu."""
    return n // groups * groups if n % groups and n < NA + groups else n


@pytest.mark.parametrize("NA,ND", [(3, 3), (2, 2), (4, 2)])
@pytest.mark.parametrize("stages", range(2, 9))
def test_every_read_finds_its_stage(NA, ND, stages):
    rng = random.Random(100 * NA + 10 * ND + stages)
    for _ in range(60):
        assert run(ring_stages(stages, NA, 2), NA, ND, 2, rng.randrange(1, 60), rng) == 0


def test_the_model_sees_the_mistake():
    """Five places, four of weights, two warpgroups."""
    rng = random.Random(1)
    assert any(run(5, 4, 2, 2, 60, rng) != 0 for _ in range(200))


def test_the_library_has_the_rule():
    import os
    import re
    from paper_2607_08991_gb300 import build
    with open(os.path.join(build.CSRC, "q4.cu")) as f:
        text = f.read()
    assert re.search(r"ring_stages\(int n, int NA\) \{ return n % kDeqGroups != 0 && n < NA \+ kDeqGroups "
                     r"\? n / kDeqGroups \* kDeqGroups : n; \}", text)
    assert "p.stages = ring_stages(p.stages, NA);" in text and "constexpr int kDeqGroups = 2;" in text
    wide = text[text.index("constexpr int kWideStages"):text.index("constexpr int kWideStages") + 40]
    assert "= 4;" in wide                                    # the kernel for many tokens: an even number, always the same


def test_what_the_kernel_before_wrote_is_waited_for_where_it_is_read():
    """The tokens' powers of two, by plain loads of the warps that write results: behind a wait of their own, in both kernels."""
    import os
    from paper_2607_08991_gb300 import build
    with open(os.path.join(build.CSRC, "q4.cu")) as f:
        text = f.read()
    reads = [i for i in range(len(text)) if text.startswith("p.tok_exp[", i)][1:]          # (the first: the kernel that writes them)
    assert len(reads) == 2
    for i in reads:
        role = max(text.rindex("// ---- sums", 0, i), text.rindex("__launch_bounds__", 0, i))
        assert "// ---- sums" in text[role:i] and "grid_dependency_wait();" in text[role:i]
