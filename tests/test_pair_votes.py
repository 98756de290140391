"""The chunk form's two warps that share rows vote through a named barrier.
PTX leaves undefined what a barrier.red does beside barrier.sync or
barrier.arrive on the same barrier, and a vote has no limit of its own, so both
warps have to come to the same votes however their bounded waits end."""
import itertools
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_23805_gb300", "csrc")


def test_reductions_are_not_mixed_with_other_barriers():
    for f in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, f)) as fh:
            text = re.sub(r"//[^\n]*", "", fh.read())
        if re.search(r"barrier\.cta\.red|\bbar\.red", text):
            assert not re.search(r"barrier\.cta\.(arrive|sync)|\bbar\.(arrive|sync)", text), f


def softmax_role():
    """One D = 256 softmax warp of kv_chunk_kernel over two parts of two tiles:
    its bounded waits and its votes, in order."""
    ops = []
    for part in range(2):
        ops.append("vote")                       # query maxima
        if part:
            ops += ["wait olast", "vote"]        # sums of the part before
        for tile in range(2):
            ops += ["wait sfull"]
            if tile == 0:                        # the reference is found first
                ops += ["vote"]
            else:                                # a pass that asks for another one
                ops += ["vote", "vote", "wait ofull"]
            ops += ["vote"]
    return ops + ["wait olast", "vote"]


def run(ops, fails):
    """Warps as generators of votes; warp w's wait number fails[w] runs out.
    Returns the votes that each took part in; None: one of them waits forever."""
    def warp(w):
        waits = 0
        for op in ops:
            if op == "vote":
                leave = yield False
                if leave:
                    return
            else:
                waits += 1
                if waits - 1 == fails[w]:
                    yield True
                    return
    live = [warp(0), warp(1)]
    said = [next(x, None) for x in live]
    votes = 0
    while said != [None, None]:
        if None in said:
            return None  # alone at the barrier
        votes += 1
        leave = any(said)
        for w in range(2):
            try:
                said[w] = live[w].send(leave)
            except StopIteration:
                said[w] = None
    return votes


def test_both_warps_meet_every_vote():
    ops = softmax_role()
    waits = sum(op != "vote" for op in ops)
    whole = run(ops, (-1, -1))
    assert whole == ops.count("vote")
    for fails in itertools.product(range(-1, waits), repeat=2):
        assert run(ops, fails) is not None, fails


def test_every_wait_is_followed_by_a_vote():
    """What the rule rests on: a warp that stops at a wait has a vote left."""
    ops = softmax_role()
    for i, op in enumerate(ops):
        if op != "vote":
            assert "vote" in ops[i + 1:]
