"""The barrier protocol of the projections with adapters, every interleaving of it, without a GPU.

The kernel's warps meet on mbarriers, whose wait names the parity of a phase: a thread that looks again only after the
barrier has gone two phases on takes the phase it waits for as not yet over, and waits for good.  So no barrier may
be able to run two phases ahead of a thread that still has to see the first.  The model below holds the waits,
arrivals and commits of each role in the order the kernel has them (the tensor core's commits arrive later, in order);
the search visits every state that some order of execution reaches and returns those from which nothing can move though
a role is not done.
"""
import itertools
import os
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                      "paper_2502_01681_b200", "csrc", "dg4_adapters.cu")
RING = 4                                        # item descriptors in flight


def u_barriers():
    """How many barriers the kernel announces U's product on, in turn (an array's length; a plain member is one)."""
    text = open(SOURCE).read()
    m = re.search(r"uint64_t u_full\[(\w+)\]", text)
    if not m:
        return 1
    return int(m.group(1)) if m.group(1).isdigit() else int(re.search(r"constexpr int %s = (\d+);" % m.group(1), text).group(1))


def ring_length():
    return int(re.search(r"constexpr int kRing = (\d+);", open(SOURCE).read()).group(1))


class Protocol:
    """Programs of the roles for a list of items (the adapter of each, -1: none).  An instruction is a tuple:
    ("wait", barrier, k): until k phases are over, as far as the parity of the present one tells; ("arrive", barrier);
    ("commit", barrier); ("look", ((barrier, k), ...), item): remember whether the item's second product is owed and one
    of these waits would not pass; ("owe", item); ("paid",); and ("if", item, flag, instruction): only if that item is
    owed (and, with flag, the last look said so)."""

    def __init__(self, adapters, blocks, sets, stages, n_u, u_warps, residual):
        slots = 3 if blocks == 3 else sets
        acc_of = lambda i, j: (j, i) if blocks == 3 else (i % slots, i // slots)            # slot, round  # noqa: E731
        last = [i + 1 == len(adapters) or adapters[i + 1] != a for i, a in enumerate(adapters)]
        order = [i for i, a in enumerate(adapters) if a >= 0]
        nth = {i: k for k, i in enumerate(order)}                                            # adapter items, counted
        fresh, held, load_of, loads = True, -1, {}, 0
        for i, a in enumerate(adapters):                                                     # which load an item waits for
            if a >= 0:
                if fresh:
                    load_of[i] = loads
                    loads += 1
                fresh = last[i]

        producer, mma, epilogue, u = [], [], [], []
        n_loads = 0
        for i, a in enumerate(adapters):
            q, s, turn = i % RING, i % stages, i // stages
            if i >= RING:
                producer.append(("wait", ("item_empty", q), i // RING))
            producer.append(("arrive", ("item_full", q)))
            if i >= stages:
                producer.append(("wait", ("a_empty", s), turn))
            producer.append(("arrive", ("a_full", s)))
            if a >= 0 and a != held:
                if n_loads:
                    producer.append(("wait", ("la_empty", 0), n_loads))
                producer.append(("arrive", ("la_full", 0)))
                if n_loads:
                    producer.append(("wait", ("lb_empty", 0), n_loads))
                producer.append(("arrive", ("lb_full", 0)))
                n_loads += 1
                held = a
            if last[i]:
                held = -1
            if residual:
                if i >= stages:
                    producer.append(("wait", ("r_empty", s), turn))
                producer.append(("arrive", ("r_full", s)))
        assert n_loads == loads

        def u_wait(i):
            out = [("wait", ("u_ready", 0), nth[i] + 1)]
            if i in load_of:
                out.append(("wait", ("lb_full", 0), load_of[i] + 1))
            return out

        def u_done(i):
            return [("commit", ("ub_empty", 0))] + ([("commit", ("lb_empty", 0))] if last[i] else [])

        def settle(i):
            return u_wait(i) + [("commit", ("acc_full", acc_of(i, 0)[0]))] + u_done(i) + [("paid",)]

        before = None                                                                        # the last adapter item
        for i, a in enumerate(adapters):
            q, s, turn = i % RING, i % stages, i // stages
            slot, round_ = acc_of(i, 0)
            mma += [("wait", ("item_full", q), i // RING + 1), ("arrive", ("item_empty", q))]
            if blocks == 1 and before is not None:
                tests = [(("a_full", s), turn + 1), (("acc_empty", slot), round_)]
                if i in load_of:
                    tests.append((("la_full", 0), load_of[i] + 1))
                mma.append(("look", tuple(tests), before))
                mma += [("if", before, True, x) for x in settle(before)]
            mma.append(("wait", ("a_full", s), turn + 1))
            if i in load_of:
                mma.append(("wait", ("la_full", 0), load_of[i] + 1))
            mma.append(("wait", ("acc_empty", slot), round_))
            if a >= 0:
                mma.append(("commit", ("u_full", nth[i] % n_u)))
                if last[i]:
                    mma.append(("commit", ("la_empty", 0)))
            if blocks == 1:
                mma.append(("commit", ("a_empty", s)))
                if before is not None:
                    mma += [("if", before, False, x) for x in settle(before)]
                mma.append(("owe", i) if a >= 0 else ("commit", ("acc_full", slot)))
            else:
                if a >= 0:
                    mma += u_wait(i)
                mma.append(("commit", ("acc_full", 0)))
                mma += [("wait", ("acc_empty", j), i) for j in (1, 2)]
                mma.append(("commit", ("a_empty", s)))
                if a >= 0:
                    mma += u_done(i)
                mma += [("commit", ("acc_full", j)) for j in (1, 2)]
            if a >= 0:
                before = i
        if blocks == 1 and before is not None:
            mma += [("if", before, False, x) for x in settle(before)]

        for i, a in enumerate(adapters):
            q, s, turn = i % RING, i % stages, i // stages
            epilogue += [("wait", ("item_full", q), i // RING + 1), ("arrive", ("item_empty", q))]
            for j in range(blocks):
                slot, round_ = acc_of(i, j)
                epilogue.append(("wait", ("acc_full", slot), round_ + 1))
                if residual:
                    epilogue.append(("wait", ("r_full", s), turn + 1))
                epilogue.append(("arrive", ("acc_empty", slot)))
                if residual:
                    epilogue.append(("arrive", ("r_empty", s)))
            u += [("wait", ("item_full", q), i // RING + 1), ("arrive", ("item_empty", q))]
            if a >= 0:
                k = nth[i]
                u += [("wait", ("u_full", k % n_u), k // n_u + 1), ("wait", ("ub_empty", 0), k), ("arrive", ("u_ready", 0))]

        self.programs = [producer, mma, epilogue] + [list(u) for _ in range(u_warps)]
        arrivals = {"item_empty": 2 + u_warps, "u_ready": u_warps}
        names = {op[1] for p in self.programs for op in self.flat(p) if op[0] in ("wait", "arrive", "commit")}
        self.bars = {b: k for k, b in enumerate(sorted(names))}
        self.need = [arrivals.get(b[0], 1) for b in sorted(names)]

    @staticmethod
    def flat(program):
        return [op[3] if op[0] == "if" else op for op in program]

    def search(self, most=2_000_000):
        """States in which nothing moves and a role is not done, and waits that pass before their phase is over."""
        bars, need, programs = self.bars, self.need, self.programs
        passes = lambda st, b, k: (st[bars[b]][0] & 1) != (k - 1 & 1)          # what a wait by parity sees  # noqa: E731

        def arrive(st, b):
            k = bars[b]
            phase, got = st[k]
            phase, got = (phase + 1, 0) if got + 1 == need[k] else (phase, got + 1)
            return st[:k] + ((phase, got),) + st[k + 1:]

        start = (tuple([0] * len(programs)), tuple([(0, 0)] * len(need)), (), -1, False)
        seen, todo, stuck = {start}, [start], []
        while todo:
            pcs, st, pipe, owed, now = todo.pop()
            moves = []
            if pipe:                                                           # the tensor core's next commit arrives
                moves.append((pcs, arrive(st, pipe[0]), pipe[1:], owed, now))
            for r, pc in enumerate(pcs):
                if pc == len(programs[r]):
                    continue
                op, st2, pipe2, owed2, now2 = programs[r][pc], st, pipe, owed, now
                if op[0] == "if":
                    op = op[3] if owed == op[1] and (now or not op[2]) else ("skip",)
                if op[0] == "wait":
                    if not passes(st, op[1], op[2]):
                        continue
                    if st[bars[op[1]]][0] < op[2]:
                        stuck.append((op, st[bars[op[1]]]))
                if op[0] == "arrive":
                    st2 = arrive(st, op[1])
                elif op[0] == "commit":
                    pipe2 = pipe + (op[1],)
                elif op[0] == "look":
                    now2 = owed == op[2] and not all(passes(st, b, k) for b, k in op[1])
                elif op[0] == "owe":
                    owed2 = op[1]
                elif op[0] == "paid":
                    owed2, now2 = -1, False
                moves.append((pcs[:r] + (pc + 1,) + pcs[r + 1:], st2, pipe2, owed2, now2))
            if not moves and any(pc < len(p) for pc, p in zip(pcs, programs)):
                stuck.append(pcs)
            for m in moves:
                if m not in seen:
                    seen.add(m)
                    todo.append(m)
            assert len(seen) < most, "the search has become too large"
        return stuck


SAME, EACH, MIXED = [0] * 5, [0, 1, 2, 3, 4], [0, -1, 0, 1, -1, 2]


def stuck_states(items, blocks=1, sets=2, stages=2, n_u=2, u_warps=1, residual=False):
    return Protocol(items, blocks, sets, stages, n_u, u_warps, residual).search()


def test_the_ring_is_the_kernels():
    assert ring_length() == RING


@pytest.mark.parametrize("sets", [2, 3])
def test_one_barrier_for_u_can_be_passed_twice(sets):
    """The search finds what a single barrier does: the next item's product is committed before this item's U is waited
    for, so a U warp that is late for this item's phase finds the barrier two phases on."""
    assert stuck_states(SAME, sets=sets, n_u=1)


@pytest.mark.parametrize("items", [SAME, EACH, MIXED], ids=["same", "each", "mixed"])
@pytest.mark.parametrize("sets,stages", [(1, 1), (2, 1), (2, 2), (3, 2)])
def test_one_block_form_has_no_stuck_state(items, sets, stages):
    assert not stuck_states(items, sets=sets, stages=stages, n_u=u_barriers())


def test_one_block_form_with_residual_and_two_u_warps():
    assert not stuck_states([0, 0, 1, -1], sets=2, stages=1, n_u=u_barriers(), residual=True)
    assert not stuck_states([0, 0, 0, 1], sets=2, stages=2, n_u=u_barriers(), u_warps=2)


@pytest.mark.parametrize("items", [SAME, EACH, MIXED], ids=["same", "each", "mixed"])
def test_three_block_form_has_no_stuck_state(items):
    for stages, n_u in itertools.product((1, 2), {1, u_barriers()}):
        assert not stuck_states(items[:4], blocks=3, stages=stages, n_u=n_u)
