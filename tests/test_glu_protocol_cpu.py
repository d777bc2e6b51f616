"""The barriers of the gated sub-layer's kernels, modelled on the CPU: every role of glu_fwd_kernel, glu_dx_kernel and
glu_dw_kernel (csrc/dg4_glu.cu) as a sequence of waits and arrivals, run in random orders over all small numbers of tiles and
blocks.  No order may stop, and no wait may pass on another phase than the one it means: a wait goes by the phase's parity
alone, so one that comes two phases late or early would be let through (or held) wrongly."""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0            # `done`: completed phases

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.done = self.count, self.done + 1


class Model:
    """Roles are generators that yield ("wait", barrier, phase) and ("go",); what they start (copies, products) ends later:
    copies in any order, products in the order of their issue."""
    def __init__(self, rng):
        self.rng, self.roles, self.copies, self.products = rng, [], [], []

    def copy(self, bar):
        self.copies.append(bar)

    def commit(self, *bars):
        self.products.append(bars)

    def run(self):
        live, steps = [[r, None] for r in self.roles], 0
        while live or self.copies or self.products:
            moves, steps = [], steps + 1
            assert steps < 100000, "goes round in circles"
            for role in live:
                want = role[1]
                if want is None or want[0].done % 2 != want[1] % 2:   # the phase's parity has passed
                    moves.append(role)
            moves += ["copy"] if self.copies else []
            moves += ["product"] if self.products else []
            assert moves, "stopped: " + str([(r[0].__name__, r[1][1], r[1][0].done) for r in live])
            move = self.rng.choice(moves)
            if move == "copy":
                self.copies.pop(self.rng.randrange(len(self.copies))).arrive()
            elif move == "product":
                for bar in self.products.pop(0):
                    bar.arrive()
            else:
                if move[1] is not None:
                    bar, phase = move[1]
                    assert bar.done == phase + 1, (move[0].__name__, phase, bar.done)
                try:
                    step = next(move[0])
                    move[1] = None if step[0] == "go" else (step[1], step[2])
                    if step[0] == "wait" and step[2] < 0:               # the wait for a place never used passes at once
                        move[1] = None
                except StopIteration:
                    live.remove(move)


def wait(bar, phase):
    return ("wait", bar, phase)


def bars(n, count):
    return [Barrier(count) for _ in range(n)]


WARPS = 2                                                              # of a set, in the model (eight in the kernel)


def pair_kernel(rng, tiles, nb, res, split, dx):
    """glu_fwd_kernel (dx False) or glu_dx_kernel: two CTAs, rank 0 issues."""
    m = Model(rng)
    stages, bufs, total = (4, 2, tiles * nb) if dx else (5, 3, tiles * nb)
    ready, a_ready, y_empty = bars(stages, 2), bars(bufs, 2 * WARPS), Barrier(2 * WARPS)
    gu_read, dy_ready = bars(bufs, 2 * WARPS), Barrier(2)
    ctas = []
    for _ in range(2):
        x_places = 1 if dx else 2
        ctas.append(dict(x_full=bars(x_places, 1), x_empty=bars(x_places, 1), r_full=bars(2, 1), r_empty=bars(2, WARPS), w_full=bars(stages, 1),
                         w_empty=bars(stages, 1), acc_full=bars(bufs, 1), y_full=bars(2, 1), dy_full=Barrier(1), dy_empty=Barrier(1)))
    both = lambda name, i=None: [c[name] if i is None else c[name][i] for c in ctas]  # noqa: E731

    def weights(c):
        for k in range(total):
            yield wait(c["w_empty"][k % stages], k // stages - 1)
            m.copy(c["w_full"][k % stages])

    def tells(c):
        for k in range(total):
            t, b = divmod(k, nb)
            if b == 0:
                yield wait(c["x_full"][t % len(c["x_full"])], t // len(c["x_full"]))
            yield wait(c["w_full"][k % stages], k // stages)
            ready[k % stages].arrive()
            if dx and b == 0:
                yield wait(c["dy_full"], t)
                dy_ready.arrive()

    def rows(c):
        if dx:
            for t in range(tiles):
                yield wait(c["x_empty"][0], t - 1)
                m.copy(c["x_full"][0])
                yield wait(c["dy_empty"], t - 1)
                m.copy(c["dy_full"])
            return
        for t in range(tiles + 1):
            if t < tiles:
                yield wait(c["x_empty"][t % 2], t // 2 - 1)
                m.copy(c["x_full"][t % 2])
            if t >= 1 and res:
                yield wait(c["r_empty"][t % 2], t // 2 - 1)
                m.copy(c["r_full"][(t - 1) % 2])

    def lead():
        for c in range(total + 2):
            t1, b1 = divmod(c, nb)
            if dx:
                if c < total:
                    yield wait(ready[c % stages], c // stages)
                    yield wait(gu_read[c % bufs], c // bufs - 1)
                    m.commit(*(both("x_empty", 0) if b1 + 1 == nb else []))
                if c >= 2:
                    yield from second(c - 2)
                if c < total:
                    if b1 == 0:
                        yield wait(dy_ready, t1)
                    m.commit(*both("acc_full", c % bufs), *(both("dy_empty") if b1 + 1 == nb else []))
            else:
                early = c >= 2 and (c - 2) % nb != 0 and rng.random() < 0.5      # where its activations have come already
                if early:
                    yield from second(c - 2)
                if c < total:
                    yield wait(ready[c % stages], c // stages)
                    m.commit(*both("acc_full", c % bufs), *(both("x_empty", t1 % 2) if b1 + 1 == nb else []))
                if c >= 2 and not early:
                    yield from second(c - 2)

    def second(k):
        t, b = divmod(k, nb)
        yield wait(a_ready[k % bufs], k // bufs)
        if b == 0:
            yield wait(y_empty, t - 1)
        m.commit(*both("w_empty", k % stages), *(both("y_full", t % 2) if b + 1 == nb else []))

    def epilogue(c, set_):
        turn, owed = set_, []

        def leave():
            if owed:
                c["r_empty"][owed.pop() % 2].arrive()

        def finish(t):
            yield wait(c["y_full"][t % 2], t // 2)
            y_empty.arrive()
            if not dx:
                yield wait(c["r_full"][t % 2], t // 2) if res else wait(c["r_empty"][(t - 1) % 2], (t - 1) // 2 if t else -1)
        for t in range(tiles):
            leave()
            is_open = t > 0 and turn == 0
            for b in range(nb):
                k = t * nb + b
                if turn == 0:
                    yield wait(c["acc_full"][k % bufs], k // bufs)
                    if dx:
                        gu_read[k % bufs].arrive()
                        yield ("go",)
                    a_ready[k % bufs].arrive()
                    leave()
                    if is_open:
                        is_open = False
                        yield from finish(t - 1)
                        if not dx:
                            owed.append(t - 1)
                turn ^= 1
        leave()
        if turn == 0 and not split:
            yield from finish(tiles - 1)
    for c in ctas:
        m.roles += [weights(c), tells(c), rows(c)] + [epilogue(c, s) for s in (0, 1) for _ in range(WARPS)]
    m.roles.append(lead())
    m.run()


def weights_kernel(rng, tiles):
    """glu_dw_kernel."""
    m = Model(rng)
    x_full, x_empty, dy_full, dy_empty = bars(2, 1), bars(2, 1), bars(2, 1), bars(2, 1)
    w_full, acc_full, acc_empty, a_full, a_empty, w_done = (Barrier(n) for n in (1, 1, WARPS, WARPS, 1, 1))

    def load(full, empty, first):
        if first:
            m.copy(w_full)
        for t in range(tiles):
            yield wait(empty[t % 2], t // 2 - 1)
            m.copy(full[t % 2])

    def lead():
        yield wait(w_full, 0)
        t1 = t2 = 0
        half = False
        while t2 < tiles:
            if t2 < t1 and a_full.done > t2:
                m.commit(x_empty[t2 % 2])
                m.commit(dy_empty[t2 % 2], a_empty)
                t2 += 1
            elif not half and t1 < tiles and x_full[t1 % 2].done > t1 // 2 and acc_empty.done >= t1:
                half = True
            elif half and dy_full[t1 % 2].done > t1 // 2:
                m.commit(acc_full)
                half, t1 = False, t1 + 1
            else:
                yield ("go",)
                continue
            yield ("go",)
        m.commit(w_done)

    def epilogue():
        for t in range(tiles):
            yield wait(acc_full, t)
            acc_empty.arrive()
            yield wait(a_empty, t - 1)
            a_full.arrive()
        yield wait(w_done, 0)
    m.roles = [load(x_full, x_empty, True), load(dy_full, dy_empty, False), lead()] + [epilogue() for _ in range(WARPS)]
    m.run()


@pytest.mark.parametrize("dx", [False, True])
@pytest.mark.parametrize("nb", [1, 2, 3, 4, 5, 8])
def test_pairs_of_ctas_never_stop_and_never_take_one_phase_for_another(nb, dx):
    for tiles in (1, 2, 3, 4, 5, 7):
        for res in ((False,) if dx else (False, True)):
            for seed in range(12):
                pair_kernel(random.Random(seed * 1000 + tiles), tiles, nb, res, False, dx)
    for seed in range(6):
        pair_kernel(random.Random(seed), 1, nb, False, True, dx)      # few rows: one tile, joined behind the roles


def test_the_weights_kernel_never_stops_and_never_takes_one_phase_for_another():
    for tiles in (1, 2, 3, 4, 5, 9):
        for seed in range(30):
            weights_kernel(random.Random(seed), tiles)
