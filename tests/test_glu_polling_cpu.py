"""What the model of the gated sub-layer's barriers (test_glu_protocol_cpu.py) takes for granted, checked: the sizes of the rings
and the numbers of arrivals as they stand in csrc/dg4_glu.cu, and the weights' kernel's issuing warp, which goes by the parities of
the phases alone: whatever can go first goes first, and a parity seen must be that of the phase it means."""
import os
import random
import re

import pytest

from test_glu_protocol_cpu import Barrier, Model, WARPS, bars, wait

SOURCE = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_01681_b200", "csrc", "dg4_glu.cu")).read()


def part(name):
    """The namespace of a kernel's sizes, and the kernel."""
    sizes = re.search(r"namespace %s \{(.*?)\}  // namespace %s" % (name, name), SOURCE, re.S).group(1)
    kernel = re.search(r"\nglu_%s_kernel\(const(.*?)\n\}\n" % name, SOURCE, re.S).group(1)
    return sizes, kernel


def arrivals(kernel):
    return {name: count for name, count in re.findall(r"mbar_init\(bar\(bars->(\w+)(?:\[\w+\])?\), ([^()]+)\)", kernel)}


def number(name, sizes):
    return int(re.search(r"\b%s = (\d+)" % name, sizes).group(1))


def test_the_model_has_the_rings_and_arrivals_of_the_source():
    sets, both = "kSetWarps", "2 * kSetWarps"
    sizes, kernel = part("fwd")
    assert (number("kStages", sizes), number("kBufs", sizes)) == (5, 3)
    assert re.search(r"x_full\[2\], x_empty\[2\], r_full\[2\], r_empty\[2\]", sizes) and "y_full[2]" in sizes
    assert arrivals(kernel) == dict(x_full="1", x_empty="1", r_full="1", r_empty=sets, w_full="1", w_empty="1", ready="2", acc_full="1",
                                    a_ready=both, y_full="1", y_empty=both, drain="1")
    sizes, kernel = part("dx")
    assert (number("kStages", sizes), number("kBufs", sizes)) == (4, 2)
    assert re.search(r"x_full, x_empty, dy_full, dy_empty,", sizes) and "y_full[2]" in sizes
    assert arrivals(kernel) == dict(x_full="1", x_empty="1", dy_full="1", dy_empty="1", dy_ready="2", w_full="1", w_empty="1", ready="2",
                                    acc_full="1", gu_read=both, a_ready=both, y_full="1", y_empty=both, drain="1")
    sizes, kernel = part("dw")
    assert number("kStages", sizes) == 2
    assert arrivals(kernel) == dict(w_full="1", x_full="1", x_empty="1", dy_full="1", dy_empty="1", acc_full="1", acc_empty="kEpiWarps",
                                    a_full="kEpiWarps", a_empty="1", w_done="1", drain="1")


def polled_weights_kernel(rng, tiles, odd_a=0):
    """glu_dw_kernel with the issuing warp's tests as it makes them.  odd_a: the parity it begins with for the hidden gradients
    (another than 0 is a mistake that has to be seen)."""
    m = Model(rng)
    x_full, x_empty, dy_full, dy_empty = bars(2, 1), bars(2, 1), bars(2, 1), bars(2, 1)
    w_full, acc_full, acc_empty, a_full, a_empty, w_done, drain = (Barrier(n) for n in (1, 1, WARPS, WARPS, 1, 1, 1))
    has_come = lambda bar, parity: bar.done % 2 != parity                              # noqa: E731

    def load(full, empty, first):
        if first:
            m.copy(w_full)
        for t in range(tiles):
            if t >= 2:
                yield wait(empty[t % 2], t // 2 - 1)
            m.copy(full[t % 2])

    def lead():
        yield wait(w_full, 0)
        t1 = t2 = x1_at = x1_odd = x2_at = 0
        acc_odd, a_odd, half = 1, odd_a, False
        while t2 < tiles:
            if t2 < t1 and has_come(a_full, a_odd):
                assert a_full.done == t2 + 1, "hidden gradients of another tile"
                a_odd ^= 1
                m.commit(x_empty[x2_at])
                m.commit(dy_empty[x2_at])
                m.commit(a_empty)
                x2_at ^= 1
                t2 += 1
            elif not half and t1 < tiles and has_come(x_full[x1_at], x1_odd) and has_come(acc_empty, acc_odd):
                assert x_full[x1_at].done == t1 // 2 + 1 and acc_empty.done == t1, "rows of another tile, or values not yet taken"
                acc_odd ^= 1
                half = True
            elif half and has_come(dy_full[x1_at], x1_odd):
                assert dy_full[x1_at].done == t1 // 2 + 1, "rows of another tile"
                m.commit(acc_full)
                half = False
                x1_at, x1_odd = (0, x1_odd ^ 1) if x1_at else (1, x1_odd)
                t1 += 1
            yield ("go",)
        m.commit(w_done)
        m.commit(drain)
        yield wait(drain, 0)

    def epilogue():
        for t in range(tiles):
            yield wait(acc_full, t)
            acc_empty.arrive()
            yield wait(a_empty, t - 1)
            a_full.arrive()
        yield wait(w_done, 0)
    m.roles = [load(x_full, x_empty, True), load(dy_full, dy_empty, False), lead()] + [epilogue() for _ in range(WARPS)]
    m.run()
    assert drain.done == 1 and acc_full.done == a_full.done == a_empty.done == tiles


@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 5, 9, 14])
def test_a_parity_seen_is_that_of_the_phase_it_means(tiles):
    for seed in range(60):
        polled_weights_kernel(random.Random(seed), tiles)


def test_a_wrong_parity_is_seen():
    with pytest.raises(AssertionError):
        for seed in range(20):
            polled_weights_kernel(random.Random(seed), 4, odd_a=1)
