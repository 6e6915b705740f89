"""The marks of tiles whose V is not all finite, on the CPU: the warps of the linear-attention kernel for heads of 64 values as
coroutines (as in test_la_protocol.py), with the marks as the shared places that the kernel keeps, written by the warps of
w V, read by the masks and by the epilogue.  Whatever the order, a reader finds the mark of its own tile."""
import os
import random
import re

import pytest

from test_la_protocol import Bars, Buffers, drive

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_06938_b200", "csrc")


def places():
    """How many marks the kernel keeps, from its source."""
    with open(os.path.join(CSRC, "la_tiles.cu")) as f:
        text = f.read()
    n = re.search(r"int odd_tile\[(\w+)\]", text).group(1)
    return int(n) if n.isdigit() else int(re.search(rf"constexpr int {n} = (\d+)", text).group(1))


def run(n, ns, odd, kept, rng):
    need = {f"{k}_{x}{s}": 1 for s in range(ns) for k in ("full", "free") for x in "qkv"}
    need.update({n: 1 for n in ("qk_full", "qk_read", "p_full", "qs_done", "pv_done", "kv_read", "s_full", "o_free",
                                "vw_full0", "vw_full1", "kv_done0", "kv_done1")})
    bars, buf, async_ops, marks = Bars(need), Buffers(), [], [0] * kept

    def tma():
        for t in range(n):
            s = t % ns
            for x in "kqv":
                if t >= ns:
                    yield f"free_{x}{s}", t // ns - 1
                async_ops.append([lambda x=x, s=s, t=t: (buf.write(f"{x}{s}", t, 2), bars.arrive(f"full_{x}{s}"))])

    def mma():
        queue = []
        async_ops.append(queue)

        def scores(t):
            yield f"full_k{t % ns}", t // ns
            yield f"full_q{t % ns}", t // ns
            if t:
                yield "qk_read", t - 1
            queue.append(lambda: (buf.read(f"k{t % ns}", t), buf.read(f"q{t % ns}", t), buf.write("a", t, 1),
                                  bars.arrive("qk_full")))
        yield from scores(0)
        for t in range(n):
            s = t % ns
            if t:
                yield "kv_read", t - 1
            yield "vw_full0", t
            queue.append(lambda t=t: (buf.read("vw0", t), buf.write("d", t, 1), bars.arrive("kv_done0")))
            yield "vw_full1", t
            queue.append(lambda t=t, s=s: (buf.read(f"k{s}", t), buf.read("vw1", t), bars.arrive("kv_done1"),
                                           bars.arrive(f"free_k{s}")))
            yield "s_full", t
            if t:
                yield "o_free", t - 1
            queue.append(lambda t=t, s=s: (buf.read(f"q{s}", t), buf.read("s", t), buf.write("qs", t, 1),
                                           bars.arrive("qs_done"), bars.arrive(f"free_q{s}")))
            if t + 1 < n:
                yield from scores(t + 1)
            yield f"full_v{s}", t // ns
            yield "p_full", t
            queue.append(lambda t=t, s=s: (buf.read(f"v{s}", t), buf.read("p", t), buf.write("pv", t, 1),
                                           bars.arrive("pv_done")))

    def masks():
        for t in range(n):
            yield "qk_full", t
            if t:
                yield "pv_done", t - 1
                yield None
                if marks[(t - 1) % kept] == t:
                    yield "o_free", t - 1
            buf.read("a", t)
            yield None
            bars.arrive("qk_read")
            buf.write("p", t, 1 + odd(t))                # the product, and the epilogue where V was not all finite
            yield None
            bars.arrive("p_full")

    def values():
        for t in range(n):
            yield f"full_v{t % ns}", t // ns
            buf.read(f"v{t % ns}", t)
            for half in range(2):
                if t:
                    yield f"kv_done{half}", t - 1
                buf.write(f"vw{half}", t, 1)
                yield None
                if odd(t):
                    marks[t % kept] = t + 1
                    yield None
                bars.arrive(f"vw_full{half}")

    def outputs():
        for t in range(n):
            yield "qs_done", t
            yield "pv_done", t
            yield None
            seen = marks[t % kept] == t + 1
            assert seen == odd(t), f"the epilogue of tile {t} finds {marks}"
            buf.read("qs", t)
            buf.read("pv", t)
            yield None
            if seen:
                buf.read("p", t)
            yield None
            bars.arrive("o_free")
            buf.write(f"v{t % ns}", f"o{t}", 1)           # staged where V stood
            yield None
            buf.read(f"v{t % ns}", f"o{t}")               # the copy to memory
            bars.arrive(f"free_v{t % ns}")

    def state():
        for t in range(n):
            if t:
                yield "qs_done", t - 1
            buf.write("s", t, 1)
            yield None
            bars.arrive("s_full")
            yield "kv_done1", t
            buf.read("d", t)
            yield None
            bars.arrive("kv_read")

    drive([tma(), mma(), state(), values(), masks(), outputs()], bars, async_ops, rng)


PATTERNS = {"all": lambda t: True, "even": lambda t: t % 2 == 0, "neighbours": lambda t: t % 4 < 2, "third": lambda t: t % 3 == 1,
            "one": lambda t: t == 2, "none": lambda t: False}


@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("ns", [2, 3])
@pytest.mark.parametrize("n", [2, 5, 16])
def test_readers_find_the_mark_of_their_tile(n, ns, pattern):
    rng = random.Random(n * 10 + ns)
    for _ in range(150):
        run(n, ns, PATTERNS[pattern], places(), rng)


def test_two_places_are_too_few():
    """The model is fine enough to see what the places are for: with one for even tiles and one for odd ones, marks get lost."""
    rng = random.Random(1)
    lost = 0
    for _ in range(300):
        try:
            run(16, 3, PATTERNS["all"], 2, rng)
        except AssertionError:
            lost += 1
    assert lost > 30
