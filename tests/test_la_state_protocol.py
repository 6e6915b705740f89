"""The waits of the linear-attention tile kernels where tiles only carry the state, on the CPU (as in test_la_protocol.py, whose
barriers, buffers and random orders these use): their additions stand in regions of two tiles in turn until the state's warps
have added them up; and the tiles behind them, whose state is handed over with what its copy holds taken out."""
import random

import pytest

from test_la_protocol import Bars, Buffers, drive


def run_states(n, ns, rng):
    """The states alone, heads of 64 values: D of two tiles in turn."""
    need = {f"{k}_{x}{s}": 1 for s in range(ns) for k in ("full", "free") for x in "kv"}
    need.update({f"free_v{s}": 2 for s in range(ns)})
    need.update({f"{x}{u}": 1 for x in ("vw_full", "kv_done") for u in range(4)} | {"d_free0": 1, "d_free1": 1})
    slot = lambda t, half: (t & 1) * 2 + half
    bars, buf, async_ops = Bars(need), Buffers(), []

    def tma():
        for t in range(n):
            s = t % ns
            for x, readers in (("k", 1), ("v", 2)):
                if t >= ns:
                    yield f"free_{x}{s}", t // ns - 1
                async_ops.append([lambda x=x, s=s, t=t, r=readers: (buf.write(f"{x}{s}", t, r), bars.arrive(f"full_{x}{s}"))])

    def mma():
        queue = []
        async_ops.append(queue)
        for t in range(n):
            s, a, b = t % ns, slot(t, 0), slot(t, 1)
            yield f"full_k{s}", t // ns
            if t > 1:
                yield f"d_free{t & 1}", (t >> 1) - 1
            yield f"vw_full{a}", t >> 1
            queue.append(lambda t=t, a=a: (buf.read(f"vw{a}", t), buf.write(f"d{t & 1}", t, 1), bars.arrive(f"kv_done{a}")))
            yield f"vw_full{b}", t >> 1
            queue.append(lambda t=t, s=s, b=b: (buf.read(f"k{s}", t), buf.read(f"vw{b}", t), bars.arrive(f"kv_done{b}"),
                                                bars.arrive(f"free_k{s}")))

    def values(half):
        for t in range(n):
            u = slot(t, half)
            yield f"full_v{t % ns}", t // ns
            buf.read(f"v{t % ns}", t)
            if t > 1:
                yield f"kv_done{u}", (t >> 1) - 1
            buf.write(f"vw{u}", t, 1)
            yield None
            bars.arrive(f"vw_full{u}")
            bars.arrive(f"free_v{t % ns}")

    def state():
        for t in range(n):
            yield f"kv_done{slot(t, 1)}", t >> 1
            buf.read(f"d{t & 1}", t)
            yield None
            bars.arrive(f"d_free{t & 1}")

    drive([tma(), mma(), state(), values(0), values(1)], bars, async_ops, rng)


def run_wide(n, nq, state_only, rng):
    n_pre = n if state_only else rng.choice([0, 0, rng.randrange(n)])      # tiles that only carry the state
    ns = {"q": nq, "k": nq + 1, "v": 3}
    need = {f"{k}_{x}{s}": 1 for x in "qkv" for s in range(ns[x]) for k in ("full", "free")}
    need.update({n: 1 for n in ("qk_full", "p_full", "qs_done", "o_scaled", "pv_done", "o_free", "s_full", "s_scaled", "kv_done")})
    ring = rng.choice([2, 4])                             # quarters of w V there is room for
    need.update({f"vw_{k}{i}": 1 for i in range(ring) for k in ("full", "done")})
    need.update({f"d_full{i}": 1 for i in range(2)} | {f"d_free{i}": 2 if state_only else 1 for i in range(2)})
    apart = rng.random() < 0.5                            # (the state is a result)
    bars, buf = Bars(need), Buffers()
    odd = lambda t: t >= n_pre and t % 3 == 1
    async_ops = []
    region = lambda t: "o" if t & 1 else "qk"             # D of tiles that only carry the state
    slot = lambda x, t: f"{x}{(t - n_pre if x == 'q' else t) % ns[x]}"

    def tma():
        def load(x, t):
            i = t - n_pre if x == "q" else t
            if i < 0 or t >= n or (state_only and x == "q"):
                return
            if i >= ns[x]:
                yield f"free_{slot(x, t)}", i // ns[x] - 1
            readers = {"q": 2, "k": 1 if t < n_pre else 2, "v": 1 if t < n_pre else 2}[x]
            async_ops.append([lambda: (buf.write(slot(x, t), t, readers), bars.arrive(f"full_{slot(x, t)}"))])
        for t in range(-3, n):
            for x in "qkv":
                yield from load(x, t + ns[x])

    def mma():
        queue = []
        async_ops.append(queue)

        def scores(t):
            yield f"full_{slot('k', t)}", t // ns["k"]
            yield f"full_{slot('q', t)}", (t - n_pre) // ns["q"]
            queue.append(lambda: (buf.read(slot("k", t), t), buf.read(slot("q", t), t), buf.write("qk", ("a", t), 1),
                                  bars.arrive("qk_full")))

        def add(t):
            for qd in range(4):
                yield f"vw_full{qd % ring}", (4 * t + qd) // ring

                def ready(t=t, qd=qd):
                    buf.read(f"vw{qd % ring}", 4 * t + qd)
                    bars.arrive(f"vw_done{qd % ring}")
                    if qd == 0 and t == 0 < n_pre and not apart and not state_only:
                        buf.read("s_entry", 0)
                    if qd == 0 and t < n_pre and apart:   # (the first product of a tile clears D)
                        buf.write(region(t), ("d", t), 2 if state_only else 1)
                    if qd == 3:
                        buf.read(slot("k", t), t)
                        if t < n_pre:
                            if apart or t == n_pre - 1:
                                bars.arrive(f"d_full{t & 1 if apart else 0}")
                        else:
                            buf.read("s_scaled", t)
                            buf.write("s", t + 1, 1)
                            bars.arrive("kv_done")
                        bars.arrive(f"free_{slot('k', t)}")
                queue.append(ready)
        for t in range(n_pre):
            yield f"full_{slot('k', t)}", t // ns["k"]
            if t > 1 if apart else t == 0 and not state_only:
                yield f"d_free{t & 1}", (t >> 1) - 1 if apart else 0
            yield from add(t)
        if n > n_pre:
            for t in range(max(0, n_pre - 2) if apart else n_pre, n_pre):
                yield f"d_free{t & 1}", t >> 1
            yield from scores(n_pre)
        for t in range(n_pre, n):
            f = t - n_pre
            yield "s_full", f
            if f:
                yield "o_free", f - 1
            queue.append(lambda t=t: (buf.read(slot("q", t), t), buf.read("s16", t), buf.write("o", ("s", t), 1),
                                      bars.arrive("qs_done"), bars.arrive(f"free_{slot('q', t)}")))
            yield "s_scaled", f
            yield from add(t)
            yield f"full_{slot('v', t)}", t // ns["v"]
            yield "p_full", f
            yield "o_scaled", f
            queue.append(lambda t=t: (buf.read(slot("v", t), ("z", t) if odd(t) else t), buf.read("qk", ("p", t)),
                                      buf.read("o", ("w", t)), buf.write("o", ("o", t), 1), bars.arrive("pv_done")))
            if t + 1 < n:
                yield "pv_done", f
                if odd(t):
                    yield "o_free", f
                yield from scores(t + 1)

    def masks():                                          # and the state
        def hand_over(t):
            if t > n_pre:
                buf.read("s", t)                          # with what the copy holds of it, which QS has read
                assert buf.v["s16"] == [t - 1, 0]
            buf.write("s16", t, 1)
            yield None
            bars.arrive("s_full")
            buf.write("s_scaled", t, 1)
            yield None
            bars.arrive("s_scaled")
        if not apart and n_pre:                           # the state that enters is there; tiles add to it in place
            if not state_only:
                buf.write("s_entry", 0, 1)
                yield None
                bars.arrive("d_free0")
            yield "d_full0", 0
        for t in range(n_pre if apart else 0):
            yield f"d_full{t & 1}", t >> 1
            buf.read(region(t), ("d", t))
            yield None
            bars.arrive(f"d_free{t & 1}")
        if state_only:
            return
        yield from hand_over(n_pre)
        for t in range(n_pre, n):
            f = t - n_pre
            yield "qk_full", f
            buf.read("qk", ("a", t))
            buf.write("qk", ("p", t), 1 + odd(t))
            yield None
            bars.arrive("p_full")
            if t + 1 < n:
                yield "kv_done", f
                yield "qs_done", f
                yield from hand_over(t + 1)

    def values():
        for t in range(n):
            v = slot("v", t)
            yield f"full_{v}", t // ns["v"]
            for qd in range(4):
                if 4 * t + qd >= ring:
                    yield f"vw_done{qd % ring}", (4 * t + qd) // ring - 1
                assert buf.v[v][0] == t, "w V from what replaced V"
                buf.write(f"vw{qd % ring}", 4 * t + qd, 1)
                yield None
                if qd == 3:
                    buf.read(v, t)
                    if odd(t):                            # what is not finite gives way to zeros
                        assert buf.v[v][1] == 1
                        buf.v[v] = [("z", t), 1]
                bars.arrive(f"vw_full{qd % ring}")
            if t < n_pre:
                bars.arrive(f"free_{v}")

    def outputs():
        for t in range(n_pre, n):
            f = t - n_pre
            v = slot("v", t)
            yield "qs_done", f
            buf.read("o", ("s", t))
            buf.write("o", ("w", t), 1)
            yield None
            bars.arrive("o_scaled")
            yield "pv_done", f
            buf.read("o", ("o", t))
            yield None
            if odd(t):
                buf.read("qk", ("p", t))
            bars.arrive("o_free")
            buf.write(v, f"o{t}", 1)
            yield None
            buf.read(v, f"o{t}")
            bars.arrive(f"free_{v}")

    drive([tma(), mma(), values(), masks()] + [masks() if state_only else outputs()], bars, async_ops, rng)


@pytest.mark.parametrize("state_only", [False, True])
@pytest.mark.parametrize("ns", [2, 3])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 7, 20])
def test_every_wait_ends_and_no_buffer_is_lost(n, ns, state_only):
    rng = random.Random(n * 10 + ns)
    for _ in range(250):
        run_wide(n, ns - 1, state_only, rng)
        if state_only:
            run_states(n, ns, rng)
