"""The waits of the linear-attention tile kernels, on the CPU: their warps as coroutines over counted barriers, run in random
orders.  Every wait ends, no barrier gets two phases ahead of a waiter (parities would alias), and no buffer is written while
its last contents are still to be read."""
import random

import pytest


class Bars:
    def __init__(self, need):
        self.need, self.got, self.done = need, {n: 0 for n in need}, {n: 0 for n in need}

    def arrive(self, n):
        self.got[n] += 1
        if self.got[n] == self.need[n]:
            self.got[n], self.done[n] = 0, self.done[n] + 1

    def ready(self, n, phase):
        assert self.done[n] <= phase + 1, f"{n}: phase {self.done[n]} with a waiter on {phase}"
        return self.done[n] > phase


class Buffers:
    """name -> (version held, readers still to come)."""

    def __init__(self):
        self.v = {}

    def write(self, name, version, readers):
        old = self.v.get(name)
        assert old is None or old[1] == 0, f"{name}: version {version} over {old}"
        self.v[name] = [version, readers]

    def read(self, name, version):
        assert self.v[name][0] == version and self.v[name][1] > 0, f"{name}: {version} wanted, {self.v[name]} held"
        self.v[name][1] -= 1


def run(n, ns, state_only, rng):
    need = {f"{k}_{x}{s}": 1 for s in range(ns) for k in ("full", "free") for x in "qkv"}
    for s in range(ns):
        need[f"free_v{s}"] = 2 if state_only else 1
    need.update({n: 1 for n in ("qk_full", "qk_read", "p_full", "qs_done", "pv_done", "kv_read", "s_full", "o_free")})
    need.update({f"{x}{u}": 1 for x in ("vw_full", "kv_done") for u in range(4)})
    slot = lambda t, half: (t & 1) * 2 + half if state_only else half
    phase = lambda t: t >> 1 if state_only else t
    bars, buf = Bars(need), Buffers()
    odd = lambda t: t % 3 == 1
    async_ops = []                       # products and copies, each queue in order: callables

    def tma():
        for t in range(n):
            s = t % ns
            for x in "kv" if state_only else "kqv":
                if t >= ns:
                    yield f"free_{x}{s}", t // ns - 1
                readers = {"q": 2, "k": 1 if state_only else 2, "v": 2}[x]
                async_ops.append([lambda x=x, s=s, t=t, r=readers: (buf.write(f"{x}{s}", t, r), bars.arrive(f"full_{x}{s}"))])

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
        if not state_only and n:
            yield from scores(0)
        for t in range(n):
            s = t % ns
            if state_only:
                yield f"full_k{s}", t // ns
            elif t:
                yield "kv_read", t - 1
            a, b = slot(t, 0), slot(t, 1)
            yield f"vw_full{a}", phase(t)
            queue.append(lambda t=t, a=a: (buf.read(f"vw{a}", t), state_only or buf.write("d", t, 1), bars.arrive(f"kv_done{a}")))
            yield f"vw_full{b}", phase(t)
            queue.append(lambda t=t, s=s, b=b: (buf.read(f"k{s}", t), buf.read(f"vw{b}", t), bars.arrive(f"kv_done{b}"),
                                           bars.arrive(f"free_k{s}"),
                                           bars.arrive("qs_done") if state_only and t == n - 1 else None))
            if state_only:
                continue
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
                if odd(t - 1):
                    yield "o_free", t - 1
            buf.read("a", t)
            yield None
            bars.arrive("qk_read")
            buf.write("p", t, 1 + odd(t))                # the product, and the epilogue where V was not all finite
            yield None
            bars.arrive("p_full")

    def values(halves):
        for t in range(n):
            yield f"full_v{t % ns}", t // ns
            buf.read(f"v{t % ns}", t)
            for half in halves:
                u = slot(t, half)
                if phase(t):
                    yield f"kv_done{u}", phase(t) - 1
                buf.write(f"vw{u}", t, 1)
                yield None
                bars.arrive(f"vw_full{u}")
            if state_only:
                bars.arrive(f"free_v{t % ns}")

    def outputs():
        for t in range(n):
            yield "qs_done", t
            yield "pv_done", t
            buf.read("qs", t)
            buf.read("pv", t)
            yield None
            if odd(t):
                buf.read("p", t)
            yield None
            bars.arrive("o_free")
            buf.write(f"v{t % ns}", f"o{t}", 1)           # staged where V stood
            yield None
            buf.read(f"v{t % ns}", f"o{t}")               # the copy to memory
            bars.arrive(f"free_v{t % ns}")

    def state():
        if state_only:
            if n:
                yield "qs_done", 0
            return
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

    drive([tma(), mma(), state()] + ([values((0,)), values((1,))] if state_only else [values((0, 1)), masks(), outputs()]),
          bars, async_ops, rng)


def run_wide(n, nq, state_only, rng):
    n_pre = n if state_only else rng.choice([0, 0, rng.randrange(n)])      # tiles that only carry the state
    pre = 1 if n_pre else 0
    ns = {"q": nq, "k": nq + 1, "v": 3}
    need = {f"{k}_{x}{s}": 1 for x in "qkv" for s in range(ns[x]) for k in ("full", "free")}
    need.update({n: 1 for n in ("qk_full", "p_full", "qs_done", "o_scaled", "pv_done", "o_free", "s_full", "s_scaled", "kv_done")})
    ring = rng.choice([2, 4])                             # quarters of w V there is room for
    need.update({f"vw_{k}{i}": 1 for i in range(ring) for k in ("full", "done")})
    bars, buf = Bars(need), Buffers()
    odd = lambda t: t >= n_pre and t % 3 == 1
    async_ops = []
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

        def add(t, done):
            for qd in range(4):
                yield f"vw_full{qd % ring}", (4 * t + qd) // ring

                def ready(t=t, qd=qd):
                    buf.read(f"vw{qd % ring}", 4 * t + qd)
                    bars.arrive(f"vw_done{qd % ring}")
                    if qd == 3:
                        buf.read(slot("k", t), t)
                        if t >= n_pre or (t == 0 and not state_only):
                            buf.read("s_scaled", t)
                        if done and not (state_only and t < n - 1):
                            buf.write("s", t + 1, 1)
                            bars.arrive("kv_done")
                        bars.arrive(f"free_{slot('k', t)}")
                queue.append(ready)
        if pre and not state_only:
            yield "s_scaled", 0
        for t in range(n_pre):
            yield f"full_{slot('k', t)}", t // ns["k"]
            yield from add(t, t == n_pre - 1)
        if n > n_pre:
            yield from scores(n_pre)
        for t in range(n_pre, n):
            f = t - n_pre
            yield "s_full", f
            if f:
                yield "o_free", f - 1
            queue.append(lambda t=t: (buf.read(slot("q", t), t), buf.read("s16", t), buf.write("o", ("s", t), 1),
                                      bars.arrive("qs_done"), bars.arrive(f"free_{slot('q', t)}")))
            yield "s_scaled", f + pre
            yield from add(t, True)
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
            if t:
                buf.read("s", t)
            buf.write("s16", t, 1)
            yield None
            bars.arrive("s_full")
            buf.write("s_scaled", t, 1)
            yield None
            bars.arrive("s_scaled")
        if state_only:
            if n:
                yield "kv_done", 0
            return
        if pre:
            buf.write("s_scaled", 0, 1)
            yield None
            bars.arrive("s_scaled")
            yield "kv_done", 0
        yield from hand_over(n_pre)
        for t in range(n_pre, n):
            f = t - n_pre
            yield "qk_full", f
            buf.read("qk", ("a", t))
            buf.write("qk", ("p", t), 1 + odd(t))
            yield None
            bars.arrive("p_full")
            if t + 1 < n:
                yield "kv_done", f + pre
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

    drive([tma(), mma(), values(), masks()] + ([] if state_only else [outputs()]), bars, async_ops, rng)


def drive(roles, bars, async_ops, rng):
    live = [[g, next(g, "end")] for g in roles]
    live = [x for x in live if x[1] != "end"]
    while live or any(async_ops):
        steps = [x for x in live if x[1] is None or bars.ready(*x[1])]
        queues = [q for q in async_ops if q]
        assert steps or queues, [x[1] for x in live]
        pick = rng.randrange(len(steps) + len(queues))
        if pick < len(steps):
            x = steps[pick]
            x[1] = next(x[0], "end")
            if x[1] == "end":
                live.remove(x)
        else:
            queues[pick - len(steps)].pop(0)()


@pytest.mark.parametrize("state_only", [False, True])
@pytest.mark.parametrize("ns", [2, 3])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 7, 20])
def test_every_wait_ends_and_no_buffer_is_lost(n, ns, state_only):
    rng = random.Random(n * 10 + ns)
    for _ in range(60):
        run(n, ns, state_only, rng)
        run_wide(n, ns - 1, state_only, rng)
