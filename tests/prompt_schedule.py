"""The prompt kernel's barriers and who waits for what, as coroutines: random runs, the roles, products and loads
advancing in any order. Every wait is by parity, as on the device, and says which phase it means."""
import random


class Barrier:
    def __init__(self, count):
        self.count, self.pending, self.done = count, 0, 0

    def arrive(self):
        self.pending += 1
        assert self.pending <= self.count, "more arrivals than a phase has"
        if self.pending == self.count:
            self.pending, self.done = 0, self.done + 1

    def passed(self, phase):
        """Whether a wait for this phase (-1: the one before the first) returns; it may only if it is complete."""
        by_parity = (self.done - 1) & 1 == phase & 1
        assert not by_parity or self.done > phase, "a wait passed ahead of its phase"
        return by_parity


def runs_of(spec):
    """(tiles, tiles of block 0, two blocks, keys that every row sees) of each run, as the producer publishes them."""
    runs, use, singles = [], 0, 0
    for tiles, end0, two, least in spec:
        if two:
            blocks, end = 3, [end0, tiles]
        else:
            x, singles = singles & 1, singles + 1
            blocks, end = 1 << x, [tiles if x == 0 else 0, tiles if x else 0]
        runs.append({"s1": tiles, "end": end, "blocks": blocks, "least": least, "use": use})
        use += 2 if two else 1
    return runs


def simulate(seed, stages, spec, q_places=3, ring=4):
    rng = random.Random(seed)
    runs, end_mark = runs_of(spec), {"blocks": 0}
    readers = 15
    bars = lambda n, count=1: [Barrier(count) for _ in range(n)]  # noqa: E731
    full, empty, q_full, q_empty = bars(stages), bars(stages), bars(q_places), bars(q_places)
    s_ready, p_ready = bars(2), bars(2, 4)
    o_ready, o_free, l_ready, (ask, clean) = bars(2), bars(2, 4), bars(2, 4), bars(2)
    run_full, run_empty, slots = bars(ring), bars(ring, readers), [None] * ring
    products, loads = [], []                       # in order; in any order
    has = lambda r, x: r["blocks"] >> x & 1  # noqa: E731
    q_use = lambda r, x: r["use"] + (x if r["blocks"] == 3 else 0)  # noqa: E731

    def publish(i):
        yield lambda: run_empty[i % ring].passed(i // ring - 1)
        slots[i % ring] = runs[i] if i < len(runs) else end_mark
        run_full[i % ring].arrive()

    def producer():
        fills = 0
        yield from publish(0)
        for i, r in enumerate(runs):
            yield from publish(i + 1)
            for _ in range(2 * r["s1"]):
                at, n = fills % stages, fills // stages
                yield lambda: empty[at].passed(n - 1)
                loads.append(full[at])
                fills += 1

    def read(walk):
        at, n = walk[0] % ring, walk[0] // ring
        yield lambda: run_full[at].passed(n)
        r = slots[at]
        run_empty[at].arrive()
        walk[0] += 1
        return r

    def issuer():
        walk, tile, seen, freed, cleaned = [0], 0, [0, 0], [-1, -1], 0   # tiles whose K was taken; of the blocks' P, O

        def issue_s(r, x, q, first, last):
            if first:
                yield lambda: q_full[q % q_places].passed(q // q_places)
            products.append([s_ready[x]] + ([q_empty[q % q_places]] if last else []))

        def k_there():
            at, n = 2 * tile % stages, 2 * tile // stages
            yield lambda: full[at].passed(n)

        r = yield from read(walk)
        if r["blocks"]:
            yield from k_there()
            for x in range(2):
                if has(r, x):
                    yield from issue_s(r, x, q_use(r, x), True, r["end"][x] == 1)
            products.append([empty[2 * tile % stages]])
            tile += 1
        while r["blocks"]:
            n = yield from read(walk)
            for s in range(r["s1"]):
                at, fill, k_seen, last = (2 * tile - 1) % stages, (2 * tile - 1) // stages, False, s + 1 == r["s1"]
                masked = s >= r["least"] // 128
                yield lambda: full[at].passed(fill)
                if masked:
                    ask.arrive()
                for x in range(2):
                    end = r["end"][x]
                    if s < end:
                        if s == 0:
                            yield lambda: o_free[x].passed(freed[x])
                            freed[x] += 1
                        yield lambda: p_ready[x].passed(seen[x])
                        seen[x] += 1
                        if masked:
                            yield lambda: clean.passed(cleaned)
                            cleaned, masked = cleaned + 1, False
                        products.append(([o_ready[x]] if s + 1 == end else [])
                                        + ([empty[at]] if x or s >= r["end"][1] else []))
                    if n["blocks"] and has(n, x) if last else s + 1 < end:
                        if not k_seen:
                            yield from k_there()
                        k_seen = True
                        if last:
                            yield from issue_s(n, x, q_use(n, x), True, n["end"][x] == 1)
                        else:
                            yield from issue_s(r, x, q_use(r, x), False, s + 2 == end)
                if not last or n["blocks"]:
                    products.append([empty[2 * tile % stages]])
                    tile += 1
            r = n

    def softmax(x):
        walk, freed, seen = [0], -1, 0
        while True:
            r = yield from read(walk)
            if not r["blocks"]:
                return
            for _ in range(r["end"][x] if has(r, x) else 0):
                yield lambda: s_ready[x].passed(seen)
                seen += 1
                p_ready[x].arrive()
            if has(r, x):
                yield lambda: o_free[x].passed(freed)
                freed += 1
                l_ready[x].arrive()

    def cleaner():
        walk, asked = [0], 0
        while True:
            r = yield from read(walk)
            if not r["blocks"]:
                return
            for s in range(r["s1"]):
                if (s + 1) * 128 > r["least"]:
                    yield lambda: ask.passed(asked)
                    asked += 1
                    clean.arrive()

    def loader():
        walk = [0]
        while True:
            r = yield from read(walk)
            if not r["blocks"]:
                return
            for x in range(2):
                if has(r, x):
                    q = q_use(r, x)
                    yield lambda: q_empty[q % q_places].passed(q // q_places - 1)
                    loads.append(q_full[q % q_places])

    def finisher():
        walk, n = [0], [0, 0]
        while True:
            r = yield from read(walk)
            if not r["blocks"]:
                return
            for x in range(2):
                if has(r, x):
                    yield lambda: l_ready[x].passed(n[x])
                    yield lambda: o_ready[x].passed(n[x])
                    n[x] += 1
                    o_free[x].arrive()

    tasks = [producer(), issuer(), cleaner(), loader()] + [softmax(x) for x in (0, 1) for _ in range(4)] \
        + [finisher() for _ in range(4)]
    waits = [None] * len(tasks)

    def go(i):
        waits[i] = next(tasks[i], None)

    for i in range(len(tasks)):
        go(i)
    # a role that is slow now and then: it moves only when nothing else can
    slow = rng.randrange(len(tasks) + 3)
    while any(w is not None for w in waits):
        ready = [i for i, w in enumerate(waits) if w is not None and w()]
        choices = ready + (["product"] if products else []) + (["load"] if loads else [])
        assert choices, "every role waits"
        others = [c for c in choices if c != slow]
        c = rng.choice(others if others and rng.random() < 0.95 else choices)
        if c == "product":
            for b in products.pop(0):
                b.arrive()
        elif c == "load":
            loads.pop(rng.randrange(len(loads))).arrive()
        else:
            go(c)
