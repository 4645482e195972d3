"""The ragged-batch operators used together, as a serving loop uses them: reserve, rope_append, extend over two layers,
branching, leaving, trimming, compaction, and the same step captured into a graph; against a model in float64 that keeps
every sequence's keys and values apart."""
import random

import pytest
import torch

from ragged import BF16, F32, HALF_STEP, Step, attend64, ints

pytestmark = pytest.mark.gpu

N_Q, N_K, N_V, D = 8, 2, 4, 64
LAYERS, SLOTS, PAGE, ROW, PAGES = 2, 6, 16, 20, 90
SCALE = D ** -0.5


@pytest.fixture(scope="module")
def api():
    from paper_2501_13629_b200 import api as _api
    return _api


class Loop:
    """Layers are slices of the head axis of one pool pair: upkeep sees all heads, rope_append and extend their layer's."""

    def __init__(self, api, capacity):
        self.api = api
        self.gen = torch.Generator("cuda").manual_seed(7)
        self.table = torch.full((SLOTS, ROW), -1, dtype=torch.int32, device="cuda")
        self.lens, self.refs = ints([0] * SLOTS), ints([0] * PAGES)
        nan = float("nan")
        k = torch.full((PAGES, LAYERS * N_K, PAGE, D), nan, dtype=BF16, device="cuda")
        v = torch.full((PAGES, LAYERS * N_V, PAGE, D), nan, dtype=BF16, device="cuda")
        make = lambda k, v: api.KVCache(k, v, self.lens, ROW * PAGE, page_table=self.table, page_size=PAGE)  # noqa: E731
        self.both = make(k, v)
        self.caches = [make(k[:, i * N_K:(i + 1) * N_K], v[:, i * N_V:(i + 1) * N_V]) for i in range(LAYERS)]
        self.inv, self.mag = api.rope_frequencies(D, 10000.0, "yarn", factor=4.0, original_length=64, fast=32, slow=1,
                                                  device="cuda")
        self.status = ints([0])
        self.capacity = capacity
        self.cu = ints([0] * (SLOTS + 1))
        self.granted = ints([0] * SLOTS)
        make = lambda h: torch.zeros((LAYERS, capacity, h, D), dtype=BF16, device="cuda")  # noqa: E731
        self.q, self.k, self.v, self.turned, self.out = make(N_Q), make(N_K), make(N_V), make(N_Q), make(N_Q)
        self.ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        # the model: per slot and layer lists of turned keys and values, float64 of the rounded values
        self.keys = [[[] for _ in range(LAYERS)] for _ in range(SLOTS)]
        self.values = [[[] for _ in range(LAYERS)] for _ in range(SLOTS)]
        self.length = [0] * SLOTS

    def enqueue(self):
        api = self.api
        api.diffqkv_pages_reserve(self.cu, self.both, self.refs, N_K * LAYERS, N_V * LAYERS, granted=self.granted,
                                  workspace=self.ws, dev_status=self.status)
        for l, c in enumerate(self.caches):
            api.diffqkv_rope_append(self.q[l], self.k[l], self.v[l], self.cu, c, self.inv, magnitude=self.mag,
                                    q_out=self.turned[l], dev_status=self.status)
            api.diffqkv_extend(self.turned[l], self.cu, c, N_K, N_V, SCALE, out=self.out[l], workspace=self.ws,
                               dev_status=self.status)

    def feed(self, new):
        """New rows of every slot; what the model expects of them."""
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        assert cu[-1] <= self.capacity
        self.cu.copy_(ints(cu))
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, generator=self.gen, device="cuda").to(BF16))
        self.new, self.bounds = new, cu

    def turn(self, x, first):
        n, half = x.shape[0], D // 2
        a = torch.outer(torch.arange(first, first + n, device="cuda").double(), self.inv)[:, None]
        u, v = x[..., :half].double(), x[..., half:].double()
        return torch.cat([u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()], -1) * self.mag

    def check(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0 and self.granted.tolist() == [1] * SLOTS
        for s, n in enumerate(self.new):
            if n == 0:
                continue
            lo, first = self.bounds[s], self.length[s]
            for l in range(LAYERS):
                k, v = self.turn(self.k[l, lo:lo + n], first), self.v[l, lo:lo + n].double()
                self.keys[s][l].append(k)
                self.values[s][l].append(v)
                q = self.turn(self.q[l, lo:lo + n], first)
                keys, values = torch.cat(self.keys[s][l]), torch.cat(self.values[s][l])
                ref, _, mean_abs, big = attend64(q, keys, values, SCALE, first)
                # q and k are rounded to bf16 once each (the values are exact): a score is off by two half steps of
                # sum |q k|, the weight by twice that through score and maximum, and once more by its own rounding;
                # the result is rounded once.  exp(x) - 1 of that, since the scores' part need not be small.
                score = 2 * HALF_STEP[BF16] * (1 + HALF_STEP[BF16]) * big + (D + 16) * 2.0 ** -24 * big
                weight = 2 * score + HALF_STEP[BF16] + (len(keys) + 16) * 2.0 ** -24
                bound = float(torch.tensor(weight).expm1()) * mean_abs
                bound = bound + HALF_STEP[BF16] * (ref.abs() + bound)
                err = (self.out[l, lo:lo + n].double() - ref).abs()
                assert bool((err <= bound).all()), f"slot {s}, layer {l}: {float((err / bound).max()):.2f} times the bound"
            self.length[s] += n
        self.lens.copy_(ints(self.length))

    def fork(self, parents, children):
        self.api.diffqkv_pages_fork(ints(parents), ints(children), self.both, self.refs, dev_status=self.status)
        old = [(list(map(list, self.keys[p])), list(map(list, self.values[p])), self.length[p]) for p in parents]
        for (k, v, n), c in zip(old, children):
            self.keys[c], self.values[c], self.length[c] = list(map(list, k)), list(map(list, v)), n

    def leave(self, slots):
        self.api.diffqkv_pages_free(ints(slots), self.both, self.refs, dev_status=self.status)
        for s in slots:
            self.keys[s], self.values[s], self.length[s] = [[] for _ in range(LAYERS)], [[] for _ in range(LAYERS)], 0

    def trim(self, slot, keep):
        self.api.diffqkv_pages_free(ints([slot]), self.both, self.refs, keep_tokens=ints([keep]), dev_status=self.status)
        for l in range(LAYERS):
            self.keys[slot][l] = [torch.cat(self.keys[slot][l])[:keep]]
            self.values[slot][l] = [torch.cat(self.values[slot][l])[:keep]]
        self.length[slot] = keep

    def compact(self):
        self.api.diffqkv_pages_compact(self.both, self.refs, N_K * LAYERS, N_V * LAYERS, workspace=self.ws,
                                       dev_status=self.status)


def test_serving_loop(api):
    loop = Loop(api, 260)

    def step(new):
        loop.feed(new)
        loop.enqueue()
        loop.check()

    step([100, 17, 0, 1, 0, 0])         # prompts
    step([1, 1, 60, 1, 0, 0])           # one more arrives, the others decode
    loop.fork([0, 0, 2], [4, 5, 3])     # two continuations of slot 0 beside it, slot 3 gives way to one of slot 2
    step([1, 5, 1, 1, 1, 1])            # shared half-filled pages are copied
    loop.leave([1])
    loop.compact()                      # pages move under the running sequences
    step([1, 140, 1, 1, 1, 3])
    loop.trim(1, 130)                   # guessed tokens are rejected
    loop.trim(0, 96)                    # back into pages that others share
    step([4, 2, 1, 1, 1, 1])
    loop.fork([4, 5, 0], [5, 0, 4])     # beams change places
    step([1, 1, 1, 1, 1, 1])


def test_captured_loop(api):
    """One graph of a step of fixed capacity, replayed through changing chunks and branching in between."""
    loop = Loop(api, 16 * SLOTS)
    loop.feed([3, 1, 0, 0, 0, 0])
    loop.enqueue()
    loop.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.enqueue()
    r = random.Random(3)
    for i in range(12):
        new = [r.choice([0, 1, 1, 5, 16]) for _ in range(SLOTS)]
        if i % 3 == 2:
            loop.fork([0, 1], [4, 5])
        loop.feed(new)
        graph.replay()
        loop.check()


def test_two_captured_loops_side_by_side(api):
    """Two loops with a workspace each, replayed on two streams at once."""
    loops = [Loop(api, 16 * SLOTS) for _ in range(2)]
    graphs = []
    for loop in loops:
        loop.feed([30, 1, 9, 0, 0, 0])
        loop.enqueue()
        loop.check()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            loop.enqueue()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in loops]
    for i in range(5):
        for loop in loops:
            loop.feed([1, 7, 1, 1, 16, i])
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        for loop in loops:
            loop.check()


def test_memory_of_a_call_belongs_to_its_stream(api, monkeypatch):
    """A workspace that a call on another stream brings itself must not be handed out on the current one while the call may
    still be waiting to run."""
    step = Step(api, [900, 40, 3], [2, 70, 1], 8, 2, 4, 64, 64, seed=1).fill()
    refs = torch.ones(step.k.shape[0], dtype=torch.int32, device="cuda")
    side, taken = torch.cuda.Stream(), []
    place = {"diffqkv_extend": 5, "diffqkv_pages_fork": 4, "diffqkv_pages_reserve": 5, "diffqkv_pages_compact": 6}
    for name, at in place.items():
        def spy(*args, call=getattr(api._raw, name), at=at):
            taken.append((args[at], args[at + 1]))
            return call(*args)
        monkeypatch.setattr(api._raw, name, spy)
    ids, none = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    k_new, v_new = step.q[:, :2].contiguous(), step.q[:, :4].contiguous()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    out = api.diffqkv_extend(step.q, step.cu, step.cache, 2, 4, 0.125, stream=side)
    api.diffqkv_pages_fork(ids, ids, step.cache, refs, stream=side)
    api.diffqkv_pages_reserve(none, step.cache, refs, 2, 4, stream=side)
    api.diffqkv_pages_compact(step.cache, refs, 2, 4, stream=side)
    turned = api.diffqkv_rope_append(step.q, k_new, v_new, step.cu, step.cache, None, stream=side)
    assert len(taken) == 4
    kept = [torch.empty(n, dtype=torch.uint8, device="cuda") for _, n in taken for _ in range(3)]
    kept += [torch.empty_like(out), torch.empty_like(turned)]
    spans = [(p, p + n) for p, n in taken]
    for x in kept:
        lo, hi = x.data_ptr(), x.data_ptr() + x.numel() * x.element_size()
        assert all(hi <= a or b <= lo for a, b in spans)
    torch.cuda.synchronize()
