"""goose_pages_evict and goose_pages_append against the simulator: which slots stay, where they go, and that nothing else changes.

Everything is exact but keys that are turned.  One of those, u half a step of its type: the angle is reduced in 64 bits and rounded to 32 (2^-23 rad),
its sine and cosine err by 2^-22 more, two products and a sum 2^-22: (|a| + |b|) 2^-20 beside the store's u |x| (fp16 below its normals 2^-25); the
simulator's own store costs the same again.
"""
import numpy as np
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, pack_pages, unpack_pages
from prompt_ref import PromptSim

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Setup:
    def __init__(self, lens, layers=2, nkv=2, d=64, dtype="bf16", seed=0, spare=4, extra=1, base=10000.0, weights="random"):
        g = torch.Generator().manual_seed(seed)
        self.dt, self.base = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype], base
        n_pages = sum((n + PAGE - 1) // PAGE for n in lens) + spare
        width = max(1, max((n + PAGE - 1) // PAGE for n in lens)) + extra
        k = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(self.dt)
        v = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(self.dt)
        self.sim = PromptSim(len(lens), width, n_pages, k, v)
        order, at = torch.randperm(n_pages, generator=g).tolist(), 0
        for q, n in enumerate(lens):
            for i in range((n + PAGE - 1) // PAGE):
                self.sim.table[q, i] = order[at]
                self.sim.refs[order[at]] = 1
                at += 1
            self.sim.len[q] = n
        shape = (layers, len(lens), nkv, width * PAGE)
        w = torch.exp(2 * torch.randn(shape, generator=g))
        if weights == "ties":
            w = torch.floor(w * 2)
        elif weights == "equal":
            w = torch.ones(shape)
        elif weights == "odd":   # signs, both zeros, infinities, NaN, denormals
            pick = torch.tensor([0.0, -0.0, 1.0, -1.0, float("inf"), float("-inf"), float("nan"), 1e-42, -1e-42, 3.4e38, 1.0000001])
            w = pick[torch.randint(0, len(pick), shape, generator=g)]
        elif weights == "close":   # they differ in the last bits only
            w = (torch.randint(0, 40, shape, generator=g) + 0x3F800000).int().view(torch.float32)
        self.w = w
        self.ctx = goose.GooseContext(goose.ModelDesc(layers, 128, nkv * 2, d, 128, 1024, base, 1e-5, dtype, nkv), 8, 128, 32)
        kp, vp = pack_pages(k, v)
        s = self.sim
        self.cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), *[torch.from_numpy(x.copy()).to(DEV) for x in (s.table, s.len, s.refs)])
        self.weight = w.to(DEV)
        self.layers, self.nkv, self.d = layers, nkv, d

    def evict(self, ev, reposition=True, flags=0):
        kept = torch.full((len(ev), self.layers, self.nkv, self.sim.table.shape[1]), 77, dtype=torch.int64, device=DEV)
        before = self.sim.k.clone()
        self.ctx.goose_pages_evict(self.cache, ev, self.weight, kept, reposition)
        got = self.ctx.goose_device_flags()
        want, words = self.sim.evict(ev, self.w, self.base, reposition)
        assert (got, want) == (flags, flags)
        kept = kept.cpu()
        for i, w in enumerate(words):
            assert (kept[i] == 77).all() if w is None else torch.equal(kept[i], w), f"kept words of {i}"
        self.check(before, reposition)
        return words

    def check(self, before=None, turned=False):
        s = self.sim
        assert np.array_equal(self.cache.table.cpu().numpy(), s.table) and np.array_equal(self.cache.len.cpu().numpy(), s.len)
        assert np.array_equal(self.cache.refs.cpu().numpy(), s.refs)
        assert torch.equal(self.weight.cpu().view(torch.int32), self.w.view(torch.int32)), "weights"
        k, v = unpack_pages(self.cache.kpool.cpu(), self.cache.vpool.cpu(), self.d)
        assert torch.equal(v.view(torch.int16), s.v.view(torch.int16)), "values"
        if not turned:
            assert torch.equal(k.view(torch.int16), s.k.view(torch.int16)), "keys"
            return
        same = s.k.view(torch.int16) == before.view(torch.int16)
        assert torch.equal(k.view(torch.int16)[same.all(-1)], s.k.view(torch.int16)[same.all(-1)]), "rows that stay"
        a, b = k.double(), s.k.double()
        u = torch.finfo(self.dt).eps / 2
        h = self.d // 2
        size = (b[..., :h] ** 2 + b[..., h:] ** 2).sqrt() * 2 ** 0.5      # |a| + |b| of the pair at most
        tol = 2 * u * b.abs() + torch.cat((size, size), -1) * 2.0 ** -20 + 2.0 ** -24
        bad = ~((a - b).abs() <= tol)
        assert not bad.any(), (bad.nonzero()[0].tolist(), float(a[bad][0]), float(b[bad][0]))
        s.k.copy_(k)   # (the next call goes on from the rounded rows)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("reposition", [True, False])
def test_types_and_head_sizes(dtype, d, reposition):
    for weights in ("random", "ties"):
        s = Setup([500, 130, 257], d=d, dtype=dtype, seed=1, weights=weights)
        s.evict([{"seq": 2, "keep": 100, "sink": 4, "recent": 30}, {"seq": 0, "keep": 333, "sink": 64, "recent": 64}], reposition)


@pytest.mark.parametrize("n,keep,sink,recent", [
    (1, 1, 0, 0), (2, 1, 0, 0), (2, 1, 1, 0), (2, 1, 0, 1), (64, 63, 0, 0), (65, 64, 0, 0), (65, 64, 64, 0), (65, 64, 0, 64), (65, 1, 0, 0),
    (200, 199, 0, 0), (200, 199, 100, 99), (200, 200, 0, 0), (200, 201, 200, 1), (200, 150, 150, 0), (200, 150, 0, 150), (129, 128, 33, 1),
    (1000, 32, 0, 0), (1000, 33, 31, 2), (1000, 999, 1, 1), (1000, 65, 64, 1), (300, 31, 0, 31), (300, 96, 95, 0), (0, 5, 1, 1), (2500, 700, 7, 77),
])
def test_lengths_and_windows(n, keep, sink, recent):
    for weights, reposition in (("random", True), ("ties", False), ("equal", True), ("odd", False), ("close", False)):
        s = Setup([n, 70], nkv=1, seed=n + keep, weights=weights)
        s.evict([{"seq": 0, "keep": keep, "sink": sink, "recent": recent}], reposition)


def test_many_slots_and_a_long_table():
    """More slots than a workgroup's threads, more pages than a wavefront's lanes."""
    s = Setup([9000, 4600], layers=1, nkv=3, seed=4, weights="ties")
    s.evict([{"seq": 0, "keep": 5000, "sink": 3, "recent": 500}, {"seq": 1, "keep": 4500}], reposition=False)


def test_again_and_again():
    """Rows that have moved move again; room is taken and appended in between, at the lowest free pages."""
    s = Setup([700, 300], seed=5, spare=6)
    for i, (keep, new) in enumerate(((400, 90), (256, 64), (300, 10), (17, 400))):
        s.evict([{"seq": 0, "keep": keep, "sink": 16, "recent": 1}, {"seq": 1, "keep": 200, "sink": 0, "recent": i}])
        assert s.sim.reserve([0, 1], [new, 5]) == 0
        s.ctx.goose_pages_reserve(s.cache, [0, 1], [new, 5])
        chunks = [{"seq": 0, "C": new}, {"seq": 1, "C": 5}]
        assert s.sim.append([0, 1], [new, 5]) == 0
        s.ctx.goose_pages_append(s.cache, chunks)
        assert s.ctx.goose_device_flags() == 0
        s.check()


def test_shared_pages_stay_or_the_sequence_does():
    s = Setup([260, 0, 0, 90], seed=6, spare=12)
    s.sim.fork(0, [1, 2], 192)
    s.ctx.goose_pages_fork(s.cache, 0, [1, 2], 192)
    assert s.sim.reserve([1, 2], [180, 100]) == 0
    s.ctx.goose_pages_reserve(s.cache, [1, 2], [180, 100])
    s.sim.append([1, 2], [180, 100])
    s.ctx.goose_pages_append(s.cache, [{"seq": 1, "C": 180}, {"seq": 2, "C": 100}])
    s.check()
    # shared pages among the sinks: they stay; one slot less and nothing is done
    s.evict([{"seq": 1, "keep": 300, "sink": 192, "recent": 20}])
    s.evict([{"seq": 2, "keep": 250, "sink": 191, "recent": 20}, {"seq": 3, "keep": 40}], flags=gb.GOOSE_FLAG_PAGES)
    # pages that only go back may be shared
    s.evict([{"seq": 0, "keep": 100, "sink": 100}])
    s.evict([{"seq": 2, "keep": 250, "sink": 192, "recent": 20}])


def test_broken_state_is_left_alone():
    s = Setup([260, 130], seed=7)
    for seq, entry, value in ((0, 1, -1), (0, 4, 10 ** 6), (0, 0, -5)):
        old = int(s.sim.table[seq, entry])
        s.sim.table[seq, entry] = value
        s.cache.table[seq, entry] = value
        s.evict([{"seq": 0, "keep": 100}], flags=gb.GOOSE_FLAG_PAGES)
        s.sim.table[seq, entry] = old
        s.cache.table[seq, entry] = old
    for n in (-1, 10 ** 9, s.sim.table.shape[1] * PAGE + 1):
        s.sim.len[0] = n
        s.cache.len[0] = n
        s.evict([{"seq": 0, "keep": 100}], flags=gb.GOOSE_FLAG_CAPACITY)
        s.ctx.goose_pages_append(s.cache, [{"seq": 0, "C": 1}])
        assert s.ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
    s.sim.len[0] = 260
    s.cache.len[0] = 260
    s.evict([{"seq": 0, "keep": 100}, {"seq": 1, "keep": 7, "recent": 7}])


def test_append_refuses_slots_that_are_not_its_own():
    s = Setup([100, 0, 64], seed=8, spare=6)
    for seq, new in ((0, 29), (0, 1), (2, 1)):   # a page that is there, and one that is not
        assert s.sim.append([seq], [new]) == (0 if (seq, new) != (2, 1) and s.sim.len[seq] + new <= 128 else 16)
        s.ctx.goose_pages_append(s.cache, [{"seq": seq, "C": new}])
        s.ctx.goose_device_flags()
        s.check()
    s.sim.fork(0, [1])
    s.ctx.goose_pages_fork(s.cache, 0, [1])
    s.sim.len[1] = 100
    s.cache.len[1] = 100
    assert s.sim.append([1], [4]) == 16
    s.ctx.goose_pages_append(s.cache, [{"seq": 1, "C": 4}])
    assert s.ctx.goose_device_flags() == 16
    s.check()
    # reserved for more than is appended: the rest goes back
    assert s.sim.reserve([2], [100]) == 0
    s.ctx.goose_pages_reserve(s.cache, [2], [100])
    assert s.sim.append([2], [30]) == 0
    s.ctx.goose_pages_append(s.cache, [{"seq": 2, "C": 30}])
    assert s.ctx.goose_device_flags() == 0
    s.check()


def test_a_graph_decides_on_the_device():
    s = Setup([400, 90], seed=9, spare=8)
    kept = torch.zeros((2, s.layers, s.nkv, s.sim.table.shape[1]), dtype=torch.int64, device=DEV)
    ev = [{"seq": 0, "keep": 200, "sink": 8, "recent": 16}, {"seq": 1, "keep": 200, "sink": 8, "recent": 16}]

    def calls():
        s.ctx.goose_pages_evict(s.cache, ev, s.weight, kept, True)
        s.ctx.goose_pages_reserve(s.cache, [0, 1], [70, 70])
        s.ctx.goose_pages_append(s.cache, [{"seq": 0, "C": 70}, {"seq": 1, "C": 70}])

    def simulate():
        before = s.sim.k.clone()
        _, words = s.sim.evict(ev, s.w, s.base, True)
        assert s.sim.reserve([0, 1], [70, 70]) == 0 and s.sim.append([0, 1], [70, 70]) == 0
        return before, words

    calls()
    before, _ = simulate()
    assert s.ctx.goose_device_flags() == 0
    s.check(before, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(4):
        before, words = simulate()
        graph.replay()
        assert s.ctx.goose_device_flags() == 0
        s.check(before, True)
        assert all(torch.equal(kept[i].cpu(), w) for i, w in enumerate(words))


def test_refusals():
    s = Setup([100, 90], seed=10)
    kept = torch.zeros((1, 2, 2, s.sim.table.shape[1]), dtype=torch.int64, device=DEV)
    good = {"seq": 0, "keep": 50, "sink": 4, "recent": 5}
    call = lambda ev, weight=s.weight, kept=kept: s.ctx.goose_pages_evict(s.cache, ev, weight, kept)  # noqa: E731
    two = torch.cat((kept, kept))
    for ev, kw in [([dict(good, seq=2)], {}), ([dict(good, seq=-1)], {}), ([dict(good, keep=0)], {}), ([dict(good, sink=-1)], {}),
                   ([dict(good, recent=-1)], {}), ([dict(good, sink=46)], {}), ([dict(good, sink=2 ** 31 - 1, recent=2 ** 31 - 1)], {}),
                   ([good, good], {"kept": two}), ([], {"kept": kept[:0]}), ([good], {"kept": two}), ([good], {"kept": kept.int()}),
                   ([good], {"kept": kept[..., :-1]}), ([good], {"weight": s.weight[..., :-64]}), ([good], {"weight": s.weight.double()}),
                   ([good], {"weight": s.weight.cpu()}), ([dict(good, keep=2 ** 40)], {})]:
        with pytest.raises(goose.GooseError) as e:
            call(ev, **kw)
        assert e.value.status == gb.GOOSE_ERR_ARG, (ev, kw)
    for c in ([{"seq": 2, "C": 1}], [{"seq": 0, "C": 0}], [{"seq": 0, "C": 40000}], [{"seq": 0, "C": 1}] * 2, []):
        with pytest.raises(goose.GooseError) as e:
            s.ctx.goose_pages_append(s.cache, c)
        assert e.value.status == gb.GOOSE_ERR_ARG, c
    s.check()
    call([good])
    assert s.ctx.goose_device_flags() == 0


@pytest.mark.parametrize("reposition", [True, False])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
def test_more_streams_than_the_card_has_units(dtype, d, reposition):
    """Four wavefronts a stream of blocks, and one where there are thousands of short ones."""
    for weights in ("random", "ties"):
        s = Setup([700, 333, 65], layers=6, nkv=16 if d == 64 else 8, d=d, dtype=dtype, seed=11, weights=weights)
        s.evict([{"seq": 1, "keep": 300, "sink": 40, "recent": 64}, {"seq": 0, "keep": 129, "sink": 65, "recent": 1}, {"seq": 2, "keep": 64}], reposition)
    for keep in (1, 33, 64, 127):
        s = Setup([130, 192, 129, 128, 191, 7], layers=6, nkv=16 if d == 64 else 8, d=d, dtype=dtype, seed=keep)
        s.evict([{"seq": r, "keep": keep, "sink": min(keep, r), "recent": min(keep - min(keep, r), 3)} for r in range(6)], reposition)


def test_long_sequences_of_many_streams():
    """More pages than a wavefront's lanes, blocks of which nothing stays, a window that ends with the pages."""
    for n, keep, sink, recent in ((4500, 4096, 3, 100), (4500, 70, 64, 2), (8300, 40, 0, 33), (4096, 4000, 4000, 0), (4161, 66, 1, 65)):
        s = Setup([n], layers=9, nkv=15, seed=keep, weights="ties")
        s.evict([{"seq": 0, "keep": keep, "sink": sink, "recent": recent}], reposition=False)
        s = Setup([n, 100], layers=1, nkv=2, seed=keep)
        s.evict([{"seq": 0, "keep": keep, "sink": sink, "recent": recent}])
