"""Pages of a paged cache on the GPU against a simulator of the tables: every entry, length, count and stored bit."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, PageSim, pack_pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(layers=2, heads=2, d=64, n_seqs=6, width=5, n_pages=17, dtype="bf16", max_B=128, seed=0, nh=None):
    desc = goose.ModelDesc(layers, 128, nh or heads, d, 128, 1024, dtype=dtype, n_kv_heads=heads)
    ctx = goose.GooseContext(desc, max_B, 128, 512)
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    k = torch.randn((layers, n_pages, heads, PAGE, d), generator=g).to(dt)
    v = torch.randn((layers, n_pages, heads, PAGE, d), generator=g).to(dt)
    sim = PageSim(n_seqs, width, n_pages, k, v)
    kp, vp = pack_pages(k, v)
    i32 = dict(dtype=torch.int32, device=DEV)
    cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), torch.full((n_seqs, width), 9, **i32), torch.full((n_seqs,), 3, **i32),
                             torch.full((n_pages,), 5, **i32))
    ctx.goose_pages_clear(cache)
    return ctx, cache, sim


def same(cache, sim, what=""):
    torch.cuda.synchronize()
    assert np.array_equal(cache.table.cpu().numpy(), sim.table), what
    assert np.array_equal(cache.len.cpu().numpy(), sim.len), what
    assert np.array_equal(cache.refs.cpu().numpy(), sim.refs), what
    kp, vp = pack_pages(sim.k, sim.v)
    assert torch.equal(cache.kpool.cpu().view(torch.int16), kp.view(torch.int16)), what
    assert torch.equal(cache.vpool.cpu().view(torch.int16), vp.view(torch.int16)), what


def commit(ctx, cache, sim, seqs, paths, B):
    path = torch.full((len(seqs), 128), -1, dtype=torch.int32)
    for r, p in enumerate(paths):
        path[r, :len(p)] = torch.tensor(p)
    path = path.to(DEV)
    L = torch.tensor([len(p) - 1 for p in paths], dtype=torch.int32, device=DEV)
    ctx.goose_pages_commit(cache, [{"seq": q, "B": b, "path": path[r], "accept_len": L[r:]} for r, (q, b) in enumerate(zip(seqs, B))])
    return sim.commit(seqs, paths)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16")])
def test_a_run_of_calls_matches_the_simulator(d, dtype):
    ctx, cache, sim = make(d=d, dtype=dtype)
    same(cache, sim, "clear")
    ctx.goose_pages_reserve(cache, [0], [100])
    assert sim.reserve([0], [100]) == 0
    same(cache, sim, "first reservation")
    commit(ctx, cache, sim, [0], [list(range(100))], [100])
    same(cache, sim, "prompt")
    ctx.goose_pages_fork(cache, 0, [1, 3])
    assert sim.fork(0, [1, 3]) == 0
    ctx.goose_pages_fork(cache, 0, [4], 64)  # ends with a page
    assert sim.fork(0, [4], 64) == 0
    ctx.goose_pages_fork(cache, 0, [5], 0)
    assert sim.fork(0, [5], 0) == 0
    same(cache, sim, "forks")
    # all three sharers of the last page at once: two leave it, the last keeps it
    ctx.goose_pages_reserve(cache, [3, 0, 1, 4], [128, 1, 28, 64])
    assert sim.reserve([3, 0, 1, 4], [128, 1, 28, 64]) == 0
    same(cache, sim, "copies on write")
    commit(ctx, cache, sim, [3, 0, 1], [[0, 3, 4, 9, 11, 40, 41, 63, 64, 100, 101, 127], [0], [0, 1, 2, 27]], [128, 1, 28])
    same(cache, sim, "commit")
    ctx.goose_pages_free(cache, [4, 0])
    sim.free([4, 0])
    same(cache, sim, "free")
    ctx.goose_pages_free(cache, [4, 0, 2])  # empty already
    same(cache, sim, "free again")
    ctx.goose_pages_reserve(cache, [2], [300])
    assert sim.reserve([2], [300]) == 0
    same(cache, sim, "lowest free pages first")
    assert ctx.goose_device_flags() == 0
    ctx.close()


@pytest.mark.parametrize("seed", range(4))
def test_random_runs(seed):
    rng = np.random.default_rng(seed)
    ctx, cache, sim = make(layers=1, heads=1, n_seqs=16, width=6, n_pages=40, seed=seed)
    want = 0
    for step in range(60):
        kind = rng.choice(["reserve", "fork", "commit", "free"], p=[0.45, 0.25, 0.1, 0.2])
        seqs = [int(x) for x in rng.permutation(16)[:rng.integers(1, 9)]]
        if kind == "fork":
            src, dst = seqs[0], seqs[1:] or [(seqs[0] + 1) % 16]
            n = -1 if rng.random() < 0.5 else int(rng.integers(0, 200))
            ctx.goose_pages_fork(cache, src, dst, n)
            want |= sim.fork(src, dst, n)
        elif kind == "free":
            ctx.goose_pages_free(cache, seqs[:2])
            sim.free(seqs[:2])
        else:
            new = [int(x) for x in rng.integers(1, 129, len(seqs))]
            ctx.goose_pages_reserve(cache, seqs, new)
            got = sim.reserve(seqs, new)
            want |= got
            if got == 0:  # a reservation is followed by the commit of an increasing path
                paths = [[0] + sorted(int(x) + 1 for x in rng.permutation(b - 1)[:rng.integers(0, b)]) for b in new]
                commit(ctx, cache, sim, seqs, paths, new)
        same(cache, sim, (seed, step, kind))
    assert ctx.goose_device_flags() == want
    ctx.close()


def test_many_pages_in_one_call():
    """A prompt of more pages than threads, in a pool whose low pages are partly taken."""
    ctx, cache, sim = make(layers=1, heads=1, n_seqs=3, width=2100, n_pages=9001, nh=1)
    for i in (1, 5, 2000):  # a few pages that belong to somebody
        sim.refs[i] = 1
    cache.refs.copy_(torch.from_numpy(sim.refs))
    ctx.goose_pages_reserve(cache, [0, 2], [2050 * 64 + 7, 1900 * 64])
    assert sim.reserve([0, 2], [2050 * 64 + 7, 1900 * 64]) == 0
    same(cache, sim)
    with pytest.raises(goose.GooseError) as e:
        ctx.goose_pages_reserve(cache, [1], [4096 * 64])
    assert e.value.status == gb.GOOSE_ERR_CAPACITY
    ctx.close()


def test_what_cannot_be_done_is_flagged_and_left_undone():
    ctx, cache, sim = make(n_pages=4, width=3)
    for call, args in (("reserve", ([0, 1], [128, 192])),):  # five pages of four: all or nothing
        ctx.goose_pages_reserve(cache, *args)
        assert sim.reserve(*args) == 16
    same(cache, sim)
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    ctx.goose_pages_reserve(cache, [0], [193])  # beyond the table
    same(cache, sim)
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
    ctx.goose_pages_reserve(cache, [0], [70])
    sim.reserve([0], [70])
    commit(ctx, cache, sim, [0], [list(range(70))], [70])
    ctx.goose_pages_fork(cache, 0, [1])
    sim.fork(0, [1])
    ctx.goose_pages_fork(cache, 0, [1, 2])  # 1 is not empty, 2 gets its pages
    assert sim.fork(0, [1, 2]) == 16
    same(cache, sim)
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    ctx.goose_pages_fork(cache, 0, [3], 71)  # longer than the source
    same(cache, sim)
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
    # an entry and a count out of range
    cache.table[1, 1] = 4
    sim.table[1, 1] = 4
    ctx.goose_pages_reserve(cache, [1], [5])
    same(cache, sim)
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    cache.table[1, 1] = -7
    ctx.goose_pages_free(cache, [1])
    torch.cuda.synchronize()
    assert (cache.table[1].cpu() == -1).all() and int(cache.len[1]) == 0
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    # a path longer than the tree leaves the length alone
    L = torch.tensor([9], dtype=torch.int32, device=DEV)
    path = torch.arange(128, dtype=torch.int32, device=DEV)
    ctx.goose_pages_commit(cache, [{"seq": 0, "B": 5, "path": path, "accept_len": L}])
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY and int(cache.len[0]) == 70
    ctx.close()


def test_refusals():
    ctx, cache, _ = make()
    lib, h, pages = ctx.lib, ctx._h, C.byref(cache._c)
    p1 = torch.zeros(256, dtype=torch.int32, device=DEV)
    m1 = torch.zeros(1024, dtype=torch.int64, device=DEV)
    one = [{"seq": 0, "B": 1, "P_max": 0, "path": p1, "accept_len": p1, "pos": p1, "mask": m1}]

    def status(fn, *a, **k):
        with pytest.raises(goose.GooseError) as e:
            fn(*a, **k)
        return e.value.status

    assert status(ctx.goose_pages_reserve, cache, [0, 0], [1, 1]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_reserve, cache, [6], [1]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_reserve, cache, [-1], [1]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_reserve, cache, [0], [0]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_reserve, cache, [0, 1], [1]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_reserve, cache, [], []) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_free, cache, [1, 1]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_fork, cache, 0, [0]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_fork, cache, 6, [0]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_commit, cache, [dict(one[0], path=None)]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_commit, cache, [dict(one[0], accept_len=None)]) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_commit, cache, one * 2) == gb.GOOSE_ERR_ARG
    assert status(ctx.goose_pages_commit, cache, [dict(one[0], B=129)]) == gb.GOOSE_ERR_CAPACITY
    part = torch.zeros((2, 32, 6 * 64), device=DEV)
    q = torch.zeros((32, 256), dtype=torch.bfloat16, device=DEV)
    g = torch.ones(64, dtype=torch.bfloat16, device=DEV)

    def rope(part=part, gq=None, gk=None, reqs=one, q=q, terms=1, layer=0):
        return status(ctx.goose_qk_norm_rope_paged, cache, layer, part, gq, gk, reqs, q, terms)

    assert rope(terms=3) == gb.GOOSE_ERR_ARG
    assert rope(layer=2) == gb.GOOSE_ERR_ARG and rope(layer=-1) == gb.GOOSE_ERR_ARG
    assert rope(gq=g) == gb.GOOSE_ERR_ARG
    assert rope(gq=g.half(), gk=g.half()) == gb.GOOSE_ERR_ARG
    assert rope(q=q[:, :120]) == gb.GOOSE_ERR_ARG and rope(q=q.half()) == gb.GOOSE_ERR_ARG and rope(q=q[:0]) == gb.GOOSE_ERR_ARG
    assert rope(q=q[:, 4:]) == gb.GOOSE_ERR_ARG                                       # alignment
    assert rope(part=part[:, :, :200].contiguous()) == gb.GOOSE_ERR_ARG
    assert rope(part=torch.zeros((17, 32, 6 * 64), device=DEV)) == gb.GOOSE_ERR_ARG
    assert rope(part=part.double()) == gb.GOOSE_ERR_ARG
    assert rope(reqs=[dict(one[0], pos=None)]) == gb.GOOSE_ERR_ARG
    assert rope(reqs=[dict(one[0], P_max=5 * 64)]) == gb.GOOSE_ERR_CAPACITY
    assert rope(reqs=[dict(one[0], P_max=-1)]) == gb.GOOSE_ERR_ARG
    o = torch.zeros((32, 128), dtype=torch.float16, device=DEV)

    def attn(q=q, terms=1, reqs=one, shared=0, o=o, oterms=1, layer=0):
        return status(ctx.goose_attn_paged, cache, layer, q, terms, reqs, shared, o, oterms)

    assert attn(shared=1) == gb.GOOSE_ERR_CAPACITY and attn(shared=-1) == gb.GOOSE_ERR_ARG and attn(shared=6) == gb.GOOSE_ERR_ARG
    assert attn(oterms=2) == gb.GOOSE_ERR_ARG and attn(terms=0) == gb.GOOSE_ERR_ARG
    assert attn(o=o.float()) == gb.GOOSE_ERR_ARG and attn(reqs=[dict(one[0], mask=None)]) == gb.GOOSE_ERR_ARG
    assert attn(reqs=[]) == gb.GOOSE_ERR_ARG
    many = [{"seq": i, "B": 128, "P_max": 0, "mask": m1} for i in range(5)]
    assert attn(q=q.new_zeros((640, 256)), o=o.new_zeros((640, 128)), reqs=many) == gb.GOOSE_ERR_CAPACITY
    # C callers: no context, no descriptor, no arrays
    assert lib.goose_pages_clear(None, pages, None) == gb.GOOSE_ERR_ARG
    assert lib.goose_pages_clear(h, None, None) == gb.GOOSE_ERR_ARG
    assert lib.goose_pages_free(h, pages, None, 1, None) == gb.GOOSE_ERR_ARG
    assert lib.goose_pages_reserve(h, pages, gb._seqs([0]), None, 1, None) == gb.GOOSE_ERR_ARG
    assert lib.goose_pages_commit(h, pages, None, 1, None) == gb.GOOSE_ERR_ARG
    bad = gb._Pages(cache.kpool.data_ptr() + 2, *[x.data_ptr() for x in (cache.vpool, cache.table, cache.len, cache.refs)], 17, 6, 5)
    assert lib.goose_pages_clear(h, C.byref(bad), None) == gb.GOOSE_ERR_ARG
    f32 = goose.GooseContext(goose.ModelDesc(2, 128, 2, 64, 128, 1024, dtype="f32"), 32, 128)
    assert status(f32.goose_pages_clear, cache) == gb.GOOSE_ERR_SHAPE
    assert ctx.goose_device_flags() == 0
    f32.close()
    ctx.close()


def test_two_streams_and_a_graph():
    """Reserve and commit, captured once, take and give back other pages at every replay; on a stream of its own."""
    ctx, cache, sim = make(n_pages=17, width=5)
    st = torch.cuda.Stream()
    path = torch.tensor([0, 2, 5] + [-1] * 125, dtype=torch.int32, device=DEV)
    L = torch.tensor([2], dtype=torch.int32, device=DEV)
    reqs = goose.PagedRequests([{"seq": 0, "B": 40, "path": path, "accept_len": L}])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.goose_pages_reserve(cache, [0], [40])
        ctx.goose_pages_commit(cache, reqs)
    same(cache, sim, "captured, not run")
    for i in range(60):
        with torch.cuda.stream(st):
            graph.replay()
        sim.reserve([0], [40])
        sim.commit([0], [[0, 2, 5]])
        if i == 20:
            st.synchronize()
            ctx.goose_pages_fork(cache, 0, [2])
            sim.fork(0, [2])
            torch.cuda.synchronize()
        if i % 7 == 0:
            same(cache, sim, i)
    same(cache, sim)
    assert ctx.goose_device_flags() == 0
    ctx.close()


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16")])
def test_a_commit_is_done_as_a_whole_or_not_at_all(d, dtype):
    """Slots that were not reserved, in a page of another sequence or in none, paths longer than the tree: rows, lengths and tables stay, also those of the
    sequence that shares the page; a request beside them is committed."""
    ctx, cache, sim = make(d=d, dtype=dtype)
    ctx.goose_pages_reserve(cache, [0], [100])
    sim.reserve([0], [100])
    commit(ctx, cache, sim, [0], [list(range(100))], [100])
    ctx.goose_pages_fork(cache, 0, [1], 70)
    sim.fork(0, [1], 70)
    ctx.goose_pages_reserve(cache, [2], [40])
    sim.reserve([2], [40])
    ctx.goose_pages_fork(cache, 0, [3], 64)
    sim.fork(0, [3], 64)
    same(cache, sim, "before")
    assert ctx.goose_device_flags() == 0

    def refused(seq, path, B, L, flag):
        p = torch.full((128,), -1, dtype=torch.int32)
        p[:len(path)] = torch.tensor(path)
        ctx.goose_pages_commit(cache, [{"seq": seq, "B": B, "path": p.to(DEV), "accept_len": torch.tensor([L], dtype=torch.int32, device=DEV)}])
        same(cache, sim, (seq, path, B, L))
        assert ctx.goose_device_flags() == flag, (seq, path, B, L)

    refused(1, [0, 5], 8, 1, gb.GOOSE_FLAG_PAGES)                  # slot 75 over 71 of a page that sequence 0 has committed rows in
    refused(1, [0], 1, 0, gb.GOOSE_FLAG_PAGES)                     # nothing moves, but slot 70 is sequence 0's
    refused(0, [0, 1, 2], 3, 2, gb.GOOSE_FLAG_PAGES)               # and the other way round
    refused(3, [0, 2], 5, 1, gb.GOOSE_FLAG_PAGES)                  # no page at slot 64
    refused(2, [0] + list(range(70, 128)), 128, 30, gb.GOOSE_FLAG_PAGES)   # destinations reserved, sources not
    refused(2, [0, 3, 9], 2, 2, gb.GOOSE_FLAG_CAPACITY)            # longer than the tree
    refused(2, [0, 3], 9, -1, gb.GOOSE_FLAG_CAPACITY)
    refused(0, list(range(128)), 128, 127, gb.GOOSE_FLAG_PAGES)
    # a refused one beside one that can be done
    path = torch.tensor([[0, 5] + [-1] * 126, [0, 2, 7, 30] + [-1] * 124], dtype=torch.int32, device=DEV)
    L = torch.tensor([1, 3], dtype=torch.int32, device=DEV)
    ctx.goose_pages_commit(cache, [{"seq": 1, "B": 8, "path": path[0], "accept_len": L}, {"seq": 2, "B": 40, "path": path[1], "accept_len": L[1:]}])
    sim.commit([2], [[0, 2, 7, 30]])
    same(cache, sim, "beside")
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    # a fork taken between the reservation and the commit shares the page again: refused until slots are reserved anew
    ctx.goose_pages_reserve(cache, [2], [10])
    sim.reserve([2], [10])
    ctx.goose_pages_fork(cache, 2, [4])
    sim.fork(2, [4])
    refused(2, [0, 3], 10, 1, gb.GOOSE_FLAG_PAGES)
    ctx.goose_pages_reserve(cache, [2], [10])
    sim.reserve([2], [10])
    commit(ctx, cache, sim, [2], [[0, 3]], [10])
    same(cache, sim, "reserved anew")
    # a path that leaves the order is followed up to there
    ctx.goose_pages_reserve(cache, [1], [128])
    sim.reserve([1], [128])
    p = torch.tensor([0, 4, 9, 9, 20] + [-1] * 123, dtype=torch.int32, device=DEV)
    ctx.goose_pages_commit(cache, [{"seq": 1, "B": 128, "path": p, "accept_len": torch.tensor([4], dtype=torch.int32, device=DEV)}])
    sim.commit([1], [[0, 4, 9, 3, 4]])
    same(cache, sim, "malformed")
    ctx.goose_pages_reserve(cache, [1], [128])
    sim.reserve([1], [128])
    long = [0, 2] + list(range(4, 66)) + list(range(67, 126))      # over both halves of the path, into the third page
    commit(ctx, cache, sim, [1], [long], [128])
    same(cache, sim, "long")
    assert ctx.goose_device_flags() == 0
    ctx.close()


def test_a_fork_over_a_hole_is_left_undone():
    """A source with a page missing, out of range or counted as free among its committed ones: no sequence gets any of them; up to the hole it can be forked."""
    ctx, cache, sim = make(width=40, n_pages=60)
    ctx.goose_pages_reserve(cache, [0], [2300])
    sim.reserve([0], [2300])
    cache.len[0] = 2300
    sim.len[0] = 2300
    same(cache, sim)
    for at, value in ((0, -1), (17, 60), (35, -5)):
        good = int(sim.table[0, at])
        cache.table[0, at] = sim.table[0, at] = value
        ctx.goose_pages_fork(cache, 0, [1, 3])
        same(cache, sim, (at, value))
        assert ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
        ctx.goose_pages_fork(cache, 0, [1], at * 64)
        sim.fork(0, [1], at * 64)
        same(cache, sim, (at, value, "up to there"))
        assert ctx.goose_device_flags() == 0
        ctx.goose_pages_free(cache, [1])
        sim.free([1])
        cache.table[0, at] = sim.table[0, at] = good
    cache.refs[int(sim.table[0, 20])] = 0
    sim.refs[sim.table[0, 20]] = 0
    ctx.goose_pages_fork(cache, 0, [2])
    same(cache, sim, "count")
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    ctx.close()
