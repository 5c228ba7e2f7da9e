"""goose_attn_weight_paged against 64-bit sums.

Error bound of a slot's sum: every weight exp(score - lse) errs by its score, (d + 4) 2^-24 sum|q||k| / sqrt(d), by the change to base 2,
2^-22 |lse|, and by the exponential, 2^-20, relative each; the sum over n rows by n 2^-24; a decayed old weight by 2^-22; flushed weights 2^-126 each.
"""
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, pack_pages, rows_of
from prompt_ref import chunk_attention64, slot_weights64
from test_gpu_chunk_attn import Case as AttnCase

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case(AttnCase):
    def setup(self, first=None, bound=None):
        self.place(bound)
        self.first = [0] * len(self.Cs) if first is None else first
        self.chunks = goose.PagedChunks([{"seq": r, "C": c, "P_max": bound or p, "first": f}
                                         for r, (c, p, f) in enumerate(zip(self.Cs, self.Ps, self.first))])
        self.k64 = [rows_of(self.k[self.layer], self.table[r], p + c).double() for r, (c, p) in enumerate(zip(self.Cs, self.Ps))]
        for r, (C, P) in enumerate(zip(self.Cs, self.Ps)):
            at = self.row0[r]
            lse = chunk_attention64(self.q64[at:at + C], self.k64[r], self.k64[r], P)[2]
            self.lse[:, at:at + C] = lse.to(DEV)
        g = torch.Generator().manual_seed(self.seed + 99)
        shape = (self.layers, len(self.Cs), self.nkv, self.cache.table.shape[1] * PAGE)
        self.old = torch.rand(shape, generator=g)
        self.weight = self.old.to(DEV)

    def weigh(self, decay=1.0):
        self.ctx.goose_attn_weight_paged(self.cache, self.layer, self.q, self.terms, self.chunks, self.lse, self.weight, decay)

    def check_weights(self, decay, times=1):
        got = self.weight.cpu()
        lse = self.lse.cpu().double()
        for l in range(self.layers):
            if l != self.layer:
                assert torch.equal(got[l], self.old[l])
        for r, (C, P) in enumerate(zip(self.Cs, self.Ps)):
            at = self.row0[r]
            new, err = slot_weights64(self.q64[at:at + C], self.k64[r], lse[:, at:at + C], P, self.first[r])
            old = self.old[self.layer, r].double()
            w, n = old[:, :P + C].clone(), (C - self.first[r]) * (self.nh // self.nkv)
            for _ in range(times):
                w[:, :P] = (w[:, :P] * decay if decay else 0.0) + new[:, :P]
                w[:, P:] = new[:, P:]
            tol = times * (err + new * (n + 1) * 2.0 ** -24 + w * 2.0 ** -22 + n * 2.0 ** -126)
            x = got[self.layer, r].double()
            bad = ~((x[:, :P + C] - w).abs() <= tol * 1.001)
            assert not bad.any(), (r, bad.nonzero()[0].tolist(), float(x[:, :P + C][bad][0]), float(w[bad][0]), float(tol[bad][0]))
            assert torch.equal(got[self.layer, r, :, P + C:], self.old[self.layer, r, :, P + C:]), "slots behind the chunk"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("terms", [1, 2])
def test_types_and_terms(dtype, d, terms):
    for Cs, Ps in (([37, 1, 70], [130, 64, 261]), ([150, 300], [333, 0])):
        c = Case(4, 2, d, dtype, Cs, Ps, seed=1, terms=terms)
        c.setup()
        c.weigh(0.5)
        c.check_weights(0.5)
        assert c.ctx.goose_device_flags() == 0


@pytest.mark.parametrize("nh,nkv,Cs,Ps,first", [
    (1, 1, [1], [0], [0]), (1, 1, [1], [63], [0]), (2, 1, [2], [63], [1]), (14, 2, [1, 3], [65, 127], [0, 2]), (40, 1, [5], [200], [3]),
    (8, 8, [129, 65], [31, 700], [100, 64]), (8, 2, [32] * 16, [192 + 7 * i for i in range(16)], [2 * i for i in range(16)]),
    (8, 1, [1] * 16, [320 + i for i in range(16)], [0] * 16), (3, 1, [500], [0], [250]), (2, 2, [511, 513], [1, 31], [0, 512]),
    (4, 2, [300], [5000], [268]), (8, 2, [1100], [900], [0]),
])
def test_head_layouts_lengths_and_windows(nh, nkv, Cs, Ps, first):
    for d, dtype in ((128, "bf16"), (64, "f16")):
        c = Case(nh, nkv, d, dtype, Cs, Ps, seed=nh + len(Cs))
        c.setup(first)
        c.weigh()
        c.check_weights(1.0)


@pytest.mark.parametrize("C", [30, 31, 32, 33, 63, 64, 65, 127, 128, 129])
def test_every_end_of_a_tile(C):
    for P in (0, 1, 31, 32, 33, 63, 64, 65):
        c = Case(2, 2, 64, "f16", [C], [P], seed=C)
        c.setup([C // 3])
        c.weigh(0.0)
        c.check_weights(0.0)


def test_the_weights_of_a_row_add_up_to_one():
    """Behind the attention itself: with all tokens counted the weights of a KV head add up to its rows."""
    c = Case(8, 2, 128, "bf16", [200], [500], seed=3, terms=2)
    c.setup()
    c.call()
    c.weight.zero_()
    c.weigh(0.0)
    total = c.weight[0, 0].double().sum(-1).cpu()
    assert ((total - 800).abs() <= 800 * (2.0 ** -19 + 700 * 2.0 ** -23)).all()   # (both roundings of a score, the sums over 700 slots)


def test_old_weights_are_not_read_without_decay():
    c = Case(4, 2, 64, "bf16", [40], [100], seed=4)
    c.setup()
    c.weight.fill_(float("nan"))
    c.old.fill_(0.0)
    c.weigh(0.0)
    c.weight[0, 0, :, 140:] = 0.0
    c.check_weights(0.0)
    # slots of the chunk are new whatever the decay
    c.weight[0, 0, :, 100:] = float("nan")
    c.weight[0, 0, :, :100] = 0.0
    c.weigh(1.0)
    c.weight[0, 0, :, 140:] = 0.0
    c.check_weights(1.0)


def test_junk_behind_a_token_and_rows_that_do_not_count():
    c = Case(4, 2, 64, "f16", [70], [90], seed=5, layers=2, layer=1)
    for s in range(160, 192):
        c.k[1, c.table[0, s // PAGE], :, s % PAGE] = float("nan")
    c.setup([20])
    c.q[:20] = float("nan")
    c.lse[:, :20] = float("nan")
    c.weigh(0.5)
    got = c.weight.clone()
    c.lse[:, :20] = 0.0
    c.check_weights(0.5)
    # a token of which nothing is left weighs nothing; a NaN concerns the slots that the token sees, under its KV head
    c.lse[0, 69] = float("-inf")
    c.weight.copy_(c.old)
    c.weigh(0.5)
    c.check_weights(0.5)
    c.lse[0, 60] = float("nan")
    c.weight.copy_(c.old)
    c.weigh(0.5)
    w = c.weight[1, 0].cpu()
    assert w[0, :151].isnan().all() and w[0, 151:].isfinite().all() and torch.equal(w[1], got[1, 0, 1].cpu())


def test_replays_accumulate():
    c = Case(8, 2, 128, "bf16", [130, 3], [400, 70], seed=6)
    c.setup(bound=700)
    c.weigh(0.75)
    c.weight.copy_(c.old)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.weigh(0.75)
    for i in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        c.check_weights(0.75, times=i)
    want = c.weight.clone()
    c.weight.copy_(c.old)
    for _ in range(3):
        c.weigh(0.75)
    assert torch.equal(c.weight, want) and c.ctx.goose_device_flags() == 0


def test_flags_leave_the_weights_alone():
    c = Case(4, 2, 64, "bf16", [40, 5], [100, 60], seed=7)
    c.setup()
    for n in (-1, 61):
        c.cache.len[1] = n
        c.weight.copy_(c.old)
        c.weigh()
        assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
        assert torch.equal(c.weight[0, 1].cpu(), c.old[0, 1]) and not torch.equal(c.weight[0, 0].cpu(), c.old[0, 0])
    c.cache.len[1] = 60
    c.cache.table[1, 0] = len(c.refs)
    c.weight.copy_(c.old)
    c.weigh()
    assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    assert torch.equal(c.weight[0, 1, :, :64].cpu(), c.old[0, 1, :, :64])


def test_refusals():
    c = Case(4, 2, 64, "bf16", [40], [100], seed=8)
    c.setup()
    ctx, good = c.ctx, [{"seq": 0, "C": 40, "P_max": 100, "first": 3}]
    call = lambda chunks=good, layer=0, q=c.q, terms=1, lse=c.lse, weight=c.weight, decay=1.0: ctx.goose_attn_weight_paged(  # noqa: E731
        c.cache, layer, q, terms, chunks, lse, weight, decay)
    for b in [dict(chunks=[dict(good[0], first=40)]), dict(chunks=[dict(good[0], first=-1)]), dict(layer=1), dict(terms=3), dict(decay=-0.1),
              dict(decay=float("nan")), dict(decay=float("inf")), dict(lse=c.lse[:, :39]), dict(lse=c.lse[:3]), dict(lse=c.lse.half()),
              dict(weight=c.weight[..., :-1]), dict(weight=c.weight.double()), dict(weight=c.weight[:, :, :1]), dict(weight=c.weight.cpu()),
              dict(q=c.q[:39]), dict(chunks=[dict(good[0], C=0)]), dict(chunks=good * 2), dict(chunks=[])]:
        with pytest.raises(goose.GooseError) as e:
            call(**b)
        assert e.value.status == gb.GOOSE_ERR_ARG, b
    with pytest.raises(goose.GooseError) as e:
        call(chunks=[dict(good[0], P_max=10000)])
    assert e.value.status == gb.GOOSE_ERR_CAPACITY
    call()
    c.first = [3]
    c.check_weights(1.0)


def test_many_heads_under_one_and_many_rows():
    """1991 query heads of one KV head x 1200 tokens: the row count times the heads passes 32 bits.  (lse: any numbers serve.)"""
    C, P, first = 1200, 70, 1140
    c = Case(1991, 1, 64, "bf16", [C], [P], seed=9, scale=0.5)
    c.place()
    c.first = [first]
    c.chunks = goose.PagedChunks([{"seq": 0, "C": C, "P_max": P, "first": first}])
    c.lse[:, :C] = torch.linspace(2.0, 6.0, 1991).view(-1, 1) + torch.arange(C).view(1, -1) * 1e-3
    c.k64 = [rows_of(c.k[0], c.table[0], P + C).double()]
    c.old = torch.zeros((1, 1, 1, c.cache.table.shape[1] * PAGE))
    c.weight = c.old.to(DEV)
    c.weigh()
    c.check_weights(1.0)


def test_the_longest_table():
    """2^31 - 64 slots, all of them in one page: every page of 64 entries gets the same sums."""
    slots, C, d = 2 ** 31 - 64, 3, 64
    g = torch.Generator().manual_seed(10)
    k = torch.randn((1, 1, 1, PAGE, d), generator=g).half()
    kp, vp = pack_pages(k, k)
    table = torch.zeros((1, slots // PAGE), dtype=torch.int32, device=DEV)
    P = slots - C
    cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), table, torch.tensor([P], dtype=torch.int32, device=DEV),
                             torch.full((1,), slots // PAGE, dtype=torch.int32, device=DEV))
    ctx = goose.GooseContext(goose.ModelDesc(1, 128, 1, d, 128, 1024, dtype="f16", n_kv_heads=1), 8, 64, 32)
    q = torch.randn((C, d), generator=g).half()
    lse = torch.full((1, C), 3.0)
    weight = torch.full((1, 1, 1, slots), 7.0, device=DEV)
    ctx.goose_attn_weight_paged(cache, 0, q.to(DEV), 1, [{"seq": 0, "C": C, "P_max": P}], lse.to(DEV), weight, 0.0)
    assert ctx.goose_device_flags() == 0
    ctx.close()
    new, err = slot_weights64(q.double().view(C, 1, d), k[0, 0].double().repeat(1, 2, 1), lse.double(), 2 * PAGE - C, 0)
    tol = (err + new * 4 * 2.0 ** -24 + C * 2.0 ** -126) * 1.001
    w = weight.view(-1, PAGE)
    assert ((w[0].cpu().double() - new[0, :PAGE]).abs() <= tol[0, :PAGE]).all()
    assert ((w[-1].cpu().double() - new[0, PAGE:]).abs() <= tol[0, PAGE:]).all()
    for at in range(0, w.shape[0] - 1, 1 << 22):
        assert (w[at:min(at + (1 << 22), w.shape[0] - 1)] == w[0]).all()


def test_more_rows_under_a_head_than_are_counted():
    """2^30 rows at most; refused before anything is looked at."""
    n = 32769
    c = Case(4, 2, 64, "bf16", [40], [100], seed=8)
    c.setup()
    table = torch.zeros((1, 600), dtype=torch.int32, device=DEV)
    pool = torch.zeros((1, 1, 1, PAGE * 64), dtype=torch.bfloat16, device=DEV)
    one = torch.ones(1, dtype=torch.int32, device=DEV)
    cache = goose.PagedCache(pool, pool.clone(), table, one * 0, one)
    ctx = goose.GooseContext(goose.ModelDesc(1, 128, n, 64, 128, 1024, dtype="bf16", n_kv_heads=1), 1, 64, 32)
    chunks = goose.PagedChunks([{"seq": 0, "C": 32768, "P_max": 0}])
    at = c.q.data_ptr()
    rc = ctx.lib.goose_attn_weight_paged(ctx._h, cache._ref, 0, at, n * 64, 1, chunks._c, 1, at, 32768, 1.0, at, 0)
    assert rc == gb.GOOSE_ERR_CAPACITY
    rc = ctx.lib.goose_attn_chunk_paged(ctx._h, cache._ref, 0, at, n * 64, 1, chunks._c, 1, at, n * 64, gb.GOOSE_DTYPE_BF16, 1, 0, 0, 0)
    assert rc == gb.GOOSE_ERR_CAPACITY
    ctx.close()


@pytest.mark.parametrize("dtype,d,terms", [("bf16", 128, 2), ("f16", 64, 1), ("f16", 128, 1), ("bf16", 64, 2)])
def test_rows_in_parts(dtype, d, terms):
    """Many rows over few pages: parts of the rows, joined afterwards."""
    for nh, nkv, Cs, Ps, first, bound in ((4, 2, [900], [0], [0], None), (8, 1, [600, 3, 700], [70, 900, 0], [5, 0, 699], None), (4, 4, [520, 513], [64, 63], [0, 500], 2000),
                                          (2, 1, [1025], [640], [0], 800)):
        for decay in (0.0, 0.75):
            c = Case(nh, nkv, d, dtype, Cs, Ps, seed=11, terms=terms)
            c.setup(first, bound)
            c.weigh(decay)
            assert c.ctx.goose_device_flags() == 0
            c.check_weights(decay)


def test_rows_in_parts_flags_and_a_graph():
    c = Case(8, 2, 128, "f16", [800, 1], [200, 100], seed=12)
    c.setup(bound=400)
    c.weigh(0.5)
    want = c.weight.clone()
    c.check_weights(0.5)
    # a page out of range: its slots stay, and the others are the same bits
    old = int(c.cache.table[0, 4])
    c.cache.table[0, 4] = -1
    c.weight.copy_(c.old)
    c.weigh(0.5)
    assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    got = c.weight.clone()
    assert torch.equal(got[0, 0, :, 256:320].cpu(), c.old[0, 0, :, 256:320])
    got[0, 0, :, 256:320] = want[0, 0, :, 256:320]
    assert torch.equal(got, want)
    c.cache.table[0, 4] = old
    for n in (-1, 401):
        c.cache.len[0] = n
        c.weight.copy_(c.old)
        c.weigh(0.5)
        assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
        assert torch.equal(c.weight[0, 0].cpu(), c.old[0, 0]) and torch.equal(c.weight[0, 1], want[0, 1])
    c.cache.len[0] = 200
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.weigh(0.5)
    for _ in range(3):
        c.weight.copy_(c.old)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.weight, want)
        # what the context's workspace holds in between does not matter
        c.call(lse=False)
        torch.cuda.synchronize()
