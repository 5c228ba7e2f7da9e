"""goose_attn_chunk_paged against 64-bit attention: head layouts, lengths, strides, several chunks, and what lies behind a token.

Error bound of one output, with A = sum p |v| / sum p and u_o half a step of the output's type:
  * probabilities are rounded before the second product, one term of the cache's type where the output keeps no more bits (bf16 2^-8 A, fp16
    2^-11 A), two terms otherwise (2^-16 A, 2^-21 A); under fp16 besides 2^-25 each below its normals, sum|v| 2^-25 in all;
  * a score errs by (d + 4) 2^-24 sum|q||k| / sqrt(d), which moves a probability by that relative amount and the quotient by twice it;
    exponentials, rescales and the final product add 2^-20 A; sums over N keys N 2^-24 A, twice;
  * the store: u_o |o| (two terms: u_o^2), fp16 2^-25.
The logarithm: the score's error, N 2^-24 + 2^-20 of the sum, 2^-22 |lse|.
"""
import numpy as np
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, pack_pages, rows_of
from prompt_ref import chunk_attention64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF = torch.bfloat16, torch.float16
U = {t: torch.finfo(t).eps / 2 for t in (BF, HF)}


def weight_rounding(dt, o_dtype, o_terms):
    one = o_terms == 1 and (o_dtype == BF or dt == HF)
    return {BF: 2.0 ** -8, HF: 2.0 ** -11}[dt] if one else {BF: 2.0 ** -16, HF: 2.0 ** -21}[dt]


class Case:
    def __init__(self, nh, nkv, d, dtype, Cs, Ps, seed=0, terms=1, o_dtype=HF, o_terms=1, layers=1, layer=0, scale=1.5, shared=0):
        self.__dict__.update(locals())
        g = torch.Generator().manual_seed(seed)
        self.dt = dt = BF if dtype == "bf16" else HF
        counts = [(p + c + PAGE - 1) // PAGE for p, c in zip(Ps, Cs)]
        self.width, n_pages = max(counts) + 1, sum(counts) + 2
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table, self.refs, at = np.full((len(Cs), self.width), -1, np.int32), np.zeros(n_pages, np.int32), shared
        for r, c in enumerate(counts):
            row = order[:shared] + order[at:at + c - shared]
            at += c - shared
            self.table[r, :c] = row
            self.refs[row] += 1
        self.k = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(dt)
        self.v = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(dt)
        self.row0 = np.cumsum([0] + [(c + 31) // 32 * 32 for c in Cs]).tolist()
        self.rows = self.row0[-2] + Cs[-1]
        self.q32 = torch.randn((self.rows, nh, d), generator=g) * scale

    def q_rows(self):
        hi = self.q32.to(self.dt)
        if self.terms == 1:
            return hi.reshape(self.rows, -1), hi.double()
        lo = (self.q32 - hi.float()).to(self.dt)
        n = self.nh * self.d
        both = torch.stack((hi.view(self.rows, n // 8, 8), lo.view(self.rows, n // 8, 8)), 2)
        return both.reshape(self.rows, 2 * n), hi.double() + lo.double()

    def place(self, bound=None, max_rows=512):
        table = self.table
        if bound is not None:
            table = np.full((len(self.Cs), (bound + max(self.Cs)) // PAGE + 1), -1, np.int32)
            table[:, :self.width] = self.table
        q, self.q64 = self.q_rows()
        desc = goose.ModelDesc(self.layers, 128, self.nh, self.d, 128, 1024, dtype=self.dtype, n_kv_heads=self.nkv)
        self.ctx = goose.GooseContext(desc, 128, 256, max_rows)
        kp, vp = pack_pages(self.k, self.v)
        self.cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), torch.from_numpy(table).to(DEV),
                                      torch.tensor(self.Ps, dtype=torch.int32, device=DEV), torch.from_numpy(self.refs).to(DEV))
        self.cols = self.nh * self.d * self.o_terms
        # rows further apart than their columns; the logarithms too
        self.q = torch.full((self.rows, q.shape[1] + 8), 55.0, dtype=self.dt, device=DEV)
        self.q[:, :q.shape[1]] = q.to(DEV)
        self.o = torch.full((self.rows + 3, self.cols + 8), 77.0, dtype=self.o_dtype, device=DEV)
        self.lse = torch.full((self.nh, self.rows + 5), 77.0, device=DEV)
        self.chunks = goose.PagedChunks([{"seq": r, "C": c, "P_max": bound or p} for r, (c, p) in enumerate(zip(self.Cs, self.Ps))])

    def call(self, lse=True):
        self.ctx.goose_attn_chunk_paged(self.cache, self.layer, self.q, self.terms, self.chunks, self.o, self.o_terms, self.lse if lse else None)

    def run(self, flags=0, bound=None, lse=True, max_rows=512):
        self.place(bound, max_rows)
        self.call(lse)
        assert self.ctx.goose_device_flags() == flags
        self.ctx.close()
        return self.o.cpu(), self.lse.cpu()

    def check(self, out, lse=True, heads=None):
        o, got_lse = out
        assert (o[:, self.cols:] == 77).all() and (o[self.rows:] == 77).all() and (got_lse[:, self.rows:] == 77).all()
        N, u, uo = self.nh * self.d, weight_rounding(self.dt, self.o_dtype, self.o_terms), U[self.o_dtype] ** self.o_terms
        pick = list(range(self.nh)) if heads is None else heads
        G = self.nh // self.nkv
        for r, (C, P) in enumerate(zip(self.Cs, self.Ps)):
            at = self.row0[r]
            k = rows_of(self.k[self.layer], self.table[r], P + C).double()[[h // G for h in pick]]
            v = rows_of(self.v[self.layer], self.table[r], P + C).double()[[h // G for h in pick]]
            want, A, want_lse, qk, vs = chunk_attention64(self.q64[at:at + C][:, pick], k, v, P)
            got = o[at:at + C, :self.cols].double()
            if self.o_terms == 2:
                got = got.view(C, N // 8, 2, 8).sum(2)
            got = got.reshape(C, self.nh, self.d)[:, pick]
            e_s = (self.d + 4) * 2.0 ** -24 * qk
            n = (P + C) * 2.0 ** -24 + 2.0 ** -20
            tol = A * (u + 2 * e_s.unsqueeze(-1) + 2 * n) + uo * want.abs() + 2.0 ** -25
            if self.dt == HF:
                tol = tol + vs * 2.0 ** -25
            same = (want.isnan() & got.isnan()) | (want == got)
            bad = ~((got - want).abs() <= tol * 1.001) & ~same
            assert not bad.any(), (r, bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]), float(tol[bad][0]))
            if lse:
                gl, tl = got_lse[pick, at:at + C].double(), e_s.T + n + 2.0 ** -22 * want_lse.abs()
                bad = ~((gl - want_lse).abs() <= tl * 1.001) & ~((want_lse.isnan() & gl.isnan()) | (want_lse == gl))
                assert not bad.any(), ("lse", r, bad.nonzero()[0].tolist(), float(gl[bad][0]), float(want_lse[bad][0]))
            else:
                assert (got_lse == 77).all()
            end = self.row0[r + 1] if r + 1 < len(self.Cs) else self.rows
            assert (o[at + C:end] == 77).all() and (got_lse[:, at + C:end] == 77).all(), "rows between chunks"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("terms", [1, 2])
def test_types_and_terms(dtype, d, terms):
    for o_dtype, o_terms in ((HF, 1), (BF, 1), (BF, 2), (HF, 2)):
        for Cs, Ps in (([37, 1, 70], [130, 64, 261]), ([150, 300], [333, 0])):
            c = Case(4, 2, d, dtype, Cs, Ps, seed=1, terms=terms, o_dtype=o_dtype, o_terms=o_terms)
            c.check(c.run())


@pytest.mark.parametrize("nh,nkv,Cs,Ps", [
    (1, 1, [1], [0]), (1, 1, [1], [1]), (2, 1, [2], [63]), (4, 4, [1], [64]), (14, 2, [1, 3], [65, 127]), (40, 1, [5], [200]),
    (8, 2, [128], [0]), (8, 8, [129, 65], [31, 700]), (8, 2, [32] * 16, [192 + 7 * i for i in range(16)]),
    (8, 1, [1] * 16, [320 + i for i in range(16)]), (6, 3, [64, 64, 33], [127, 128, 129]), (4, 4, [1, 257, 1], [64, 64, 64]),
    (3, 1, [500], [0]), (2, 2, [511, 513], [1, 31]), (5, 1, [1, 400, 7], [1000, 3, 0]), (8, 2, [1, 2, 3, 300], [2000, 0, 63, 500]),
])
def test_head_layouts_and_lengths(nh, nkv, Cs, Ps):
    for d, dtype in ((128, "bf16"), (64, "f16")):
        c = Case(nh, nkv, d, dtype, Cs, Ps, seed=nh + len(Cs))
        c.check(c.run(), heads=sorted({0, nh // 2, nh - 1}))


@pytest.mark.parametrize("C", list(range(30, 36)) + list(range(62, 67)) + list(range(126, 131)) + [255, 256, 257])
def test_every_end_of_a_tile(C):
    for P in (0, 1, 31, 32, 33, 63, 64, 65):
        c = Case(2, 2, 64, "f16", [C], [P], seed=C)
        c.check(c.run())


@pytest.mark.parametrize("blocks", range(1, 14))
def test_every_number_of_blocks(blocks):
    for dtype, o in (("f16", HF), ("bf16", BF), ("bf16", HF)):
        c = Case(4, 1, 128, dtype, [130], [blocks * 32 - 31 + 7 * blocks % 32], seed=blocks, o_dtype=o)
        c.check(c.run())


def test_long_prefix_over_many_pages():
    """More than 64 pages in a table, splits of few rows, and a chunk of many."""
    for Cs, Ps, heads in (([3], [9000], [0, 3]), ([300], [8300], [1]), ([1, 260], [12000, 4500], [2])):
        c = Case(4, 2, 128, "f16", Cs, Ps, seed=6)
        c.check(c.run(), heads=heads)


def test_a_long_chunk():
    """More rows than a context's passes have."""
    c = Case(8, 2, 64, "bf16", [2500], [77], seed=7, terms=2)
    c.check(c.run(max_rows=128), heads=[5])


def test_another_layer_and_pages_of_several_sequences():
    c = Case(4, 2, 64, "f16", [40, 200, 3], [130, 128, 190], layers=3, layer=2, shared=2, seed=8)
    c.check(c.run())


def test_bounds_above_the_lengths_and_no_logarithms():
    c = Case(8, 2, 128, "bf16", [70, 1, 200], [100, 500, 0], seed=9)
    c.check(c.run(bound=3000))
    c = Case(8, 2, 128, "bf16", [70, 1, 200], [100, 500, 0], seed=9)
    c.check(c.run(lse=False), lse=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Cs,Ps", [([70, 5], [100, 33]), ([300], [65])])
def test_what_lies_behind_a_token_has_no_effect(dtype, Cs, Ps):
    """NaN and infinities in slots behind the chunk, and in rows of the chunk that earlier tokens do not see."""
    plain = Case(4, 2, 128, dtype, Cs, Ps, seed=10)
    want = plain.run()
    c = Case(4, 2, 128, dtype, Cs, Ps, seed=10)
    for r, (C, P) in enumerate(zip(Cs, Ps)):
        last = (P + C + PAGE - 1) // PAGE
        for s in range(P + C, last * PAGE):
            c.k[0, c.table[r, s // PAGE], :, s % PAGE] = float("nan")
            c.v[0, c.table[r, s // PAGE], :, s % PAGE] = float("inf") if s % 2 else float("nan")
    got = c.run()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    # a value row of the last token: all rows in front of it are the same numbers
    C, P = Cs[0], Ps[0]
    s = P + C - 1
    c.v[0, c.table[0, s // PAGE], :, s % PAGE] = float("nan")
    got = c.run()
    assert got[0][C - 1, :c.cols].isnan().all() and torch.equal(want[0][:C - 1], got[0][:C - 1]) and torch.equal(want[1], got[1])
    c.v[0, c.table[0, s // PAGE], :, s % PAGE] = 0
    c.v[0, c.table[0, s // PAGE], 0, s % PAGE, 5] = float("-inf")
    c.k[0, c.table[0, s // PAGE], 1, s % PAGE] = float("nan")
    got = c.run()
    c.check(got)
    o = got[0][:C, :c.cols].view(C, 4, 128)
    assert (o[C - 1, :2, 5] == -float("inf")).all() and o[C - 1, 2:].isnan().all() and o[:C - 1].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_maxima_that_grow_in_every_block(dtype):
    """Keys whose scores rise block by block, by less and by more than a maximum is left behind; and fall."""
    for step in (0.6, 5.0, -5.0):
        c = Case(2, 1, 64, dtype, [200], [300], seed=11, scale=1.0, o_dtype=BF if dtype == "bf16" else HF)
        c.q32 = torch.ones_like(c.q32) + 0.01 * c.q32
        for s in range(500):
            c.k[0, c.table[0, s // PAGE], :, s % PAGE] = c.k[0, c.table[0, s // PAGE], :, s % PAGE] * 0.1 + step * (s // 32) / 8.0
        c.check(c.run())


def test_scores_of_minus_infinity():
    """Keys of -infinity over whole blocks count for nothing; a token that sees only such is zero, its logarithm -infinity."""
    for first in (32, 70, 200):
        c = Case(2, 2, 64, "bf16", [150], [100], seed=12)
        c.q32 = c.q32.abs() + 0.1
        for s in range(first):
            c.k[0, c.table[0, s // PAGE], :, s % PAGE] = float("-inf")
        o, lse = c.run()
        n = max(0, first - 100)
        assert (o[:n, :c.cols] == 0).all() and (lse[:, :n] == float("-inf")).all()
        c.check((o, lse))


def test_infinite_and_nan_scores():
    c = Case(2, 1, 64, "bf16", [60], [70], seed=13)
    c.q32 = c.q32.abs() + 0.1
    c.k[0, c.table[0, 0], :, 10] = float("inf")
    o, lse = c.run()
    assert o[:60, :c.cols].isnan().all()
    c.k[0, c.table[0, 0], :, 10] = float("nan")
    o, lse = c.run()
    assert o[:60, :c.cols].isnan().all() and lse[:, :60].isnan().all()


def test_large_scores_and_one_dominating_key():
    for scale in (40.0, 4000.0):
        c = Case(4, 4, 128, "bf16", [90], [140], seed=14, scale=scale)
        c.check(c.run())
    c = Case(2, 2, 64, "f16", [140], [300], seed=15, scale=60000.0 / 6)
    c.check(c.run())


def test_the_same_bits_again_and_on_another_stream():
    c = Case(8, 2, 128, "bf16", [300, 1, 45], [700, 2000, 0], seed=16, terms=2)
    c.place()
    c.call()
    torch.cuda.synchronize()
    want = c.o.clone(), c.lse.clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        c.o.fill_(77.0)
        c.lse.fill_(77.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            c.call()
        side.synchronize()
        assert torch.equal(c.o, want[0]) and torch.equal(c.lse, want[1])


def test_a_graph_follows_the_lengths():
    """Captured with bounds: replays go by the lengths and tables on the device."""
    c = Case(4, 2, 128, "f16", [100, 2], [800, 600], seed=17)
    c.place(bound=900)
    c.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call()
    for Ps in ([800, 600], [0, 1], [500, 598], [800, 600]):
        c.Ps = Ps
        c.cache.len.copy_(torch.tensor(Ps, dtype=torch.int32))
        c.o.fill_(77.0)
        c.lse.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = c.o.cpu(), c.lse.cpu()
        c.check(replayed)
        c.call()
        assert c.ctx.goose_device_flags() == 0
        assert torch.equal(c.o.cpu(), replayed[0]) and torch.equal(c.lse.cpu(), replayed[1])


def test_flags():
    c = Case(4, 2, 64, "bf16", [40, 5], [100, 60], seed=18)
    c.Ps = [100, 61]
    c.place()
    c.cache.len[1] = 62
    c.call()
    assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
    c.cache.len[1] = -1
    c.call()
    assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
    c.cache.len[1] = 61
    c.cache.table[0, 0] = len(c.refs)
    c.call()
    assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    c.cache.table[0, 0] = -1
    c.call()
    assert c.ctx.goose_device_flags() == gb.GOOSE_FLAG_PAGES
    c.cache.table[0, 0] = int(c.table[0, 0])
    c.call()
    assert c.ctx.goose_device_flags() == 0


def test_refusals():
    c = Case(4, 2, 64, "bf16", [40, 5], [100, 60], seed=19)
    c.place()
    ctx, good = c.ctx, [{"seq": 0, "C": 40, "P_max": 100}, {"seq": 1, "C": 5, "P_max": 60}]
    call = lambda chunks, layer=0, q=c.q, terms=1, o=c.o, o_terms=1, lse=c.lse: ctx.goose_attn_chunk_paged(  # noqa: E731
        c.cache, layer, q, terms, chunks, o, o_terms, lse)
    cap = c.cache.table.shape[1] * PAGE
    bad = [dict(chunks=[]), dict(chunks=good * 9), dict(chunks=[good[0], dict(good[1], seq=0)]), dict(chunks=[dict(good[0], seq=2)]),
           dict(chunks=[dict(good[0], seq=-1)]), dict(chunks=[dict(good[0], C=0)]), dict(chunks=[dict(good[0], C=32769)]),
           dict(chunks=[dict(good[0], P_max=-1)]), dict(chunks=[dict(good[0], seq=1 << 32)]), dict(layer=1), dict(layer=-1), dict(terms=0),
           dict(terms=3), dict(o_terms=3), dict(q=c.q[:20]), dict(o=c.o[:20]), dict(o=c.o.float()), dict(q=c.q.half()), dict(lse=c.lse.double()),
           dict(lse=c.lse[:3]), dict(lse=c.lse[:, :20]), dict(lse=c.lse.t()), dict(q=c.q[:, 4:]), dict(o=c.o[:, 4:]), dict(o=c.o.cpu()),
           dict(q=c.q.t()), dict(chunks=goose.PagedRequests([{"seq": 0, "B": 1}]))]
    for b in bad:
        with pytest.raises(goose.GooseError) as e:
            call(**dict(dict(chunks=good), **b))
        assert e.value.status == gb.GOOSE_ERR_ARG, b
    with pytest.raises(goose.GooseError) as e:
        call([dict(good[0], P_max=cap - 39)])
    assert e.value.status == gb.GOOSE_ERR_CAPACITY
    call([dict(good[0], P_max=cap - 40)])
    assert ctx.goose_device_flags() == 0


@pytest.mark.parametrize("nh,nkv,C", [(8, 2, 64), (8, 2, 65), (8, 1, 32), (8, 1, 33), (4, 4, 32), (4, 4, 33), (6, 2, 85), (6, 2, 86), (512, 2, 1), (514, 2, 1)])
def test_both_sides_of_few_rows(nh, nkv, C):
    for Cs, Ps in (([C], [1500]), ([C, 1, 200, C], [70, 900, 33, 0])):
        c = Case(nh, nkv, 64, "bf16", Cs, Ps, seed=C)
        c.check(c.run(), heads=sorted({0, nh // 2, nh - 1}))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("terms,o_terms", [(1, 1), (2, 1), (2, 2)])
def test_odd_values_where_the_keys_are_split(dtype, d, terms, o_terms):
    """NaN and infinities among the values of a long prefix, in a slot in the midst of the chunk and in its last one: only rows that see them have them."""
    want = Case(4, 2, d, dtype, [290], [2501], seed=20, terms=terms, o_terms=o_terms)
    o = want.run()[0]
    for slot in (5, 1300, 2500, 2600, 2790):
        c = Case(4, 2, d, dtype, [290], [2501], seed=20, terms=terms, o_terms=o_terms)
        c.v[0, c.table[0, slot // PAGE], 0, slot % PAGE, 7] = float("nan")
        c.v[0, c.table[0, slot // PAGE], 1, slot % PAGE, 9] = float("inf") if o_terms == 1 else float("nan")   # (two terms of infinity add up to NaN)
        got = c.run()
        c.check(got)
        first = max(0, slot - 2501)
        assert torch.equal(got[0][:first], o[:first])
        x = got[0][first:290, :c.cols].view(-1, 4 * d // 8, o_terms, 8)[:, :, 0].reshape(-1, 4, d)
        assert x[:, :2, 7].isnan().all() and (x[:, 2:, 9].isinf() if o_terms == 1 else x[:, 2:, 9].isnan()).all() and int((~x.isfinite()).sum()) == 4 * x.shape[0]


# A bound of more than 256 blocks: workgroups of eight wavefronts and the longer ring, whatever the lengths.
LONG = 8400


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("terms,o_dtype,o_terms", [(1, HF, 1), (2, HF, 2), (2, BF, 1), (1, BF, 2)])
def test_the_longer_ring_types_and_terms(dtype, d, terms, o_dtype, o_terms):
    for Cs, Ps in (([37, 1, 70], [130, 64, 261]), ([150, 300], [333, 0])):
        c = Case(4, 1, d, dtype, Cs, Ps, seed=21, terms=terms, o_dtype=o_dtype, o_terms=o_terms)
        c.check(c.run(bound=LONG))


@pytest.mark.parametrize("blocks", range(1, 14))
def test_the_longer_ring_every_number_of_blocks(blocks):
    for dtype, o in (("f16", HF), ("bf16", HF)):
        c = Case(4, 1, 128, dtype, [130], [blocks * 32 - 31 + 7 * blocks % 32], seed=blocks, o_dtype=o)
        c.check(c.run(bound=LONG))


@pytest.mark.parametrize("C", [65, 127, 128, 129, 255, 256, 257])
def test_the_longer_ring_every_end_of_a_tile(C):
    for P in (0, 31, 32, 33, 1000):
        c = Case(4, 2, 64, "f16", [C], [P], seed=C)
        c.check(c.run(bound=LONG))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_the_longer_ring_odd_values(dtype):
    o = Case(4, 2, 128, dtype, [290], [2501], seed=22).run(bound=LONG)[0]
    for slot in (5, 2500, 2600, 2790):
        c = Case(4, 2, 128, dtype, [290], [2501], seed=22)
        c.v[0, c.table[0, slot // PAGE], 0, slot % PAGE, 7] = float("nan")
        for s in range(2791, 2816):
            c.k[0, c.table[0, s // PAGE], :, s % PAGE] = float("nan")
            c.v[0, c.table[0, s // PAGE], :, s % PAGE] = float("inf")
        got = c.run(bound=LONG)
        c.check(got)
        assert torch.equal(got[0][:max(0, slot - 2501)], o[:max(0, slot - 2501)])


def test_all_at_once_and_more_than_fit():
    """Work items in pairs (more than 256, at most 512), with one range of the keys and with several, and in rounds."""
    for nh, nkv, C, P in ((8, 8, 4200, 0), (4, 4, 2100, 1500), (24, 8, 1500, 700), (16, 16, 4097, 31)):
        c = Case(nh, nkv, 64, "f16", [C], [P], seed=C)
        c.check(c.run(), heads=[0, nh - 1])
