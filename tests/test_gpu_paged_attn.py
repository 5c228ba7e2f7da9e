"""goose_attn_paged against 64-bit attention: head layouts, lengths, shared prefixes, masks, and what lies behind them.

Error bound of one output, u_o = half a step of the output's type: with A = sum p |v| / sum p,
  * probabilities are rounded before the second product: fp16 2^-11 A and 2^-25 each below its normals, sum|v| 2^-25 in all, as the
    largest probability of a row is one in the item that holds it and every rescale only shrinks both; bf16 in two terms, 2^-16 A;
  * a score errs by (d + 4) 2^-24 sum|q||k| / sqrt(d) (products exact in 32 bits, d additions, scale), which moves a probability by the same relative
    amount and the quotient by twice that: 2 A (d + 4) 2^-24 max sum|q||k|/sqrt(d); exponentials and rescales add 2^-20 A;
  * sums over N keys: N 2^-24 A, twice;
  * the store: u_o |o| (two terms: u_o^2), fp16 2^-25.
"""
import math

import numpy as np
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, attention64, mask_words, pack_pages, rows_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U_P = {torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -11}
U = {torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2, torch.float16: torch.finfo(torch.float16).eps / 2}


def parents(B, rng):
    return [-1] + [int(rng.integers(0, i)) if rng.random() < 0.5 else i - 1 for i in range(1, B)]


class Case:
    def __init__(self, nh, nkv, d, dtype, Bs, Ps, S, seed=0, terms=1, o_dtype=torch.float16, o_terms=1, layers=1, layer=0, scale=1.5):
        self.__dict__.update(locals())
        rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.dt = dt = torch.bfloat16 if dtype == "bf16" else torch.float16
        n_sh = S // PAGE
        counts = [(p + b + PAGE - 1) // PAGE for p, b in zip(Ps, Bs)]
        self.width, n_pages = max(counts) + 1, n_sh + sum(c - n_sh for c in counts) + 2
        order = torch.randperm(n_pages, generator=g).tolist()
        self.table, self.refs, at = np.full((len(Bs), self.width), -1, np.int32), np.zeros(n_pages, np.int32), n_sh
        for r, c in enumerate(counts):
            row = order[:n_sh] + order[at:at + c - n_sh]
            at += c - n_sh
            self.table[r, :c] = row
            self.refs[row] += 1
        self.k = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(dt)
        self.v = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(dt)
        self.rows = sum((b + 31) // 32 * 32 for b in Bs)
        self.q32 = torch.randn((self.rows, nh, d), generator=g) * scale
        self.masks = [mask_words(parents(b, rng)) for b in Bs]

    def q_rows(self):
        hi = self.q32.to(self.dt)
        if self.terms == 1:
            return hi.reshape(self.rows, -1), hi.double()
        lo = (self.q32 - hi.float()).to(self.dt)
        n = self.nh * self.d
        both = torch.stack((hi.view(self.rows, n // 8, 8), lo.view(self.rows, n // 8, 8)), 2)
        return both.reshape(self.rows, 2 * n), hi.double() + lo.double()

    def run(self, S=None, flags=0, bound=None):
        """bound: P_max of all requests instead of their lengths (launches go by it; the tables are widened to hold it)."""
        S = self.S if S is None else S
        table = self.table
        if bound is not None:
            table = np.full((len(self.Bs), (bound + max(self.Bs)) // PAGE + 1), -1, np.int32)
            table[:, :self.width] = self.table
        q, self.q64 = self.q_rows()
        desc = goose.ModelDesc(self.layers, 128, self.nh, self.d, 128, 1024, dtype=self.dtype, n_kv_heads=self.nkv)
        ctx = goose.GooseContext(desc, max(self.Bs), 256, 512)
        kp, vp = pack_pages(self.k, self.v)
        self.cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), torch.from_numpy(table).to(DEV),
                                      torch.tensor(self.Ps, dtype=torch.int32, device=DEV), torch.from_numpy(self.refs).to(DEV))
        o = torch.full((self.rows, self.nh * self.d * self.o_terms + 8), 77.0, dtype=self.o_dtype, device=DEV)
        reqs = [{"seq": r, "B": b, "P_max": bound or p, "mask": self.masks[r][0].to(DEV)} for r, (b, p) in enumerate(zip(self.Bs, self.Ps))]
        ctx.goose_attn_paged(self.cache, self.layer, q.to(DEV), self.terms, reqs, S // PAGE, o, self.o_terms)
        assert ctx.goose_device_flags() == flags
        ctx.close()
        o = o.cpu()
        assert (o[:, self.nh * self.d * self.o_terms:] == 77).all()
        return o[:, :self.nh * self.d * self.o_terms]

    def check(self, o, nodes=None):
        at, N = 0, self.nh * self.d
        u, uo = U_P[self.dt], U[self.o_dtype] ** self.o_terms
        for r, (B, P) in enumerate(zip(self.Bs, self.Ps)):
            k = rows_of(self.k[self.layer], self.table[r], P + B).double()
            v = rows_of(self.v[self.layer], self.table[r], P + B).double()
            pick = list(range(B)) if nodes is None or B <= nodes else sorted({0, B - 1, *range(1, B, max(1, B // nodes))})
            see = np.concatenate([np.ones((B, P), bool), self.masks[r][1]], 1)
            want, A, qk, vs = attention64(self.q64[at:at + B][pick], k, v, torch.from_numpy(see[pick]))
            got = o[at:at + B].double()
            if self.o_terms == 2:
                got = got.view(B, N // 8, 2, 8).sum(2)
            got = got.reshape(B, self.nh, self.d)[pick]
            tol = A * (u + 2 * (self.d + 4) * 2.0 ** -24 * qk.unsqueeze(-1) + 2.0 ** -20 + 2 * (P + B) * 2.0 ** -24) + uo * want.abs() + 2.0 ** -25
            if self.dt == torch.float16:
                tol = tol + vs * 2.0 ** -25
            bad = ~((got - want).abs() <= tol * 1.001) & ~(want.isnan() & got.isnan())
            assert not bad.any(), (r, bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]), float(tol[bad][0]))
            assert (o[at + B:at + (B + 31) // 32 * 32] == 77).all(), "rows between requests"
            at += (B + 31) // 32 * 32


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("terms", [1, 2])
def test_types_and_terms(dtype, d, terms):
    for o_dtype, o_terms in ((torch.float16, 1), (torch.bfloat16, 2)):
        c = Case(4, 2, d, dtype, [21, 1, 40], [130, 128, 261], 128, seed=1, terms=terms, o_dtype=o_dtype, o_terms=o_terms)
        c.check(c.run())


@pytest.mark.parametrize("nh,nkv,Bs,Ps,S", [
    (1, 1, [1], [0], 0), (1, 1, [1], [1], 0), (2, 1, [2], [63], 0), (4, 4, [1], [64], 64), (14, 2, [1, 3], [65, 127], 64), (40, 1, [5], [200], 0),
    (8, 2, [128], [0], 0), (8, 8, [128, 65], [31, 700], 0), (8, 2, [32] * 16, [192 + 7 * i for i in range(16)], 192),
    (8, 1, [1] * 16, [320 + i for i in range(16)], 320), (6, 3, [64, 64, 33], [127, 128, 129], 0), (4, 4, [1, 128, 1], [64, 64, 64], 64),
])
def test_head_layouts_and_lengths(nh, nkv, Bs, Ps, S):
    for d, dtype in ((128, "bf16"), (64, "f16")):
        c = Case(nh, nkv, d, dtype, Bs, Ps, S, seed=nh + len(Bs))
        c.check(c.run(), nodes=9)


def test_the_result_does_not_depend_on_the_sharing():
    """The same tables with 0 to 5 of the common pages given as shared."""
    c = Case(8, 2, 128, "bf16", [9, 30, 1], [320, 350, 401], 320, seed=5)
    for S in (0, 64, 192, 320):
        c.check(c.run(S), nodes=6)


def test_long_prefix_over_many_pages():
    """A prefix of several splits, each wavefront crossing more than 64 pages."""
    c = Case(32, 32, 128, "f16", [32] * 16, [20480 + 3 * i for i in range(16)], 20480, seed=6, layers=1)
    o = c.run()
    # two requests, a few rows and heads of the whole (the 64-bit form of all of it would take minutes)
    k = c.k[0][torch.as_tensor(c.table[7, :(c.Ps[7] + 32 + 63) // 64].astype(np.int64))]
    v = c.v[0][torch.as_tensor(c.table[7, :(c.Ps[7] + 32 + 63) // 64].astype(np.int64))]
    N = c.Ps[7] + 32
    for h in (0, 13, 31):
        kk, vv = k[:, h].reshape(-1, 128)[:N].double(), v[:, h].reshape(-1, 128)[:N].double()
        see = torch.from_numpy(np.concatenate([np.ones((32, c.Ps[7]), bool), c.masks[7][1]], 1))
        s = c.q64[7 * 32:8 * 32, h] @ kk.t().contiguous() / math.sqrt(128)
        p = torch.softmax(s.masked_fill(~see, -math.inf), 1)
        want = p @ vv
        qk = (c.q64[7 * 32:8 * 32, h].abs() @ kk.abs().t().contiguous()).max() / math.sqrt(128)
        tol = (p @ vv.abs()) * (U[torch.float16] + 2 * 132 * 2.0 ** -24 * qk + 2.0 ** -20 + 2 * N * 2.0 ** -24) + want.abs() * 2.0 ** -11 \
            + 2.0 ** -25 + vv.abs().sum(0) * 2.0 ** -25
        got = o[7 * 32:8 * 32].view(32, 32, 128)[:, h].double()
        assert ((got - want).abs() <= tol).all()


def test_scores_far_apart():
    """Scores of thousands, a running maximum that grows with every block, and one key that takes all the weight."""
    c = Case(4, 2, 128, "bf16", [17], [500], 0, seed=7, scale=200.0)
    c.check(c.run(), nodes=6)
    c = Case(2, 1, 64, "f16", [3], [256], 64, seed=8)
    ramp = torch.arange(256 + 3, dtype=torch.float32) * 0.2
    for i in range(259):
        c.k[0, c.table[0, i // 64], 0, i % 64] = ramp[i] * c.q32[0, 0].sign()
    c.check(c.run())


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_lies_behind_a_mask_has_no_effect(junk, dtype):
    """Slots behind the tree, siblings' keys and values, mask bits beyond the tree."""
    for d, Bs, Ps in ((128, [20, 70], [40, 100]), (64, [3, 33], [0, 31])):
        c = Case(4, 2, d, dtype, Bs, Ps, 0, seed=9)
        for r, (B, P) in enumerate(zip(Bs, Ps)):
            for s in range(P + B, (P + B + 63) // 64 * 64):
                c.k[0, c.table[r, s // 64], :, s % 64] = junk
                c.v[0, c.table[r, s // 64], :, s % 64] = junk
            # node 1 is a leaf that only itself sees
            see = c.masks[r][1]
            see[2:, 1] = False
            words = np.zeros((B, (B + 63) // 64), np.uint64)
            for i in range(B):
                for j in np.nonzero(see[i])[0]:
                    words[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
                if B % 64:
                    words[i, -1] |= ~np.uint64(0) << np.uint64(B % 64)  # bits beyond the tree
            c.masks[r] = (torch.from_numpy(words.view(np.int64)), see)
            s = P + 1
            c.v[0, c.table[r, s // 64], :, s % 64, ::3] = junk
            c.k[0, c.table[r, s // 64], :, s % 64, 5] = junk
        o = c.run()
        # rows that see node 1: itself.  Its own row is what IEEE arithmetic makes of it; all others are finite and right
        at = 0
        for B in Bs:
            c.q64[at + 1] = 0
            at += (B + 31) // 32 * 32
        at = 0
        for r, (B, P) in enumerate(zip(Bs, Ps)):
            keep = [i for i in range(B) if i != 1]
            k = rows_of(c.k[0], c.table[r], P + B).double()
            v = rows_of(c.v[0], c.table[r], P + B).double()
            see = np.concatenate([np.ones((B, P), bool), c.masks[r][1]], 1)[keep]
            want, A, qk, vs = attention64(c.q64[at:at + B][keep], k, v, torch.from_numpy(see))
            got = o[at:at + B].double().view(B, 4, d)[keep]
            u = U_P[c.dt]
            tol = A * (u + 2 * (d + 4) * 2.0 ** -24 * qk.unsqueeze(-1) + 2.0 ** -20 + (P + B) * 2.0 ** -23) + want.abs() * 2.0 ** -11 + 2.0 ** -25 + vs * 2.0 ** -25
            assert ((got - want).abs() <= tol).all(), (r, d)
            at += (B + 31) // 32 * 32


def test_rows_that_see_nothing_and_visible_infinities():
    c = Case(4, 2, 64, "bf16", [5], [0], 0, seed=10)
    c.masks[0] = (torch.tensor([[0], [2], [1], [0], [31]]), np.array([[0] * 5, [0, 1, 0, 0, 0], [1, 0, 0, 0, 0], [0] * 5, [1] * 5], bool))
    o = c.run()
    assert (o[0] == 0).all() and (o[3] == 0).all()
    c.check(o)
    # a key of -infinity scores for every query that sees it (one column, positive queries): no weight; with no other key, zero
    c = Case(2, 2, 64, "f16", [2], [0], 0, seed=11)
    c.masks[0] = (torch.tensor([[1], [3]]), np.array([[1, 0], [1, 1]], bool))
    c.q32 = c.q32.abs() + 0.1
    c.k[0, c.table[0, 0], :, 0, 3] = -float("inf")
    o = c.run()
    assert (o[0] == 0).all()
    assert torch.equal(o[1].view(2, 64), c.v[0, c.table[0, 0], :, 1])  # the one key with weight
    c.k[0, c.table[0, 0], :, 0, 3] = float("inf")
    o = c.run()
    assert o[:2].isnan().all()
    c.k[0, c.table[0, 0], :, 0, 3] = float("nan")
    assert c.run()[:2].isnan().all()


def test_offsets_beyond_32_bits():
    """A pool of more than 2^31 elements: the last pages of the last layer."""
    nkv, d, n_pages = 32, 128, 4300
    g = torch.Generator().manual_seed(12)
    kp = torch.zeros((2, n_pages, nkv, PAGE * d), dtype=torch.bfloat16, device=DEV)
    vp = torch.zeros_like(kp)
    k = torch.randn((1, 3, nkv, PAGE, d), generator=g).to(torch.bfloat16)
    v = torch.randn((1, 3, nkv, PAGE, d), generator=g).to(torch.bfloat16)
    a, b = pack_pages(k, v)
    kp[1, n_pages - 3:], vp[1, n_pages - 3:] = a[0].to(DEV), b[0].to(DEV)
    c = Case(nkv, nkv, d, "bf16", [9], [150], 128, seed=13)
    c.k, c.v = k, v
    c.table, c.refs = np.array([[2, 0, 1, -1]], np.int32), np.ones(3, np.int32)
    q, c.q64 = c.q_rows()
    ctx = goose.GooseContext(goose.ModelDesc(2, 128, nkv, d, 128, 1024, n_kv_heads=nkv), 32, 256, 512)
    i32 = dict(dtype=torch.int32, device=DEV)
    table = torch.tensor([[n_pages - 1, n_pages - 3, n_pages - 2, -1]], **i32)
    cache = goose.PagedCache(kp, vp, table, torch.tensor([150], **i32), torch.ones(n_pages, **i32))
    o = torch.full((32, nkv * d), 77.0, dtype=torch.float16, device=DEV)
    ctx.goose_attn_paged(cache, 1, q.to(DEV), 1, [{"seq": 0, "B": 9, "P_max": 150, "mask": c.masks[0][0].to(DEV)}], 2, o)
    assert ctx.goose_device_flags() == 0
    c.check(o.cpu())
    ctx.close()


def test_bad_tables_and_lengths_are_flagged():
    c = Case(4, 2, 64, "bf16", [3, 4], [70, 75], 64, seed=14)
    c.table[1, 0] = c.table[1, 1]  # not the shared page
    c.run(flags=gb.GOOSE_FLAG_PAGES)
    c = Case(4, 2, 64, "bf16", [3, 4], [70, 75], 64, seed=15)
    c.table[1, 1] = 99
    c.run(flags=gb.GOOSE_FLAG_PAGES)
    c = Case(4, 2, 64, "bf16", [3], [70], 0, seed=16)
    q, _ = c.q_rows()
    c.run()
    ctx = goose.GooseContext(goose.ModelDesc(1, 128, 4, 64, 128, 1024, n_kv_heads=2), 32, 256, 512)
    o = torch.full((32, 256), 77.0, dtype=torch.float16, device=DEV)
    req = [{"seq": 0, "B": 3, "P_max": 69, "mask": c.masks[0][0].to(DEV)}]
    ctx.goose_attn_paged(c.cache, 0, q.to(DEV), 1, req, 0, o)
    assert ctx.goose_device_flags() == gb.GOOSE_FLAG_CAPACITY
    req[0]["P_max"] = 100  # a bound above the length is what it is for
    ctx.goose_attn_paged(c.cache, 0, q.to(DEV), 1, req, 0, o)
    assert ctx.goose_device_flags() == 0
    c.check(o.cpu())
    ctx.close()


def test_a_captured_call_follows_the_lengths():
    """One graph, replayed while the device-resident length grows, with eager calls of the same context in between."""
    c = Case(8, 2, 128, "bf16", [12, 6], [64, 70], 64, seed=17)
    long = Case(8, 2, 128, "bf16", [12, 6], [250, 300], 64, seed=17)
    q, q64 = long.q_rows()
    long.q64 = q64
    desc = goose.ModelDesc(1, 128, 8, 128, 128, 1024, n_kv_heads=2)
    ctx = goose.GooseContext(desc, 32, 256, 512)
    kp, vp = pack_pages(long.k, long.v)
    length = torch.tensor([64, 70], dtype=torch.int32, device=DEV)
    cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), torch.from_numpy(long.table).to(DEV), length, torch.from_numpy(long.refs).to(DEV))
    o = torch.zeros((64, 1024), dtype=torch.float16, device=DEV)
    qd = q.to(DEV)
    reqs = goose.PagedRequests([{"seq": r, "B": b, "P_max": 300, "mask": long.masks[r][0].to(DEV)} for r, b in enumerate([12, 6])])
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        ctx.goose_attn_paged(cache, 0, qd, 1, reqs, 1, o)
    for Ps in ([64, 70], [100, 64], [250, 300], [127, 128]):
        length.copy_(torch.tensor(Ps, dtype=torch.int32))
        o.fill_(77.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        first = o.clone()
        long.Ps = Ps
        long.check(first.cpu())
        ctx.goose_attn_paged(cache, 0, qd, 1, reqs, 1, o)
        torch.cuda.synchronize()
        assert torch.equal(first, o)  # the same launch, the same order of sums
    assert ctx.goose_device_flags() == 0 and c is not None
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [128, 256])
def test_many_rows_over_every_number_of_blocks(dtype, rows):
    """128 rows a KV head (two key groups) and 256 (one): no whole block, then 1 to 14 of them, with and without a partial one behind."""
    for n in range(15):
        P = 32 * n + (0, 0, 17)[n % 3]
        c = Case(8, 1, 128 if n % 2 else 64, dtype, [rows // 8], [P], 0, seed=40 + n, terms=1 + n // 2 % 2)
        c.check(c.run(), nodes=4)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [24, 128, 256])
def test_maxima_that_grow_in_every_block(dtype, rows):
    """Keys along one direction, longer by the slot: some queries' maxima grow by up to 2^13 a block (others' shrink or stay), from one and from two
    requests that share the first pages."""
    B, d = rows // 8, 64
    c = Case(8, 1, d, dtype, [B, B], [389, 400], 128, seed=60)
    way = torch.randn(d, generator=torch.Generator().manual_seed(61))
    turn = torch.linspace(-3.0, 3.0, c.rows * 8).view(c.rows, 8, 1)  # of the queries along it
    c.q32 = turn * way / way.norm() ** 2 * math.sqrt(d) + 0.05 * c.q32
    for r in range(2):
        for s in range(c.Ps[r] + B):
            c.k[0, c.table[r, s // 64], 0, s % 64] = (0.05 * c.k[0, c.table[r, s // 64], 0, s % 64].float() + way * (s / 11.0)).to(c.dt)
    c.check(c.run(), nodes=8)
    c.check(c.run(64), nodes=8)


def test_keys_of_minus_infinity_over_whole_blocks():
    """The first 300 keys score -infinity for queries with a positive entry: rows that first see nothing, block after block; the others see a +infinity."""
    for rows in (16, 128, 256):
        c = Case(8, 1, 64, "f16", [rows // 8], [420], 128, seed=70)
        c.q32[..., 5] = c.q32[..., 5].abs() + 0.1
        c.q32[1, 3, 5] = -0.5
        for s in range(300):
            c.k[0, c.table[0, s // 64], 0, s % 64, 5] = -float("inf")
        o = c.run()
        assert o.view(-1, 8, 64)[1, 3].isnan().all()
        o.view(-1, 8, 64)[1, 3] = float("nan")
        # against the 64-bit form without those keys: they have no weight
        k, v = (rows_of(x[0], c.table[0], 420 + rows // 8).double()[:, 300:] for x in (c.k, c.v))
        see = np.concatenate([np.ones((rows // 8, 120), bool), c.masks[0][1]], 1)
        want, A, qk, vs = attention64(c.q64[:rows // 8], k, v, torch.from_numpy(see))
        tol = A * (2.0 ** -11 + 2 * 68 * 2.0 ** -24 * qk.unsqueeze(-1) + 2.0 ** -20 + 2 * 430 * 2.0 ** -24) + want.abs() * 2.0 ** -11 + 2.0 ** -25 + vs * 2.0 ** -25
        off = (o[:rows // 8].view(-1, 8, 64).double() - want).abs()
        off[1, 3] = 0
        assert (off <= tol * 1.001).all()


def test_two_graphs_of_one_context():
    """They share the context's workspace: replayed in turn, between eager calls, each gives what it gave alone."""
    few, many = (Case(8, 2, 128, "bf16", Bs, Ps, 256, seed=80) for Bs, Ps in (([1] * 5, [2000 + i for i in range(5)]), ([64, 64, 31], [800, 900, 1000])))
    ctx = goose.GooseContext(goose.ModelDesc(1, 128, 8, 128, 128, 1024, n_kv_heads=2), 64, 256, 512)
    st, calls = torch.cuda.Stream(), []
    for c in (few, many):
        q, c.q64 = c.q_rows()
        kp, vp = pack_pages(c.k, c.v)
        cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), torch.from_numpy(c.table).to(DEV), torch.tensor(c.Ps, dtype=torch.int32, device=DEV),
                                 torch.from_numpy(c.refs).to(DEV))
        reqs = goose.PagedRequests([{"seq": r, "B": b, "P_max": p, "mask": c.masks[r][0].to(DEV)} for r, (b, p) in enumerate(zip(c.Bs, c.Ps))])
        o, qd, graph = torch.full((c.rows, 1024), 77.0, dtype=torch.float16, device=DEV), q.to(DEV), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=st):
            ctx.goose_attn_paged(cache, 0, qd, 1, reqs, 4, o)
        calls.append((c, graph, o, (cache, 0, qd, 1, reqs, 4, o)))
    first = [None, None]
    for turn in range(6):
        with torch.cuda.stream(st):
            for _, graph, o, _ in calls:
                o.fill_(77.0)
                graph.replay()
            if turn % 2:
                ctx.goose_attn_paged(*calls[0][3])
        st.synchronize()
        for i, (c, _, o, _) in enumerate(calls):
            if turn == 0:
                c.check(o.cpu(), nodes=6)
                first[i] = o.clone()
            assert torch.equal(o, first[i]), (turn, i)
    assert ctx.goose_device_flags() == 0
    ctx.close()


# Sixteen requests that may have 16384 slots are many rows over many keys, so that the ring takes them; their real lengths give its items (two of a
# request, each half the keys) from no block to some thirty.
RING = dict(Bs=[32] * 16, Ps=[0, 31, 32, 33, 64, 95, 130, 200, 300, 420, 555, 700, 901, 1111, 1500, 2050])


@pytest.mark.parametrize("dtype,terms", [("bf16", 1), ("bf16", 2), ("f16", 1), ("f16", 2)])
@pytest.mark.parametrize("nh", [32, 64])
def test_the_ring_over_every_number_of_blocks(dtype, terms, nh):
    """128 rows a KV head (two key groups) and 256 (one)."""
    for d in (128, 64):
        c = Case(nh, 8, d, dtype, S=0, seed=90 + nh, terms=terms, **RING)
        c.check(c.run(bound=16384), nodes=3)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nh", [32, 64])
def test_the_ring_with_maxima_that_grow_and_keys_of_minus_infinity(dtype, nh):
    """As test_maxima_that_grow_in_every_block; the odd requests' first 200 keys score -infinity."""
    c = Case(nh, 8, 64, dtype, S=0, seed=95, **RING)
    way = torch.randn(64, generator=torch.Generator().manual_seed(96))
    way[5] = 0
    turn = torch.linspace(-3.0, 3.0, c.rows * nh).view(c.rows, nh, 1)
    c.q32 = turn * way / way.norm() ** 2 * 8 + 0.05 * c.q32
    c.q32[..., 5] = 0.25
    for r, P in enumerate(c.Ps):
        for s in range(P + 32):
            at = (0, c.table[r, s // 64], slice(None), s % 64)
            c.k[at] = (0.05 * c.k[at].float() + way * (s % 450 / 11.0)).to(c.dt)
            c.k[at][:, 5] = -float("inf") if r % 2 and s < min(P, 200) else 0.0
    o, N, at = c.run(bound=16384), nh * 64, 0
    for r, P in enumerate(c.Ps):
        skip = min(P, 200) if r % 2 else 0   # (keys without weight: the 64-bit form goes without them)
        k, v = (rows_of(x[0], c.table[r], P + 32).double()[:, skip:] for x in (c.k, c.v))
        pick = [0, 1, 17, 31]
        see = np.concatenate([np.ones((32, P - skip), bool), c.masks[r][1]], 1)[pick]
        want, A, qk, vs = attention64(c.q64[at:at + 32][pick], k, v, torch.from_numpy(see))
        tol = A * (U_P[c.dt] + 2 * 68 * 2.0 ** -24 * qk.unsqueeze(-1) + 2.0 ** -20 + 2 * (P + 32) * 2.0 ** -24) + want.abs() * 2.0 ** -11 + 2.0 ** -25
        if dtype == "f16":
            tol = tol + vs * 2.0 ** -25
        got = o[at:at + 32][pick].double().view(4, nh, 64)
        assert ((got - want).abs() <= tol * 1.001).all(), (r, float(((got - want).abs() / tol).max()))
        at += 32


@pytest.mark.parametrize("nh,nkv,B,S,dtype,terms", [(32, 32, 16, 8192, "f16", 1), (32, 32, 16, 8192, "bf16", 2), (16, 2, 1, 4096, "bf16", 2),
                                                    (16, 2, 4, 4096, "f16", 1), (8, 8, 3, 4096, "bf16", 1)])
def test_long_shared_prefixes_by_items_of_their_own(nh, nkv, B, S, dtype, terms):
    """Few rows of a request over many shared keys, where the shared keys are worked on once for all sixteen: 256 rows of them, 128, 64 and 48."""
    c = Case(nh, nkv, 64, dtype, [B] * 16, [S + 5 * i + (i == 3) * 200 for i in range(16)], S, seed=100 + B, terms=terms)
    c.check(c.run(), nodes=1 if nh == 32 else 2)


@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
@pytest.mark.parametrize("nh,d,dtype", [(32, 128, "bf16"), (32, 64, "f16"), (64, 128, "f16"), (64, 64, "bf16")])
def test_the_ring_and_what_lies_behind_a_mask(junk, nh, d, dtype):
    """As test_what_lies_behind_a_mask_has_no_effect: stale slots, a node that only itself sees, mask bits beyond the tree."""
    c = Case(nh, 8, d, dtype, S=0, seed=97, **RING)
    for r, P in enumerate(c.Ps):
        for s in range(P + 32, (P + 32 + 63) // 64 * 64):
            c.k[0, c.table[r, s // 64], :, s % 64] = junk
            c.v[0, c.table[r, s // 64], :, s % 64] = junk
        see = c.masks[r][1]
        see[2:, 1] = False
        words = np.full((32, 1), 0xFFFFFFFF00000000, np.uint64)
        for i in range(32):
            for j in np.nonzero(see[i])[0]:
                words[i, 0] |= np.uint64(1) << np.uint64(j)
        c.masks[r] = (torch.from_numpy(words.view(np.int64)), see)
        s = P + 1
        c.v[0, c.table[r, s // 64], :, s % 64, ::3] = junk
        c.k[0, c.table[r, s // 64], :, s % 64, 5] = junk
    o = c.run(bound=16384)
    pick = [0, 2, 9, 31]
    for r, P in enumerate(c.Ps):
        k, v = (rows_of(x[0], c.table[r], P + 32).double() for x in (c.k, c.v))
        see = np.concatenate([np.ones((32, P), bool), c.masks[r][1]], 1)[pick]
        want, A, qk, vs = attention64(c.q64[r * 32:r * 32 + 32][pick], k, v, torch.from_numpy(see))
        got = o[r * 32:r * 32 + 32].double().view(32, nh, d)[pick]
        tol = A * (U_P[c.dt] + 2 * (d + 4) * 2.0 ** -24 * qk.unsqueeze(-1) + 2.0 ** -20 + (P + 32) * 2.0 ** -23) + want.abs() * 2.0 ** -11 + 2.0 ** -25 + vs * 2.0 ** -25
        assert ((got - want).abs() <= tol).all(), (r, P)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_the_ring_with_the_largest_trees(dtype):
    """Trees of 128 nodes reach over five blocks, with an odd whole one in front six: more than the ring has copied ahead."""
    for nh, d in ((32, 128), (64, 64)):
        c = Case(nh, 32, d, dtype, [128] * 4, [45, 100, 333, 610], 0, seed=110 + nh)
        c.check(c.run(bound=16384), nodes=5)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nh,nkv,Bs,bound", [(8, 4, [7], None), (16, 4, [12, 9], None), (32, 8, [32] * 16, 16384), (64, 8, [32] * 16, 16384)])
def test_a_weight_above_one_keeps_its_bits(dtype, nh, nkv, Bs, bound):
    """All scores are zero but one key's, t < 8 ln 2 in a later block than a wavefront's first: its weight e^t is not one, as the reference stays at the
    first maximum.  All other values are zero, so the output is p v of that key and what is lost of the weight is lost of it.  One product makes a score,
    so it errs by its scale's and the reference's rounding only (4 steps of 2^-24 t); p in two terms (fp16 2^-21, bf16 2^-16); sums, exponential, store as above."""
    d, P = 64, 560
    c = Case(nh, nkv, d, dtype, Bs, [P] * len(Bs), 0, seed=120, o_dtype=torch.float16, o_terms=2)
    c.k.zero_()
    c.v.mul_(0)
    values = torch.randn((nkv, d), generator=torch.Generator().manual_seed(121)).to(c.dt)
    c.q32 = torch.linspace(0.5, 5.4, c.rows * nh).view(c.rows, nh, 1) * torch.eye(d)[5]
    for r in range(len(Bs)):
        for h in range(nkv):
            s = 40 + 32 * h
            c.k[0, c.table[r, s // 64], h, s % 64, 5] = 8.0
            c.v[0, c.table[r, s // 64], h, s % 64] = values[h]
    o, at = c.run(bound=bound).double(), 0
    o = o.view(c.rows, nh * d // 8, 2, 8).sum(2).view(c.rows, nh, d)
    u = 2.0 ** -21 if dtype == "f16" else 2.0 ** -16
    v = values.double().repeat_interleave(nh // nkv, 0)
    for B, (_, see) in zip(Bs, c.masks):
        t = c.q64[at:at + B, :, 5:6]                                             # (the key's 8 over sqrt(64))
        N = torch.from_numpy(P + see.sum(1)).view(B, 1, 1)
        want = torch.exp(t) / (N - 1 + torch.exp(t)) * v
        tol = want.abs() * (u + 8 * 2.0 ** -24 * t + 2.0 ** -20 + 2 * N * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -24 + v.abs() * 2.0 ** -25
        off = (o[at:at + B] - want).abs() / tol
        assert off.max() <= 1, (float(off.max()), off.argmax())
        at += (B + 31) // 32 * 32


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nh,nkv,Bs,P,S,bound", [(8, 4, [7], 600, 0, None), (16, 4, [12, 9], 600, 0, None), (32, 8, [32] * 16, 600, 0, 16384),
                                                 (64, 8, [32] * 16, 600, 0, 16384), (8, 4, [1] * 8, 4500, 4096, None), (8, 4, [2], 9000, 0, None)])
def test_large_scores_join_by_their_differences(dtype, nh, nkv, Bs, P, S, bound):
    """Two keys score 2^27 and 2^27 + 16 (over sqrt(64): 2 apart), all others 0, wherever the two lie: in one block, one wavefront's share, two of them, two
    splits, or the shared pages and a request's own.  The sums of products are multiples of 16 up to 2^27 + 16, so exact in 32 bits in any order; the difference is exact too, and
    its scale and exponential err by 2^-21 and 2^-22 of the weight: with p, output (one term) and store tol = |v| sums (u + 2^-19) + u_o |o| + 2^-25."""
    d = 64
    c = Case(nh, nkv, d, dtype, Bs, [P + i for i in range(len(Bs))], S, seed=130)
    c.k.zero_()
    c.v.mul_(0.5)
    c.q32.zero_()
    c.q32[..., 3], c.q32[..., 9] = 2.0 ** 13, 4.0
    first = [[40 if h == 0 else (P - 33 * h if S else 40 + (P // 16 * h)) for h in range(nkv)], [20 + 3 * h for h in range(nkv)]]
    for r in range(len(Bs)):
        for h in range(nkv):
            for s, nine in ((first[1][h], 0.0), (first[0][h], 4.0)):
                c.k[0, c.table[r, s // 64], h, s % 64, 3] = 2.0 ** 14
                c.k[0, c.table[r, s // 64], h, s % 64, 9] = nine
    o, at, u = c.run().double() if bound is None else c.run(bound=bound).double(), 0, U_P[c.dt]
    for r, B in enumerate(Bs):
        got = o[at:at + B].view(B, nh, d)
        for h in range(nkv):
            lo, hi = (c.v[0, c.table[r, s // 64], h, s % 64].double() for s in (first[1][h], first[0][h]))
            w = math.exp(2.0)
            want, mag = (lo + w * hi) / (1 + w), (lo.abs() + w * hi.abs()) / (1 + w)
            tol = mag * (u + 2.0 ** -19) + U[torch.float16] * want.abs() + 2.0 ** -25
            off = (got[:, h * nh // nkv:(h + 1) * nh // nkv] - want).abs() / tol
            assert off.max() <= 1, (r, h, float(off.max()))
        at += (B + 31) // 32 * 32
