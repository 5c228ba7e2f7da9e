"""goose_qk_norm_rope_paged against the 64-bit formula: queries, K/V rows in the pages, and everything it must leave alone.

Error bound of one value, u32 = 2^-24, u = half a step of the storage type (bf16 2^-9 of the value's own binade is at most
2^-8 relative, fp16 2^-11): the sum of ks slices errs by at most ks u32 sum|x|; the norm multiplies by a factor with a relative error of
(d/2 + 8) u32 or less (sum of squares of positive terms: at most d + 2 roundings, halved by the root; root, quotient, two products); angle,
cosine and sine err by at most 2e-7 in all (reduced in 64 bits, rounded to 32: pi 2^-24 = 1.9e-7 at most, evaluated to 2 ulp); the rotation adds 3 u32.  So
|err| <= (|a| + |b|) (2.0e-7 + 2.4e-7 + (ks + d/2 + 12) u32) with a, b the pair in slices' absolute sums, plus u |value| for the store.
"""
import numpy as np
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, pack_pages, rope64, unpack_pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2, torch.float16: torch.finfo(torch.float16).eps / 2}


def setup(nh, nkv, d, dtype, Bs, Ps, ks, norm, seed, base=10000.0, layers=1, layer=0, pad=0):
    """A cache whose pages for the trees are the sequences' own, in shuffled order; other entries are empty."""
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float16
    width = max((p + b + PAGE - 1) // PAGE for p, b in zip(Ps, Bs)) + 1
    n_pages = sum((p + b - 1) // PAGE - p // PAGE + 1 for p, b in zip(Ps, Bs)) + 2
    order = torch.randperm(n_pages, generator=g).tolist()
    table, refs, at = np.full((len(Bs), width), -1, np.int32), np.zeros(n_pages, np.int32), 0
    for r, (p, b) in enumerate(zip(Ps, Bs)):
        for i in range(p // PAGE, (p + b - 1) // PAGE + 1):
            table[r, i] = order[at]
            refs[order[at]] = 1
            at += 1
    desc = goose.ModelDesc(layers, 128, nh, d, 128, 1024, base, 1e-6, dtype, nkv, norm)
    ctx = goose.GooseContext(desc, max(Bs), 256, 512)
    k = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(dt)
    v = torch.randn((layers, n_pages, nkv, PAGE, d), generator=g).to(dt)
    kp, vp = pack_pages(k, v)
    cache = goose.PagedCache(kp.to(DEV), vp.to(DEV), torch.from_numpy(table).to(DEV), torch.tensor(Ps, dtype=torch.int32, device=DEV),
                             torch.from_numpy(refs).to(DEV))
    rows = sum((b + 31) // 32 * 32 for b in Bs)
    part = torch.randn((ks, rows, (nh + 2 * nkv) * d + pad), generator=g)
    gains = [(1 + 0.2 * torch.randn(d, generator=g)).to(dt) for _ in range(2)]
    return ctx, cache, table, k, v, part, gains


def check(nh, nkv, d, dtype, Bs, Ps, ks, norm, terms, seed=0, base=10000.0, layers=1, layer=0, pad=0, pos=None, part_fn=None):
    ctx, cache, table, k, v, part, gains = setup(nh, nkv, d, dtype, Bs, Ps, ks, norm, seed, base, layers, layer, pad)
    dt, u = cache.kpool.dtype, HALF_STEP[cache.kpool.dtype]
    if part_fn:
        part = part_fn(part)
    rows = part.shape[1]
    q = torch.full((rows, nh * d * terms + 8), 77.0, dtype=dt, device=DEV)
    g = torch.Generator().manual_seed(seed + 1)
    poss = pos or [[p + int(x) for x in torch.randint(0, b, (b,), generator=g)] for p, b in zip(Ps, Bs)]
    reqs = [{"seq": r, "B": b, "P_max": p, "pos": torch.tensor(poss[r], dtype=torch.int32, device=DEV)}
            for r, (p, b) in enumerate(zip(Ps, Bs))]
    gq, gk = [x.to(DEV) for x in gains] if norm else (None, None)
    ctx.goose_qk_norm_rope_paged(cache, layer, part.to(DEV), gq, gk, reqs, q, terms)
    assert ctx.goose_device_flags() == 0
    qc = q.cpu()
    assert (qc[:, nh * d * terms:] == 77).all()
    kk, vv = unpack_pages(cache.kpool.cpu(), cache.vpool.cpu(), d)
    kw, vw = k.clone(), v.clone()  # what the pools must hold: written rows are compared, then copied over before the bit test
    row0 = 0
    g64 = [x.double() for x in gains] if norm else (None, None)
    for r, (p, b) in enumerate(zip(Ps, Bs)):
        x = part[:, row0:row0 + b, :(nh + 2 * nkv) * d].double()
        qe, ke, ve = rope64(x, g64[0], g64[1], poss[r], nh, nkv, d, base, 1e-6)
        a = x.abs().sum(0).view(b, nh + 2 * nkv, d)
        if norm:
            y = x.sum(0).view(b, nh + 2 * nkv, d)
            a = a / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6)
            a = torch.cat((a[:, :nh] * g64[0].abs(), a[:, nh:nh + nkv] * g64[1].abs(), a[:, nh + nkv:]), 1)
        pair = a[..., :d // 2] + a[..., d // 2:]
        pair = torch.cat((pair, pair), -1)
        slack = pair * (4.4e-7 + (ks + d // 2 + 12) * U32)
        got = qc[row0:row0 + b, :nh * d * terms].double()
        if terms == 2:
            got = got.view(b, nh * d // 8, 2, 8).sum(2)
        got = got.view(b, nh, d)
        # two terms: the second rounds a remainder of at most u |x|
        store = u * u if terms == 2 else u
        tiny = 2.0 ** -25 if dt == torch.float16 else 0.0  # half a step of fp16's subnormals
        assert ((got - qe).abs() <= slack[:, :nh] + store * qe.abs() + tiny).all(), (r, "q", float((got - qe).abs().max()))
        for i in range(b):
            page, slot = table[r, (p + i) // PAGE], (p + i) % PAGE
            gk_, gv_ = kk[layer, page, :, slot].double(), vv[layer, page, :, slot].double()
            assert ((gk_ - ke[i]).abs() <= slack[i, nh:nh + nkv] + u * ke[i].abs() * 1.0001 + tiny).all(), (r, i, "k")
            vs = a[i, nh + nkv:] * ks * U32 if not norm else x[:, i].abs().sum(0).view(-1, d)[nh + nkv:] * ks * U32
            assert ((gv_ - ve[i]).abs() <= vs * 1.01 + u * ve[i].abs() * 1.0001 + tiny).all(), (r, i, "v")
            kw[layer, page, :, slot] = kk[layer, page, :, slot]
            vw[layer, page, :, slot] = vv[layer, page, :, slot]
        pad_rows = qc[row0 + b:row0 + (b + 31) // 32 * 32]
        assert (pad_rows == 77).all(), "rows between requests"
        row0 += (b + 31) // 32 * 32
    assert torch.equal(kk.view(torch.int16), kw.view(torch.int16)) and torch.equal(vv.view(torch.int16), vw.view(torch.int16))
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm", [False, True])
def test_against_the_formula(dtype, d, norm):
    check(8, 2, d, dtype, [21, 1, 64, 40], [5, 0, 100, 63], 4, norm, 1, seed=1)
    check(8, 2, d, dtype, [33, 7], [61, 122], 3, norm, 2, seed=2, pad=4)


@pytest.mark.parametrize("nh,nkv,Bs,Ps,ks", [(4, 4, [1], [0], 1), (17, 1, [1], [63], 16), (3, 3, [8], [56], 5), (20, 5, [9], [57], 2),
                                             (52, 52, [3], [127], 7), (40, 40, [128], [1], 8), (32, 8, [32] * 16, list(range(1000, 1016)), 4)])
def test_head_counts_and_ragged_ends(nh, nkv, Bs, Ps, ks):
    check(nh, nkv, 128, "bf16", Bs, Ps, ks, False, 1, seed=3)


def test_far_positions_and_other_layers():
    """Angles of positions near 2^24 and beyond, where a 32-bit product has lost its fraction; layer 2 of 3."""
    check(4, 2, 64, "f16", [5], [70], 2, True, 2, seed=4, base=500000.0, layers=3, layer=2,
          pos=[[0, 131071, 16777217, 1 << 30, (1 << 31) - 1]])


def test_large_and_small_rows():
    """Rows whose squares are far from one: 1e-12 (the norm's eps decides) and 1e15."""
    def scaled(p):
        p = p.clone()
        p[:, 0] *= 1e-12
        p[:, 1] *= 1e15
        p[:, 2] = 0
        return p
    check(2, 2, 128, "bf16", [4], [9], 2, True, 1, seed=5, part_fn=scaled)


def test_pages_that_are_missing_or_shared_are_not_written():
    ctx, cache, table, k, v, part, _ = setup(4, 2, 64, "bf16", [40], [50], 1, False, 6)
    pos = torch.arange(50, 90, dtype=torch.int32, device=DEV)
    q = torch.zeros((64, 256), dtype=torch.bfloat16, device=DEV)
    before = cache.kpool.clone(), cache.vpool.clone()
    own = int(cache.table[0, 0]), int(cache.table[0, 1])

    def call(p_max=50):
        ctx.goose_qk_norm_rope_paged(cache, 0, part.to(DEV), None, None, [{"seq": 0, "B": 40, "P_max": p_max, "pos": pos}], q, 1)
        return ctx.goose_device_flags()

    cache.refs[own[0]] = 2
    cache.table[0, 1] = -1
    assert call() == gb.GOOSE_FLAG_PAGES
    cache.table[0, 1] = cache.refs.numel()
    assert call() == gb.GOOSE_FLAG_PAGES
    assert torch.equal(cache.kpool, before[0]) and torch.equal(cache.vpool, before[1])
    cache.refs[own[0]] = 1
    cache.table[0, 1] = own[1]
    assert call(p_max=49) == gb.GOOSE_FLAG_CAPACITY  # the length is above the host's bound
    assert torch.equal(cache.kpool, before[0]) and torch.equal(cache.vpool, before[1])
    assert call() == 0 and not torch.equal(cache.kpool, before[0])
    ctx.close()
