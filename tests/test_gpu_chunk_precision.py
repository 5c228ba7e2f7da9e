"""goose_attn_chunk_paged: weights enter the second product in two terms of the cache's type, whatever the output's type and terms.

The bound of tests/test_gpu_chunk_attn.py with 2^-16 A (bf16: half a step 2^-8 of a remainder of 2^-8) or 2^-21 A (fp16) for the weights' rounding
throughout, A = sum p |v| / sum p: less than the store of a one-term output by 2^8 and 2^10.
"""
import pytest
import torch

import paper_2604_02047_amd as goose
import test_gpu_chunk_attn as chunk_attn
from test_gpu_chunk_attn import BF, HF, LONG, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def two_terms(monkeypatch):
    monkeypatch.setattr(chunk_attn, "weight_rounding", lambda dt, o_dtype, o_terms: {BF: 2.0 ** -16, HF: 2.0 ** -21}[dt])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("terms", [1, 2])
@pytest.mark.parametrize("bound", [None, LONG])
def test_every_output_has_the_bits_of_two_terms(dtype, d, terms, bound):
    """Many rows (both rings) and few."""
    for o_dtype, o_terms in ((HF, 1), (BF, 1), (BF, 2), (HF, 2)):
        for Cs, Ps in (([150, 300], [333, 0]), ([3, 1], [260, 70])):
            c = Case(4, 1, d, dtype, Cs, Ps, seed=31, terms=terms, o_dtype=o_dtype, o_terms=o_terms)
            c.check(c.run(bound=bound))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rise", [0.7, 2.3, 3.5])
@pytest.mark.parametrize("nh,nkv,C,bound", [(2, 1, 200, None), (32, 8, 4096, 4200)])
def test_a_dominating_key_that_raises_no_maximum(dtype, rise, nh, nkv, C, bound):
    """Block 0 has a key of score 0 and all others lie 30 below; block 1, of the same range of keys, has one whose score is `rise` times one to 1.25: by less than maxima
    lag behind (8 log 2 = 5.5), so that its weight may be any number from one to 256, and not a sum of few bits.  Both rings: the larger call has more than 256 blocks by
    its bound, and too many rows for its keys to be split."""
    P, d = 64, 64
    c = Case(nh, nkv, d, dtype, [C], [P], seed=32, scale=0.0, o_dtype=BF if dtype == "bf16" else HF)
    g = torch.Generator().manual_seed(32)
    # column 0 carries the scores (times sqrt(d) = 8), every row with a factor of its own
    c.q32[:, :, 0] = 1.0 + 0.25 * torch.rand((c.rows, nh), generator=g)
    c.k.zero_()
    c.k[..., 0] = -240.0
    c.k[0, c.table[0, 0], :, 3, 0] = 0.0
    c.k[0, c.table[0, 0], :, 40, 0] = 8.0 * rise
    c.check(c.run(bound=bound), heads=sorted({0, nh - 1}))


@pytest.mark.parametrize("dtype,o_dtype", [("bf16", BF), ("f16", HF), ("bf16", HF)])
@pytest.mark.parametrize("nh,nkv,C,P", [(32, 8, 64, 200), (32, 8, 33, 70), (40, 40, 1, 600), (40, 40, 16, 300), (8, 2, 300, 100)])
def test_a_chunk_alone_and_among_others(dtype, o_dtype, nh, nkv, C, P):
    """Which kernel takes a chunk and how its keys are split goes by the whole call and by P_max (alone: few rows, the tree kernels; with fifteen others: the ring; with
    a far bound: more parts): the bits may differ, the precision does not."""
    n = 16 if C < 100 else 4
    Cs, Ps = [C] + [max(1, C - r) for r in range(1, n)], [P] + [P + 3 * r for r in range(1, n)]
    heads = sorted({0, nh - 1})
    for count, bound in ((n, None), (1, None), (1, 3000), (1, LONG)):
        c = Case(nh, nkv, 64, dtype, Cs, Ps, seed=33, o_dtype=o_dtype)
        c.place(bound)
        c.chunks = goose.PagedChunks([{"seq": r, "C": Cs[r], "P_max": bound or Ps[r]} for r in range(count)])
        c.call()
        assert c.ctx.goose_device_flags() == 0
        c.ctx.close()
        if count == 1:
            assert (c.o[C:] == 77).all()
            c.Cs, c.Ps, c.rows = Cs[:1], Ps[:1], C
        c.check((c.o.cpu(), c.lse.cpu()), heads=heads)
