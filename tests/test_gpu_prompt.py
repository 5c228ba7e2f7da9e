"""Prompts on a paged cache as they are used: chunk layers beside chains of nodes, weights, eviction and what runs on after it, graphs, decoding."""
import numpy as np
import pytest
import torch

import goose_inputs as gi
import paper_2604_02047_amd as goose
from paged_ref import PAGE, mask_words, unpack_pages
from prompt_ref import chunk_attention64
from util import gpu_model, torch_model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def chain(gm, seq, P, n):
    """A request that is a chain of n nodes behind P slots, all of it accepted."""
    words, _ = mask_words(list(range(-1, n - 1)))
    i32 = dict(dtype=torch.int32, device=DEV)
    return {"seq": seq, "B": n, "P_max": P, "mask": words.to(DEV), "pos": torch.arange(P, P + n, **i32), "path": torch.arange(n, **i32),
            "accept_len": torch.tensor([n - 1], **i32)}


def rows_of_layer(cache, seq, l, d):
    """Logical K and V rows [head][n][d] of a sequence's committed slots."""
    n = int(cache.len[seq])
    pages = cache.table[seq, :(n + PAGE - 1) // PAGE].long()
    out = []
    for x in unpack_pages(cache.kpool[l:l + 1], cache.vpool[l:l + 1], d):
        x = x[0, pages].transpose(0, 1)
        out.append(x.reshape(x.shape[0], -1, d)[:, :n])
    return out


def fill(gm, cache, seq, n, seed):
    """n committed slots of random rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    if seed == 0:
        cache.kpool.normal_(generator=g)
        cache.vpool.normal_(generator=g)
    gm.ctx.goose_pages_reserve(cache, [seq], [n])
    gm.ctx.goose_pages_append(cache, [{"seq": seq, "C": n}])


@pytest.mark.parametrize("name,act_mode", [("small_bf16", 0), ("tiny_gqa_bf16", 0), ("small_gqa_qknorm_bf16", 1), ("small_gqa_qknorm_f16", 0)])
def test_a_layer_over_chunks_beside_chains(name, act_mode):
    """Chunks that are chains of up to 64 nodes as well: the same K/V rows, bit for bit, and the same outputs up to what 16-bit operands leave open."""
    import dataclasses

    from paper_2604_02047_amd.runner import GooseModel
    shape = gi.SHAPES[name]
    tm = torch_model(shape, seed=3, gain_jitter=0.1)
    desc = dataclasses.replace(goose.ModelDesc.from_shape(shape), act_mode=act_mode)
    gm = GooseModel(desc, 64, 512, lambda l: tm["layers"][l], tm["embed"], tm["lm_head"], tm["final_norm"], max_rows=256)
    Ps, Cs = [150, 1, 63], [33, 64, 7]
    rows = 32 + 32 + 64 + 7
    x0 = torch.randn((rows, shape.hidden), generator=torch.Generator().manual_seed(1)).to(DEV)
    out = []
    for way in (0, 1, 2):
        cache = gm.paged_cache(16, 3, 320)
        for r, p in enumerate(Ps):
            fill(gm, cache, r, p, r)
        gm.ctx.goose_pages_reserve(cache, [0, 1, 2], Cs)
        x = x0.clone()
        if way == 0:
            gm.ctx.goose_verify_layer_paged(gm.packed_layer(1), cache, 1, x, [chain(gm, r, p, c) for r, (p, c) in enumerate(zip(Ps, Cs))])
        else:
            pos = lambda p, c: torch.arange(p, p + c, dtype=torch.int32, device=DEV) if way == 2 else None  # noqa: E731
            gm.ctx.goose_chunk_layer_paged(gm.packed_layer(1), cache, 1, x, [{"seq": r, "C": c, "P_max": p, "pos": pos(p, c)}
                                                                           for r, (p, c) in enumerate(zip(Ps, Cs))])
        assert gm.ctx.goose_device_flags() == 0
        gm.ctx.goose_pages_append(cache, [{"seq": r, "C": c} for r, c in enumerate(Cs)])
        out.append((x, [rows_of_layer(cache, r, 1, shape.head_dim) for r in range(3)]))
    scale = (out[0][0] - x0).abs().max()
    at = 0
    for r, c in enumerate(Cs):
        assert (out[1][0][at:at + c] - out[0][0][at:at + c]).abs().max() <= 5e-3 * scale
        assert torch.equal(out[1][0][at:at + c], out[2][0][at:at + c])
        for a, b in zip(out[0][1][r], out[1][1][r]):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        for a, b in zip(out[1][1][r], out[2][1][r]):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        at += (c + 31) // 32 * 32
    assert all(o[0].isfinite().all() for o in out)
    gm.ctx.close()


def test_a_chunk_layer_refuses_what_does_not_fit():
    shape = gi.SHAPES["tiny_gqa_bf16"]
    gm = gpu_model(shape, torch_model(shape), max_B=32, cap=512, max_rows=128)
    cache = gm.paged_cache(16, 3, 320)
    x = torch.zeros((160, shape.hidden), device=DEV)
    w = gm.slot_weights(cache)
    call = lambda chunks, layer=0, x=x, weight=None, decay=1.0: gm.ctx.goose_chunk_layer_paged(gm.packed_layer(0), cache, layer, x, chunks, weight, decay)  # noqa: E731
    for chunks, kw, status in [([{"seq": 0, "C": 129}], {}, -3), ([{"seq": 0, "C": 97}, {"seq": 1, "C": 1}], {}, -3), ([{"seq": 0, "C": 10, "P_max": 311}], {}, -3),
                               ([{"seq": 0, "C": 10}], {"layer": 2}, -1), ([{"seq": 0, "C": 10}], {"x": x[:9]}, -1), ([{"seq": 3, "C": 10}], {}, -1),
                               ([{"seq": 0, "C": 10, "first": 10}], {"weight": w}, -1), ([{"seq": 0, "C": 10}], {"weight": w, "decay": -1.0}, -1),
                               ([{"seq": 0, "C": 10}], {"weight": w[:1]}, -1), ([{"seq": 0, "C": 10}, {"seq": 0, "C": 10}], {}, -1)]:
        with pytest.raises(goose.GooseError) as e:
            call(chunks, **kw)
        assert e.value.status == status, (chunks, kw)
    # slots that were not reserved: flagged, and no row is written
    call([{"seq": 0, "C": 10}])
    assert gm.ctx.goose_device_flags() == 16 and int(cache.kpool.count_nonzero()) == 0
    gm.ctx.close()


def test_prompt_weights_eviction_and_a_step_after_it():
    """A prompt in three passes, its weights, the cut, and then: attention over the cut rows against 64 bits, a verification step, another chunk."""
    shape = gi.SHAPES["small_gqa_qknorm_bf16"]
    d, G = shape.head_dim, shape.n_heads // shape.kv_heads
    gm = gpu_model(shape, torch_model(shape, seed=5, gain_jitter=0.1), max_B=32, cap=512, max_rows=256)
    c, cache = gm.ctx, gm.paged_cache(40, 2, 1024)
    weight = gm.slot_weights(cache)
    weight.fill_(float("nan"))       # (nothing of it is read before it is written)
    tokens = torch.as_tensor(gi.prefix_tokens(3, 600, shape.vocab).astype(np.int32), device=DEV)
    x = torch.zeros((256, shape.hidden), device=DEV)
    done = 0
    for n in (256, 250, 94):
        chunk = goose.PagedChunks([{"seq": 1, "C": n, "P_max": done}])
        c.goose_pages_reserve(cache, [1], [n])
        for a in range(0, n, 32):
            c.goose_embed(gm.embed, tokens[done + a:], min(32, n - a), x[a:])
        for l in range(shape.n_layers):
            c.goose_chunk_layer_paged(gm.packed_layer(l), cache, l, x, chunk, weight, 1.0)
        c.goose_pages_append(cache, chunk)
        done += n
    assert c.goose_device_flags() == 0 and int(cache.len[1]) == 600
    total = weight[:, 1, :, :600].double().sum(-1)
    assert ((total - 600 * G).abs() <= 1e-4 * 600 * G).all()      # every row of every query head gives one, to the rounding of its scores
    assert weight[:, 0].isnan().all() and weight[:, 1, :, 600:].isnan().all()
    before = [rows_of_layer(cache, 1, l, d) for l in range(shape.n_layers)]
    w0 = weight.clone()
    kept = torch.zeros((1, shape.n_layers, shape.kv_heads, cache.table.shape[1]), dtype=torch.int64, device=DEV)
    c.goose_pages_evict(cache, [{"seq": 1, "keep": 200, "sink": 4, "recent": 50}], weight, kept)
    assert c.goose_device_flags() == 0 and int(cache.len[1]) == 200
    bits = (kept[0].unsqueeze(-1) >> torch.arange(64, device=DEV)) & 1
    for l in range(shape.n_layers):
        k, v = rows_of_layer(cache, 1, l, d)
        for h in range(shape.kv_heads):
            mine = torch.nonzero(bits[l, h].reshape(-1)).reshape(-1)
            others = torch.argsort(-w0[l, 1, h, 4:550], stable=True)[:146] + 4
            want = torch.cat((torch.arange(4, device=DEV), others.sort().values, torch.arange(550, 600, device=DEV)))
            assert torch.equal(mine, want) and torch.equal(weight[l, 1, h, :200], w0[l, 1, h, mine])
            assert torch.equal(v[h].view(torch.int16), before[l][1][h, mine].view(torch.int16))
            # turned keys: a rotation keeps the length of every pair, to the rounding of both terms
            a, b = before[l][0][h, mine].float(), k[h].float()
            r0, r1 = (a[:, :d // 2] ** 2 + a[:, d // 2:] ** 2).sqrt(), (b[:, :d // 2] ** 2 + b[:, d // 2:] ** 2).sqrt()
            assert ((r0 - r1).abs() <= 2.0 ** -7 * r0 + 1e-6).all() and torch.equal(a[:4], b[:4])
    # attention over what is left
    q = torch.randn((5, shape.n_heads * d), generator=torch.Generator().manual_seed(2)).to(gm.dt).to(DEV)
    o = torch.zeros((5, shape.n_heads * d), dtype=torch.float16, device=DEV)
    c.goose_pages_reserve(cache, [1], [5])
    c.goose_attn_chunk_paged(cache, 0, q, 1, [{"seq": 1, "C": 5, "P_max": 200}], o)
    c.goose_pages_append(cache, [{"seq": 1, "C": 5}])
    k, v = rows_of_layer(cache, 1, 0, d)
    want, A = chunk_attention64(q.cpu().double().view(5, shape.n_heads, d), k.cpu().double(), v.cpu().double(), 200)[:2]
    assert ((o.cpu().double().view(5, shape.n_heads, d) - want).abs() <= 2.0 ** -10 * want.abs() + 2.0 ** -14 * A + 2.0 ** -24).all()
    # a verification step, and a chunk again: positions are slots
    i32 = dict(dtype=torch.int32, device=DEV)
    t, p, s = gm.stage_tree([5, 6, 7, 8], [-1, 0, 1, 0], np.ones(4, np.uint8))
    req = [{"seq": 1, "B": 4, "P_max": 205, "tokens": t, "parent": p, "is_spine": s, "accept_len": torch.zeros(1, **i32), "path": torch.zeros(4, **i32),
            "bonus": torch.zeros(1, **i32)}]
    c.goose_verify_step_paged(gm.model_ptrs(), cache, req, 0, torch.zeros(32, **i32))
    assert c.goose_device_flags() == 0 and int(cache.len[1]) == 206 + int(req[0]["accept_len"])
    c.close()


def test_a_captured_pass_follows_the_sequence():
    """One graph: room, a layer pass with weights, the commit, a cut.  Replays equal eager calls on a second cache, bit for bit."""
    shape = gi.SHAPES["tiny_gqa_bf16"]
    gm = gpu_model(shape, torch_model(shape, seed=7, gain_jitter=0.1), max_B=32, cap=512, max_rows=128)
    c = gm.ctx
    caches = [gm.paged_cache(20, 3, 512) for _ in range(2)]
    weights = [gm.slot_weights(x) for x in caches]
    kept = [torch.zeros((2, shape.n_layers, shape.kv_heads, 8), dtype=torch.int64, device=DEV) for _ in range(2)]
    x0 = torch.randn((83, shape.hidden), generator=torch.Generator().manual_seed(1)).to(DEV)
    xs = [x0.clone(), x0.clone()]
    chunks = goose.PagedChunks([{"seq": 0, "C": 50, "P_max": 400}, {"seq": 2, "C": 19, "P_max": 400, "first": 5}])
    ev = [{"seq": 0, "keep": 170, "sink": 2, "recent": 30}, {"seq": 2, "keep": 90, "recent": 20}]

    def one(i):
        xs[i].copy_(x0)
        c.goose_pages_reserve(caches[i], [0, 2], [50, 19])
        for l in range(shape.n_layers):
            c.goose_chunk_layer_paged(gm.packed_layer(l), caches[i], l, xs[i], chunks, weights[i], 0.9)
        c.goose_pages_append(caches[i], chunks)
        c.goose_pages_evict(caches[i], ev, weights[i], kept[i])

    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        one(0)
    for i in range(9):
        with torch.cuda.stream(st):
            graph.replay()
        st.synchronize()
        torch.zeros(1000, device=DEV).sum().item()
        one(1)
        torch.cuda.synchronize()
        a, b = caches
        for u, v in ((a.table, b.table), (a.len, b.len), (a.refs, b.refs), (weights[0], weights[1]), (kept[0], kept[1]), (xs[0][:50], xs[1][:50]),
                     (xs[0][64:], xs[1][64:]), (a.kpool.view(torch.int16), b.kpool.view(torch.int16)), (a.vpool.view(torch.int16), b.vpool.view(torch.int16))):
            assert torch.equal(u, v), i
        assert int(a.len[0]) == min(170, 50 * (i + 1)) and int(a.len[2]) == min(90, 19 * (i + 1))
    assert c.goose_device_flags() == 0
    c.close()


def _prompts(vocab, n, common):
    pat = gi.prefix_tokens(31, 12, vocab).tolist()
    head = (pat * (common // 12 + 1))[:common]
    return [head + gi.prefix_tokens(40 + r, 10 + 37 * r, vocab).tolist() + pat[:6] for r in range(n)]


@pytest.mark.parametrize("common", [0, 150])
def test_prompts_in_chunks_give_the_tokens_of_chains(common):
    """16-bit near-ties may be decided differently where launches differ in shape: long agreement is the check, as for the decoders elsewhere."""
    from paper_2604_02047_amd.decoder import PagedGooseDecoder
    shape = gi.SHAPES["small_bf16"]
    tm = torch_model(shape, seed=6, gain_jitter=0.1)
    prompts = _prompts(shape.vocab, 3, common)
    outs = []
    for options in ({}, {"prompt_rows": 192}, {"prompt_rows": 50}, {"prompt_rows": 192, "keep": 440}):
        gm = gpu_model(shape, tm, max_B=64, cap=512, max_rows=192)
        pd = PagedGooseDecoder(gm, 3, n_pages=24, max_slots=448, B=40, min_score=0.0, **options)
        outs.append(pd.generate(prompts, 50))
        assert int(pd.cache.refs.sum()) == (common + 63) // 64
        if options:
            assert pd.generate(prompts, 50) == outs[-1]
        gm.ctx.close()
    for other in outs[1:]:
        for r in range(3):
            n = min(len(outs[0][r]), len(other[r]))
            same = next((i for i in range(n) if outs[0][r][i] != other[r][i]), n)
            assert same >= 30, (r, same)
    assert outs[3] == outs[1]      # nothing had to go


def test_decoding_goes_on_over_a_cut_prompt():
    """Caches of unlike prompts cut to one size: they hold that many slots, share what they shared, decode to the end and give everything back."""
    from paper_2604_02047_amd.binding import GOOSE_ERR_ARG, GooseError
    from paper_2604_02047_amd.decoder import PagedGooseDecoder
    shape = gi.SHAPES["small_gqa_qknorm_f16"]
    gm = gpu_model(shape, torch_model(shape, seed=6, gain_jitter=0.1), max_B=64, cap=512, max_rows=192)
    prompts = _prompts(shape.vocab, 3, 130)                        # 146, 183, 220 tokens
    pd = PagedGooseDecoder(gm, 3, n_pages=24, max_slots=448, B=40, min_score=0.0, prompt_rows=100, keep=160, recent=20)
    pd.prefill(prompts)
    assert pd.cache.len.tolist() == [130, 146, 160, 160] and [q.P for q in pd.reqs] == [146, 160, 160]
    table, refs = pd.cache.table.cpu(), pd.cache.refs.cpu()
    assert refs[table[0, :2].long()].tolist() == [4, 4] and int(refs.sum()) == 3 * 4
    outs = pd.generate(prompts, 60)
    assert all(len(o) >= 60 for o in outs) and int(pd.cache.refs.sum()) == 3
    pd = PagedGooseDecoder(gm, 3, n_pages=24, max_slots=448, B=40, prompt_rows=100, keep=140, recent=20)
    with pytest.raises(GooseError) as e:
        pd.prefill(prompts)
    assert e.value.status == GOOSE_ERR_ARG
    gm.ctx.close()
