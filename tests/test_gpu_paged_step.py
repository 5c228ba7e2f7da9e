"""Whole passes on a paged cache: the layer and the step beside their contiguous forms, graphs, and decoding loops that share a prompt."""
import numpy as np
import pytest
import torch

import goose_inputs as gi
from paged_ref import PAGE, unpack_pages
from util import gpu_model, torch_model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _page_rows(cache, table_row, n, d):
    """Logical K and V rows [layer][head][n][d] of a sequence."""
    k, v = unpack_pages(cache.kpool, cache.vpool, d)
    pages = torch.as_tensor(table_row[:(n + PAGE - 1) // PAGE].astype(np.int64), device=cache.kpool.device)
    out = []
    for x in (k, v):
        x = x[:, pages].transpose(1, 2)
        out.append(x.reshape(x.shape[0], x.shape[1], -1, d)[:, :, :n])
    return out


def _fill(gm, cache, Ps, common, seed):
    """Random rows for prefixes with `common` equal slots: contiguous caches per request, and the same in pages (sequence r + 1 of a fork)."""
    from paper_2604_02047_amd import layout
    d, L, H = gm.desc.head_dim, gm.desc.n_layers, gm.desc.kv_heads
    g = torch.Generator().manual_seed(seed)
    base = [torch.randn((L, H, common, d), generator=g).to(gm.dt) for _ in range(2)]
    rows = [[torch.cat((b, torch.randn((L, H, p - common, d), generator=g).to(gm.dt)), 2).to(DEV) for b in base] for p in Ps]
    caches = []
    for k, v in rows:
        kc, vc = torch.zeros_like(gm.kcache), torch.zeros_like(gm.vcache)
        s = torch.arange(k.shape[2], device=DEV)
        kc[:, :, layout.k_offsets(s, d)] = k
        vc[:, :, layout.v_offsets(s, d)] = v
        caches.append((kc, vc))
    c = gm.ctx
    one = lambda seq, n: {"seq": seq, "B": n, "path": torch.arange(n, dtype=torch.int32, device=DEV),  # noqa: E731
                          "accept_len": torch.tensor([n - 1], dtype=torch.int32, device=DEV)}

    def grow(seq, n):
        while n > 0:
            step = min(n, gm.max_B)
            c.goose_pages_reserve(cache, [seq], [step])
            c.goose_pages_commit(cache, [one(seq, step)])
            n -= step

    if common:
        grow(0, common)
        c.goose_pages_fork(cache, 0, list(range(1, len(Ps) + 1)))
    for r, p in enumerate(Ps):
        grow(r + 1, p - common)
    table = cache.table.cpu().numpy()
    for r, (k, v) in enumerate(rows):
        for i in range((Ps[r] + PAGE - 1) // PAGE):
            n = min(PAGE, Ps[r] - i * PAGE)
            s = torch.arange(n, device=DEV)
            cache.kpool[:, table[r + 1, i]][:, :, layout.k_offsets(s, d)] = k[:, :, i * PAGE:i * PAGE + n]
            cache.vpool[:, table[r + 1, i]][:, :, layout.v_offsets(s, d)] = v[:, :, i * PAGE:i * PAGE + n]
    assert c.goose_device_flags() == 0
    return caches


def _requests(gm, n, B, seed):
    rng = np.random.default_rng(seed)
    out = []
    for r in range(n):
        parent = np.array([-1] + [int(rng.integers(0, i)) for i in range(1, B[r])], np.int32)
        tokens = rng.integers(0, gm.desc.vocab, B[r])
        t, p, s = gm.stage_tree(tokens, parent, np.ones(B[r], np.uint8))
        i32 = dict(dtype=torch.int32, device=DEV)
        out.append({"tokens": t, "parent": p, "is_spine": s, "B": B[r], "accept_len": torch.zeros(1, **i32), "path": torch.zeros(128, **i32),
                    "bonus": torch.zeros(1, **i32), "next_root": torch.zeros(1, **i32)})
    return out


@pytest.mark.parametrize("name,act_mode", [("small_bf16", 0), ("tiny_gqa_bf16", 0), ("small_gqa_qknorm_bf16", 1), ("small_gqa_qknorm_f16", 0)])
def test_a_step_on_pages_beside_the_batched_step(name, act_mode):
    import dataclasses

    import paper_2604_02047_amd as goose
    from paper_2604_02047_amd.runner import GooseModel
    shape = gi.SHAPES[name]
    tm = torch_model(shape, seed=3, gain_jitter=0.1)
    desc = dataclasses.replace(goose.ModelDesc.from_shape(shape), act_mode=act_mode)
    gm = GooseModel(desc, 64, 512, lambda l: tm["layers"][l], tm["embed"], tm["lm_head"], tm["final_norm"], max_rows=256)
    Ps, B, common = [150, 201, 129], [33, 7, 64], 129
    cache = gm.paged_cache(24, 5, 400)
    caches = _fill(gm, cache, Ps, common, 1)
    rq = _requests(gm, 3, B, 2)
    d_P = [torch.tensor([p], dtype=torch.int32, device=DEV) for p in Ps]
    am0, am1 = torch.zeros(256, dtype=torch.int32, device=DEV), torch.zeros(256, dtype=torch.int32, device=DEV)
    K = 8
    tables = [[(torch.full((shape.vocab, K), -1, dtype=torch.int32, device=DEV), torch.zeros((shape.vocab, K), device=DEV))
               for _ in range(3)] for _ in range(2)]
    batch = [dict(q, P_max=p, P=dp, kcache=kc, vcache=vc, succ_ids=t[0], succ_scores=t[1])
             for q, p, dp, (kc, vc), t in zip(rq, Ps, d_P, caches, tables[0])]
    gm.ctx.goose_verify_step_batched(gm.model_ptrs(), batch, am0)
    want = [(int(q["accept_len"]), q["path"].clone(), int(q["bonus"])) for q in rq]
    paged = [dict(q, seq=r + 1, P_max=p, succ_ids=t[0], succ_scores=t[1]) for r, (q, p, t) in enumerate(zip(rq, Ps, tables[1]))]
    gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, paged, common // PAGE, am1)
    assert gm.ctx.goose_device_flags() == 0
    # the softmax weights of the successor tables are logits of the two passes side by side: equal to what 16-bit operands leave open
    for (i0, s0), (i1, s1) in zip(*tables):
        assert (i0 == i1).float().mean() > 0.98
        assert (s0 - s1).abs().max() < 2e-2
    row0, agree, total = 0, 0, 0
    for b in B:
        agree += int((am0[row0:row0 + b] == am1[row0:row0 + b]).sum())
        total += b
        row0 += (b + 31) // 32 * 32
    assert agree >= total - 2
    table, lens, refs = cache.table.cpu().numpy(), cache.len.cpu().numpy(), cache.refs.cpu().numpy()
    for r, (q, p) in enumerate(zip(rq, Ps)):
        L = int(q["accept_len"])
        assert lens[r + 1] == p + L + 1
        if want[r][0] != L or not torch.equal(want[r][1], q["path"]):
            continue  # (a near tie decided otherwise)
        assert want[r][2] == int(q["bonus"]) == int(q["next_root"])
        n = p + L + 1
        k, v = _page_rows(cache, table[r + 1], n, desc.head_dim)
        from paper_2604_02047_amd import layout
        s = torch.arange(n, device=DEV)
        for got, ref in ((k, caches[r][0][:, :, layout.k_offsets(s, desc.head_dim)]), (v, caches[r][1][:, :, layout.v_offsets(s, desc.head_dim)])):
            assert torch.equal(got[:, :, :p], ref[:, :, :p])                          # the prefix, bit for bit
            assert (got - ref).abs().max() <= 2e-2 * ref.abs().max()                  # the committed rows
            assert (got[0] - ref[0]).abs().max() <= torch.finfo(gm.dt).eps * ref[0].abs().max()   # layer 0: the same projection, one rounding
    # shared pages are held by the prompt and all three; nothing beyond the lengths is held
    assert list(refs[table[0, :2]]) == [4, 4] and refs.sum() == sum((int(x) + 63) // 64 for x in lens)
    gm.ctx.close()


def test_a_layer_does_not_depend_on_the_sharing():
    shape = gi.SHAPES["small_bf16"]
    tm = torch_model(shape, seed=5)
    gm = gpu_model(shape, tm, max_B=64, cap=512, max_rows=128)
    cache = gm.paged_cache(20, 3, 320)
    _fill(gm, cache, [130, 180], 128, 4)
    B = [20, 40]
    from paged_ref import mask_words
    rng = np.random.default_rng(0)
    masks = [mask_words([-1] + [int(rng.integers(0, i)) for i in range(1, b)]) for b in B]
    gm.ctx.goose_pages_reserve(cache, [1, 2], B)
    reqs = []
    for r, (b, p) in enumerate(zip(B, [130, 180])):
        depth = masks[r][1].sum(1) - 1
        reqs.append({"seq": r + 1, "B": b, "P_max": p, "mask": masks[r][0].to(DEV), "pos": torch.tensor(p + depth, dtype=torch.int32, device=DEV)})
    x0 = torch.randn((96, shape.hidden), generator=torch.Generator().manual_seed(1)).to(DEV)
    out = []
    for shared in (0, 1, 2):
        x = x0.clone()
        gm.ctx.goose_verify_layer_paged(gm.packed_layer(1), cache, 1, x, reqs, shared)
        out.append(x)
    assert gm.ctx.goose_device_flags() == 0
    scale = (out[0] - x0).abs().max()
    for x in out[1:]:
        assert (x - out[0]).abs().max() <= 5e-3 * scale
        assert torch.equal(x[20:32], out[0][20:32]) or (x[20:32] - out[0][20:32]).abs().max() <= 1e-2 * scale  # rows between requests: finite
    gm.ctx.close()


def test_a_captured_step_follows_pages_and_lengths():
    """One graph of a whole step; replays advance the sequences, take and give back pages, and equal the eager steps of a second cache."""
    shape = gi.SHAPES["tiny_gqa_bf16"]
    tm = torch_model(shape, seed=7, gain_jitter=0.1)
    gm = gpu_model(shape, tm, max_B=32, cap=512, max_rows=64)
    c0, c1 = gm.paged_cache(16, 3, 256), gm.paged_cache(16, 3, 256)
    for c in (c0, c1):
        _fill(gm, c, [70, 90], 64, 9)
    rq = _requests(gm, 2, [12, 20], 11)
    am = [torch.zeros(64, dtype=torch.int32, device=DEV) for _ in range(2)]
    table = [dict(q, seq=r + 1, P_max=230) for r, q in enumerate(rq)]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        gm.ctx.goose_verify_step_paged(gm.model_ptrs(), c0, table, 1, am[0])
    for i in range(8):
        with torch.cuda.stream(st):
            graph.replay()
        st.synchronize()
        got = [(int(q["accept_len"]), int(q["bonus"])) for q in rq]
        torch.zeros(1000, device=DEV).sum().item()
        gm.ctx.goose_verify_step_paged(gm.model_ptrs(), c1, table, 1, am[1])
        torch.cuda.synchronize()
        assert got == [(int(q["accept_len"]), int(q["bonus"])) for q in rq], i
        assert torch.equal(am[0][:12], am[1][:12]) and torch.equal(am[0][32:52], am[1][32:52])
        for a, b in ((c0.table, c1.table), (c0.len, c1.len), (c0.refs, c1.refs)):
            assert torch.equal(a, b), i
    assert torch.equal(c0.kpool, c1.kpool) and torch.equal(c0.vpool, c1.vpool)
    assert gm.ctx.goose_device_flags() == 0
    gm.ctx.close()


def _prompts(vocab, n, common):
    pat = gi.prefix_tokens(31, 12, vocab).tolist()
    head = (pat * (common // 12 + 1))[:common]
    return [head + gi.prefix_tokens(40 + r, 10 + 7 * r, vocab).tolist() + pat[:6] for r in range(n)]


@pytest.mark.parametrize("common", [0, 40, 150])
def test_paged_decoding_gives_each_request_its_own_tokens(common):
    """Requests that share a prompt, decoded over one paged cache, against each decoded alone over a contiguous one.  16-bit near-ties may be
    decided differently where launches differ in shape: long agreement is the check, as for the batched decoder."""
    from paper_2604_02047_amd.decoder import GooseDecoder, PagedGooseDecoder
    shape = gi.SHAPES["small_bf16"]
    tm = torch_model(shape, seed=6, gain_jitter=0.1)
    prompts = _prompts(shape.vocab, 3, common)
    gm = gpu_model(shape, tm, max_B=64, cap=512, max_rows=192)
    pd = PagedGooseDecoder(gm, 3, n_pages=24, max_slots=448, B=40, min_score=0.0)
    outs = pd.generate(prompts, 60)
    assert pd.shared_pages == common // 64 and pd.passes < sum(len(o) for o in outs) / 3
    refs = pd.cache.refs.cpu()
    assert int(refs.sum()) == (common + 63) // 64      # all requests have given their pages back, the prompt's are held
    again = pd.generate(prompts, 60)                   # and the pool serves a second round
    assert again == outs
    gm.ctx.close()
    for r, prompt in enumerate(prompts):
        gm = gpu_model(shape, tm, max_B=64, cap=512)
        y = GooseDecoder(gm, B=40, min_score=0.0).generate(prompt, 60)
        gm.ctx.close()
        n = min(len(y), len(outs[r]))
        same = next((i for i in range(n) if y[i] != outs[r][i]), n)
        assert same >= 40, (r, same, y[:same + 2], outs[r][:same + 2])


def test_a_full_pool_stops_decoding_with_an_error():
    from paper_2604_02047_amd.binding import GOOSE_ERR_CAPACITY, GooseError
    from paper_2604_02047_amd.decoder import PagedGooseDecoder
    shape = gi.SHAPES["tiny_bf16"]
    tm = torch_model(shape, seed=4, gain_jitter=0.1)
    gm = gpu_model(shape, tm, max_B=64, cap=512, max_rows=128)
    for pages, slots in ((5, 512), (40, 128)):      # the pool, and a sequence's table
        pd = PagedGooseDecoder(gm, 2, n_pages=pages, max_slots=slots, B=24, min_score=0.0)
        with pytest.raises(GooseError) as e:
            pd.generate(_prompts(shape.vocab, 2, 70), 400)
        assert e.value.status == GOOSE_ERR_CAPACITY
    gm.ctx.close()


def test_a_step_without_room_is_left_undone_and_can_be_run_again():
    """Six pages, three of them held by a third sequence, three by the prompt and the requests: the step finds no room for one request, commits nothing for either, and after the third has given
    its pages back it does what it does in a pool with room."""
    from paper_2604_02047_amd import binding as gb
    shape = gi.SHAPES["tiny_gqa_bf16"]
    tm = torch_model(shape, seed=7, gain_jitter=0.1)
    gm = gpu_model(shape, tm, max_B=32, cap=512, max_rows=64)
    rq = _requests(gm, 2, [12, 20], 13)
    am = torch.zeros(64, dtype=torch.int32, device=DEV)
    seen = []
    for pages in (6, 16):
        cache = gm.paged_cache(pages, 4, 256)
        _fill(gm, cache, [50, 60], 40, 12)                 # one page each, the prompt's page beside them
        if pages == 6:
            gm.ctx.goose_pages_reserve(cache, [3], [3 * PAGE])
            before = [x.clone() for x in (cache.table, cache.len, cache.refs)]
            table = [dict(q, seq=r + 1, P_max=p) for r, (q, p) in enumerate(zip(rq, (50, 60)))]
            gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, table, 0, am)
            assert gm.ctx.goose_device_flags() & gb.GOOSE_FLAG_PAGES
            assert all(torch.equal(a, b) for a, b in zip(before, (cache.table, cache.len, cache.refs)))
            gm.ctx.goose_pages_free(cache, [3])
        gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, table, 0, am)
        assert gm.ctx.goose_device_flags() == 0
        seen.append(([(int(q["accept_len"]), int(q["bonus"])) for q in rq], cache.len.tolist(), am[:12].clone(), am[32:52].clone()))
    assert seen[0][:2] == seen[1][:2] and torch.equal(seen[0][2], seen[1][2]) and torch.equal(seen[0][3], seen[1][3])
    gm.ctx.close()


def _layer_requests(Bs, Ps, seed=0):
    from paged_ref import mask_words
    rng = np.random.default_rng(seed)
    reqs = []
    for r, (b, p) in enumerate(zip(Bs, Ps)):
        words, see = mask_words([-1] + [int(rng.integers(0, i)) for i in range(1, b)])
        reqs.append({"seq": r + 1, "B": b, "P_max": p, "mask": words.to(DEV), "pos": torch.tensor(p + see.sum(1) - 1, dtype=torch.int32, device=DEV)})
    return reqs


@pytest.mark.parametrize("Bs", [[5], [5, 5], [20, 40], [64, 64, 33], [33, 1]])
def test_a_layer_writes_no_row_behind_the_last_request(Bs):
    """x of exactly the rows that the call asks for, at the front of a larger allocation whose rest must stay."""
    shape = gi.SHAPES["small_bf16"]
    gm = gpu_model(shape, torch_model(shape, seed=5), max_B=64, cap=512, max_rows=256)
    cache = gm.paged_cache(24, len(Bs) + 1, 320)
    Ps = [130 + 9 * r for r in range(len(Bs))]
    _fill(gm, cache, Ps, 128, 4)
    gm.ctx.goose_pages_reserve(cache, list(range(1, len(Bs) + 1)), Bs)
    reqs = _layer_requests(Bs, Ps)
    rows = sum((b + 31) // 32 * 32 for b in Bs[:-1]) + Bs[-1]
    x0 = torch.randn((256, shape.hidden), generator=torch.Generator().manual_seed(1)).to(DEV)
    big, exact = x0.clone(), x0.clone()
    gm.ctx.goose_verify_layer_paged(gm.packed_layer(1), cache, 1, big, reqs, 2)
    gm.ctx.goose_verify_layer_paged(gm.packed_layer(1), cache, 1, exact[:rows], reqs, 2)
    assert gm.ctx.goose_device_flags() == 0
    assert torch.equal(exact[rows:], x0[rows:]) and torch.equal(big[rows:], x0[rows:])
    assert torch.equal(exact, big) and not torch.equal(exact[rows - 1], x0[rows - 1]) and exact[:rows].isfinite().all()
    gm.ctx.close()


@pytest.mark.parametrize("Bs", [[1], [5], [20, 12], [64, 64, 33], [33, 1]])
def test_a_step_writes_no_prediction_behind_the_last_request(Bs):
    """argmax_all of exactly the entries that the call asks for, at the front of a larger allocation whose rest must stay."""
    shape = gi.SHAPES["small_bf16"]
    gm = gpu_model(shape, torch_model(shape, seed=5), max_B=64, cap=512, max_rows=256)
    n = len(Bs)
    rows = sum((b + 31) // 32 * 32 for b in Bs[:-1]) + Bs[-1]
    Ps, seen = [130 + 9 * r for r in range(n)], []
    rq = _requests(gm, n, Bs, 3)
    for size in (256, rows):
        cache = gm.paged_cache(24, n + 1, 320)
        _fill(gm, cache, Ps, 128, 4)
        am = torch.full((256,), -9, dtype=torch.int32, device=DEV)
        gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, [dict(q, seq=r + 1, P_max=p) for r, (q, p) in enumerate(zip(rq, Ps))], 2, am[:size])
        assert gm.ctx.goose_device_flags() == 0
        assert (am[rows:] == -9).all()
        seen.append((am.clone(), [(int(q["accept_len"]), int(q["bonus"])) for q in rq]))
    at = 0
    for b in Bs:
        assert (seen[0][0][at:at + b] >= 0).all() and torch.equal(seen[0][0][at:at + b], seen[1][0][at:at + b])
        at += (b + 31) // 32 * 32
    assert seen[0][1] == seen[1][1]
    with pytest.raises(Exception) as e:
        gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, [dict(q, seq=r + 1, P_max=p) for r, (q, p) in enumerate(zip(rq, Ps))], 2, am[:rows - 1])
    assert e.value.status == -1
    gm.ctx.close()


def _state(cache):
    torch.cuda.synchronize()
    return [x.clone() for x in (cache.table, cache.len, cache.refs)]


@pytest.mark.parametrize("what", ["P_max", "shared_len", "shared_more", "shared_pages", "hole", "P_max in a graph"])
def test_a_step_that_its_arguments_do_not_fit_is_left_undone(what):
    """A length above P_max, shared pages beyond a length, tables that differ in them, an entry out of range: flagged; tables, lengths, counts and committed
    rows stay, and with arguments that fit the step does what it does in a fresh cache."""
    from paper_2604_02047_amd import binding as gb
    shape = gi.SHAPES["tiny_gqa_bf16"]
    gm = gpu_model(shape, torch_model(shape, seed=7, gain_jitter=0.1), max_B=32, cap=512, max_rows=64)
    rq = _requests(gm, 2, [12, 20], 11)
    am = torch.zeros(64, dtype=torch.int32, device=DEV)
    Ps, seen = [140, 170], []
    for trial in range(2):
        cache = gm.paged_cache(24, 3, 320)
        _fill(gm, cache, Ps, 130, 9)
        table = [dict(q, seq=r + 1, P_max=p) for r, (q, p) in enumerate(zip(rq, Ps))]
        if trial == 0:
            bad, shared, flag, entry = [dict(q) for q in table], 2, gb.GOOSE_FLAG_CAPACITY, None
            if what.startswith("P_max"):
                bad[1]["P_max"] = 169
            elif what == "shared_len":
                cache.len[1] = 127
            elif what == "shared_more":   # three pages of 140 and 170 slots
                shared = 3
                bad[0]["P_max"] = bad[1]["P_max"] = 200
            else:
                flag, entry = gb.GOOSE_FLAG_PAGES, (2, 0, 7 if what == "shared_pages" else -1)
                shared = 2 if what == "shared_pages" else 0
            if entry:
                kept = int(cache.table[entry[:2]])
                cache.table[entry[:2]] = entry[2]
            before, rows = _state(cache), [x.clone() for x in _page_rows(cache, cache.table[1].cpu().numpy(), 127, 64)]
            if what.endswith("graph"):
                st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.graph(graph, stream=st):
                    gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, bad, shared, am)
                for _ in range(3):
                    graph.replay()
            else:
                gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, bad, shared, am)
            torch.cuda.synchronize()
            assert gm.ctx.goose_device_flags() & flag
            assert all(torch.equal(a, b) for a, b in zip(before, _state(cache)))
            assert all(torch.equal(a, b) for a, b in zip(rows, _page_rows(cache, cache.table[1].cpu().numpy(), 127, 64)))
            if what == "shared_len":
                break   # (rows behind the length that it was given here, 127, are nobody's: the undone step may have written there)
            if entry:
                cache.table[entry[:2]] = kept
        gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, table, 2, am)
        assert gm.ctx.goose_device_flags() == 0
        seen.append(([(int(q["accept_len"]), int(q["bonus"])) for q in rq], cache.len.tolist(), am[:12].clone(), am[32:52].clone()))
    if seen:
        assert seen[0][:2] == seen[1][:2] and torch.equal(seen[0][2], seen[1][2]) and torch.equal(seen[0][3], seen[1][3])
    gm.ctx.close()


@pytest.mark.parametrize("vocab_chunks", [1, 2])
def test_an_undone_step_touches_neither_roots_nor_successor_tables(vocab_chunks):
    """No room for one of two requests: next roots (which may be the trees' own first tokens), paths, accept lengths and the harvested tables stay as they
    were for both, with a vocabulary of one chunk of the harvest and of several; with room, a second step over the same buffers writes them."""
    import dataclasses

    import paper_2604_02047_amd as goose
    from paper_2604_02047_amd import binding as gb
    from paper_2604_02047_amd.runner import GooseModel
    shape = dataclasses.replace(gi.SHAPES["tiny_gqa_bf16"], vocab=1024 if vocab_chunks == 1 else 9000)
    tm = torch_model(shape, seed=7, gain_jitter=0.1)
    gm = GooseModel(goose.ModelDesc.from_shape(shape), 32, 512, lambda l: tm["layers"][l], tm["embed"], tm["lm_head"], tm["final_norm"], max_rows=64)
    rq, K = _requests(gm, 2, [12, 20], 13), 4
    cache = gm.paged_cache(6, 4, 256)
    _fill(gm, cache, [50, 60], 40, 12)
    gm.ctx.goose_pages_reserve(cache, [3], [3 * PAGE])             # (two pages held, the prompt's and three: none is left)
    g = torch.Generator().manual_seed(1)
    reqs, kept = [], []
    for r, q in enumerate(rq):
        ids = torch.randint(0, shape.vocab, (shape.vocab, K), generator=g).to(torch.int32).to(DEV)
        scores = torch.rand((shape.vocab, K), generator=g).to(DEV)
        for name in ("accept_len", "path", "bonus"):
            q[name].fill_(-77)
        reqs.append(dict(q, seq=r + 1, P_max=50 + 10 * r, succ_ids=ids, succ_scores=scores, next_root=q["tokens"][:1]))
        kept.append([reqs[r][k].clone() for k in ("tokens", "accept_len", "path", "bonus", "succ_ids", "succ_scores")])
    am = torch.zeros(64, dtype=torch.int32, device=DEV)
    for room in (False, True):
        if room:
            gm.ctx.goose_pages_free(cache, [3])
        gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, reqs, 0, am)
        flags = gm.ctx.goose_device_flags()
        assert flags == 0 if room else flags & gb.GOOSE_FLAG_PAGES
        for q, before in zip(reqs, kept):
            for k, x in zip(("tokens", "accept_len", "path", "bonus", "succ_ids", "succ_scores"), before):
                assert torch.equal(q[k], x) == (not room) or (room and k == "tokens" and int(q["bonus"]) == int(x[0])), (room, k)
    gm.ctx.close()


@pytest.mark.parametrize("name", ["small_bf16", "small_gqa_qknorm_f16"])
def test_committed_rows_of_accepted_paths(name):
    """Trees whose path 0, 3, 8, 14, 21 carries the model's own predictions, so that it is accepted; the committed rows begin in one page and end in the
    next.  They are compared for every request with those of the batched step: the walk must be the same, with at least four nodes accepted."""
    from paper_2604_02047_amd import layout
    shape = gi.SHAPES[name]
    tm = torch_model(shape, seed=3, gain_jitter=0.1)
    gm = gpu_model(shape, tm, max_B=64, cap=512, max_rows=256)
    d, Ps, B, way = gm.desc.head_dim, [190, 254, 318], [24, 33, 40], [0, 3, 8, 14, 21]
    cache = gm.paged_cache(24, 4, 448)
    caches = _fill(gm, cache, Ps, 129, 1)
    rq = _requests(gm, 3, B, 2)
    am = torch.zeros(256, dtype=torch.int32, device=DEV)
    for q, b in zip(rq, B):
        for up, node in zip(way, way[1:]):
            q["parent"][node] = up
        for node in range(1, b):    # (a child of the path that is not on it must not be accepted before its turn)
            if node not in way and int(q["parent"][node]) in way:
                q["parent"][node] = 1 if node > 2 else 0

    def batched():
        d_P = [torch.tensor([p], dtype=torch.int32, device=DEV) for p in Ps]
        gm.ctx.goose_verify_step_batched(gm.model_ptrs(), [dict(q, P_max=p, P=dp, kcache=kc, vcache=vc)
                                                            for q, p, dp, (kc, vc) in zip(rq, Ps, d_P, caches)], am)
        torch.cuda.synchronize()

    start = [(kc.clone(), vc.clone()) for kc, vc in caches]
    for up, node in zip(way, way[1:]):
        batched()
        at = 0
        for q, b in zip(rq, B):
            q["tokens"][node] = am[at + up]
            at += (b + 31) // 32 * 32
    for (kc, vc), (k0, v0) in zip(caches, start):
        kc.copy_(k0)
        vc.copy_(v0)
    batched()
    want = [(int(q["accept_len"]), q["path"].clone(), int(q["bonus"])) for q in rq]
    gm.ctx.goose_verify_step_paged(gm.model_ptrs(), cache, [dict(q, seq=r + 1, P_max=p) for r, (q, p) in enumerate(zip(rq, Ps))], 2, am)
    assert gm.ctx.goose_device_flags() == 0
    table = cache.table.cpu().numpy()
    for r, (q, p) in enumerate(zip(rq, Ps)):
        L = int(q["accept_len"])
        assert L >= 4 and want[r][0] == L and torch.equal(want[r][1][:L + 1], q["path"][:L + 1]) and want[r][2] == int(q["bonus"])
        assert q["path"][:5].tolist() == way and int(cache.len[r + 1]) == p + L + 1
        n = p + L + 1
        s = torch.arange(n, device=DEV)
        k, v = _page_rows(cache, table[r + 1], n, d)
        for got, ref in ((k, caches[r][0][:, :, layout.k_offsets(s, d)]), (v, caches[r][1][:, :, layout.v_offsets(s, d)])):
            assert torch.equal(got[:, :, :p], ref[:, :, :p])
            assert (got - ref).abs().max() <= 2e-2 * ref.abs().max()
            assert (got[0] - ref[0]).abs().max() <= torch.finfo(gm.dt).eps * ref[0].abs().max()
    gm.ctx.close()
