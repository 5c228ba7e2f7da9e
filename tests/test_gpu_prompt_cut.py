"""When the paged decoder cuts its prompts: each before the next one is fed, and not at all where the sizes do not fit."""
import pytest
import torch

import goose_inputs as gi
from paper_2604_02047_amd.binding import GOOSE_ERR_ARG, GooseError
from paper_2604_02047_amd.decoder import PagedGooseDecoder
from util import gpu_model, torch_model

pytestmark = pytest.mark.gpu
SHAPE = "small_gqa_qknorm_f16"


def prompts_of(vocab, n, common, rest):
    head = gi.prefix_tokens(51, common, vocab).tolist() if common else []
    return [head + gi.prefix_tokens(60 + r, rest, vocab).tolist() for r in range(n)]


@pytest.mark.parametrize("common", [0, 70, 128])
def test_a_pool_for_cut_requests_and_one_whole_prompt(common):
    """Four prompts of 400 further tokens, cut to 200 slots.  The pages of the common beginning, of three cut requests and of one whole prompt are enough (whole ones
    would be more than twice as many), and the tokens and caches are those of a pool that holds everything."""
    shape = gi.SHAPES[SHAPE]
    gm = gpu_model(shape, torch_model(shape, seed=6, gain_jitter=0.1), max_B=64, cap=512, max_rows=192)
    prompts = prompts_of(shape.vocab, 4, common, 400)
    pages = lambda n: (n + 63) // 64  # noqa: E731
    shared = common // 64
    few = pages(common) + 3 * (pages(200) - shared) + pages(common + 400) - shared
    assert few < pages(common) + 4 * (pages(common + 400) - shared)
    outs, lens = [], []
    for n_pages in (64, few):
        pd = PagedGooseDecoder(gm, 4, n_pages=n_pages, max_slots=704, B=32, min_score=0.0, prompt_rows=192, keep=200, sink=4, recent=40)
        outs.append(pd.prefill(prompts))
        lens.append(pd.cache.len.tolist())
        assert [q.P for q in pd.reqs] == [200] * 4 and lens[-1] == [common] + [200] * 4
        assert int(pd.cache.refs.clamp(max=1).sum()) == pages(common) + 4 * (pages(200) - shared)
        outs.append(pd.generate(prompts, 12) if n_pages == 64 else None)
    assert outs[0] == outs[2] and [o[0] for o in outs[1]] == outs[0]
    gm.ctx.close()


def test_sizes_that_do_not_fit_are_refused_before_anything_is_fed():
    shape = gi.SHAPES[SHAPE]
    gm = gpu_model(shape, torch_model(shape, seed=6, gain_jitter=0.1), max_B=64, cap=512, max_rows=192)
    pd = PagedGooseDecoder(gm, 2, n_pages=32, max_slots=448, B=40, prompt_rows=100, keep=140, sink=4, recent=20)
    short = prompts_of(shape.vocab, 2, 0, 90)
    pd.prefill(short)
    before = [x.clone() for x in (pd.cache.table, pd.cache.len, pd.cache.refs, pd.cache.kpool)], [(q.P, list(q.seq)) for q in pd.reqs]
    with pytest.raises(GooseError) as e:
        pd.prefill(prompts_of(shape.vocab, 2, 130, 60))     # 128 shared slots and 20 last ones
    assert e.value.status == GOOSE_ERR_ARG
    for x, y in zip(before[0], (pd.cache.table, pd.cache.len, pd.cache.refs, pd.cache.kpool)):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    assert before[1] == [(q.P, list(q.seq)) for q in pd.reqs]
    # nothing to cut: as many shared slots as there are
    pd.prefill(prompts_of(shape.vocab, 2, 130, 10))
    assert [q.P for q in pd.reqs] == [140, 140]
    gm.ctx.close()
