"""Paged caches without a GPU: what the binding and the entry points refuse before anything is launched, and the simulator itself."""
import numpy as np
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, PageSim, mask_words, pack_pages, unpack_pages


def tensors(**kw):
    t = {"kpool": torch.zeros((2, 7, 3, 64 * 64), dtype=torch.bfloat16), "vpool": torch.zeros((2, 7, 3, 64 * 64), dtype=torch.bfloat16),
         "table": torch.zeros((4, 5), dtype=torch.int32), "len": torch.zeros(4, dtype=torch.int32), "refs": torch.zeros(7, dtype=torch.int32)}
    t.update(kw)
    return t


def test_the_cache_checks_its_tensors():
    goose.PagedCache(**tensors())
    bad = [dict(vpool=torch.zeros((2, 7, 3, 64 * 128), dtype=torch.bfloat16)), dict(vpool=torch.zeros((2, 7, 3, 64 * 64), dtype=torch.float16)),
           dict(kpool=torch.zeros((2, 7, 3, 64 * 64)), vpool=torch.zeros((2, 7, 3, 64 * 64))), dict(table=torch.zeros((4, 5))),
           dict(len=torch.zeros(3, dtype=torch.int32)), dict(refs=torch.zeros(8, dtype=torch.int32)),
           dict(table=torch.zeros((5, 4), dtype=torch.int32).t())]
    for b in bad:
        with pytest.raises(goose.GooseError) as e:
            goose.PagedCache(**tensors(**b))
        assert e.value.status == gb.GOOSE_ERR_ARG


def test_requests_check_their_tensors():
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    good = {"seq": 0, "B": 70, "P_max": 5, "tokens": i32(70), "parent": i32(70), "is_spine": torch.zeros(70, dtype=torch.uint8), "pos": i32(80),
            "path": i32(128), "mask": torch.zeros((70, 2), dtype=torch.int64), "accept_len": i32(1), "bonus": i32(1), "next_root": i32(1),
            "succ_ids": torch.zeros((9, 4), dtype=torch.int32), "succ_scores": torch.zeros((9, 4))}
    r = goose.PagedRequests([good, dict(good, seq=1, B=3, is_spine=None, succ_ids=None, succ_scores=None)])
    assert len(r) == 2 and r.rows == 96 + 3 and r._c[0].harvest_k == 4 and r._c[1].harvest_k == 0
    bad = [dict(tokens=i32(69)), dict(tokens=torch.zeros(70, dtype=torch.int64)), dict(parent=i32(140)[::2]), dict(pos=torch.zeros(70)),
           dict(path=i32(64)), dict(mask=torch.zeros((70, 1), dtype=torch.int64)), dict(mask=i32(280)), dict(is_spine=i32(70)),
           dict(accept_len=i32(0)), dict(accept_len=torch.zeros(1, dtype=torch.int64)), dict(bonus=torch.zeros(1)), dict(succ_ids=None),
           dict(succ_scores=None), dict(succ_scores=torch.zeros((9, 5))), dict(succ_ids=torch.zeros((9, 4))),
           dict(succ_ids=torch.zeros((4, 9), dtype=torch.int32).t())]
    for b in bad:
        with pytest.raises(goose.GooseError) as e:
            goose.PagedRequests([good, dict(good, seq=1, **b)])
        assert e.value.status == gb.GOOSE_ERR_ARG, b


def test_a_cache_in_host_memory_or_on_another_device_is_refused(monkeypatch):
    """Before the library is called: the context here has none."""
    ctx = object.__new__(goose.GooseContext)
    ctx._device = 0
    ctx.desc = goose.ModelDesc(2, 192, 3, 64, 128, 1024)
    ctx._cache_shape = (torch.bfloat16, 2, 3, 64 * 64)
    cache = goose.PagedCache(**tensors())
    for device, current in ((-1, 0), (1, 0), (1, 1), (0, 1)):
        cache._device = device
        monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
        for call in (lambda: ctx.goose_pages_clear(cache), lambda: ctx.goose_pages_free(cache, [0]), lambda: ctx.goose_pages_fork(cache, 0, [1]),
                     lambda: ctx.goose_pages_reserve(cache, [0], [1]), lambda: ctx.goose_pages_commit(cache, [{"seq": 0, "B": 1}])):
            with pytest.raises(goose.GooseError) as e:
                call()
            assert e.value.status == gb.GOOSE_ERR_ARG


def test_entry_points_refuse_a_missing_context():
    lib = goose.load_library()
    import ctypes as C
    pages = C.byref(goose.PagedCache(**tensors())._c)
    s = gb._seqs([0])
    r = goose.PagedRequests([{"seq": 0, "B": 1}])._c
    assert lib.goose_pages_clear(None, pages, None) == -1
    assert lib.goose_pages_fork(None, pages, 1, -1, s, 1, None) == -1
    assert lib.goose_pages_reserve(None, pages, s, s, 1, None) == -1
    assert lib.goose_pages_commit(None, pages, r, 1, None) == -1
    assert lib.goose_pages_free(None, pages, s, 1, None) == -1
    assert lib.goose_qk_norm_rope_paged(None, pages, 0, None, 1, 4, 4, None, None, r, 1, None, 8, 1, None) == -1
    assert lib.goose_attn_paged(None, pages, 0, None, 8, 1, r, 1, 0, None, 8, 0, 1, None) == -1
    assert lib.goose_verify_layer_paged(None, None, pages, 0, None, r, 1, 0, None) == -1
    assert lib.goose_verify_step_paged(None, None, pages, r, 1, 0, None, None) == -1


def test_request_structs_match_the_header(tmp_path):
    """Size and field offsets of the two descriptors as a C compiler lays them out."""
    import ctypes as C
    import os
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [("goose_pages", gb._Pages), ("goose_paged_request", gb._PagedRequest)]
    body = "".join(f'printf("%zu ", sizeof({c}));' + "".join(f'printf("%zu ", offsetof({c}, {f[0]}));' for f in t._fields_) for c, t in names)
    src = tmp_path / "o.c"
    src.write_text('#include <stdio.h>\n#include "goose.h"\nint main(void){' + body + "return 0;}\n")
    subprocess.run([gcc, "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "o")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "o")], capture_output=True, text=True).stdout.split()]
    want = []
    for _, t in names:
        want += [C.sizeof(t)] + [getattr(t, f[0]).offset for f in t._fields_]
    assert got == want


def test_simulator_and_layout():
    k = torch.arange(2 * 3 * 1 * PAGE * 64, dtype=torch.float32).view(2, 3, 1, PAGE, 64)
    kp, vp = pack_pages(k, -k)
    a, b = unpack_pages(kp, vp, 64)
    assert torch.equal(a, k) and torch.equal(b, -k)
    s = PageSim(4, 3, 5)
    assert s.reserve([0], [70]) == 0 and list(s.table[0]) == [0, 1, -1]
    s.len[0] = 70
    assert s.fork(0, [1, 2]) == 0 and list(s.refs) == [3, 3, 0, 0, 0]
    assert s.reserve([1, 2, 0], [1, 60, 1]) == 0
    assert list(s.table[1]) == [0, 2, -1] and list(s.table[2]) == [0, 3, 4] and list(s.table[0]) == [0, 1, -1]
    assert list(s.refs) == [3, 1, 1, 1, 1] and s.reserve([3], [1]) == 16
    s.free([2])
    assert list(s.refs) == [2, 1, 1, 0, 0]
    words, see = mask_words([-1, 0, 1, 0])
    assert words.tolist() == [[1], [3], [7], [9]] and see[3].tolist() == [True, False, False, True]
    assert np.array_equal(see, np.tril(see))


class AnyCall:
    """A library that does whatever it is told."""

    def __getattr__(self, name):
        return lambda *a: 0


def test_integers_beyond_32_bits_are_refused(monkeypatch):
    """Sequence 2^32 is not sequence 0, nor a layer, a length or a count of shared pages the rest of its division by 2^32."""
    path = torch.zeros(128, dtype=torch.int32)
    far = (1 << 32, (1 << 32) + 1, 1 << 31, -(1 << 31) - 1, (1 << 64) - 1)

    def refused(call):
        with pytest.raises(goose.GooseError) as e:
            call()
        assert e.value.status == gb.GOOSE_ERR_ARG

    ctx = object.__new__(goose.GooseContext)
    ctx._h, ctx._device, ctx.desc = None, 0, goose.ModelDesc(2, 192, 3, 64, 128, 1024)
    ctx._cache_shape, ctx.lib = (torch.bfloat16, 2, 3, 64 * 64), AnyCall()
    cache = goose.PagedCache(**tensors())
    cache._device = 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(gb, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(gb.GooseContext, "_paged", lambda self, cache, reqs, *t: (reqs, 0))
    rows = torch.zeros((32, 9 * 64), dtype=torch.bfloat16)
    reqs = goose.PagedRequests([{"seq": 0, "B": 1}])
    for x in far:
        refused(lambda: goose.PagedRequests([{"seq": x, "B": 1, "path": path}]))
        refused(lambda: goose.PagedRequests([{"seq": 0, "B": 1, "P_max": x, "path": path}]))
        refused(lambda: goose.PagedRequests([{"seq": 0, "B": x}]))
        refused(lambda: gb._seqs([0, x]))
        refused(lambda: ctx.goose_pages_free(cache, [x]))
        refused(lambda: ctx.goose_pages_reserve(cache, [0], [x]))
        refused(lambda: ctx.goose_pages_fork(cache, x, [1]))
        refused(lambda: ctx.goose_pages_fork(cache, 0, [1], x))
        refused(lambda: ctx.goose_attn_paged(cache, x, rows, 1, reqs, 0, rows))
        refused(lambda: ctx.goose_attn_paged(cache, 0, rows, 1, reqs, x, rows))
        refused(lambda: ctx.goose_qk_norm_rope_paged(cache, x, torch.zeros((1, 32, 9 * 64)), None, None, reqs, rows))
        refused(lambda: ctx.goose_verify_layer_paged(rows, cache, x, torch.zeros((32, 192)), reqs))
    assert list(gb._seqs([0, 2 ** 31 - 1, -2 ** 31])) == [0, 2 ** 31 - 1, -2 ** 31]
