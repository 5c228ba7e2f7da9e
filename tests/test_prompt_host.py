"""Prompts on a paged cache without a GPU: what the binding and the entry points refuse before anything is launched, and the simulator itself."""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2604_02047_amd as goose
from paper_2604_02047_amd import binding as gb
from paged_ref import PAGE, attention64
from prompt_ref import PromptSim, chunk_attention64, slot_weights64


def test_chunks_check_their_tensors():
    pos = torch.zeros(70, dtype=torch.int32)
    c = goose.PagedChunks([{"seq": 0, "C": 70, "P_max": 5, "pos": pos}, {"seq": 1, "C": 3, "first": 2}])
    assert len(c) == 2 and c.rows == 96 + 3 and c._c[0].d_pos == pos.data_ptr() and c._c[1].d_pos is None and c._c[1].first == 2
    for bad in (dict(pos=pos[:69]), dict(pos=pos.long()), dict(pos=torch.zeros(140, dtype=torch.int32)[::2]), dict(C=1 << 31), dict(seq=1 << 32),
                dict(P_max=1 << 31), dict(first=-(1 << 31) - 1)):
        with pytest.raises(goose.GooseError) as e:
            goose.PagedChunks([dict({"seq": 0, "C": 70, "P_max": 5, "pos": pos}, **bad)])
        assert e.value.status == gb.GOOSE_ERR_ARG, bad


def test_entry_points_refuse_a_missing_context():
    lib = goose.load_library()
    t = {"kpool": torch.zeros((2, 7, 3, 64 * 64), dtype=torch.bfloat16), "vpool": torch.zeros((2, 7, 3, 64 * 64), dtype=torch.bfloat16),
         "table": torch.zeros((4, 5), dtype=torch.int32), "len": torch.zeros(4, dtype=torch.int32), "refs": torch.zeros(7, dtype=torch.int32)}
    pages = C.byref(goose.PagedCache(**t)._c)
    c = goose.PagedChunks([{"seq": 0, "C": 1}])._c
    e = (gb._Eviction * 1)(gb._Eviction(0, 1, 0, 0))
    assert lib.goose_attn_chunk_paged(None, pages, 0, None, 8, 1, c, 1, None, 8, 0, 1, None, 0, None) == -1
    assert lib.goose_attn_weight_paged(None, pages, 0, None, 8, 1, c, 1, None, 0, 1.0, None, None) == -1
    assert lib.goose_pages_append(None, pages, c, 1, None) == -1
    assert lib.goose_pages_evict(None, pages, e, 1, None, None, 0, None) == -1
    assert lib.goose_chunk_layer_paged(None, None, pages, 0, None, c, 1, None, 1.0, None) == -1


def test_structs_match_the_header(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [("goose_chunk", gb._Chunk), ("goose_eviction", gb._Eviction)]
    body = "".join(f'printf("%zu ", sizeof({c}));' + "".join(f'printf("%zu ", offsetof({c}, {f[0]}));' for f in t._fields_) for c, t in names)
    src = tmp_path / "o.c"
    src.write_text('#include <stdio.h>\n#include "goose.h"\nint main(void){' + body + 'printf("%d", GOOSE_MAX_CHUNK); return 0;}\n')
    subprocess.run([gcc, "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "o")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "o")], capture_output=True, text=True).stdout.split()]
    want = []
    for _, t in names:
        want += [C.sizeof(t)] + [getattr(t, f[0]).offset for f in t._fields_]
    assert got == want + [32768]


def test_the_plain_forms_agree():
    """Causal attention against the masked form, weights against its probabilities."""
    g = torch.Generator().manual_seed(1)
    q, k = torch.randn((9, 4, 16), generator=g).double(), torch.randn((2, 14, 16), generator=g).double()
    v = torch.randn((2, 14, 16), generator=g).double()
    see = torch.from_numpy(np.concatenate([np.ones((9, 5), bool), np.tril(np.ones((9, 9), bool))], 1))
    a = attention64(q, k, v, see)
    out, mag, lse, qk, vs = chunk_attention64(q, k, v, 5)
    for x, y in ((out, a[0]), (mag, a[1]), (qk, a[2]), (vs, a[3])):
        assert torch.allclose(x, y, rtol=1e-12, atol=1e-12)
    w, err = slot_weights64(q, k, lse, 5, 0)
    assert torch.allclose(w.sum(1), torch.full((2,), 18.0, dtype=torch.float64)) and (err > 0).all()
    last = slot_weights64(q, k, lse, 5, 8)[0]
    s = torch.softmax((q[8].view(2, 2, 16) @ k.transpose(1, 2)) / 4.0, -1).sum(1)
    assert torch.allclose(last, s)
    # a NaN in a row that only the last token sees
    v[:, 13] = math.nan
    out = chunk_attention64(q, k, v, 5)[0]
    assert out[8].isnan().all() and torch.allclose(out[:8], a[0][:8])


def test_the_simulator():
    k = torch.randn(1, 4, 1, PAGE, 4)
    s = PromptSim(2, 3, 4, k.clone(), -k.clone())
    assert s.append([0], [3]) == 16 and s.reserve([0], [70]) == 0 and s.append([0], [70]) == 0 and s.len[0] == 70
    w = torch.zeros(1, 2, 1, 3 * PAGE)
    w[0, 0, 0, [5, 30, 69]] = torch.tensor([2.0, 3.0, 1.0])
    flags, words = s.evict([{"seq": 0, "keep": 4, "sink": 1}], w, 10000.0, False)
    assert flags == 0 and s.len[0] == 4 and list(s.table[0]) == [0, -1, -1] and list(s.refs) == [1, 0, 0, 0]
    assert words[0][0, 0, 0] == (1 << 0) | (1 << 5) | (1 << 30) and words[0][0, 0, 1] == 1 << 5
    assert torch.equal(s.k[0, 0, 0, :4], torch.stack((k[0, 0, 0, 0], k[0, 0, 0, 5], k[0, 0, 0, 30], k[0, 1, 0, 5])))
    assert torch.equal(s.k[0, 0, 0, 4:], k[0, 0, 0, 4:]) and w[0, 0, 0, :4].tolist() == [0.0, 2.0, 3.0, 1.0]
    # turned by a position that is given up: the product with a query at the new distance is that at the old one
    s = PromptSim(1, 2, 2, torch.randn(1, 2, 1, PAGE, 4).double(), torch.zeros(1, 2, 1, PAGE, 4).double())
    s.reserve([0], [10])
    s.append([0], [10])
    x = s.k[0, 0, 0, 9].clone()
    w = torch.zeros(1, 1, 1, 2 * PAGE)
    s.evict([{"seq": 0, "keep": 1, "recent": 1}], w, 100.0, True)
    ang = torch.tensor([9.0, 9.0 * 100.0 ** -0.5], dtype=torch.float64)
    a, b = x[:2], x[2:]
    assert torch.allclose(s.k[0, 0, 0, 0], torch.cat((a * torch.cos(ang) + b * torch.sin(ang), b * torch.cos(ang) - a * torch.sin(ang))))
