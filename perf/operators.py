"""Operators of a paged KV cache, as cases that can be timed and checked.

Three operators that work on one data structure, a pool of 64-slot pages with a table of page ids per sequence:

  pages   goose_pages_free, goose_pages_fork, goose_pages_reserve, goose_pages_commit: several requests start from one
          prompt, get room for a tree (the shared last page is copied), and keep the accepted path of the tree.
  rope    goose_qk_norm_rope_paged: from the split-K slices of the q|k|v projection to rotated (and, where the
          model has it, per-head normalised) queries and to K/V rows in the pages.
  attn    goose_attn_paged: tree attention of requests that share the first pages of their tables, the shared pages
          read once for all of them.

Head layouts are those of the repository's own model shapes.  The plain forms are elementary torch operations in
32 bits (64 for angles), rounded once.
"""
import math

import torch

own = False

DEV = "cuda:0"
PAGE = 64
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
#          heads, KV heads, head_dim, rotary base, eps, q/k norm
HEADS = {
    "tiny": (4, 4, 64, 10000.0, 1e-5, False),
    "tiny_gqa": (4, 2, 64, 10000.0, 1e-5, False),
    "7b": (32, 32, 128, 10000.0, 1e-5, False),
    "13b": (40, 40, 128, 10000.0, 1e-5, False),
    "33b": (52, 52, 128, 10000.0, 1e-5, False),
    "llama3_8b": (32, 8, 128, 500000.0, 1e-5, False),
    "qwen3_8b": (32, 8, 128, 1000000.0, 1e-6, True),
}


def listed():
    return [
        # two short chats of the two-layer model, one token each: launches and latency
        {"name": "attn_tiny_2x1_S64", "kind": "attn", "model": "tiny_gqa", "dtype": "f16", "q_terms": 1, "n": 2, "B": 1,
         "ragged": False, "S": 64, "own": 17},
        # sixteen chats behind one long system prompt, one token each (no drafts found)
        {"name": "attn_llama3_16x1_S8192", "kind": "attn", "model": "llama3_8b", "dtype": "bf16", "q_terms": 2, "n": 16, "B": 1,
         "ragged": False, "S": 8192, "own": 400},
        # the batch sweep of the paper (trees of 32 nodes) behind a system prompt
        {"name": "attn_llama3_16x32_S4096", "kind": "attn", "model": "llama3_8b", "dtype": "bf16", "q_terms": 2, "n": 16, "B": 32,
         "ragged": False, "S": 4096, "own": 500},
        # the same behind a whole document, fp16 storage: the largest call
        {"name": "attn_llama3_f16_16x32_S16384", "kind": "attn", "model": "llama3_8b", "dtype": "f16", "q_terms": 1, "n": 16,
         "B": 32, "ragged": False, "S": 16384, "own": 700},
        # multi-head model, requests of unlike trees (a bypass chain, a single token, a spine tree) in fp16
        {"name": "attn_7b_f16_5_ragged_S1984", "kind": "attn", "model": "7b", "dtype": "f16", "q_terms": 1, "n": 5, "B": 61,
         "ragged": True, "S": 1984, "own": 333},
        # four requests of the largest model with its tree budget; 52 heads
        {"name": "attn_33b_4x80_S4096", "kind": "attn", "model": "33b", "dtype": "bf16", "q_terms": 1, "n": 4, "B": 80,
         "ragged": False, "S": 4096, "own": 150},
        # an autoregressive cycle of one request of the model with q/k norms
        {"name": "rope_qwen3_1x1", "kind": "rope", "model": "qwen3_8b", "dtype": "bf16", "n": 1, "B": 1, "ragged": False,
         "P": 1337, "ks": 4},
        # a full batch, late in a long context
        {"name": "rope_llama3_16x32", "kind": "rope", "model": "llama3_8b", "dtype": "bf16", "n": 16, "B": 32, "ragged": False,
         "P": 30011, "ks": 4},
        # unlike trees of a multi-head model, fp16
        {"name": "rope_7b_f16_5_ragged", "kind": "rope", "model": "7b", "dtype": "f16", "n": 5, "B": 61, "ragged": True,
         "P": 2041, "ks": 2},
        # one request forks off a short prompt
        {"name": "pages_tiny_1_P100", "kind": "pages", "model": "tiny", "dtype": "bf16", "layers": 2, "n": 1, "B": 8, "P": 100,
         "L": 2, "pages": 40},
        # sixteen requests fork off a prompt that ends inside a page (eight layers, as the batched passes elsewhere here)
        {"name": "pages_llama3_16_P4133", "kind": "pages", "model": "llama3_8b", "dtype": "bf16", "layers": 8, "n": 16, "B": 32,
         "P": 4133, "L": 5, "pages": 160},
        # four samples of the largest model from one prompt
        {"name": "pages_33b_4_P1000", "kind": "pages", "model": "33b", "dtype": "f16", "layers": 4, "n": 4, "B": 80, "P": 1000,
         "L": 9, "pages": 48},
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["attn", "attn", "attn", "rope", "pages"])
    dtype = rng.choice(["bf16", "f16"])
    model = rng.choice(["tiny_gqa", "7b", "13b", "33b", "llama3_8b", "qwen3_8b"])
    if kind == "pages":
        B = log_int(2, 128)
        L = rng.randint(0, min(12, (B - 1) // 2))
        n, P = rng.randint(1, 16), log_int(1, 6000)
        layers = rng.randint(1, 8) if model in ("llama3_8b", "qwen3_8b", "tiny_gqa") else rng.randint(1, 2)
        return {"kind": kind, "model": model, "dtype": dtype, "layers": layers, "n": n, "B": B, "P": P, "L": L,
                "pages": (P + PAGE - 1) // PAGE + 4 * n + rng.randint(3, 30)}
    B = rng.choice([1, log_int(1, 32), log_int(1, 32), rng.randint(33, 128)])
    n = rng.randint(1, min(16, 512 // ((B + 31) // 32 * 32)))
    ragged = rng.random() < 0.5
    if kind == "rope":
        return {"kind": kind, "model": model, "dtype": dtype, "n": n, "B": B, "ragged": ragged, "P": log_int(1, 100000),
                "ks": rng.randint(1, 8)}
    S = PAGE * rng.choice([0, log_int(1, 128), log_int(1, 128), log_int(1, 128)])
    return {"kind": kind, "model": model, "dtype": dtype, "q_terms": rng.choice([1, 2]), "n": n, "B": B, "ragged": ragged, "S": S,
            "own": log_int(1, 1500) if S else log_int(1, 5000)}


# ---- inputs: everything from the seed alone -----------------------------------------------------------------
def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1013 + tag)
    return g


def _randn(g, shape, std, dt=torch.float32):
    t = torch.empty(shape, dtype=dt, device=DEV)
    t.normal_(0.0, std, generator=g)
    return t


def _ints(seed, tag, n, lo, hi):
    """n host integers of [lo, hi]."""
    g = torch.Generator()
    g.manual_seed(int(seed) * 1013 + tag)
    return torch.randint(lo, hi + 1, (n,), generator=g).tolist()


def _tree_sizes(case):
    """Sizes belong to the case, values to the seed."""
    n, B = case["n"], case["B"]
    if not case["ragged"]:
        return [B] * n
    return [B] + _ints(n * 131 + B, 1, n - 1, 1, B)


def _lengths(case, Bs):
    """Committed slots per request: the shared part and an own part of about case["own"] (attn), about P (rope)."""
    if case["kind"] == "attn":
        return [case["S"] + x for x in _ints(case["own"], 2, len(Bs), max(0, case["own"] * 3 // 4), case["own"])]
    return _ints(case["P"], 2, len(Bs), case["P"] * 3 // 4, case["P"])


def _parents(seed, r, B):
    """A random tree in topological order that is mostly a chain at first, as a spine tree is."""
    u = _ints(seed, 100 + r, B, 0, 1 << 20)
    return [-1] + [i - 1 if i <= B // 3 or u[i] % 3 == 0 else u[i] % i for i in range(1, B)]


def _ancestors(parent):
    """Per node the list of itself and its ancestors."""
    out = []
    for i, p in enumerate(parent):
        out.append([i] if p < 0 else out[p] + [i])
    return out


def _row0s(Bs):
    out, at = [], 0
    for b in Bs:
        out.append(at)
        at += (b + 31) // 32 * 32
    return out, at


def _shuffled(seed, n):
    g = torch.Generator()
    g.manual_seed(int(seed) * 1013 + 7)
    return torch.randperm(n, generator=g).tolist()


# one head's part of a page in operand order: flat element offsets of [slot][column]
def _page_offsets(d):
    slot = torch.arange(PAGE).view(-1, 1)
    c = torch.arange(d).view(1, -1)
    blk, kk = slot // 32, slot % 32
    row = (kk // 4) % 4 * 8 + kk // 16 * 4 + kk % 4
    k = ((blk * (d // 16) + c // 16) * 64 + row + 32 * (c // 8 % 2)) * 8 + c % 8
    v = (((blk * (d // 32) + c // 32) * 2 + kk // 8 % 2) * 64 + c % 32 + 32 * (kk // 16)) * 8 + kk % 8
    return k.to(DEV), v.to(DEV)


def _pack(rows, off):
    """rows [..., 64, d] -> [..., 64 * d] in operand order."""
    out = torch.empty(rows.shape[:-2] + (PAGE * rows.shape[-1],), dtype=rows.dtype, device=rows.device)
    out[..., off.reshape(-1)] = rows.reshape(out.shape)
    return out


def _tables(seed, n_pages, counts, width, first=()):
    """Tables of len(counts) sequences: `first` shared page ids, then own ones, from a shuffled pool; reference counts."""
    order = [p for p in _shuffled(seed, n_pages) if p not in set(first)]
    rows, refs, at = [], [0] * n_pages, 0
    for c in counts:
        row = list(first) + order[at:at + c - len(first)]
        at += c - len(first)
        rows.append(row + [-1] * (width - c))
        for p in row:
            refs[p] += 1
    return rows, refs


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _attn_inputs(case, seed):
    nh, nkv, d = HEADS[case["model"]][:3]
    Bs = _tree_sizes(case)
    Ps = _lengths(case, Bs)
    counts = [(p + b + PAGE - 1) // PAGE for p, b in zip(Ps, Bs)]
    n_sh = case["S"] // PAGE
    n_pages = n_sh + sum(c - n_sh for c in counts) + 3
    table, refs = _tables(seed, n_pages, counts, max(counts) + 1, _shuffled(seed, n_pages)[:n_sh])
    g, dt = _gen(seed, 10), DTYPES[case["dtype"]]
    row0, rows = _row0s(Bs)
    q = _randn(g, (rows, nh, d), 1.5)
    k = _randn(g, (n_pages, nkv, PAGE, d), 1.0, dt)
    v = _randn(g, (n_pages, nkv, PAGE, d), 1.0, dt)
    anc = [_ancestors(_parents(seed, r, b)) for r, b in enumerate(Bs)]
    hi = q.to(dt)
    lo = (q - hi.float()).to(dt) if case["q_terms"] == 2 else None
    return {"Bs": Bs, "Ps": Ps, "table": table, "refs": refs, "n_pages": n_pages, "rows": rows, "row0": row0, "hi": hi, "lo": lo,
            "k": k, "v": v, "anc": anc}


def _rope_inputs(case, seed):
    nh, nkv, d = HEADS[case["model"]][:3]
    Bs = _tree_sizes(case)
    Ps = _lengths(case, Bs)
    # the pool holds the pages that the trees reach into; the rest of a long context is not touched
    first = [p // PAGE for p in Ps]
    counts = [(p + b + PAGE - 1) // PAGE for p, b in zip(Ps, Bs)]
    n_pages = sum(c - f for c, f in zip(counts, first)) + 3
    order, at, table, refs = _shuffled(seed, n_pages), 0, [], [0] * n_pages
    for f, c in zip(first, counts):
        mine = order[at:at + c - f]
        at += c - f
        table.append([-1] * f + mine + [-1] * (max(counts) - c))
        for p in mine:
            refs[p] = 1
    g, dt = _gen(seed, 20), DTYPES[case["dtype"]]
    row0, rows = _row0s(Bs)
    anc = [_ancestors(_parents(seed, r, b)) for r, b in enumerate(Bs)]
    pos = [p + len(a) - 1 for p, aa in zip(Ps, anc) for a in aa]
    return {"Bs": Bs, "Ps": Ps, "table": table, "refs": refs, "n_pages": n_pages, "rows": rows, "row0": row0, "pos": pos,
            "part": _randn(g, (case["ks"], rows, (nh + 2 * nkv) * d), 1.0 / math.sqrt(case["ks"])),
            "gq": (1.0 + _randn(g, (d,), 0.1)).to(dt), "gk": (1.0 + _randn(g, (d,), 0.1)).to(dt),
            "k": _randn(g, (n_pages, nkv, PAGE, d), 1.0, dt), "v": _randn(g, (n_pages, nkv, PAGE, d), 1.0, dt)}


def _pages_inputs(case, seed):
    """Sequence 0 holds the prompt, sequence n + 1 belongs to somebody else, 1 .. n are the forks; n_pages from the case."""
    nkv, d = HEADS[case["model"]][1:3]
    n, P, n_pages = case["n"], case["P"], case["pages"]
    np_src = (P + PAGE - 1) // PAGE
    order = _shuffled(seed, n_pages)
    width = (P + case["B"] + PAGE - 1) // PAGE + 2
    table = [[-1] * width for _ in range(n + 2)]
    table[0][:np_src] = order[:np_src]
    table[n + 1][:2] = order[np_src:np_src + 2]
    refs = [0] * n_pages
    for p in order[:np_src + 2]:
        refs[p] = 1
    # accepted paths: node 0, then L nodes behind the first L + 1
    paths = []
    for r in range(n):
        L, B = case["L"], case["B"]
        pick = sorted(torch.randperm(B - 1 - L, generator=torch.Generator().manual_seed(int(seed) * 31 + r))[:L].tolist())
        paths.append([0] + [L + 1 + x for x in pick])
    g, dt = _gen(seed, 30), DTYPES[case["dtype"]]
    shape = (case["layers"], n_pages, nkv, PAGE, d)
    return {"table": table, "refs": refs, "len": [P] + [0] * n + [70], "paths": paths, "k": _randn(g, shape, 1.0, dt),
            "v": _randn(g, shape, 1.0, dt)}


# ---- states -------------------------------------------------------------------------------------------------
def _ctx(case, max_B, rows, layers, width):
    from paper_2604_02047_amd import GooseContext, ModelDesc
    nh, nkv, d, base, eps, norm = HEADS[case["model"]]
    desc = ModelDesc(layers, 128, nh, d, 128, 1024, base, eps, case["dtype"], nkv, norm)
    return GooseContext(desc, max_B, max(width * PAGE, 128), rows)


def prepare(case, seed):
    nh, nkv, d, base, eps, norm = HEADS[case["model"]]
    koff, voff = _page_offsets(d)
    i = {"attn": _attn_inputs, "rope": _rope_inputs, "pages": _pages_inputs}[case["kind"]](case, seed)
    st = {"case": case, "koff": koff, "voff": voff, "kpool": _pack(i["k"], koff), "vpool": _pack(i["v"], voff),
          "table": _i32(i["table"]), "refs": _i32(i["refs"])}
    if case["kind"] == "pages":
        st["len"] = _i32(i["len"])
        st["paths"], st["L"] = i["paths"], case["L"]
        pad = [p + [-1] * (case["B"] - len(p)) for p in i["paths"]]
        st["path"] = _i32(pad)
        st["accept"] = _i32([case["L"]] * case["n"])
        max_B, rows, layers = case["B"], 32 * ((case["B"] + 31) // 32), case["layers"]
    else:
        st["len"], st["Bs"], st["Ps"], st["row0"], st["rows"] = _i32(i["Ps"]), i["Bs"], i["Ps"], i["row0"], i["rows"]
        max_B, rows, layers = max(i["Bs"]), i["rows"], 1
    if case["kind"] == "attn":
        terms = case["q_terms"]
        if terms == 1:
            st["q"] = i["hi"].reshape(i["rows"], nh * d).contiguous()
        else:  # groups of eight columns: eight high terms, then their eight low ones
            both = torch.stack((i["hi"].view(i["rows"], nh * d // 8, 8), i["lo"].view(i["rows"], nh * d // 8, 8)), dim=2)
            st["q"] = both.reshape(i["rows"], 2 * nh * d).contiguous()
        st["o"] = torch.zeros((i["rows"], nh * d), dtype=torch.float16, device=DEV)
        words = []
        for a, B in zip(i["anc"], i["Bs"]):
            W = (B + 63) // 64
            rowsw = []
            for lst in a:
                w = [0] * W
                for j in lst:
                    w[j // 64] |= 1 << (j % 64)
                rowsw.append([x - (1 << 64) if x >> 63 else x for x in w])
            words.append(torch.tensor(rowsw, dtype=torch.int64, device=DEV))
        st["mask"] = words
        st["visible"] = []
        for a, B in zip(i["anc"], i["Bs"]):
            m = torch.zeros((B, B), dtype=torch.bool)
            for r, lst in enumerate(a):
                m[r, lst] = True
            st["visible"].append(m.to(DEV))
    if case["kind"] == "rope":
        st["part"], st["gq"], st["gk"] = i["part"], i["gq"], i["gk"]
        st["q"] = torch.zeros((i["rows"], nh * d), dtype=DTYPES[case["dtype"]], device=DEV)
        st["pos"] = []
        at = 0
        for B in i["Bs"]:
            st["pos"].append(_i32(i["pos"][at:at + B]))
            at += B
    if own:
        from paper_2604_02047_amd import PagedCache, PagedRequests
        st["ctx"] = _ctx(case, max_B, rows, layers, st["table"].shape[1])
        pool = st["kpool"].shape if case["kind"] == "pages" else (1,) + tuple(st["kpool"].shape)
        st["cache"] = PagedCache(st["kpool"].view(pool), st["vpool"].view(pool), st["table"], st["len"], st["refs"])
        if case["kind"] == "attn":
            st["reqs"] = PagedRequests([{"seq": r, "B": B, "P_max": P, "mask": st["mask"][r]}
                                        for r, (B, P) in enumerate(zip(st["Bs"], st["Ps"]))])
        elif case["kind"] == "rope":
            st["reqs"] = PagedRequests([{"seq": r, "B": B, "P_max": P, "pos": st["pos"][r]}
                                        for r, (B, P) in enumerate(zip(st["Bs"], st["Ps"]))])
        else:
            st["reqs"] = PagedRequests([{"seq": r + 1, "B": case["B"], "P_max": case["P"], "path": st["path"][r],
                                         "accept_len": st["accept"][r:]} for r in range(case["n"])])
            st["forks"] = list(range(1, case["n"] + 1))
    return st


def run(state):
    return {"attn": _attn, "rope": _rope, "pages": _pages}[state["case"]["kind"]](state)


# ---- attention of requests that share a prefix ----------------------------------------------------------------
def _attn(st):
    case = st["case"]
    if own:
        st["ctx"].goose_attn_paged(st["cache"], 0, st["q"], case["q_terms"], st["reqs"], case["S"] // PAGE, st["o"])
        return st["o"]
    nh, nkv, d = HEADS[case["model"]][:3]
    G = nh // nkv
    q = st["q"].float()
    if case["q_terms"] == 2:
        q = q.view(-1, nh * d // 8, 2, 8).sum(dim=2)
    q = q.reshape(-1, nkv, G, d)
    out = torch.zeros_like(st["o"])
    for r, (B, P) in enumerate(zip(st["Bs"], st["Ps"])):
        N = P + B
        pages = st["table"][r, :(N + PAGE - 1) // PAGE].long()
        k = st["kpool"][pages][..., st["koff"]].float()       # [page][head][slot][d]
        v = st["vpool"][pages][..., st["voff"]].float()
        k = k.permute(1, 0, 2, 3).reshape(nkv, -1, d)[:, :N].contiguous()
        v = v.permute(1, 0, 2, 3).reshape(nkv, -1, d)[:, :N].contiguous()
        qr = q[st["row0"][r]:st["row0"][r] + B].permute(1, 2, 0, 3).reshape(nkv, G * B, d).contiguous()
        s = torch.matmul(qr, k.transpose(1, 2).contiguous()).view(nkv, G, B, N) * (1.0 / math.sqrt(d))
        s[..., P:] = s[..., P:].masked_fill(~st["visible"][r], float("-inf"))
        p = torch.exp(s - s.amax(dim=-1, keepdim=True))
        p = p / p.sum(dim=-1, keepdim=True)
        o = torch.matmul(p.view(nkv, G * B, N), v).view(nkv, G, B, d)
        out[st["row0"][r]:st["row0"][r] + B] = o.permute(2, 0, 1, 3).reshape(B, nh * d).to(out.dtype)
    return out


# ---- head norms, rotation, K/V rows into pages ---------------------------------------------------------------------
def _rope(st):
    case = st["case"]
    nh, nkv, d, base, eps, norm = HEADS[case["model"]]
    if own:
        st["ctx"].goose_qk_norm_rope_paged(st["cache"], 0, st["part"], st["gq"] if norm else None, st["gk"] if norm else None,
                                           st["reqs"], st["q"], 1)
        return st["q"], st["kpool"], st["vpool"]
    dt = DTYPES[case["dtype"]]
    inv = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    x = st["part"].sum(dim=0)
    for r, (B, P) in enumerate(zip(st["Bs"], st["Ps"])):
        y = x[st["row0"][r]:st["row0"][r] + B].view(B, nh + 2 * nkv, d)
        qk, v = y[:, :nh + nkv], y[:, nh + nkv:]
        if norm:
            g = torch.cat((st["gq"].float().expand(nh, d), st["gk"].float().expand(nkv, d)))
            qk = qk * torch.rsqrt((qk * qk).mean(dim=-1, keepdim=True) + eps) * g
        ang = st["pos"][r].double().view(B, 1, 1) * inv
        c, s = torch.cos(ang).float(), torch.sin(ang).float()
        a, b = qk[..., :d // 2], qk[..., d // 2:]
        qk = torch.cat((a * c - b * s, b * c + a * s), dim=-1).to(dt)
        st["q"][st["row0"][r]:st["row0"][r] + B] = qk[:, :nh].reshape(B, nh * d)
        slots = torch.arange(P, P + B, device=DEV)
        page = st["table"][r, slots // PAGE].long().view(B, 1, 1)
        head = torch.arange(nkv, device=DEV).view(1, nkv, 1)
        st["kpool"][page, head, st["koff"][slots % PAGE].view(B, 1, d)] = qk[:, nh:]
        st["vpool"][page, head, st["voff"][slots % PAGE].view(B, 1, d)] = v.to(dt)
    return st["q"], st["kpool"], st["vpool"]


# ---- pages ----------------------------------------------------------------------------------------------------------
def _pages(st):
    case = st["case"]
    n, P, B, L = case["n"], case["P"], case["B"], case["L"]
    out = (st["table"], st["len"], st["refs"], st["kpool"], st["vpool"])
    if own:
        c, cache = st["ctx"], st["cache"]
        c.goose_pages_free(cache, st["forks"])
        c.goose_pages_fork(cache, 0, st["forks"])
        c.goose_pages_reserve(cache, st["forks"], [B] * n)
        c.goose_pages_commit(cache, st["reqs"])
        return out
    table, lens, refs, kpool, vpool = out
    forks = slice(1, n + 1)
    # free
    held = table[forks].reshape(-1)
    refs.index_add_(0, held.clamp_min(0), -(held >= 0).int())
    table[forks] = -1
    lens[forks] = 0
    # fork
    full = (P + PAGE - 1) // PAGE
    table[forks, :full] = table[0, :full]
    refs[table[0, :full].long()] += n
    lens[forks] = P
    # reserve: the page that holds slot P is shared and becomes an own one, further pages are new; lowest free ids first
    shared = P % PAGE != 0
    first, last = P // PAGE, (P + B - 1) // PAGE
    new = last - first + 1
    free = torch.argsort((refs > 0).int(), stable=True)[:n * new].view(n, new)
    if shared:
        src = table[0, first].long()
        used = (P % PAGE + 31) // 32 * 32 * HEADS[case["model"]][2]
        kpool[:, free[:, 0], :, :used] = kpool[:, src, :, :used].unsqueeze(1)
        vpool[:, free[:, 0], :, :used] = vpool[:, src, :, :used].unsqueeze(1)
        refs[src] -= n
    table[forks, first:last + 1] = free.int()
    refs[free.reshape(-1)] = 1
    # commit: slot P + path[j] -> slot P + j, later pages are given back
    if L > 0:
        src = P + st["path"][:, 1:L + 1].long()
        dst = P + torch.arange(1, L + 1, device=DEV).expand(n, L)
        seq = torch.arange(1, n + 1, device=DEV).view(n, 1)
        sp, dp = table[seq, src // PAGE].long().unsqueeze(-1), table[seq, dst // PAGE].long().unsqueeze(-1)
        for pool, off in ((kpool, st["koff"]), (vpool, st["voff"])):
            so, do = off[src % PAGE], off[dst % PAGE]
            for l in range(pool.shape[0]):
                for h in range(pool.shape[2]):
                    pool[l, :, h][dp, do] = pool[l, :, h][sp, so]
    lens[forks] = P + L + 1
    keep = (P + L + PAGE) // PAGE
    rest = table[forks, keep:].reshape(-1)
    refs.index_add_(0, rest.clamp_min(0), -(rest >= 0).int())
    table[forks, keep:] = -1
    return out


def work(case):
    nh, nkv, d, _, _, norm = HEADS[case["model"]]
    if case["kind"] == "pages":
        row = case["layers"] * 2 * nkv * d * 2                      # one slot, K and V of all layers
        per = row * 2 * (case["P"] % PAGE + case["L"])              # read and written: the copied slots, the moved ones
        tables = case["n"] * ((case["P"] + case["B"]) // PAGE + 1) * 4 * 3 + case["pages"] * 4
        return {"bytes": case["n"] * per + tables, "flops": 0}
    Bs = _tree_sizes(case)
    rows = sum(Bs)
    if case["kind"] == "rope":
        cols = (nh + 2 * nkv) * d
        return {"bytes": int(rows * cols * (4 * case["ks"] + 2)), "flops": int(rows * cols * (case["ks"] + 3 + 4 * norm))}
    Ps = _lengths(case, Bs)
    pairs = sum(b * (p + (b + 1) / 3) for b, p in zip(Bs, Ps))  # (a node sees about a third of its tree)
    kv = case["S"] + sum(p + b - case["S"] for b, p in zip(Bs, Ps))
    return {"bytes": int(2 * 2 * kv * nkv * d + rows * nh * d * 2 * (case["q_terms"] + 1)), "flops": int(4 * nh * d * pairs)}


# ---- the definitions in 64 bits, from the logical inputs --------------------------------------------------------------
def exact(case, seed):
    return {"attn": _exact_attn, "rope": _exact_rope, "pages": _exact_pages}[case["kind"]](case, seed)


def _exact_attn(case, seed):
    nh, nkv, d = HEADS[case["model"]][:3]
    i = _attn_inputs(case, seed)
    q = i["hi"].double() + (i["lo"].double() if i["lo"] is not None else 0.0)
    out = torch.zeros((i["rows"], nh, d), dtype=torch.float64, device=DEV)
    for r, (B, P) in enumerate(zip(i["Bs"], i["Ps"])):
        pages = i["table"][r][:(P + B + PAGE - 1) // PAGE]
        idx = torch.tensor(pages, device=DEV)
        see = torch.zeros((B, P + B), dtype=torch.bool)
        see[:, :P] = True
        for node, lst in enumerate(i["anc"][r]):
            see[node, [P + j for j in lst]] = True
        see = see.to(DEV)
        for h in range(nkv):
            k = i["k"][idx, h].reshape(-1, d)[:P + B].double()
            v = i["v"][idx, h].reshape(-1, d)[:P + B].double()
            kt = k.t().contiguous()
            for x in range(h * (nh // nkv), (h + 1) * (nh // nkv)):
                s = q[i["row0"][r]:i["row0"][r] + B, x] @ kt / math.sqrt(d)
                e = torch.where(see, torch.exp(s - torch.where(see, s, -1e300).max(dim=1, keepdim=True).values), 0.0)
                out[i["row0"][r]:i["row0"][r] + B, x] = (e @ v) / e.sum(dim=1, keepdim=True)
    return out.view(i["rows"], nh * d)


def _exact_rope(case, seed):
    nh, nkv, d, base, eps, norm = HEADS[case["model"]]
    i = _rope_inputs(case, seed)
    koff, voff = _page_offsets(d)
    k, v = i["k"].double(), i["v"].double()
    q = torch.zeros((i["rows"], nh, d), dtype=torch.float64, device=DEV)
    freq = torch.tensor([base ** (-2.0 * j / d) for j in range(d // 2)], dtype=torch.float64, device=DEV)
    at = 0
    for r, (B, P) in enumerate(zip(i["Bs"], i["Ps"])):
        x = i["part"][:, i["row0"][r]:i["row0"][r] + B].double().sum(dim=0).view(B, nh + 2 * nkv, d)
        if norm:
            rms = torch.sqrt((x ** 2).sum(dim=-1, keepdim=True) / d + eps)
            x = torch.cat((x[:, :nh] / rms[:, :nh] * i["gq"].double(), x[:, nh:nh + nkv] / rms[:, nh:nh + nkv] * i["gk"].double(),
                           x[:, nh + nkv:]), dim=1)
        pos = torch.tensor(i["pos"][at:at + B], dtype=torch.float64, device=DEV).view(B, 1, 1)
        at += B
        z = torch.complex(x[:, :nh + nkv, :d // 2], x[:, :nh + nkv, d // 2:]) * torch.polar(torch.ones_like(pos * freq), pos * freq)
        y = torch.cat((z.real, z.imag), dim=-1)
        q[i["row0"][r]:i["row0"][r] + B] = y[:, :nh]
        for node in range(B):
            page, slot = i["table"][r][(P + node) // PAGE], (P + node) % PAGE
            k[page, :, slot] = y[node, nh:]
            v[page, :, slot] = x[node, nh + nkv:]
    return q.view(i["rows"], nh * d), _pack(k, koff), _pack(v, voff)


def _exact_pages(case, seed):
    d = HEADS[case["model"]][2]
    i = _pages_inputs(case, seed)
    koff, voff = _page_offsets(d)
    table, refs, lens, k, v = i["table"], i["refs"], i["len"], i["k"], i["v"]
    P, B, L = case["P"], case["B"], case["L"]
    for s in range(1, case["n"] + 1):
        for j in range((P + PAGE - 1) // PAGE):
            table[s][j] = table[0][j]
            refs[table[0][j]] += 1
        lens[s] = P
    for s in range(1, case["n"] + 1):
        for j in range(P // PAGE, (P + B - 1) // PAGE + 1):
            old, got = table[s][j], refs.index(0)
            refs[got] = 1
            table[s][j] = got
            if old >= 0:
                refs[old] -= 1
                used = (P % PAGE + 31) // 32 * 32
                k[:, got, :, :used] = k[:, old, :, :used]
                v[:, got, :, :used] = v[:, old, :, :used]
    for s in range(1, case["n"] + 1):
        for j in range(1, L + 1):
            a, b = P + i["paths"][s - 1][j], P + j
            k[:, table[s][b // PAGE], :, b % PAGE] = k[:, table[s][a // PAGE], :, a % PAGE]
            v[:, table[s][b // PAGE], :, b % PAGE] = v[:, table[s][a // PAGE], :, a % PAGE]
        lens[s] = P + L + 1
        for j in range((lens[s] + PAGE - 1) // PAGE, len(table[s])):
            if table[s][j] >= 0:
                refs[table[s][j]] -= 1
                table[s][j] = -1
    return _i32(table), _i32(lens), _i32(refs), _pack(k, koff).double(), _pack(v, voff).double()
