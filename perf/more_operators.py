"""Operators of prompts on a paged KV cache, as cases that can be timed and checked.

A prompt comes into the pages chunk by chunk, the attention of its tokens says which slots matter, and a cache that has become too
long is cut down to the slots that do:

  attn    goose_attn_chunk_paged: causal attention of chunks of new tokens (one token to thousands, several requests) over the
          committed slots of their sequences and over themselves, with the logarithm of every row's sum of exponentials.
  weight  goose_attn_weight_paged: the attention weight that every slot has received, summed over rows and over the query heads of
          its KV head, added to what earlier calls have left.
  evict   goose_pages_evict, goose_pages_reserve, goose_pages_append: per layer and KV head the heaviest slots are kept beside the
          first and the last ones, moved to the front (keys turned to their new positions), and the room is taken for new slots.

Head layouts are those of the repository's own model shapes.  The plain forms are elementary torch operations in 32 bits (64 for
angles), rounded once.
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
        # two short chats of the two-layer model go on by a token each: launches and latency
        {"name": "attn_tiny_2x1_P81", "kind": "attn", "model": "tiny_gqa", "dtype": "f16", "q_terms": 1, "o": "f16", "n": 2, "C": 1,
         "ragged": False, "P": 81},
        # one pass of the framework's stacked rows late in a prompt, bf16 storage as its layers run it (queries in two terms)
        {"name": "attn_llama3_1x512_P3500", "kind": "attn", "model": "llama3_8b", "dtype": "bf16", "q_terms": 2, "o": "f16", "n": 1,
         "C": 512, "ragged": False, "P": 3500},
        # unlike chunks of five requests of a multi-head model (a whole short prompt, the rest of one, a few tokens), fp16
        {"name": "attn_7b_f16_5_ragged", "kind": "attn", "model": "7b", "dtype": "f16", "q_terms": 1, "o": "f16", "n": 5, "C": 333,
         "ragged": True, "P": 1984},
        # a document in one chunk behind another one: the largest call
        {"name": "attn_llama3_f16_1x4096_P12288", "kind": "attn", "model": "llama3_8b", "dtype": "f16", "q_terms": 1, "o": "f16", "n": 1,
         "C": 4096, "ragged": False, "P": 12288},
        # a prompt from its first token on, 52 heads, outputs in bf16
        {"name": "attn_33b_1x2000_P0", "kind": "attn", "model": "33b", "dtype": "bf16", "q_terms": 1, "o": "bf16", "n": 1, "C": 2000,
         "ragged": False, "P": 0},
        # sixteen chats go on by a token each: which slots have they looked at
        {"name": "weight_llama3_16x1_P4000", "kind": "weight", "model": "llama3_8b", "dtype": "bf16", "q_terms": 2, "n": 16, "C": 1,
         "first": 0, "ragged": True, "P": 4000, "decay": 0.98},
        # the last 32 tokens of a chunk of 300 look back over a document
        {"name": "weight_7b_f16_1x300_last32_P7000", "kind": "weight", "model": "7b", "dtype": "f16", "q_terms": 1, "n": 1, "C": 300,
         "first": 268, "ragged": False, "P": 7000, "decay": 0.0},
        # all tokens of a long chunk count
        {"name": "weight_llama3_f16_1x2048_P6144", "kind": "weight", "model": "llama3_8b", "dtype": "f16", "q_terms": 1, "n": 1, "C": 2048,
         "first": 0, "ragged": False, "P": 6144, "decay": 1.0},
        # a short cache of the two-layer model loses a few slots
        {"name": "evict_tiny_1_P200", "kind": "evict", "model": "tiny", "dtype": "bf16", "layers": 2, "n": 1, "P": 200, "keep": 150,
         "sink": 4, "recent": 32, "reposition": True, "spare": 5, "ties": False},
        # four documents are cut to a quarter (eight layers, as the batched passes elsewhere here)
        {"name": "evict_llama3_4_P8192_keep2048", "kind": "evict", "model": "llama3_8b", "dtype": "bf16", "layers": 8, "n": 4, "P": 8192,
         "keep": 2048, "sink": 64, "recent": 256, "reposition": True, "spare": 9, "ties": False},
        # a multi-head model makes room for the next chunk; keys stay as they are, many slots of equal weight
        {"name": "evict_7b_f16_2_P3001_keep2500", "kind": "evict", "model": "7b", "dtype": "f16", "layers": 4, "n": 2, "P": 3001,
         "keep": 2500, "sink": 0, "recent": 100, "reposition": False, "spare": 3, "ties": True},
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["attn", "attn", "weight", "evict"])
    dtype = rng.choice(["bf16", "f16"])
    model = rng.choice(["tiny_gqa", "7b", "13b", "33b", "llama3_8b", "qwen3_8b"])
    nh, nkv, d = HEADS[model][:3]
    if kind == "evict":
        P = log_int(2, 8192)
        n, layers = rng.randint(1, 8), rng.randint(1, 8)
        while n * layers * P * nkv * d > 4 * 8 * 8192 * 8 * 128 and n * layers > 1:
            n, layers = (n - 1, layers) if n >= layers else (n, layers - 1)
        keep = rng.randint(1, P) if rng.random() < 0.9 else P + rng.randint(0, 9)
        sink = rng.randint(0, min(keep, 130))
        return {"kind": kind, "model": model, "dtype": dtype, "layers": layers, "n": n, "P": P, "keep": keep, "sink": sink,
                "recent": rng.randint(0, min(keep - sink, 300)), "reposition": rng.random() < 0.6, "spare": rng.randint(0, 20),
                "ties": rng.random() < 0.3}
    C = rng.choice([1, log_int(1, 128), log_int(1, 4096), log_int(1, 4096)])
    n = rng.randint(1, max(1, min(16, 2048 // C)))
    P = rng.choice([0, log_int(1, 16384), log_int(1, 16384)])
    most = 32 * 4096 * (12288 + 2048) if kind == "attn" else 32 * 2048 * (6144 + 1024)
    while n * nh * C * (P + C // 2 + 1) > most:
        P, C = P // 2, max(1, C * 3 // 4)
    case = {"kind": kind, "model": model, "dtype": dtype, "q_terms": rng.choice([1, 2]), "n": n, "C": C, "ragged": rng.random() < 0.5, "P": P}
    if kind == "attn":
        case["o"] = rng.choice(["bf16", "f16"])
    else:
        case["first"] = rng.choice([0, max(0, C - log_int(1, 64))])
        case["decay"] = rng.choice([0.0, 1.0, round(rng.uniform(0.5, 1.0), 3)])
    return case


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


def _shuffled(seed, n):
    g = torch.Generator()
    g.manual_seed(int(seed) * 1013 + 7)
    return torch.randperm(n, generator=g).tolist()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _sizes(case):
    """Tokens of every request's chunk, and its committed slots.  Sizes belong to the case, values to the seed."""
    n, C, P = case["n"], case["C"], case["P"]
    if not case["ragged"]:
        return [C] * n, [P] * n
    return [C] + _ints(n * 131 + C, 1, n - 1, 1, C), _ints(P, 2, n, P // 2, P)


def _row0s(Cs):
    out, at = [], 0
    for c in Cs:
        out.append(at)
        at += (c + 31) // 32 * 32
    return out, at


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


def _tables(seed, counts, spare):
    """Tables of sequences with pages of their own from a shuffled pool, `spare` free ones in it; reference counts."""
    n_pages = sum(counts) + spare
    order, at, rows, refs = _shuffled(seed, n_pages), 0, [], [0] * n_pages
    for c in counts:
        rows.append(order[at:at + c] + [-1] * (max(counts) + 1 - c))
        for p in order[at:at + c]:
            refs[p] = 1
        at += c
    return rows, refs, n_pages


def _chunk_inputs(case, seed):
    nh, nkv, d = HEADS[case["model"]][:3]
    Cs, Ps = _sizes(case)
    table, refs, n_pages = _tables(seed, [(p + c + PAGE - 1) // PAGE for p, c in zip(Ps, Cs)], 3)
    g, dt = _gen(seed, 10), DTYPES[case["dtype"]]
    row0, rows = _row0s(Cs)
    q = _randn(g, (rows, nh, d), 1.5)
    k = _randn(g, (n_pages, nkv, PAGE, d), 1.0, dt)
    v = _randn(g, (n_pages, nkv, PAGE, d), 1.0, dt)
    hi = q.to(dt)
    lo = (q - hi.float()).to(dt) if case["q_terms"] == 2 else None
    i = {"Cs": Cs, "Ps": Ps, "table": table, "refs": refs, "n_pages": n_pages, "rows": rows, "row0": row0, "hi": hi, "lo": lo, "k": k,
         "v": v, "w": None}
    if case["kind"] == "weight":
        i["w"] = _randn(g, (1, case["n"], nkv, PAGE * len(table[0])), 1.0).abs()
        # what the attention of the same rows has left: an input of the weights
        i["lse"] = torch.zeros((nh, rows), dtype=torch.float32, device=DEV)
        for r, (C, P) in enumerate(zip(Cs, Ps)):
            at, first = row0[r], min(case["first"], C - 1)
            keys = k[torch.tensor(table[r][:(P + C + PAGE - 1) // PAGE], device=DEV)].transpose(1, 2).flatten(0, 1)[:P + C]
            unseen = torch.arange(P + C, device=DEV).view(1, -1) > P + torch.arange(first, C, device=DEV).view(-1, 1)
            for x in range(nh):
                s = q[at + first:at + C, x] @ keys[:, x * nkv // nh].float().t().contiguous() / math.sqrt(d)
                i["lse"][x, at + first:at + C] = torch.logsumexp(s.masked_fill(unseen, -math.inf), dim=1)
    return i


def _evict_inputs(case, seed):
    nkv, d = HEADS[case["model"]][1:3]
    n, P, layers = case["n"], case["P"], case["layers"]
    table, refs, n_pages = _tables(seed, [(P + PAGE - 1) // PAGE] * n, case["spare"])
    g, dt = _gen(seed, 30), DTYPES[case["dtype"]]
    # weights as attention leaves them: most slots little, a few much; with ties as coarse a scale as counts
    w = torch.exp(_randn(g, (layers, n, nkv, PAGE * len(table[0])), 2.0))
    if case["ties"]:
        w = torch.floor(4.0 * w)
    shape = (layers, n_pages, nkv, PAGE, d)
    return {"table": table, "refs": refs, "len": [P] * n, "w": w, "k": _randn(g, shape, 1.0, dt), "v": _randn(g, shape, 1.0, dt)}


# ---- states -------------------------------------------------------------------------------------------------
def _ctx(case, layers, width):
    from paper_2604_02047_amd import GooseContext, ModelDesc
    nh, nkv, d, base, eps, norm = HEADS[case["model"]]
    desc = ModelDesc(layers, 128, nh, d, 128, 1024, base, eps, case["dtype"], nkv, norm)
    return GooseContext(desc, 128, max(width * PAGE, 128), 512)


def prepare(case, seed):
    nh, nkv, d = HEADS[case["model"]][:3]
    koff, voff = _page_offsets(d)
    i = _evict_inputs(case, seed) if case["kind"] == "evict" else _chunk_inputs(case, seed)
    st = {"case": case, "koff": koff, "voff": voff, "kpool": _pack(i["k"], koff), "vpool": _pack(i["v"], voff),
          "table": _i32(i["table"]), "refs": _i32(i["refs"]), "weight": i["w"]}
    if case["kind"] == "evict":
        st["len"], layers = _i32(i["len"]), case["layers"]
        st["kept"] = torch.zeros((case["n"], layers, nkv, st["table"].shape[1]), dtype=torch.int64, device=DEV)
        st["seqs"] = list(range(case["n"]))
        st["new"] = [max(0, case["P"] - case["keep"])] * case["n"]
    else:
        layers = 1
        st["kpool"], st["vpool"] = st["kpool"].unsqueeze(0), st["vpool"].unsqueeze(0)
        st["len"], st["Cs"], st["Ps"], st["row0"], st["rows"] = _i32(i["Ps"]), i["Cs"], i["Ps"], i["row0"], i["rows"]
        if case["q_terms"] == 1:
            st["q"] = i["hi"].reshape(i["rows"], nh * d).contiguous()
        else:  # groups of eight columns: eight high terms, then their eight low ones
            both = torch.stack((i["hi"].view(i["rows"], nh * d // 8, 8), i["lo"].view(i["rows"], nh * d // 8, 8)), dim=2)
            st["q"] = both.reshape(i["rows"], 2 * nh * d).contiguous()
        if case["kind"] == "attn":
            st["o"] = torch.zeros((i["rows"], nh * d), dtype=DTYPES[case["o"]], device=DEV)
            st["lse"] = torch.zeros((nh, i["rows"]), dtype=torch.float32, device=DEV)
        else:
            st["lse"] = i["lse"]
    if own:
        from paper_2604_02047_amd import PagedCache, PagedChunks
        st["ctx"] = _ctx(case, layers, st["table"].shape[1])
        st["cache"] = PagedCache(st["kpool"], st["vpool"], st["table"], st["len"], st["refs"])
        if case["kind"] == "evict":
            st["evictions"] = [{"seq": r, "keep": case["keep"], "sink": case["sink"], "recent": case["recent"]} for r in st["seqs"]]
            if st["new"][0]:
                st["chunks"] = PagedChunks([{"seq": r, "C": st["new"][r], "P_max": case["keep"]} for r in st["seqs"]])
        else:
            st["chunks"] = PagedChunks([{"seq": r, "C": c, "P_max": p, "first": min(case.get("first", 0), c - 1)}
                                        for r, (c, p) in enumerate(zip(st["Cs"], st["Ps"]))])
    return st


def run(state):
    return {"attn": _attn, "weight": _weight, "evict": _evict}[state["case"]["kind"]](state)


def _logical(pool, pages, off, n):
    """Rows [heads][n][d] of the pages of one layer, in 32 bits."""
    x = pool[pages][..., off].float()                               # [page][head][slot][d]
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[-1])[:, :n].contiguous()


def _scores(st, r, first=0):
    """Scores [KV head][group][C - first][P + C] of request r from token `first` on, -infinity where one does not see a slot."""
    case = st["case"]
    nh, nkv, d = HEADS[case["model"]][:3]
    G, C, P = nh // nkv, st["Cs"][r], st["Ps"][r]
    N = P + C
    pages = st["table"][r, :(N + PAGE - 1) // PAGE].long()
    k = _logical(st["kpool"][0], pages, st["koff"], N)
    R = C - first
    q = st["q"][st["row0"][r] + first:st["row0"][r] + C].float()
    if case["q_terms"] == 2:
        q = q.view(R, nh * d // 8, 2, 8).sum(dim=2)
    q = q.reshape(R, nkv, G, d).permute(1, 2, 0, 3).reshape(nkv, G * R, d).contiguous()
    s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(nkv, G, R, N).mul_(1.0 / math.sqrt(d))
    s[..., P:].masked_fill_(torch.ones((R, C), dtype=torch.bool, device=DEV).triu(1 + first), float("-inf"))
    return pages, s


# ---- attention of chunks --------------------------------------------------------------------------------------
def _attn(st):
    case = st["case"]
    if own:
        st["ctx"].goose_attn_chunk_paged(st["cache"], 0, st["q"], case["q_terms"], st["chunks"], st["o"], lse=st["lse"])
        return st["o"], st["lse"]
    nh, nkv, d = HEADS[case["model"]][:3]
    G = nh // nkv
    for r, (C, P) in enumerate(zip(st["Cs"], st["Ps"])):
        at = st["row0"][r]
        pages, s = _scores(st, r)
        v = _logical(st["vpool"][0], pages, st["voff"], P + C)
        top = s.amax(dim=-1, keepdim=True)
        p = s.sub_(top).exp_()
        total = p.sum(dim=-1, keepdim=True)
        o = torch.matmul(p.view(nkv, G * C, P + C), v).view(nkv, G, C, d) / total
        st["o"][at:at + C] = o.permute(2, 0, 1, 3).reshape(C, nh * d).to(st["o"].dtype)
        st["lse"][:, at:at + C] = (top + torch.log(total)).view(nh, C)
    return st["o"], st["lse"]


# ---- weights of slots -----------------------------------------------------------------------------------------
def _weight(st):
    case = st["case"]
    if own:
        st["ctx"].goose_attn_weight_paged(st["cache"], 0, st["q"], case["q_terms"], st["chunks"], st["lse"], st["weight"], case["decay"])
        return st["weight"]
    nh, nkv, d = HEADS[case["model"]][:3]
    for r, (C, P) in enumerate(zip(st["Cs"], st["Ps"])):
        at, first = st["row0"][r], min(case["first"], C - 1)
        _, s = _scores(st, r, first)
        lse = st["lse"][:, at + first:at + C].reshape(nkv, nh // nkv, C - first, 1)
        new = torch.exp(s - lse).sum(dim=(1, 2))
        w = st["weight"][0, r]
        w[:, :P] = w[:, :P] * case["decay"] + new[:, :P]
        w[:, P:P + C] = new[:, P:]
    return st["weight"]


# ---- eviction, room for new slots, and their commit -------------------------------------------------------------
def _evict(st):
    case = st["case"]
    nh, nkv, d, base = HEADS[case["model"]][:4]
    n, P, keep, sink, recent, L = (case[x] for x in ("n", "P", "keep", "sink", "recent", "layers"))
    table, lens, refs, kpool, vpool, weight, kept = out = tuple(st[x] for x in ("table", "len", "refs", "kpool", "vpool", "weight", "kept"))
    if own:
        c, cache = st["ctx"], st["cache"]
        c.goose_pages_evict(cache, st["evictions"], weight, kept, case["reposition"])
        if st["new"][0]:
            c.goose_pages_reserve(cache, st["seqs"], st["new"])
            c.goose_pages_append(cache, st["chunks"])
        return out
    bits = (torch.ones((), dtype=torch.int64, device=DEV) << torch.arange(PAGE, device=DEV))
    full = (P + PAGE - 1) // PAGE
    if keep >= P:
        kept.zero_()
        every = torch.zeros((full * PAGE,), dtype=torch.int64, device=DEV)
        every[:P] = 1
        kept[..., :full] = (every.view(full, PAGE) * bits).sum(dim=-1)
        return out
    # which slots
    w = weight[..., :P]                                                                # [layer][seq][head][slot]
    heavy = torch.argsort(-w[..., sink:P - recent], dim=-1, stable=True)[..., :keep - sink - recent] + sink
    mask = torch.zeros((L, n, nkv, full * PAGE), dtype=torch.bool, device=DEV)
    mask[..., :sink] = True
    mask[..., P - recent:P] = True
    mask.scatter_(-1, heavy, True)
    kept.zero_()
    kept[..., :full] = (mask.view(L, n, nkv, full, PAGE).long() * bits).sum(dim=-1).permute(1, 0, 2, 3)
    idx = mask.nonzero()[:, 3].view(L, n, nkv, keep)
    weight[..., :keep] = torch.gather(w, -1, idx)
    # their rows to the front
    inv = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    for r in range(n):
        pages = table[r, :full].long()
        for pool, off in ((kpool, st["koff"]), (vpool, st["voff"])):
            x = pool[:, pages][..., off].permute(0, 2, 1, 3, 4).reshape(L, nkv, full * PAGE, d)  # [layer][head][slot][d]
            y = torch.gather(x, 2, idx[:, r].unsqueeze(-1).expand(L, nkv, keep, d))
            if pool is kpool and case["reposition"]:
                ang = (torch.arange(keep, device=DEV) - idx[:, r]).double().unsqueeze(-1) * inv
                co, si = torch.cos(ang).float(), torch.sin(ang).float()
                a, b = y[..., :d // 2].float(), y[..., d // 2:].float()
                y = torch.cat((a * co - b * si, b * co + a * si), dim=-1).to(y.dtype)
            x[:, :, :keep] = y
            pool[:, pages] = _pack(x.view(L, nkv, full, PAGE, d).permute(0, 2, 1, 3, 4), off)
    # pages behind them go back, and the room is taken again: lowest free ids first
    left = (keep + PAGE - 1) // PAGE
    refs.index_add_(0, table[:n, left:full].reshape(-1).long(), torch.full((n * (full - left),), -1, dtype=torch.int32, device=DEV))
    free = torch.argsort((refs > 0).int(), stable=True)[:n * (full - left)].view(n, full - left)
    table[:n, left:full] = free.int()
    refs[free.reshape(-1)] = 1
    return out


def _pairs(case):
    Cs, Ps = _sizes(case)
    return sum((c - f) * p + (c * (c + 1) - f * (f + 1)) // 2 for c, p, f in zip(Cs, Ps, (min(case.get("first", 0), c - 1) for c in Cs)))


def work(case):
    nh, nkv, d = HEADS[case["model"]][:3]
    if case["kind"] == "evict":
        rows = max(0, case["keep"] - case["sink"]) if case["keep"] < case["P"] else 0
        per = case["layers"] * nkv * (rows * 2 * 2 * d * 2 + case["P"] * 4 + rows * 4 + case["P"] // 8)
        return {"bytes": int(case["n"] * (per + 8 * (case["P"] // PAGE + 1))), "flops": 0}
    Cs, Ps = _sizes(case)
    rows, slots = sum(Cs), sum(p + c for p, c in zip(Ps, Cs))
    if case["kind"] == "weight":
        rows = sum(c - min(case["first"], c - 1) for c in Cs)
        once = 2 if case["decay"] else 1
        return {"bytes": int(2 * slots * nkv * d + rows * nh * (d * 2 * case["q_terms"] + 4) + 4 * nkv * (once * sum(Ps) + sum(Cs))),
                "flops": int(2 * nh * d * _pairs(case))}
    return {"bytes": int(2 * 2 * slots * nkv * d + rows * nh * (d * 2 * (case["q_terms"] + 1) + 4)), "flops": int(4 * nh * d * _pairs(case))}


# ---- the definitions in 64 bits, from the logical inputs --------------------------------------------------------------
def exact(case, seed):
    return {"attn": _exact_attn, "weight": _exact_weight, "evict": _exact_evict}[case["kind"]](case, seed)


def _exact_rows(i, r, x, n):
    """Rows [n][head][d] of request r in 64 bits."""
    return i[x][torch.tensor(i["table"][r][:(n + PAGE - 1) // PAGE], device=DEV)].transpose(1, 2).flatten(0, 1)[:n].double()


def _exact_attn(case, seed):
    nh, nkv, d = HEADS[case["model"]][:3]
    i = _chunk_inputs(case, seed)
    q = i["hi"].double() + (i["lo"].double() if i["lo"] is not None else 0.0)
    out = torch.zeros((i["rows"], nh, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((nh, i["rows"]), dtype=torch.float64, device=DEV)
    for r, (C, P) in enumerate(zip(i["Cs"], i["Ps"])):
        k, v = _exact_rows(i, r, "k", P + C), _exact_rows(i, r, "v", P + C)
        at = i["row0"][r]
        for a in range(0, C, 1024):
            b = min(C, a + 1024)
            see = torch.arange(P + C, device=DEV).view(1, -1) <= P + torch.arange(a, b, device=DEV).view(-1, 1)
            for x in range(nh):
                y = x * nkv // nh
                s = torch.where(see, q[at + a:at + b, x] @ k[:, y].t() / math.sqrt(d), -math.inf)
                lse[x, at + a:at + b] = torch.logsumexp(s, dim=1)
                out[at + a:at + b, x] = torch.exp(s - lse[x, at + a:at + b].view(-1, 1)) @ v[:, y]
    return out.view(i["rows"], nh * d), lse


def _exact_weight(case, seed):
    nh, nkv, d = HEADS[case["model"]][:3]
    i = _chunk_inputs(case, seed)
    given = i["lse"].double()
    q = i["hi"].double() + (i["lo"].double() if i["lo"] is not None else 0.0)
    w = i["w"].double()
    for r, (C, P) in enumerate(zip(i["Cs"], i["Ps"])):
        w[0, r, :, :P] *= case["decay"]
        w[0, r, :, P:P + C] = 0.0
        k = _exact_rows(i, r, "k", P + C)
        at = i["row0"][r]
        for a in range(min(case["first"], C - 1), C, 1024):
            b = min(C, a + 1024)
            see = torch.arange(P + C, device=DEV).view(1, -1) <= P + torch.arange(a, b, device=DEV).view(-1, 1)
            for x in range(nh):
                y = x * nkv // nh
                s = q[at + a:at + b, x] @ k[:, y].t() / math.sqrt(d)
                w[0, r, y, :P + C] += torch.where(see, torch.exp(s - given[x, at + a:at + b].view(-1, 1)), 0.0).sum(dim=0)
    return w


def _exact_evict(case, seed):
    nh, nkv, d, base = HEADS[case["model"]][:4]
    i = _evict_inputs(case, seed)
    koff, voff = _page_offsets(d)
    n, P, keep, sink, recent, L = (case[x] for x in ("n", "P", "keep", "sink", "recent", "layers"))
    table, refs, w, k, v = i["table"], i["refs"], i["w"].double(), i["k"].double(), i["v"].double()
    old = i["w"].cpu().double()
    kept = torch.zeros((n, L, nkv, len(table[0])), dtype=torch.int64)
    freq = torch.tensor([base ** (-2.0 * j / d) for j in range(d // 2)], dtype=torch.float64, device=DEV)
    for r in range(n):
        place = torch.tensor([table[r][s // PAGE] * PAGE + s % PAGE for s in range(P)], device=DEV)
        for l in range(L):
            for h in range(nkv):
                mine = list(range(P))
                if keep < P:
                    x = old[l, r, h].tolist()
                    rest = sorted(range(sink, P - recent), key=lambda s: (-x[s], s))[:keep - sink - recent]
                    mine = sorted(list(range(sink)) + rest + list(range(P - recent, P)))
                    at = torch.tensor(mine, device=DEV)
                    w[l, r, h, :keep] = i["w"][l, r, h, at].double()
                    for pool in (k, v):
                        flat = pool[l, :, h].reshape(-1, d)
                        y = flat[place[at]]
                        if pool is k and case["reposition"]:
                            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                                               (torch.arange(keep, device=DEV) - at).double().view(-1, 1) * freq)
                            z = torch.complex(y[:, :d // 2], y[:, d // 2:]) * turn
                            y = torch.cat((z.real, z.imag), dim=1)
                        flat[place[:keep]] = y
                        pool[l, :, h] = flat.view(-1, PAGE, d)
                words = [0] * len(table[0])
                for s in mine:
                    words[s // PAGE] |= 1 << (s % PAGE)
                kept[r, l, h] = torch.tensor([x - (1 << 64) if x >> 63 else x for x in words])
    if keep < P:
        for r in range(n):
            for j in range((keep + PAGE - 1) // PAGE, (P + PAGE - 1) // PAGE):
                refs[table[r][j]] = 0
        for r in range(n):
            for j in range((keep + PAGE - 1) // PAGE, (P + PAGE - 1) // PAGE):
                table[r][j] = refs.index(0)
                refs[table[r][j]] = 1
    return _i32(table), _i32(i["len"]), _i32(refs), _pack(k, koff), _pack(v, voff), w, kept.to(DEV)
