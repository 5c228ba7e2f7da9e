"""Plain forms of the operators that prompts on a paged cache need: 64-bit causal attention and slot weights, a simulator of append and eviction."""
import math

import numpy as np
import torch

from paged_ref import PAGE, PageSim


def chunk_attention64(q, k, v, P):
    """q [C][nh][d], k and v [nkv][P + C][d], all 64-bit; token i sees slots [0, P + i].  Returns the output, sum p |v| per element, lse [nh][C],
    the largest sum |q||k| / sqrt(d) of a row's visible scores [C][nh] and sum |v| over its visible slots (for error bounds)."""
    C, nh, d = q.shape
    nkv, N = k.shape[:2]
    out, mag, vs = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    lse, qk = torch.zeros((nh, C), dtype=torch.float64), torch.zeros((C, nh), dtype=torch.float64)
    see = torch.arange(N).view(1, -1) <= P + torch.arange(C).view(-1, 1)
    for x in range(nh):
        kk, vv = k[x * nkv // nh], v[x * nkv // nh]
        # masked places are left out, whatever they hold
        s = torch.where(see, (q[:, x] @ torch.nan_to_num(kk, 0.0, 0.0, 0.0).T) / math.sqrt(d), -math.inf)
        bad = ~torch.isfinite(kk).all(1)
        for n in torch.nonzero(bad).reshape(-1).tolist():
            s[:, n] = torch.where(see[:, n], (q[:, x] * kk[n]).sum(1) / math.sqrt(d), -math.inf)
        top = s.max(1, keepdim=True).values
        e = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
        total = e.sum(1, keepdim=True)
        p = torch.where(total == 0, 0.0, e / total)
        clean = torch.nan_to_num(vv, 0.0, 0.0, 0.0)
        o = p @ clean
        for n in torch.nonzero(~torch.isfinite(vv).all(1)).reshape(-1).tolist():
            odd = torch.where(torch.isfinite(vv[n]), 0.0, vv[n])
            o = o + torch.where(see[:, n:n + 1] & (odd != 0), p[:, n:n + 1] * odd, 0.0)
        out[:, x], mag[:, x] = o, p @ clean.abs()
        vs[:, x] = see.double() @ clean.abs()
        lse[x] = (top + torch.log(total)).reshape(-1)
        qk[:, x] = torch.where(see, q[:, x].abs() @ torch.nan_to_num(kk, 0.0, 0.0, 0.0).abs().T, 0.0).max(1).values / math.sqrt(d)
    return out, mag, lse, qk, vs


def slot_weights64(q, k, lse, P, first):
    """What the slots receive from tokens first .. C - 1: [nkv][P + C]; and per slot the sum of weight x (score magnitude), for error bounds."""
    C, nh, d = q.shape
    nkv, N = k.shape[:2]
    w, err = torch.zeros((nkv, N), dtype=torch.float64), torch.zeros((nkv, N), dtype=torch.float64)
    see = torch.arange(N).view(1, -1) <= P + torch.arange(first, C).view(-1, 1)
    for x in range(nh):
        kk = k[x * nkv // nh]
        s = q[first:, x] @ kk.T / math.sqrt(d)
        l = lse[x, first:].view(-1, 1)
        p = torch.where(see & (l != -math.inf), torch.exp(s - l), 0.0)
        size = (q[first:, x].abs() @ kk.abs().T / math.sqrt(d)) * (d + 4) * 2.0 ** -24 + l.abs() * 2.0 ** -22 + 2.0 ** -20
        w[x * nkv // nh] += p.sum(0)
        err[x * nkv // nh] += torch.where(p > 0, p * size, 0.0).sum(0)
    return w, err


class PromptSim(PageSim):
    """PageSim with append and eviction; k, v: logical rows [layers][pages][heads][64][d] of the cache's type; weight [layers][seqs][heads][slots]."""

    def append(self, seqs, new):
        flags = 0
        for q, n in zip(seqs, new):
            P, end = int(self.len[q]), int(self.len[q]) + n
            if P < 0 or end > self.table.shape[1] * PAGE:
                flags |= 2
                continue
            pages = self.table[q, P // PAGE:(end + PAGE - 1) // PAGE]
            if any(e < 0 or e >= len(self.refs) or self.refs[e] != 1 for e in pages):
                flags |= 16
                continue
            self.len[q] = end
            self._release(q, (end + PAGE - 1) // PAGE)
        return flags

    def evict(self, evictions, weight, base, reposition):
        """Returns flags and the kept words [n][layers][heads][pages of a table] (None where the sequence was left alone).  Keys that are turned are
        rounded from 64 bits."""
        L, _, nkv, _, d = self.k.shape
        flags, words = 0, []
        freq = torch.tensor([base ** (-2.0 * j / d) for j in range(d // 2)], dtype=torch.float64)
        done = []
        for e in evictions:
            q, keep, sink, recent, n = e["seq"], e["keep"], e.get("sink", 0), e.get("recent", 0), int(self.len[e["seq"]])
            used = self.table[q, :max(0, (n + PAGE - 1) // PAGE)]
            if n < 0 or n > self.table.shape[1] * PAGE:
                flags |= 2
                words.append(None)
                continue
            moves = keep < n and sink < keep
            if any(p < 0 or p >= len(self.refs) or (moves and sink // PAGE <= i <= (keep - 1) // PAGE and self.refs[p] != 1)
                   for i, p in enumerate(used)):
                flags |= 16
                words.append(None)
                continue
            out = np.zeros((L, nkv, self.table.shape[1]), np.uint64)
            place = torch.tensor([int(used[s // PAGE]) * PAGE + s % PAGE for s in range(n)], dtype=torch.int64)
            for l in range(L):
                for h in range(nkv):
                    w = weight[l, q, h, :n].tolist()
                    mine = list(range(n))
                    if keep < n:
                        rest = sorted(range(sink, n - recent), key=lambda s: (math.isnan(w[s]), 0.0 if math.isnan(w[s]) else -w[s], s))
                        mine = sorted(list(range(sink)) + rest[:keep - sink - recent] + list(range(n - recent, n)))
                        at = torch.tensor(mine, dtype=torch.int64)
                        weight[l, q, h, :keep] = weight[l, q, h, at].clone()
                        for x in (self.k, self.v):
                            flat = x[l, :, h].reshape(-1, d)
                            y = flat[place[at]].clone()
                            if x is self.k and reposition:
                                ang = (torch.arange(keep) - at).double().view(-1, 1) * freq
                                a, b = y[:, :d // 2].double(), y[:, d // 2:].double()
                                turned = torch.cat((a * torch.cos(ang) - b * torch.sin(ang), b * torch.cos(ang) + a * torch.sin(ang)), 1).to(y.dtype)
                                y = torch.where((torch.arange(keep) == at).view(-1, 1), y, turned)
                            flat[place[:keep]] = y
                            x[l, :, h] = flat.view(-1, PAGE, d)
                    for s in mine:
                        out[l, h, s // PAGE] |= np.uint64(1) << np.uint64(s % PAGE)
            words.append(torch.from_numpy(out.view(np.int64)))
            if keep < n:
                done.append((q, keep))
        for q, keep in done:
            self.len[q] = keep
            self._release(q, (keep + PAGE - 1) // PAGE)
        return flags, words
