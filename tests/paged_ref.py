"""Plain forms of the paged-cache operators for the tests: a simulator of the tables, and 64-bit attention and rotation."""
import math

import numpy as np
import torch

from paper_2604_02047_amd import layout

PAGE = 64


def pack_pages(k, v):
    """Logical rows [layers][pages][heads][64][d] -> the pools' operand order [layers][pages][heads][64 * d]."""
    d = k.shape[-1]
    slots = torch.arange(PAGE, device=k.device)
    ko, vo = layout.k_offsets(slots, d).reshape(-1), layout.v_offsets(slots, d).reshape(-1)
    kp, vp = torch.empty(k.shape[:3] + (PAGE * d,), dtype=k.dtype, device=k.device), None
    vp = torch.empty_like(kp)
    kp[..., ko] = k.reshape(kp.shape)
    vp[..., vo] = v.reshape(vp.shape)
    return kp, vp


def unpack_pages(kp, vp, d):
    slots = torch.arange(PAGE, device=kp.device)
    return kp[..., layout.k_offsets(slots, d)], vp[..., layout.v_offsets(slots, d)]


class PageSim:
    """Tables, lengths, counts and logical K/V rows of a paged cache; the same calls on the host.  Returns the flags they raise."""

    def __init__(self, n_seqs, width, n_pages, k=None, v=None):
        self.table = np.full((n_seqs, width), -1, np.int32)
        self.len = np.zeros(n_seqs, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.k, self.v = k, v  # [layers][pages][heads][64][d]

    def fork(self, src, dst, length=-1):
        n = int(self.len[src]) if length < 0 else length
        if n > self.len[src]:
            return 2
        flags = 0
        for q in dst:
            if self.len[q] != 0 or self.table[q, 0] != -1:
                flags = 16
                continue
            for i in range((n + PAGE - 1) // PAGE):
                self.table[q, i] = self.table[src, i]
                self.refs[self.table[src, i]] += 1
            self.len[q] = n
        return flags

    def reserve(self, seqs, new):
        table, refs, copies = self.table.copy(), self.refs.copy(), []
        for q, n in zip(seqs, new):
            P = int(self.len[q])
            if P + n > table.shape[1] * PAGE:
                return 2
            for i in range(P // PAGE, (P + n - 1) // PAGE + 1):
                e = int(table[q, i])
                if e >= 0 and refs[e] == 1:
                    continue
                # (a page that this call has released is not free for it)
                free = [p for p in range(len(refs)) if refs[p] == 0 and self.refs[p] == 0]
                if not free:
                    return 16
                table[q, i] = free[0]
                refs[free[0]] = 1
                if e >= 0:
                    refs[e] -= 1
                    copies.append((e, free[0], (P % PAGE + 31) // 32 * 32))
        self.table, self.refs = table, refs
        if self.k is not None:
            for a, b, n in copies:
                self.k[:, b, :, :n] = self.k[:, a, :, :n]
                self.v[:, b, :, :n] = self.v[:, a, :, :n]
        return 0

    def commit(self, seqs, paths):
        for q, path in zip(seqs, paths):
            P, L = int(self.len[q]), len(path) - 1
            for j in range(1, L + 1):
                a, b = P + path[j], P + j
                for x in (self.k, self.v):
                    x[:, self.table[q, b // PAGE], :, b % PAGE] = x[:, self.table[q, a // PAGE], :, a % PAGE]
            self.len[q] = P + L + 1
            self._release(q, (P + L + PAGE) // PAGE)
        return 0

    def free(self, seqs):
        for q in seqs:
            self._release(q, 0)
            self.len[q] = 0
        return 0

    def _release(self, q, first):
        for i in range(first, self.table.shape[1]):
            if self.table[q, i] >= 0:
                self.refs[self.table[q, i]] -= 1
                self.table[q, i] = -1


def rows_of(sim_k, table_row, n):
    """Logical rows [heads][n][d] of a sequence from one layer's [pages][heads][64][d]."""
    pages = torch.as_tensor(np.asarray(table_row[:(n + PAGE - 1) // PAGE], np.int64), device=sim_k.device)
    x = sim_k[pages].transpose(0, 1)
    return x.reshape(x.shape[0], -1, x.shape[-1])[:, :n]


def mask_words(parent):
    """uint64 words [B][ceil(B/64)] (as int64) and the boolean matrix of ancestors-or-self."""
    B = len(parent)
    see = np.zeros((B, B), bool)
    for i, p in enumerate(parent):
        if p >= 0:
            see[i] = see[p]
        see[i, i] = True
    W = (B + 63) // 64
    words = np.zeros((B, W), np.uint64)
    for i in range(B):
        for j in np.nonzero(see[i])[0]:
            words[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return torch.from_numpy(words.view(np.int64)), see


def attention64(q, k, v, see):
    """q [B][nh][d], k and v [nkv][N][d], see bool [B][N]; all 64-bit.  Returns the output and sum p |v| per element, the largest
    sum |q||k| of a row's visible scores and sum |v| over its visible keys (for error bounds).  Masked places are left out, whatever they hold."""
    B, nh, d = q.shape
    nkv, N = k.shape[0], k.shape[1]
    out, mag = torch.zeros_like(q), torch.zeros_like(q)
    qk, vs = torch.zeros((B, nh), dtype=torch.float64), torch.zeros_like(q)
    for i in range(B):
        idx = torch.nonzero(see[i]).reshape(-1)
        if len(idx) == 0:
            continue
        for h in range(nkv):
            ki, vi = k[h, idx], v[h, idx]
            for x in range(h * nh // nkv, (h + 1) * nh // nkv):
                s = (ki * q[i, x]).sum(1) / math.sqrt(d)
                top = s.max()
                if top == -math.inf:
                    continue
                e = torch.exp(s - top)
                p = e / e.sum()
                out[i, x], mag[i, x] = (p[:, None] * vi).sum(0), (p[:, None] * vi.abs()).sum(0)
                qk[i, x], vs[i, x] = (ki * q[i, x]).abs().sum(1).max() / math.sqrt(d), vi.abs().sum(0)
    return out, mag, qk, vs


def rope64(part, gq, gk, pos, nh, nkv, d, base, eps):
    """part [ks][B][(nh + 2 nkv) d] 64-bit -> rotated q [B][nh][d], k and v [B][nkv][d]."""
    x = part.sum(0).view(part.shape[1], nh + 2 * nkv, d)
    q, k, v = x[:, :nh], x[:, nh:nh + nkv], x[:, nh + nkv:]
    ang = torch.as_tensor(pos, dtype=torch.float64).view(-1, 1, 1) * torch.tensor([base ** (-2.0 * j / d) for j in range(d // 2)],
                                                                                   dtype=torch.float64)
    c, s = torch.cos(ang), torch.sin(ang)

    def turn(t, g):
        if g is not None:
            t = t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * g
        a, b = t[..., :d // 2], t[..., d // 2:]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    return turn(q, gq), turn(k, gk), v
