"""A plain host model of the paged cache, written from the header's words (test infrastructure).

State in numpy: ref, table, length as on the device, pools as raw bits [n_pages, H, page, d];
every operation walks the slots one by one.  Attention in 64 bits on the CPU, with a bound of
the kernels' rounding derived beside it."""
import math

import numpy as np
import torch

BAD, FULL = 32, 16


def pages_for(rows, page):
    return -(-rows // page)


class Model:
    def __init__(self, k, v, ref, table, length):
        self.k, self.v, self.ref, self.table, self.length = (x.copy() for x in (k, v, ref, table, length))
        self.page, self.n_pages = k.shape[2], k.shape[0]
        self.S, self.M = table.shape

    def _free(self, begun):
        return [p for p in range(self.n_pages) if begun[p] == 0]

    def resize(self, new_len):
        begun, status, need = self.ref.copy(), 0, []
        for s in range(self.S):
            L, t = int(self.length[s]), int(new_len[s])
            if t < 0:
                continue
            if t > self.M * self.page or not 0 <= L <= self.M * self.page:
                return BAD
            if t > L:
                first = pages_for(L, self.page)
                if L % self.page:
                    p = self.table[s, first - 1]
                    if not 0 <= p < self.n_pages:
                        return BAD
                    first -= int(begun[p] > 1)
                need += [(s, j) for j in range(first, pages_for(t, self.page))]
        free = self._free(begun)
        if len(need) > len(free):
            return FULL
        for (s, j), p in zip(need, free):
            L = int(self.length[s])
            if j < pages_for(L, self.page):
                old, r = self.table[s, j], L % self.page
                self.ref[old] -= 1
                self.k[p][:, :r] = self.k[old][:, :r]
                self.v[p][:, :r] = self.v[old][:, :r]
            self.table[s, j] = p
            self.ref[p] = 1
        for s in range(self.S):
            L, t = int(self.length[s]), int(new_len[s])
            if t < 0:
                continue
            for j in range(pages_for(t, self.page), pages_for(L, self.page)):
                if 0 <= self.table[s, j] < self.n_pages:
                    self.ref[self.table[s, j]] -= 1
                else:
                    status = BAD
                self.table[s, j] = -1
            self.length[s] = t
        return status

    def fork(self, parent):
        status, length = 0, self.length.copy()
        for s in range(self.S):
            p = int(parent[s])
            if p < 0:
                continue
            if p >= self.S or parent[p] >= 0 or length[s] != 0 or not 0 <= length[p] <= self.M * self.page:
                status = BAD
                continue
            n = pages_for(int(length[p]), self.page)
            row = self.table[p, :n]
            if ((row < 0) | (row >= self.n_pages)).any():
                status = BAD
                continue
            self.table[s, :n] = row
            for q in row:
                self.ref[q] += 1
            self.length[s] = length[p]
        return status

    def write(self, k_new, v_new, cu):
        status = 0
        for s in range(self.S):
            n = cu[s + 1] - cu[s]
            for i in range(n):
                row = int(self.length[s]) - n + i
                p = self.table[s, row // self.page] if 0 <= row < self.M * self.page else -1
                if not 0 <= p < self.n_pages:
                    status = BAD
                    continue
                self.k[p][:, row % self.page] = k_new[cu[s] + i]
                self.v[p][:, row % self.page] = v_new[cu[s] + i]
        return status

    def compact(self, map_, src):
        K, begun, need, moved = src.shape[2], self.ref.copy(), [], []
        for s in range(self.S):
            if map_[s] < 0:
                continue
            L = int(self.length[s])
            if map_[s] >= src.shape[0] or not K <= L <= self.M * self.page:
                return BAD
            row = self.table[s, :pages_for(L, self.page)]
            if ((row < 0) | (row >= self.n_pages)).any():
                return BAD
            need += [(s, j) for j in range(pages_for(K, self.page)) if begun[row[j]] > 1]
        free = self._free(begun)
        if len(need) > len(free):
            return FULL
        for s in range(self.S):
            if map_[s] >= 0:
                moved.append((s, [self.rows(x, s, src[map_[s]]) for x in (self.k, self.v)]))
        for (s, j), p in zip(need, free):
            self.ref[self.table[s, j]] -= 1
            self.table[s, j] = p
            self.ref[p] = 1
        for s, pair in moved:
            for x, rows in zip((self.k, self.v), pair):
                for j in range(K):
                    x[self.table[s, j // self.page]][:, j % self.page] = rows[:, j]
            for j in range(pages_for(K, self.page), pages_for(int(self.length[s]), self.page)):
                self.ref[self.table[s, j]] -= 1
                self.table[s, j] = -1
            self.length[s] = K
        return 0

    def rows(self, x, s, src=None):
        """Rows of slot s, [H, rows, d]; with src [H, K], head h's rows src[h]."""
        H = x.shape[1]
        if src is None:
            src = np.broadcast_to(np.arange(int(self.length[s])), (H, int(self.length[s])))
        p = self.table[s][src // self.page]
        return x[p, np.arange(H)[:, None], src % self.page].copy()


def attend(q, k, v, n_rows, causal):
    """Attention in 64 bits of the newest n tokens q [n, H, G, d] (float64) over the rows k, v
    [H, L, d], token i seeing rows < sees_i.  Returns out, lse and their error bounds
    (dict): `A` = sum_j p_j |v_j|, and `delta`, the most a score can be off in fp32."""
    n, H, G, d = q.shape
    out = np.zeros((n, H, G, d))
    lse = np.full((n, H, G), -math.inf)
    A = np.zeros((n, H, G, d))
    delta = np.zeros((n, H, G))
    for i in range(n):
        sees = max(n_rows - n + i + 1, 0) if causal else n_rows
        if sees == 0:
            continue
        kk, vv = k[:, :sees], v[:, :sees]
        z = np.einsum("hgd,hjd->hgj", q[i], kk) / math.sqrt(d)
        # d products and sums in fp32, in any order: d + 1 steps of sum |q_c k_c| (whole
        # ones: the matrix unit's rounding is not specified); 3 more for the scale and the
        # difference to the maximum
        mag = np.einsum("hgd,hjd->hgj", np.abs(q[i]), np.abs(kk)) / math.sqrt(d)
        delta[i] = (d + 4) * 2.0 ** -23 * mag.max(-1)
        m = z.max(-1, keepdims=True)
        e = np.exp(z - m)
        w = e.sum(-1, keepdims=True)
        lse[i] = (m + np.log(w))[..., 0]
        out[i] = np.einsum("hgj,hjd->hgd", e / w, vv)
        A[i] = np.einsum("hgj,hjd->hgd", e / w, np.abs(vv))
    return out, lse, dict(A=A, delta=delta)


def out_bound(ref, b, n_keys, bf16):
    """|out - ref| at most this.  Each probability is off by a factor e^(2 delta) (its score and
    the others', in the sum), by 2^-21 for the hardware's exponential and the products of a
    rescale, and sums of n terms in fp32 by n steps; bf16: the probability is rounded to
    2^-8 and so is the output.  The factor 1.01 covers products of these."""
    rel = 2 * b["delta"][..., None] + (2 * n_keys + 64) * 2.0 ** -23 + 2.0 ** -21
    rel = rel + 2.0 ** -8 * bf16
    return 1.01 * (rel * b["A"] + 2.0 ** -8 * bf16 * np.abs(ref)) + 1e-30


def lse_bound(lse, b, n_keys):
    return b["delta"] + (n_keys + 64) * 2.0 ** -23 + 2.0 ** -21 + 4 * 2.0 ** -24 * np.abs(np.where(np.isfinite(lse), lse, 0))


def raw(t):
    """A tensor's bits on the host: bf16 as int16, fp32 as int32."""
    t = t.detach().cpu().contiguous()
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).numpy().copy()
