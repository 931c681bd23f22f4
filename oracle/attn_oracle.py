"""Reference attention, cache writing and page bookkeeping in fp64 / plain Python -- TEST INFRASTRUCTURE ONLY (nothing in the
product path may import this).

Every query row is taken by itself: scores over the tokens it sees, softmax, weighted sum, in fp64 on the CPU.  With the result
comes how far a right kernel may be from it, from these roundings (bf16 rounds by at most 2^-8 of the value, fp32 by 2^-24):
  - weights are rounded to bf16 and normalised by the sum of the rounded ones: o moves by at most 2^-8 (sum w |v| + |o|),
    to first order; second order is below 2^-8 of that and covered by the factor 1.02
  - a score is a sum of head_dim exact products in fp32, in any order, times the scale: its error is at most
    (head_dim + 4) 2^-24 scale sum |q k|, the exponent's argument m (|s| up to |m| + the distance) is rounded to
    2^-24 of its size; a weight moves by the error of its exponent, and v_exp_f32 by 2^-22 of the value: o moves by at most
    twice the largest of these times sum w |v|
  - sums over tokens are fp32: n 2^-24 sum w |v|, and the same for the norm
  - the output is rounded to bf16: 2^-8 |o|
"""
from __future__ import annotations

from typing import List, Sequence, Tuple

import torch


def attend(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: Sequence[int], scale: float) -> Tuple[torch.Tensor, torch.Tensor]:
    """q [rows, heads, d], k and v [tokens, kv heads, d], row i sees tokens 0 .. positions[i]: (out, tolerance), fp64."""
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    rows, heads, d = q.shape
    group = heads // k.shape[1]
    out, tol = torch.zeros(rows, heads, d, dtype=torch.float64), torch.zeros(rows, heads, d, dtype=torch.float64)
    for i in range(rows):
        n = min(max(positions[i] + 1, 0), k.shape[0])
        if n == 0:
            continue
        for h in range(heads):
            kk, vv = k[:n, h // group], v[:n, h // group]
            s = (kk @ q[i, h]) * scale
            w = torch.softmax(s, 0)
            out[i, h] = w @ vv
            size = (kk.abs() @ q[i, h].abs()) * scale
            e = (d + 4) * 2.0 ** -24 * size.max() + 2.0 ** -23 * 1.5 * (s.abs().max() + 20) + 2.0 ** -22 + 2 * n * 2.0 ** -24
            a = w @ vv.abs()
            tol[i, h] = 1.02 * 2.0 ** -8 * (a + 2 * out[i, h].abs()) + 2 * e * a
    return out, tol


def rotate(x: torch.Tensor, table: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
    """x [rows, heads, d] fp32 or bf16, table fp32 [n, 2, d / 2]: every product and sum rounded to fp32."""
    c, s = table[positions][:, None, 0], table[positions][:, None, 1]
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


class Pages:
    """Page bookkeeping by its plain definition: holders are counted anew for every question."""

    def __init__(self, n_pages: int, page_tokens: int, max_seqs: int, max_seq_pages: int):
        self.n, self.t, self.most = n_pages, page_tokens, max_seq_pages
        self.pages: List[List[int]] = [[] for _ in range(max_seqs)]
        self.length = [0] * max_seqs

    def holders(self, page: int) -> int:
        return sum(own.count(page) for own in self.pages)

    def unused(self) -> List[int]:
        return [p for p in range(self.n) if not self.holders(p)]

    def grow(self, seqs, tokens):
        """Copies asked for, or None where pages run out (then nothing has changed)."""
        keep = [list(p) for p in self.pages], list(self.length)
        copies = []
        try:
            for s, n in zip(seqs, tokens):
                own = self.pages[s]
                if n > 0 and self.length[s] % self.t and self.holders(own[-1]) > 1:
                    fresh = self.unused()[0]
                    copies.append((own[-1], fresh))
                    own[-1] = fresh
                self.length[s] += n
                while len(own) * self.t < self.length[s]:
                    own.append(self.unused()[0])
        except IndexError:
            self.pages, self.length = keep
            return None
        return copies

    def fork(self, parent, child, n):
        self.pages[child] = self.pages[parent][: -(-n // self.t)]
        self.length[child] = n

    def free(self, s):
        self.pages[s], self.length[s] = [], 0
