"""Plain float64 reference of the paged cache (include/ff_paged.h) and the error bounds that its
tests hold the kernels to.  Written per sequence and token from the definitions, on the CPU."""
from __future__ import annotations

import math
from typing import List, NamedTuple, Optional, Tuple

import numpy as np
import torch

U_BF16, U_F32 = 2.0 ** -8, 2.0 ** -24     # half a step, relative (torch.finfo(t).eps / 2)


class Batch(NamedTuple):
    """A batch on the CPU."""
    q_start: List[int]
    kv_len: List[int]
    table: torch.Tensor        # int32 [n_seqs][max_pages]
    page: int                  # tokens per page
    n_pages: int               # pages of the pool

    def tokens(self, n_rows: int):
        """(row, sequence, token index) of every row that belongs to a sequence."""
        for s, length in enumerate(self.kv_len):
            a, e = self.q_start[s], self.q_start[s + 1]
            for row in range(a, e):
                yield row, s, max(length, 0) - (e - a) + row - a

    def place(self, s: int, j: int) -> Optional[Tuple[int, int]]:
        """(page, slot) of token j of sequence s, None in a hole."""
        col = j // self.page
        if not 0 <= col < self.table.shape[1]:
            return None
        p = int(self.table[s, col])
        return (p, j % self.page) if 0 <= p < self.n_pages else None


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().double().numpy()


def rope_split(d: int) -> Tuple[int, int, int]:
    return d // 2 - 2 * (d // 6), d // 6, d // 6


def rotate(x: np.ndarray, pos, pairs, theta: float) -> np.ndarray:
    """x [heads][d] turned by the position (t, h, w)."""
    angle = np.array([pos[a] * theta ** (-j / n) for a, n in enumerate(pairs) for j in range(n)])
    z = (x[:, 0::2] + 1j * x[:, 1::2]) * np.exp(1j * angle)
    out = np.empty_like(x)
    out[:, 0::2], out[:, 1::2] = z.real, z.imag
    return out


def append(b: Batch, k, v, k_pages, v_pages, q=None, q_out=None, positions=None, pairs=None,
           theta: float = 10000.0):
    """(k_pages, v_pages, q_out) after an append, float64 and unrounded where written."""
    kp, vp = f64(k_pages), f64(v_pages)
    qo = f64(q_out) if q_out is not None else None
    pairs = pairs or rope_split(k.shape[2])
    kk, vv, qq = f64(k), f64(v), f64(q) if q is not None else None
    for row, s, i in b.tokens(k.shape[0]):
        if i < 0:
            continue
        pos = [int(x) for x in positions[row]] if positions is not None else [i, i, i]
        if qq is not None:
            qo[row] = rotate(qq[row], pos, pairs, theta)
        at = b.place(s, i)
        if at is not None:
            kp[at[0], :, at[1]] = rotate(kk[row], pos, pairs, theta)
            vp[at[0], :, at[1]] = vv[row]
    return kp, vp, qo


class Attention(NamedTuple):
    out: np.ndarray     # [rows][q heads][d]
    lse: np.ndarray     # [rows][q heads], base 2
    tol: np.ndarray     # bound of |kernel - out|
    lse_tol: np.ndarray
    rows: List[int]     # rows that belong to a sequence


def attention(b: Batch, q, k_pages, v_pages, *, block=False, window=-1, anchors=0,
              scale: Optional[float] = None, rows: Optional[List[int]] = None,
              heads: Optional[List[int]] = None) -> Attention:
    """Attention by the definition.  The bound counts, relative to a weight p_j:
      u_p   its rounding as an operand (bf16 kernels: half a step of bf16),
      e_s   the float32 score: a sum of d products and the scaling, (d + 8) 2^-24 of the sum of
            the products' magnitudes, on both the key's and the reference's side, and the
            exponential (4 steps of float32),
    so a quotient of weighted sums is off by at most (u_p + e_s) (sum p |v| / sum p + |out|),
    the float32 sums over n keys by n 2^-24 of the same, the result's rounding by half a step."""
    bf16 = q.dtype == torch.bfloat16
    n_rows, hq, d = q.shape
    hk = k_pages.shape[1]
    g = hq // hk
    scale = scale if scale is not None else 1.0 / math.sqrt(d)
    u_out, u_p = (U_BF16, U_BF16) if bf16 else (U_F32, 0.0)
    res = Attention(np.zeros((n_rows, hq, d)), np.full((n_rows, hq), -np.inf), np.zeros((n_rows, hq, d)),
                    np.zeros((n_rows, hq)), [])
    kc, vc = k_pages.detach().cpu(), v_pages.detach().cpu()
    qq = f64(q)
    for row, s, i in b.tokens(n_rows):
        res.rows.append(row)
        if rows is not None and row not in rows:
            continue
        first = max(b.kv_len[s], 0) - (b.q_start[s + 1] - b.q_start[s])
        at = max(first if block else i, 0)
        end = b.kv_len[s] if block else i + 1
        seen = [b.place(s, j) for j in range(max(end, 0))
                if window < 0 or j >= at - window or j < anchors]
        seen = [x for x in seen if x is not None]
        if not seen:
            continue
        pg, sl = torch.tensor([x[0] for x in seen]), torch.tensor([x[1] for x in seen])
        for h in (range(hq) if heads is None else heads):
            k, v = f64(kc[pg, h // g, sl]), f64(vc[pg, h // g, sl])
            with np.errstate(invalid="ignore", over="ignore"):
                x = (k @ qq[row, h]) * scale
                size = float(np.max((np.abs(k) @ np.abs(qq[row, h])) * scale))
                p = np.exp(x - x.max())
                total = p.sum()
                res.out[row, h] = p @ v / total
                mean = p @ np.abs(v) / total
                res.lse[row, h] = (x.max() + math.log(total)) / math.log(2.0) if total == total else math.nan
            e_s = 2 * (d + 8) * U_F32 * size + 8 * U_F32
            e = e_s + len(seen) * U_F32
            res.tol[row, h] = 1.05 * (u_p + e) * (mean + np.abs(res.out[row, h])) + u_out * np.abs(res.out[row, h]) + 1e-30
            res.lse_tol[row, h] = 1.5 * e + 4 * U_F32 * abs(res.lse[row, h]) + 1e-6
    return res
