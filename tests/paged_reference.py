"""The operators over a paged cache in 64 bits on the CPU, row by row, and how far the kernels may be from them."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half a step, relative


def sequences(B, rows, row_start, lengths, max_rows=None, max_len=None):
    """-> [(sequence, first row, rows, length)] as the header defines a batch."""
    out = []
    for b in range(B):
        r0, r1 = (row_start[b], row_start[b + 1]) if row_start is not None else (b * (rows // B), (b + 1) * (rows // B))
        n = r1 - r0 if max_rows is None else min(r1 - r0, max_rows)
        out.append((b, r0, n, lengths[b] if max_len is None else min(lengths[b], max_len)))
    return out


def append(k_pages, v_pages, table, batch, q, k, v, inv_freq):
    """-> (q out, k pages, v pages, |error| bounds of the same shapes).  All CPU tensors; the outputs are float64."""
    S, u = k_pages.shape[1], UNIT[k.dtype]
    half = 0 if inv_freq is None else inv_freq.shape[0]
    ko, vo, qo = k_pages.double(), v_pages.double(), torch.full(q.shape, math.nan, dtype=torch.float64)
    ke, qe = torch.zeros_like(ko), torch.zeros_like(qo)

    def turn(x, pos):
        x = x.double()
        y, err = x.clone(), torch.zeros_like(x)
        if half:
            a = pos * inv_freq
            c, s, x0, x1 = torch.cos(a), torch.sin(a), x[:, :half], x[:, half:2 * half]
            y[:, :half], y[:, half:2 * half] = x0 * c - x1 * s, x1 * c + x0 * s
            # the angle in turns is rounded to fp32 (2^-26 of a turn, 9.4e-8 rad), sine and cosine are good to 2 ulp (2.4e-7), two
            # products and a sum to 2^-24 each (1.8e-7)
            e = 6e-7 * (x0.abs() + x1.abs())
            e = torch.cat([e, e], 1)
            err[:, :2 * half] = e + u * (y[:, :2 * half].abs() + e)
        return y, err

    for b, r0, n, kv in batch:
        for i in range(n):
            pos = kv - n + i
            if pos < 0:
                continue
            qo[r0 + i], qe[r0 + i] = turn(q[r0 + i], pos)
            page = int(table[b][pos // S])
            if 0 <= page < k_pages.shape[0]:
                ko[page, pos % S], ke[page, pos % S] = turn(k[r0 + i], pos)
                vo[page, pos % S] = v[r0 + i].double()
    return qo, ko, vo, qe, ke


def attention(k_pages, v_pages, table, batch, q, scale, window):
    """-> (out, |error| bound), float64, NaN in rows that no sequence owns.

    The bound: scores are sums of hd products in fp32, off by at most (hd + 8) 2^-24 sum |q_i k_i| scale, which weighs twice in a weight
    over a sum of weights; exp2, the sums over n positions and the joins of chunks are off by (n + 64) 2^-24 relative at most; weights are
    rounded once to the type (u), and so is the result (u)."""
    n_pages, S, Hk, hd = k_pages.shape
    Hq, u = q.shape[1], UNIT[q.dtype]
    G = Hq // Hk
    out, err = torch.full(q.shape, math.nan, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b, r0, n, kv in batch:
        for i in range(n):
            pos = kv - n + i
            lo = max(0, pos - window + 1) if window else 0
            at = [(int(table[b][p // S]), p % S) for p in range(lo, pos + 1)]
            at = [(g, r) for g, r in at if 0 <= g < n_pages]
            if not at:
                out[r0 + i] = 0.0
                continue
            pg, pr = (torch.tensor(x) for x in zip(*at))
            K, V = k_pages[pg, pr].double(), v_pages[pg, pr].double()  # [n][Hk][hd]
            for h in range(Hq):
                x = q[r0 + i, h].double()
                Kh, Vh = K[:, h // G], V[:, h // G]
                w = torch.softmax(Kh @ x * scale, 0)
                out[r0 + i, h] = w @ Vh
                size = w @ Vh.abs()
                e = 2 * (hd + 8) * 2.0 ** -24 * float((Kh.abs() @ x.abs()).max()) * scale + (len(at) + 64) * 2.0 ** -24
                err[r0 + i, h] = size * (e + (u if u > 2.0 ** -24 else 0.0)) * 1.01 + u * (out[r0 + i, h].abs() + u * size)
    return out, err
