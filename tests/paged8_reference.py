"""Head transforms, e4m3 caches and attention over them in 64 bits on the CPU, and the batches that their tests run.

A batch: sequences with their rows and lengths, pages in random order, dead rows (negative positions), rows behind the last sequence, absent
pages; what no call may touch carries a mark."""
import math

import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half a step, relative
LEAST = {torch.bfloat16: -100, torch.float16: -15}
MOST = {torch.bfloat16: 1.875 * 2.0 ** 127, torch.float16: 61440.0}
BEYOND = {torch.bfloat16: (2 - 2.0 ** -8) * 2.0 ** 127, torch.float16: 65520.0}  # rounds to infinity from here on
DEV = "cuda:0"


def numbers():
    """The non-negative e4m3 numbers by code, 0 .. 126."""
    out = []
    for c in range(127):
        e, m = c >> 3, c & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return torch.tensor(out, dtype=torch.float64)


def decode(codes):
    """uint8 codes -> float64, NaN for 0x7f and 0xff."""
    table = torch.cat([numbers(), torch.tensor([math.nan], dtype=torch.float64)])
    table = torch.cat([table, -table])
    return table[codes.long()]


def encode(y, td):
    """Heads [.., hd] in 64 bits -> (codes uint8, exponents, distance of |y| / 2^e from the nearest border of two codes)."""
    a = y.abs()
    odd = ~(a < BEYOND[td]).all(-1)
    top = torch.where(odd[..., None], 0.0, a).amax(-1)
    e = torch.full(top.shape, LEAST[td])
    while (more := top > 448.0 * torch.ldexp(torch.ones_like(top), e)).any():
        e = torch.where(more, e + 1, e)
    z = torch.ldexp(a.clamp(max=MOST[td]), -e[..., None])
    z = torch.where(odd[..., None], 0.0, z)
    num = numbers()
    mid = (num[1:] + num[:-1]) / 2
    up = torch.searchsorted(mid, z, right=True)   # ties upwards
    down = torch.searchsorted(mid, z, right=False)  # ties downwards
    code = torch.where(up % 2 == 0, up, down)     # they differ at a tie: the even code
    gap = torch.minimum((z - mid[(code - 1).clamp(min=0)]).abs(), (z - mid[code.clamp(max=125)]).abs())
    code = torch.where(torch.signbit(y), code + 128, code)
    code = torch.where(odd[..., None], 0x7f, code)
    return code.to(torch.uint8), torch.where(odd, LEAST[td], e), gap


def transform(x, pos, w, eps, inv_freq, interleaved):
    """[heads][hd] of one row -> (y, |error| of fp32 arithmetic), float64."""
    y = x.double()
    err = torch.zeros_like(y)
    if w is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * w.double()
        err = 4 * 2.0 ** -24 * y.abs()  # the root and two products, each rounded once, and a little
    if inv_freq is not None:
        half = inv_freq.shape[0]
        R, a = 2 * half, pos * inv_freq
        c, s = torch.cos(a), torch.sin(a)
        i0, i1 = (torch.arange(0, R, 2), torch.arange(1, R, 2)) if interleaved else (torch.arange(half), torch.arange(half, R))
        x0, x1, e0, e1 = y[:, i0], y[:, i1], err[:, i0], err[:, i1]
        z, ze = y.clone(), err.clone()
        z[:, i0], z[:, i1] = x0 * c - x1 * s, x1 * c + x0 * s
        # the angle in turns is rounded to fp32 (9.4e-8 rad), sine and cosine are good to 2 ulp (2.4e-7), two products and a sum to 2^-24 each (1.8e-7)
        ze[:, i0] = ze[:, i1] = 6e-7 * (x0.abs() + x1.abs()) + e0 + e1
        y, err = z, ze
    return y, err


class Batch:
    """rows: new rows per sequence; lens: lengths (a length below the rows makes dead rows); absent: (sequence, page index) without a page."""

    def __init__(self, rows, lens, page, seed=0, ragged=True, extra_rows=3, absent=()):
        self.g = torch.Generator().manual_seed(seed + 5)
        self.rows, self.lens, self.page, self.B, self.ragged = list(rows), list(lens), page, len(rows), ragged
        per = [(n + page - 1) // page for n in lens]
        self.n_pages = sum(per) + 2
        order = torch.randperm(self.n_pages, generator=self.g).to(torch.int32)
        self.table = torch.full((self.B, max(per + [1]) + 1), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = order[at:at + n]
            at += n
        for b, j in absent:
            self.table[b, j] = (-1, self.n_pages, 1 << 30)[j % 3]
        self.row_start = [0]
        for n in rows:
            self.row_start.append(self.row_start[-1] + n)
        self.T = self.row_start[-1] + (extra_rows if ragged else 0)

    def on_gpu(self, B, max_rows=None, max_len=None):
        start = torch.tensor(self.row_start, dtype=torch.int32, device=DEV) if self.ragged else None
        return B.PagedBatch(self.table.to(DEV), torch.tensor(self.lens, dtype=torch.int32, device=DEV), self.T, row_start=start, max_rows=max_rows,
                            max_len=max_len)

    def heads(self, n, hd, td, wide=0, size=1.0):
        """[T][n][hd]; wide: parts of rows that much wider"""
        return (size * torch.randn((self.T, n + wide, hd), generator=self.g)).to(td)[:, wide:]

    def places(self):
        """-> [(sequence, row, position, page or -1, place in it)] of the rows that are alive"""
        out = []
        for b in range(self.B):
            for i in range(self.rows[b]):
                pos = self.lens[b] - self.rows[b] + i
                if pos >= 0:
                    page = int(self.table[b, pos // self.page])
                    out.append((b, self.row_start[b] + i, pos, page if 0 <= page < self.n_pages else -1, pos % self.page))
        return out


def pool(x, layout):
    """[n_pages][page][heads][hd] on the GPU, in memory as the layout says."""
    if layout == "hnd":  # heads before positions
        return x.permute(0, 2, 1, 3).contiguous().to(DEV).permute(0, 2, 1, 3)
    return x.to(DEV)


def attention(k, v, batch, q, scale, window):
    """k, v [n_pages][page][Hk][hd] float64 -> (out, |error| bound), float64, NaN in rows that no sequence owns.

    The bound: scores are sums of hd products in fp32, off by at most (hd + 8) 2^-24 sum |q_i k_i| scale, which weighs twice in a weight
    over a sum of weights; exp2, the sums over n positions and the joins of chunks are off by (n + 64) 2^-24 relative at most; weights are
    rounded once to the type (u), and so is the result (u).  Codes times their scales are numbers of the type: they add nothing."""
    Hq, Hk, hd, u = q.shape[1], k.shape[2], k.shape[3], UNIT[q.dtype]
    G = Hq // Hk
    out, err = torch.full(q.shape, math.nan, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b in range(batch.B):
        n, kv, r0 = batch.rows[b], batch.lens[b], batch.row_start[b]
        if n == 0:
            continue
        out[r0:r0 + n] = 0.0
        at = [(int(batch.table[b, p // batch.page]), p % batch.page, p) for p in range(kv)]
        at = [x for x in at if 0 <= x[0] < batch.n_pages]
        if not at:
            continue
        pg, pr, key = (torch.tensor(x) for x in zip(*at))
        pos = torch.arange(kv - n, kv)[:, None]
        see = (key <= pos) & ((key > pos - window) if window else torch.tensor(True))
        K, V = k[pg, pr], v[pg, pr]  # [n][Hk][hd]
        odd = ~torch.isfinite(V).all(-1)  # a position with a NaN among its values makes NaN of the rows that see it
        for h in range(Hq):
            x, Kh, Vh = q[r0:r0 + n, h].double(), K[:, h // G], torch.where(odd[:, h // G, None], 0.0, V[:, h // G])
            z = torch.where(see, x @ Kh.t() * scale, -math.inf)
            some = see.any(1)
            w = torch.where(some[:, None], torch.softmax(torch.where(some[:, None], z, 0.0), 1), 0.0)
            o, size = w @ Vh, w @ Vh.abs()
            e = 2 * (hd + 8) * 2.0 ** -24 * torch.where(see, x.abs() @ torch.nan_to_num(Kh).abs().t(), 0.0).amax(1) * scale + (len(at) + 64) * 2.0 ** -24
            err[r0:r0 + n, h] = size * (e[:, None] + u) * 1.01 + u * (o.abs() + u * size)
            out[r0:r0 + n, h] = torch.where((see & odd[:, h // G]).any(1)[:, None], math.nan, o)
    return out, err
