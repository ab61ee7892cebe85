"""Operators of a caller's own verification pass, as cases that can be timed and whose outputs can be compared: queries and keys normed
and rotated on their way into a paged cache (`spec_paged_append_normed`), the same into a cache of 8 bits (`spec_paged8_append`), that
cache read back (`spec_paged8_read`) and attended over (`spec_paged8_attention`), and logits cut to what temperature, top-k, top-p and
min-p leave of them (`spec_truncate_logits`).

The cache of 8 bits holds e4m3 codes and, for every position and key head, the exponent of one power of two: the smallest with which the
largest magnitude of the head is at most 448 times it.

With `own` false, `run` computes the operators in elementary torch operations: in 32 bits and rounded once at the end, in 64 where a value
decides which of two codes or tokens it is; with `own` true it makes the calls of `paper_2310_18813_amd.binding`.  `exact` is the
definition in 64 bits, sequence by sequence.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TORCH_DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
THETA = 10000.0
EPS = 1e-5
TOP = 448.0                            # the largest e4m3 number
LEAST = {"bf16": -100, "fp16": -15}    # the least exponent of a scale
MOST = {"bf16": 1.875 * 2.0 ** 127, "fp16": 61440.0}  # the largest number of four bits that the type holds


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one user of a model with normed heads, plain decoding: one row into the cache, all latency
        dict(name="normed_b1", kind="normed", dtype="bf16", B=1, q=1, ragged=False, ctx=310, heads=32, kv_heads=8, hd=128, page=16, rot=128,
             interleaved=False, norm=True),
        # prompts of different lengths with interleaved pairs, about 8000 rows at the 33B width
        dict(name="normed_prompts", kind="normed", dtype="fp16", B=5, q=2013, ragged=True, ctx=2013, heads=52, kv_heads=52, hd=128, page=64, rot=128,
             interleaved=True, norm=True),
        # a verification of 64 sequences, four rows each, into 8 bits
        dict(name="append8_b64", kind="append8", dtype="bf16", B=64, q=4, ragged=False, ctx=450, heads=32, kv_heads=8, hd=128, page=16, rot=128,
             interleaved=False, norm=True),
        # prompts of different lengths at the 7B width into 8 bits, without norms
        dict(name="append8_prompts", kind="append8", dtype="bf16", B=5, q=2003, ragged=True, ctx=2003, heads=32, kv_heads=32, hd=128, page=64, rot=128,
             interleaved=False, norm=False),
        # the last block of eight sequences read back, heads of 64, to be written into another pool
        dict(name="read8_blocks", kind="read8", dtype="fp16", B=8, q=64, ragged=False, ctx=500, heads=16, kv_heads=16, hd=64, page=16, rot=0,
             interleaved=False, norm=False),
        # a long prefix read back whole, for a pass that wants 16 bits
        dict(name="read8_prefix", kind="read8", dtype="bf16", B=1, q=32000, ragged=False, ctx=32000, heads=32, kv_heads=8, hd=128, page=64, rot=0,
             interleaved=False, norm=False),
        # one user with a long context, one row: split over the positions and joined
        dict(name="attend8_b1_long", kind="attend8", dtype="fp16", B=1, q=1, ragged=False, ctx=32000, heads=32, kv_heads=8, hd=128, page=64, window=0),
        # the headline workload's verification over a cache of 8 bits: 64 sequences, s = 3, a key head for every query head
        dict(name="attend8_7b_b64", kind="attend8", dtype="bf16", B=64, q=4, ragged=False, ctx=1000, heads=32, kv_heads=32, hd=128, page=16, window=0),
        # chunks of long prompts that join a running batch, some sequences with single rows
        dict(name="attend8_chunks", kind="attend8", dtype="bf16", B=6, q=2048, ragged=True, ctx=8192, heads=32, kv_heads=8, hd=128, page=64, window=0),
        # one row of logits of one user
        dict(name="truncate_b1", kind="truncate", dtype="fp32", B=1, s=0, vocab=32000),
        # the logits of 64 verified sequences as a 16-bit head leaves them, each with its own wishes
        dict(name="truncate_b64", kind="truncate", dtype="bf16", B=64, s=3, vocab=50272),
        # a large vocabulary
        dict(name="truncate_large", kind="truncate", dtype="fp32", B=24, s=7, vocab=151936),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["normed", "append8", "read8", "attend8", "attend8", "truncate"])
    if kind == "truncate":
        vocab = rng.choice([32000, 50272, 151936, rng.randint(1000, 160000)])
        s = rng.randint(0, 8)
        B = _log_int(rng, 1, max(1, 24_000_000 // (vocab * (s + 1))))
        return dict(kind=kind, dtype=rng.choice(["fp32", "bf16", "fp16"]), B=min(B, 128), s=s, vocab=vocab)
    hd = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 8, 16) if kv_heads * g <= 52])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    ragged = rng.random() < 0.4
    q = _log_int(rng, 16, 2048) if ragged else rng.randint(1, 9)
    case = dict(kind=kind, dtype=dtype, ragged=ragged, heads=heads, kv_heads=kv_heads, hd=hd, page=page)
    if kind == "attend8":
        B = _log_int(rng, 1, max(1, min(64, 4000 // q)))
        ctx = max(q, _log_int(rng, 16, max(16, (400_000 if ragged else 1_200_000) // (B * kv_heads))))
        return dict(case, B=B, q=q, ctx=min(ctx, max(q, 8000 if ragged else 32000)), window=rng.choice([0, 0, rng.randint(1, 2000)]))
    B = _log_int(rng, 1, max(1, min(64, 8000 // q)))
    ctx = max(q, _log_int(rng, 16, max(16, 60000 // (B * kv_heads))))
    if kind == "read8":
        return dict(case, B=B, q=q, ctx=ctx, rot=0, interleaved=False, norm=False)
    if kind == "normed":
        case["dtype"] = rng.choice(["bf16", "fp16", "fp32"])
    return dict(case, B=B, q=q, ctx=ctx, rot=rng.choice([hd, hd, hd // 2, 0]), interleaved=rng.random() < 0.5, norm=rng.random() < 0.7)


def _part(i, step):
    return (i + 1) * step % 1.0


def _rows(case):
    """New rows of every sequence; ragged batches mix chunks of up to q rows with single rows."""
    if not case["ragged"]:
        return [case["q"]] * case["B"]
    return [1 if i % 3 == 1 else max(1, round(case["q"] * (0.3 + 0.7 * _part(i, 0.618)))) for i in range(case["B"])]


def _lengths(case):
    """Cached positions of every sequence, its new rows included: between a quarter of ctx and ctx (all of it for one sequence)."""
    if case["B"] == 1:
        return [max(case["ctx"], _rows(case)[0])]
    return [max(n, round(case["ctx"] * (0.25 + 0.75 * _part(i, 0.7549)))) for i, n in enumerate(_rows(case))]


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * seed + 29)
    return _prepare_logits(case, g) if case["kind"] == "truncate" else _prepare_paged(case, g)


def _power(e):
    """2^e for whole numbers, in 64 bits: put together from its bits, since a power function may be a last place off."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _codes(y, dtype):
    """Heads [.., hd] in 64 bits -> (the e4m3 numbers, exponents of their scales)."""
    top = y.abs().amax(dim=-1, keepdim=True)
    m, x = torch.frexp(top)  # top = m 2^x, m from 0.5 up to 1; 448 = 0.875 * 2^9
    e = (x - 9 + (m > 0.875)).clamp_(min=LEAST[dtype])
    e = torch.where(top > 0, e, LEAST[dtype])
    z = y.clamp(-MOST[dtype], MOST[dtype]) * _power(-e)
    step = _power((torch.frexp(z)[1] - 4).clamp_(min=-9))
    return torch.round(z / step) * step, e.squeeze(-1)


def _prepare_paged(case, g):
    td, hd, S = TORCH_DTYPE[case["dtype"]], case["hd"], case["page"]
    rows, lens = _rows(case), _lengths(case)
    per = [(n + S - 1) // S for n in lens]
    n_pages = sum(per) + 3

    def N(*shape):
        return torch.empty(shape, dtype=td, device=DEV).normal_(0.0, 1.0, generator=g)

    # pages of the sequences lie anywhere in the pool, as after some time of serving; what they hold behind a sequence's end is an
    # earlier sequence's
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["B"], max(per) + 2), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    T = sum(rows)
    st = dict(case=case, T=T, rows=rows, lens=lens, q_max=max(rows), len_max=max(lens), table=table,
              length=torch.tensor(lens, dtype=torch.int32, device=DEV),
              row_start=torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device=DEV) if case["ragged"] else None)
    # which sequence and position a row is, for the plain form
    st["seq"] = torch.repeat_interleave(torch.arange(case["B"]), torch.tensor(rows)).to(DEV)
    st["pos"] = torch.cat([torch.arange(n - r, n) for r, n in zip(rows, lens)]).to(DEV)
    st["in_seq"] = torch.cat([torch.arange(r) for r in rows]).to(DEV)
    # some elements of a head are larger than others throughout, keys' more than values'
    loud = torch.exp(0.7 * torch.randn(hd, generator=g, device=DEV)).to(td)
    if case["kind"] == "normed":
        st["k_pages"], st["v_pages"] = N(n_pages, S, case["kv_heads"], hd), N(n_pages, S, case["kv_heads"], hd)
    else:
        for name, by in (("k", loud), ("v", None)):
            x = N(n_pages, S, case["kv_heads"], hd)
            num, e = _codes((x if by is None else x * by).double(), case["dtype"])
            st[name + "_pages"] = num.float().to(torch.float8_e4m3fn)
            st[name + "_scale"] = (e + 127).to(torch.uint8).transpose(1, 2).contiguous()  # [n_pages][kv_heads][page]
    if case["kind"] in ("normed", "append8"):
        # q, k and v as one product leaves them, side by side
        qkv = N(T, case["heads"] + 2 * case["kv_heads"], hd)
        qkv[:, :case["heads"] + case["kv_heads"]] *= loud
        st["q"], st["k"], st["v"] = qkv.split([case["heads"], case["kv_heads"], case["kv_heads"]], dim=1)
        half = case["rot"] // 2
        st["inv_freq"] = THETA ** (-torch.arange(half, dtype=torch.float64) / half).to(DEV) if half else None
        st["q_norm"] = 1 + 0.2 * N(hd) if case["norm"] else None
        st["k_norm"] = 1 + 0.2 * N(hd) if case["norm"] else None
        st["q_out"] = torch.empty((T, case["heads"], hd), dtype=td, device=DEV)
    elif case["kind"] == "read8":
        st["k_out"] = torch.empty((T, case["kv_heads"], hd), dtype=td, device=DEV)
        st["v_out"] = torch.empty_like(st["k_out"])
    else:
        st["q"] = N(T, case["heads"], hd)
        st["out"] = torch.empty_like(st["q"])
    return st


def _prepare_logits(case, g):
    B, q, V = case["B"], case["s"] + 1, case["vocab"]

    def of(values, dtype):  # a sequence's wish, one of the values
        pick = torch.randint(0, len(values), (B,), generator=g, device=DEV)
        return torch.tensor(values, dtype=dtype, device=DEV)[pick]

    # rows from flat ones to such as know their token
    z = torch.randn((B, q, V), generator=g, device=DEV) * (1.5 + 2 * torch.rand((B, q, 1), generator=g, device=DEV))
    z += 4 * (torch.rand((B, q, V), generator=g, device=DEV) < 20.0 / V)
    return dict(case=case, logits=z.to(TORCH_DTYPE[case["dtype"]]), uniforms=torch.rand((B, q), generator=g, device=DEV),
                temperature=of([0.0, 0.6, 0.7, 0.8, 1.0, 1.0, 1.2], torch.float32), top_k=of([0, 0, 20, 50, 50, 1000], torch.int32),
                top_p=of([1.0, 0.8, 0.9, 0.95, 0.99], torch.float32), min_p=of([0.0, 0.0, 0.02, 0.1], torch.float32),
                out=torch.empty((B, q, V), dtype=torch.float32, device=DEV), tokens=torch.empty((B, q), dtype=torch.int32, device=DEV))


# ---------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"normed": _own_normed, "append8": _own_append8, "read8": _own_read8, "attend8": _own_attend8, "truncate": _own_truncate}[kind](state)
    return {"normed": _plain_normed, "append8": _plain_append8, "read8": _plain_read8, "attend8": _plain_attend8, "truncate": _plain_truncate}[kind](state)


def _plan(st):
    """The cache, the batch, the rules and the workspace that a program keeps between its calls."""
    from paper_2310_18813_amd import binding as B
    if "plan" not in st:
        case = st["case"]
        if case["kind"] == "truncate":
            rules = B.SamplingRules(temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
            n = B.spec_truncate_logits_workspace_bytes(case["B"], case["s"], case["vocab"])
            st["plan"] = (rules, torch.empty(n, dtype=torch.uint8, device=DEV))
        else:
            if case["kind"] == "normed":
                cache = B.PagedCache(st["k_pages"], st["v_pages"])
            else:
                cache = B.PagedCache8(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], TORCH_DTYPE[case["dtype"]])
            batch = B.PagedBatch(st["table"], st["length"], st["T"], row_start=st["row_start"], max_rows=st["q_max"], max_len=st["len_max"])
            more = None
            if case["kind"] == "attend8":
                more = torch.empty(B.spec_paged8_attention_workspace_bytes(cache, batch, case["heads"]), dtype=torch.uint8, device=DEV)
            elif case["kind"] != "read8":
                more = B.HeadTransform(inv_freq=st["inv_freq"], interleaved=case["interleaved"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS)
            st["plan"] = (cache, batch, more)
    return B, st["plan"]


def _own_normed(st):
    B, (cache, batch, heads) = _plan(st)
    B.spec_paged_append_normed(cache, batch, st["q"], st["k"], st["v"], heads, out=st["q_out"])
    return {"q": st["q_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _own_append8(st):
    B, (cache, batch, heads) = _plan(st)
    B.spec_paged8_append(cache, batch, st["q"], st["k"], st["v"], heads, out=st["q_out"])
    return _written8(st, st["q_out"])


def _own_read8(st):
    B, (cache, batch, _) = _plan(st)
    k, v = B.spec_paged8_read(cache, batch, k=st["k_out"], v=st["v_out"])
    return {"k": k, "v": v}


def _own_attend8(st):
    B, (cache, batch, space) = _plan(st)
    return {"out": B.spec_paged8_attention(cache, batch, st["q"], window=st["case"]["window"], out=st["out"], workspace=space)}


def _own_truncate(st):
    B, (rules, space) = _plan(st)
    out, tokens = B.spec_truncate_logits(st["logits"], rules, uniforms=st["uniforms"], out=st["out"], tokens=st["tokens"], workspace=space)
    return {"logits": out, "tokens": tokens}


def _written8(st, q):
    """The pages as e4m3 numbers and the exponents of their scales, which together are what the cache stands for."""
    return {"q": q, "k_pages": st["k_pages"], "v_pages": st["v_pages"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _transformed(st, x, weight, bits):
    """Heads normed and turned, in `bits` and not rounded."""
    case = st["case"]
    y = x.to(bits)
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + EPS) * weight.to(bits)
    R = case["rot"]
    if not R:
        return y
    angle = st["pos"].double()[:, None] * st["inv_freq"]
    cos, sin = torch.cos(angle).to(bits)[:, None, :], torch.sin(angle).to(bits)[:, None, :]
    turned, rest = y[..., :R], y[..., R:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if case["interleaved"] else (turned[..., :R // 2], turned[..., R // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([a, b], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _plain_normed(st):
    td, S = TORCH_DTYPE[st["case"]["dtype"]], st["case"]["page"]
    page, at = st["table"][st["seq"], st["pos"] // S].long(), st["pos"] % S
    st["k_pages"][page, at] = _transformed(st, st["k"], st["k_norm"], torch.float32).to(td)
    st["v_pages"][page, at] = st["v"]
    return {"q": _transformed(st, st["q"], st["q_norm"], torch.float32).to(td), "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_append8(st):
    case = st["case"]
    td, S = TORCH_DTYPE[case["dtype"]], case["page"]
    page, at = st["table"][st["seq"], st["pos"] // S].long(), st["pos"] % S

    def put(name, y):
        num, e = _codes(y, case["dtype"])
        st[name + "_pages"].view(torch.uint8)[page, at] = num.float().to(torch.float8_e4m3fn).view(torch.uint8)
        st[name + "_scale"][page, :, at] = (e + 127).to(torch.uint8)

    put("k", _transformed(st, st["k"], st["k_norm"], torch.float64))
    put("v", st["v"].double())
    return _written8(st, _transformed(st, st["q"], st["q_norm"], torch.float32).to(td))


def _numbers8(st, name, page, at):
    """What the cache stands for at pages and places, [..][kv_heads][hd], in 32 bits."""
    scale = _power(st[name + "_scale"][page, :, at].int() - 127).float()
    return st[name + "_pages"].view(torch.uint8)[page, at].view(torch.float8_e4m3fn).float() * scale[..., None]


def _plain_read8(st):
    td, S = TORCH_DTYPE[st["case"]["dtype"]], st["case"]["page"]
    page, at = st["table"][st["seq"], st["pos"] // S].long(), st["pos"] % S
    return {"k": _numbers8(st, "k", page, at).to(td), "v": _numbers8(st, "v", page, at).to(td)}


def _plain_attend8(st):
    """All sequences at once, padded to the longest; rows of a group of query heads share their key head's product."""
    case = st["case"]
    B, Hk, hd, S, Q = case["B"], case["kv_heads"], case["hd"], case["page"], st["q_max"]
    G = case["heads"] // Hk
    n = (st["len_max"] + S - 1) // S
    L = n * S
    key = torch.arange(L, device=DEV)
    live = key < st["length"][:, None]                                                          # [B][L]
    pages = st["table"][:, :n].long().clamp(min=0)

    def cached(name):  # [B][Hk][L][hd]
        x = st[name + "_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).view(B, L, Hk, hd).float()
        scale = _power(st[name + "_scale"][pages].transpose(2, 3).reshape(B, L, Hk, 1).int() - 127).float()
        return torch.where(live[:, :, None, None], x * scale, 0.0).permute(0, 2, 1, 3).contiguous()

    q = torch.zeros((B, Q, case["heads"], hd), device=DEV)
    q[st["seq"], st["in_seq"]] = st["q"].float()
    q = q.view(B, Q, Hk, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Q, hd) * (1.0 / math.sqrt(hd))
    pos = torch.full((B, Q), -1, device=DEV)
    pos[st["seq"], st["in_seq"]] = st["pos"]
    see = (key <= pos[:, :, None]) & live[:, None, :]
    if case["window"]:
        see &= key > pos[:, :, None] - case["window"]
    scores = torch.matmul(q, cached("k").transpose(2, 3).contiguous()).view(B, Hk, G, Q, L)
    scores.masked_fill_(~see[:, None, None], -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = scores.sum(dim=-1, keepdim=True)
    o = torch.matmul(scores.view(B, Hk, G * Q, L), cached("v")).view(B, Hk, G, Q, hd) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, Q, case["heads"], hd)
    return {"out": o[st["seq"], st["in_seq"]].to(st["q"].dtype)}


def _plain_truncate(st):
    V = st["case"]["vocab"]
    z, ids = torch.sort(st["logits"].float(), dim=-1, descending=True, stable=True)
    T, k, p, floor = (st[x][:, None, None] for x in ("temperature", "top_k", "top_p", "min_p"))
    x = (z.double() - z[..., :1]) / T.double()
    w = torch.exp(x)
    rank = torch.arange(V, device=DEV)
    keep = (rank < k) | (k <= 0)
    mass = torch.where(keep, w, 0.0).cumsum(dim=-1)
    before = torch.cat([torch.zeros_like(mass[..., :1]), mass[..., :-1]], dim=-1)
    keep = keep & ((before < p.double() * mass[..., -1:]) | (p >= 1))
    keep = keep & ((w >= floor.double()) | (rank == 0))
    keep = torch.where(T > 0, keep, rank == 0)
    w = torch.where(keep, torch.where(T > 0, w, 1.0), 0.0)
    out = torch.where(keep, torch.where(T > 0, x, 0.0), -math.inf).float()
    out, w = torch.empty_like(out).scatter_(-1, ids, out), torch.empty_like(w).scatter_(-1, ids, w)
    total = w.cumsum(dim=-1)
    token = (total <= st["uniforms"].double()[..., None] * total[..., -1:]).sum(dim=-1)
    return {"logits": out, "tokens": token.to(torch.int32)}


# ---------------------------------------------------------------- what a pass cannot do without
def _attended(case):
    """(pairs of a row and a position that it sees, positions that any row of their sequence sees), over all sequences."""
    pairs = keys = 0
    w = case["window"] or math.inf
    for n, kv in zip(_rows(case), _lengths(case)):
        pos = np.arange(kv - n, kv)
        pairs += int(np.minimum(pos + 1, w).sum())
        keys += int(min(kv, n - 1 + w))
    return pairs, keys


def work(case):
    e = BYTES[case["dtype"]]
    if case["kind"] == "truncate":
        rows = case["B"] * (case["s"] + 1)
        return {"bytes": rows * case["vocab"] * (e + 4) + 8 * rows + 16 * case["B"], "flops": 8 * rows * case["vocab"]}
    rows, Hq, Hk, hd = sum(_rows(case)), case["heads"], case["kv_heads"], case["hd"]
    if case["kind"] == "attend8":
        pairs, keys = _attended(case)
        return {"bytes": 2 * keys * Hk * (hd + 1) + 2 * rows * Hq * hd * e, "flops": 4 * pairs * Hq * hd}
    if case["kind"] == "read8":
        return {"bytes": 2 * rows * Hk * (hd + 1 + hd * e), "flops": 2 * rows * Hk * hd}
    flops = rows * (Hq + Hk) * (3 * case["rot"] + (4 * hd if case["norm"] else 0))
    if case["kind"] == "append8":
        return {"bytes": rows * (2 * Hq * hd * e + 2 * Hk * (hd * e + hd + 1)), "flops": flops + 4 * rows * Hk * hd}
    return {"bytes": 2 * rows * (Hq + 2 * Hk) * hd * e, "flops": flops}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"normed": _exact_append, "append8": _exact_append, "read8": _exact_read8, "attend8": _exact_attend8, "truncate": _exact_truncate}[case["kind"]](case, st)


def _exact_heads(case, x, weight, positions):
    """Heads [n][h][hd] normed and turned: a turn is a product of complex numbers."""
    x, R = x.double(), case["rot"]
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["hd"] + EPS) * weight.double()
    if not R:
        return x
    freq = torch.tensor([THETA ** (-2.0 * i / R) for i in range(R // 2)], dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones((len(positions), R // 2), dtype=torch.float64, device=DEV), positions.double()[:, None] * freq)[:, None]
    if case["interleaved"]:
        z = torch.view_as_complex(x[..., :R].reshape(*x.shape[:2], R // 2, 2).contiguous()) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), x[..., R:]], dim=-1)
    z = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous()) * turn
    return torch.cat([z.real, z.imag, x[..., R:]], dim=-1)


def _exact_codes(y, dtype):
    """The nearest e4m3 number of every element, found in the table of all of them."""
    numbers = torch.tensor(sorted(m * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in ((8 if e else 0) + i for i in range(8)) if (e, m) != (15, 15)),
                           dtype=torch.float64, device=DEV)
    low = y.abs().amax(-1).clamp(min=TOP * 2.0 ** LEAST[dtype])
    e = torch.ceil(torch.log2(low / TOP))
    e = torch.where(low > TOP * _power(e), e + 1, torch.where(low <= TOP * _power(e - 1), e - 1, e))
    x = (y.abs().clamp(max=MOST[dtype]) / _power(e)[..., None]).clamp(max=TOP)
    at = torch.searchsorted(numbers, x).clamp(min=1)
    down, up = numbers[at - 1], numbers[at]
    near = torch.where((x - down == up - x), torch.where((at - 1) % 2 == 0, down, up), torch.where(x - down < up - x, down, up))
    return near * torch.sign(y), e


def _exact_append(case, st):
    S, eight = case["page"], case["kind"] == "append8"
    out = {n: st[n].double() for n in ("k_pages", "v_pages")}
    if eight:
        out |= {n: st[n].clone() for n in ("k_scale", "v_scale")}
    q_out = st["q"].double()
    table = st["table"].tolist()
    row = 0
    for b, (n, kv) in enumerate(zip(st["rows"], st["lens"])):
        p = torch.arange(kv - n, kv, device=DEV)
        q_out[row:row + n] = _exact_heads(case, st["q"][row:row + n], st["q_norm"], p)
        k, v = _exact_heads(case, st["k"][row:row + n], st["k_norm"], p), st["v"][row:row + n].double()
        for name, y in (("k", k), ("v", v)):
            if eight:
                y, e = _exact_codes(y, case["dtype"])
            for first in range((kv - n) // S * S, kv, S):  # page by page
                lo, hi = max(first, kv - n), min(first + S, kv)
                page = table[b][first // S]
                out[name + "_pages"][page, lo - first:hi - first] = y[lo - (kv - n):hi - (kv - n)]
                if eight:
                    out[name + "_scale"][page, :, lo - first:hi - first] = (e[lo - (kv - n):hi - (kv - n)] + 127).to(torch.uint8).t()
        row += n
    return {"q": q_out, **out}


def _exact_sequence(st, name, b, lo, hi):
    """Positions lo .. hi - 1 of a sequence, [n][kv_heads][hd]."""
    S = st["case"]["page"]
    pages = st["table"][b, :(hi + S - 1) // S].long()
    x = st[name + "_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).float().double()
    scale = _power(st[name + "_scale"][pages].int() - 127)
    return (x * scale.transpose(1, 2)[..., None]).flatten(0, 1)[lo:hi]


def _exact_read8(case, st):
    at = list(enumerate(zip(st["rows"], st["lens"])))
    return {name: torch.cat([_exact_sequence(st, name, b, kv - n, kv) for b, (n, kv) in at]) for name in ("k", "v")}


def _exact_attend8(case, st):
    hd, G = case["hd"], case["heads"] // case["kv_heads"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for b, (n, kv) in enumerate(zip(st["rows"], st["lens"])):
        k, v = _exact_sequence(st, "k", b, 0, kv), _exact_sequence(st, "v", b, 0, kv)
        ahead = torch.arange(kv, device=DEV) - torch.arange(kv - n, kv, device=DEV)[:, None]
        hidden = (ahead > 0) | (ahead <= -case["window"]) if case["window"] else ahead > 0
        for h in range(case["heads"]):
            x = st["q"][row:row + n, h].double() @ k[:, h // G].t() / hd ** 0.5
            x[hidden] = -math.inf
            out[row:row + n, h] = torch.softmax(x, dim=-1) @ v[:, h // G]
        row += n
    return {"out": out}


def _exact_truncate(case, st):
    logits, out = st["logits"].double().cpu().numpy(), np.full((case["B"], case["s"] + 1, case["vocab"]), -np.inf)
    tokens = np.zeros((case["B"], case["s"] + 1), dtype=np.int32)
    u, T, k, p, floor = (st[x].double().cpu().numpy() for x in ("uniforms", "temperature", "top_k", "top_p", "min_p"))
    for b in range(case["B"]):
        for j in range(case["s"] + 1):
            z = logits[b, j]
            order = np.argsort(-z, kind="stable")
            n, x = 1, np.zeros_like(z)
            if T[b] > 0:
                x = (z - z.max()) / T[b]
                w = np.exp(x[order])
                n = int(k[b]) if 0 < k[b] < len(z) else len(z)
                if p[b] < 1:
                    mass = np.cumsum(w[:n])
                    n = 1 + int(np.count_nonzero(mass < p[b] * mass[-1]))
                n = max(1, min(n, int(np.count_nonzero(w >= floor[b]))))
            kept = np.sort(order[:n])
            out[b, j, kept] = x[kept]
            c = np.cumsum(np.exp(x[kept]))
            tokens[b, j] = kept[min(n - 1, int(np.searchsorted(c, u[b, j] * c[-1], side="right")))]
    return {"logits": torch.from_numpy(out), "tokens": torch.from_numpy(tokens)}
