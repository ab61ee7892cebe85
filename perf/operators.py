"""The operators for a caller that runs the target model itself, as cases that can be timed and whose outputs can be compared.

Such a caller verifies the s + 1 rows of every sequence over a paged cache: it appends the rows' keys and values with the position
rotation (`spec_paged_append`), attends over the pages (`spec_paged_attention`), and applies penalties, biases and a grammar's mask
to the logits (`spec_process_logits`) before the acceptance rules.

With `own` false, `run` computes the operators in elementary torch operations, in 32 bits and rounded once at the end; with `own` true
it makes the calls of `paper_2310_18813_amd.binding`.  `exact` is the definition in 64 bits, sequence by sequence.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TORCH_DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
THETA = 10000.0


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one user of the 7B width, plain decoding: one row into the cache, all latency
        dict(name="append_7b_b1", kind="append", dtype="bf16", B=1, q=1, ragged=False, ctx=230, heads=32, kv_heads=32, hd=128, page=16, rot=128),
        # a verification of 64 sequences, four rows each, grouped heads
        dict(name="append_gqa_b64", kind="append", dtype="bf16", B=64, q=4, ragged=False, ctx=448, heads=32, kv_heads=8, hd=128, page=16, rot=128),
        # the start of a batch at the 33B width: prompts of different lengths, about 8000 rows
        dict(name="append_33b_prompts", kind="append", dtype="fp16", B=5, q=2011, ragged=True, ctx=2011, heads=52, kv_heads=52, hd=128, page=64,
             rot=128),
        # a draft model's step for one user: one row, heads of 64, all latency
        dict(name="attend_draft_b1", kind="attend", dtype="fp16", B=1, q=1, ragged=False, ctx=500, heads=12, kv_heads=12, hd=64, page=16, window=0),
        # a small model served in fp32, eight sequences
        dict(name="attend_fp32_b8", kind="attend", dtype="fp32", B=8, q=5, ragged=False, ctx=200, heads=16, kv_heads=16, hd=64, page=16, window=0),
        # the headline workload's verification: 64 sequences, s = 3, a key head for every query head
        dict(name="attend_7b_b64", kind="attend", dtype="bf16", B=64, q=4, ragged=False, ctx=1000, heads=32, kv_heads=32, hd=128, page=16, window=0),
        # a few users with long contexts and grouped heads, s = 7
        dict(name="attend_gqa_long", kind="attend", dtype="bf16", B=6, q=8, ragged=False, ctx=32000, heads=32, kv_heads=8, hd=128, page=64, window=0),
        # chunks of long prompts that join a running batch: some sequences bring a chunk, some a few rows, over what is cached already
        dict(name="attend_chunks", kind="attend", dtype="bf16", B=6, q=2048, ragged=True, ctx=8192, heads=32, kv_heads=8, hd=128, page=64, window=0),
        # the same with a sliding window, heads of 64 in fp16
        dict(name="attend_window", kind="attend", dtype="fp16", B=9, q=777, ragged=True, ctx=6000, heads=16, kv_heads=4, hd=64, page=32, window=1024),
        # one row of logits of one user with a short history, all rules
        dict(name="logits_b1", kind="logits", dtype="fp32", B=1, s=0, vocab=32000, history=500, n_bias=8, allowed=0.9, mask_rows=1),
        # the logits of 64 verified sequences, as a 16-bit head leaves them
        dict(name="logits_b64", kind="logits", dtype="bf16", B=64, s=3, vocab=50272, history=1000, n_bias=32, allowed=0.3, mask_rows=4),
        # a large vocabulary, long histories, no mask
        dict(name="logits_long", kind="logits", dtype="fp32", B=24, s=7, vocab=151936, history=16000, n_bias=0, allowed=1.0, mask_rows=0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "logits"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind == "logits":
        vocab = rng.choice([32000, 50272, 151936, rng.randint(1000, 160000)])
        s = rng.randint(0, 8)
        mask_rows = rng.choice([0, 1, s + 1])
        B = _log_int(rng, 1, max(1, 24_000_000 // (vocab * (s + 1))))
        return dict(kind=kind, dtype=dtype, B=min(B, 128), s=s, vocab=vocab, history=_log_int(rng, 10, 16000), n_bias=rng.choice([0, rng.randint(1, 300)]),
                    allowed=rng.choice([0.02, 0.5, 0.95]) if mask_rows else 1.0, mask_rows=mask_rows)
    hd = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    heads = kv_heads * rng.choice([g for g in (1, 2, 3, 4, 8, 16) if kv_heads * g <= 52])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    ragged = rng.random() < 0.4
    q = _log_int(rng, 16, 2048) if ragged else rng.randint(1, 9)
    if kind == "append":
        B = _log_int(rng, 1, max(1, min(64, 8000 // q)))
        ctx = max(q, _log_int(rng, 16, max(16, 60000 // (B * kv_heads))))
        return dict(kind=kind, dtype=dtype, B=B, q=q, ragged=ragged, ctx=ctx, heads=heads, kv_heads=kv_heads, hd=hd, page=page,
                    rot=rng.choice([hd, hd, hd // 2]))
    if dtype == "fp32":
        q = min(q, 64)
    B = _log_int(rng, 1, max(1, min(64, 4000 // q)))
    ctx = max(q, _log_int(rng, 16, max(16, (400_000 if ragged else 1_200_000) // (B * kv_heads))))
    return dict(kind=kind, dtype=dtype, B=B, q=q, ragged=ragged, ctx=min(ctx, max(q, 8000 if ragged else 32000)), heads=heads, kv_heads=kv_heads, hd=hd,
                page=page, window=rng.choice([0, 0, rng.randint(1, 2000)]))


def _part(i, step):
    return (i + 1) * step % 1.0


def _rows(case):
    """New rows of every sequence; ragged batches mix chunks of up to q rows with single rows."""
    if not case["ragged"]:
        return [case["q"]] * case["B"]
    return [1 if i % 3 == 1 else max(1, round(case["q"] * (0.3 + 0.7 * _part(i, 0.618)))) for i in range(case["B"])]


def _lengths(case):
    """Cached positions of every sequence, its new rows included: between a quarter of ctx and ctx."""
    return [max(n, round(case["ctx"] * (0.25 + 0.75 * _part(i, 0.7549)))) for i, n in enumerate(_rows(case))]


def _histories(case):
    """(prompt length, length) of every sequence's tokens."""
    lens = [max(1, round(case["history"] * (0.25 + 0.75 * _part(i, 0.7549)))) for i in range(case["B"])]
    return [(round(n * (0.2 + 0.6 * _part(i, 0.618))), n) for i, n in enumerate(lens)]


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * seed + 17)
    return _prepare_logits(case, g) if case["kind"] == "logits" else _prepare_paged(case, g)


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
              row_start=torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device=DEV) if case["ragged"] else None,
              k_pages=N(n_pages, S, case["kv_heads"], hd), v_pages=N(n_pages, S, case["kv_heads"], hd))
    # which sequence and position a row is, for the plain form
    st["seq"] = torch.repeat_interleave(torch.arange(case["B"]), torch.tensor(rows)).to(DEV)
    st["pos"] = torch.cat([torch.arange(n - r, n) for r, n in zip(rows, lens)]).to(DEV)
    st["in_seq"] = torch.cat([torch.arange(r) for r in rows]).to(DEV)
    if case["kind"] == "append":
        # q, k and v as one product leaves them, side by side
        qkv = N(T, case["heads"] + 2 * case["kv_heads"], hd)
        st["q"], st["k"], st["v"] = qkv.split([case["heads"], case["kv_heads"], case["kv_heads"]], dim=1)
        half = case["rot"] // 2
        st["inv_freq"] = THETA ** (-torch.arange(half, dtype=torch.float64) / half).to(DEV)
        st["q_out"] = torch.empty((T, case["heads"], hd), dtype=td, device=DEV)
    else:
        st["q"] = N(T, case["heads"], hd)
        st["out"] = torch.empty_like(st["q"])
    return st


def _prepare_logits(case, g):
    B, q, V = case["B"], case["s"] + 1, case["vocab"]
    hist = _histories(case)
    L = max(n for _, n in hist)

    def tokens(*shape):  # some tokens come often
        return (torch.rand(shape, generator=g, device=DEV).pow(3) * V).to(torch.int32).clamp_(max=V - 1)

    def uniform(lo, hi):
        return torch.rand(B, generator=g, device=DEV) * (hi - lo) + lo

    st = dict(case=case, logits=(torch.randn((B, q, V), generator=g, device=DEV) * 3).to(TORCH_DTYPE[case["dtype"]]), tokens=tokens(B, L),
              prompt_len=torch.tensor([p for p, _ in hist], dtype=torch.int32, device=DEV),
              length=torch.tensor([n for _, n in hist], dtype=torch.int32, device=DEV),
              proposals=tokens(B, case["s"]) if case["s"] else None, repetition=uniform(1.0, 1.3), frequency=uniform(0.0, 0.5),
              presence=uniform(0.0, 0.5), bias_ids=None, bias=None, mask=None, out=torch.empty((B, q, V), dtype=torch.float32, device=DEV))
    if case["n_bias"]:
        st["bias_ids"] = torch.rand((B, V), generator=g, device=DEV).argsort(dim=1)[:, :case["n_bias"]].to(torch.int32).contiguous()
        st["bias"] = torch.randn((B, case["n_bias"]), generator=g, device=DEV) * 4
    if case["mask_rows"]:
        words = (V + 31) // 32
        bits = torch.rand((B, case["mask_rows"], words * 32), generator=g, device=DEV) < case["allowed"]
        shifts = torch.arange(32, device=DEV)
        st["mask"] = (bits.view(B, -1, words, 32).to(torch.int64) << shifts).sum(-1).to(torch.int32)
    return st


# ---------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own_logits(state) if kind == "logits" else _own_append(state) if kind == "append" else _own_attend(state)
    return _plain_logits(state) if kind == "logits" else _plain_append(state) if kind == "append" else _plain_attend(state)


def _plan(st):
    """The cache, the batch and the workspace that a program keeps between its calls."""
    from paper_2310_18813_amd import binding as B
    if "plan" not in st:
        case = st["case"]
        if case["kind"] == "logits":
            st["plan"] = B.LogitRules(tokens=st["tokens"], prompt_len=st["prompt_len"], length=st["length"], repetition=st["repetition"],
                                      frequency=st["frequency"], presence=st["presence"], bias_ids=st["bias_ids"], bias=st["bias"], mask=st["mask"])
        else:
            cache = B.PagedCache(st["k_pages"], st["v_pages"])
            batch = B.PagedBatch(st["table"], st["length"], st["T"], row_start=st["row_start"], max_rows=st["q_max"], max_len=st["len_max"])
            space = None
            if case["kind"] == "attend":
                space = torch.empty(B.spec_paged_attention_workspace_bytes(cache, batch, case["heads"]), dtype=torch.uint8, device=DEV)
            st["plan"] = (cache, batch, space)
    return B, st["plan"]


def _own_append(st):
    B, (cache, batch, _) = _plan(st)
    B.spec_paged_append(cache, batch, st["q"], st["k"], st["v"], st["inv_freq"], out=st["q_out"])
    return {"q": st["q_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _own_attend(st):
    B, (cache, batch, space) = _plan(st)
    return {"out": B.spec_paged_attention(cache, batch, st["q"], window=st["case"]["window"], out=st["out"], workspace=space)}


def _own_logits(st):
    B, rules = _plan(st)
    return {"logits": B.spec_process_logits(st["logits"], rules, st["proposals"], out=st["out"])}


def _rotate(x, cos, sin):
    half = cos.shape[-1]
    y = x.float()
    a, b = y[..., :half], y[..., half:2 * half]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., 2 * half:]], dim=-1).to(x.dtype)


def _plain_append(st):
    S = st["case"]["page"]
    angle = st["pos"].double()[:, None] * st["inv_freq"]
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    page = st["table"][st["seq"], st["pos"] // S].long()
    st["k_pages"][page, st["pos"] % S] = _rotate(st["k"], cos, sin)
    st["v_pages"][page, st["pos"] % S] = st["v"]
    return {"q": _rotate(st["q"], cos, sin), "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_attend(st):
    """All sequences at once, padded to the longest; rows of a group of query heads share their key head's product."""
    case = st["case"]
    B, Hk, hd, S, Q = case["B"], case["kv_heads"], case["hd"], case["page"], st["q_max"]
    G = case["heads"] // Hk
    n = (st["len_max"] + S - 1) // S
    L = n * S
    key = torch.arange(L, device=DEV)
    live = key < st["length"][:, None]                                                          # [B][L]

    def cached(pages):  # [B][Hk][L][hd]
        x = pages[st["table"][:, :n].long().clamp(min=0)].view(B, L, Hk, hd).float()
        return torch.where(live[:, :, None, None], x, 0.0).permute(0, 2, 1, 3).contiguous()

    q = torch.zeros((B, Q, case["heads"], hd), device=DEV)
    q[st["seq"], st["in_seq"]] = st["q"].float()
    q = q.view(B, Q, Hk, G, hd).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * Q, hd) * (1.0 / math.sqrt(hd))
    pos = torch.full((B, Q), -1, device=DEV)
    pos[st["seq"], st["in_seq"]] = st["pos"]
    see = (key <= pos[:, :, None]) & live[:, None, :]
    if case["window"]:
        see &= key > pos[:, :, None] - case["window"]
    scores = torch.matmul(q, cached(st["k_pages"]).transpose(2, 3).contiguous()).view(B, Hk, G, Q, L)
    scores.masked_fill_(~see[:, None, None], -math.inf)
    top = scores.amax(dim=-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = scores.sum(dim=-1, keepdim=True)
    o = torch.matmul(scores.view(B, Hk, G * Q, L), cached(st["v_pages"])).view(B, Hk, G, Q, hd) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, Q, case["heads"], hd)
    return {"out": o[st["seq"], st["in_seq"]].to(st["q"].dtype)}


def _plain_logits(st):
    case = st["case"]
    B, s, V = case["B"], case["s"], case["vocab"]
    at = torch.arange(st["tokens"].shape[1], device=DEV)
    emitted = ((at >= st["prompt_len"][:, None]) & (at < st["length"][:, None])).int()
    known = (at < st["length"][:, None]).int()
    ids = st["tokens"].long()
    zeros = torch.zeros((B, V), dtype=torch.int32, device=DEV)
    count = zeros.scatter_add(1, ids, emitted)[:, None].repeat(1, s + 1, 1)
    seen = zeros.scatter_add(1, ids, known)[:, None] > 0
    if s:  # row j also counts t_1 .. t_j
        before = torch.ones((s + 1, s), dtype=torch.int32, device=DEV).tril(-1)
        count.scatter_add_(2, st["proposals"].long()[:, None].expand(B, s + 1, s), before.expand(B, s + 1, s))
    z = st["logits"].float()
    r = st["repetition"][:, None, None]
    z = torch.where(seen | (count > 0), torch.where(z > 0, z / r, z * r), z)
    z = z - (st["frequency"][:, None, None] * count.float() + torch.where(count > 0, st["presence"][:, None, None], 0.0))
    if st["bias"] is not None:
        z = z + torch.zeros((B, V), device=DEV).scatter_add(1, st["bias_ids"].long(), st["bias"])[:, None]
    if st["mask"] is not None:
        bits = (st["mask"][..., None] >> torch.arange(32, device=DEV)) & 1
        z = torch.where(bits.view(B, case["mask_rows"], -1)[:, :, :V] != 0, z, -math.inf)
    return {"logits": z}


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
    if case["kind"] == "append":
        row = case["heads"] + 2 * case["kv_heads"]
        rows = sum(_rows(case))
        return {"bytes": 2 * rows * row * case["hd"] * e, "flops": 3 * rows * (case["heads"] + case["kv_heads"]) * case["rot"]}
    if case["kind"] == "attend":
        pairs, keys = _attended(case)
        return {"bytes": 2 * keys * case["kv_heads"] * case["hd"] * e + 2 * sum(_rows(case)) * case["heads"] * case["hd"] * e,
                "flops": 4 * pairs * case["heads"] * case["hd"]}
    rows = case["B"] * (case["s"] + 1)
    return {"bytes": rows * case["vocab"] * (e + 4) + case["B"] * case["mask_rows"] * ((case["vocab"] + 31) // 32) * 4
            + 4 * sum(n for _, n in _histories(case)) + 8 * case["B"] * case["n_bias"], "flops": 4 * rows * case["vocab"]}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(case, st)
    if case["kind"] == "attend":
        return _exact_attend(case, st)
    return _exact_logits(case, st)


def _exact_append(case, st):
    S, R = case["page"], case["rot"]
    k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
    q_out = st["q"].double()
    table = st["table"].tolist()
    freq = torch.tensor([THETA ** (-2.0 * i / R) for i in range(R // 2)], dtype=torch.float64, device=DEV)
    row = 0
    for b, (n, kv) in enumerate(zip(st["rows"], st["lens"])):
        p = torch.arange(kv - n, kv, device=DEV, dtype=torch.float64)
        turn = torch.polar(torch.ones((n, R // 2), dtype=torch.float64, device=DEV), p[:, None] * freq)[:, None]

        def turned(x):
            x = x.double()
            z = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous()) * turn
            return torch.cat([z.real, z.imag, x[..., R:]], dim=-1)

        q_out[row:row + n] = turned(st["q"][row:row + n])
        k, v = turned(st["k"][row:row + n]), st["v"][row:row + n].double()
        for first in range((kv - n) // S * S, kv, S):  # page by page
            lo, hi = max(first, kv - n), min(first + S, kv)
            page = table[b][first // S]
            k_pages[page, lo - first:hi - first] = k[lo - (kv - n):hi - (kv - n)]
            v_pages[page, lo - first:hi - first] = v[lo - (kv - n):hi - (kv - n)]
        row += n
    return {"q": q_out, "k_pages": k_pages, "v_pages": v_pages}


def _exact_attend(case, st):
    S, hd, G = case["page"], case["hd"], case["heads"] // case["kv_heads"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for b, (n, kv) in enumerate(zip(st["rows"], st["lens"])):
        pages = st["table"][b, :(kv + S - 1) // S].long()
        k = st["k_pages"][pages].flatten(0, 1)[:kv]
        v = st["v_pages"][pages].flatten(0, 1)[:kv]
        ahead = torch.arange(kv, device=DEV) - torch.arange(kv - n, kv, device=DEV)[:, None]
        hidden = (ahead > 0) | (ahead <= -case["window"]) if case["window"] else ahead > 0
        for h in range(case["heads"]):
            x = st["q"][row:row + n, h].double() @ k[:, h // G].double().t() / hd ** 0.5
            x[hidden] = -math.inf
            out[row:row + n, h] = torch.softmax(x, dim=-1) @ v[:, h // G].double()
        row += n
    return {"out": out}


def _exact_logits(case, st):
    V, s = case["vocab"], case["s"]
    z = st["logits"].double()
    for b, (p, n) in enumerate(_histories(case)):
        toks = st["tokens"][b].long()
        more = st["proposals"][b].long() if s else toks[:0]
        r, f, pr = (st[x][b].double() for x in ("repetition", "frequency", "presence"))
        for j in range(s + 1):
            c = torch.bincount(torch.cat([toks[p:n], more[:j]]), minlength=V).double()
            seen = (c > 0) | (torch.bincount(toks[:p], minlength=V) > 0)
            x = z[b, j]
            x = torch.where(seen, torch.where(x > 0, x / r, x * r), x) - f * c - pr * (c > 0)
            if st["bias"] is not None:
                x[st["bias_ids"][b].long()] += st["bias"][b].double()
            if st["mask"] is not None:
                words = st["mask"][b, j % case["mask_rows"]].long()
                token = torch.arange(V, device=DEV)
                x[(words[token // 32] >> (token % 32)) & 1 == 0] = -math.inf
            z[b, j] = x
    return {"logits": z}
