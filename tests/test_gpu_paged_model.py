"""The operators together, as a caller that runs the target model itself uses them: a tiny LLaMA whose products are torch's, prefilled and verified
over a paged cache round by round, its logits under rules, its tokens by the greedy rule.  What comes out is the oracle's greedy continuation under the
same rules, and what a context of the library emits."""
import numpy as np
import pytest
import torch

import helpers
import synth_inputs as si
from logit_reference import bits, ruled_greedy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Caller:
    """fp32 LLaMA over pages of `page` positions that lie in random order in one pool a layer."""

    def __init__(self, B, desc, w, nB, L_max, page, seed):
        self.B, self.desc, self.w, self.page = B, desc, w, page
        self.H, self.hd = desc["n_heads"], desc["d_model"] // desc["n_heads"]
        per = (L_max + page - 1) // page
        g = torch.Generator().manual_seed(seed)
        self.table = torch.randperm(nB * per, generator=g).view(nB, per).to(torch.int32).to(DEV)
        pool = lambda: torch.full((nB * per, page, self.H, self.hd), float("nan"), device=DEV)
        self.caches = [B.PagedCache(pool(), pool()) for _ in range(desc["n_layers"])]
        self.wqkv = [torch.cat([L["wq"], L["wk"], L["wv"]]).t().contiguous() for L in w["layers"]]
        self.freq = B.spec_rope_frequencies(desc["rope_theta"], self.hd)

    def norm(self, x, gain):
        return x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + self.desc["norm_eps"]) * gain

    def forward(self, tokens, batch):
        B, d = self.B, self.desc["d_model"]
        x = self.w["tok_emb"][tokens.long()]
        T = x.shape[0]
        for L, wqkv, cache in zip(self.w["layers"], self.wqkv, self.caches):
            q, k, v = (self.norm(x, L["attn_norm_w"]) @ wqkv).view(T, 3 * self.H, self.hd).split(self.H, dim=1)
            q = B.spec_paged_append(cache, batch, q, k, v, self.freq, out=q)  # in place, in the product's own rows
            x = x + B.spec_paged_attention(cache, batch, q).view(T, d) @ L["wo"].t()
            h = self.norm(x, L["ffn_norm_w"])
            x = x + (torch.nn.functional.silu(h @ L["w1"].t()) * (h @ L["w3"].t())) @ L["w2"].t()
        return self.norm(x, self.w["final_norm_w"]) @ self.w["lm_head"].t()


@pytest.mark.parametrize("page,s,ruled", [(8, 0, True), (16, 3, True), (32, 5, False), (64, 5, True)])
def test_verification_rounds_over_pages_give_the_oracles_continuation(page, s, ruled):
    from oracle import oracle as om
    from paper_2310_18813_amd import binding as B
    dtype, seed, desc, _ = si.CONFIGS["tiny_fp32"]
    ot, _, w, _ = helpers.build_pair(om.Oracle("f64"), desc, None, dtype, seed, DEV)
    V, N, lens = desc["vocab"], 18, [5, 40, 1, 23]
    nB, L_max = len(lens), 40 + 18 + s + 2
    prompts = [[int(t) for t in p[:n]] for p, n in zip(si.make_prompts(nB, 40, V, seed), lens)]
    rng = np.random.default_rng(9)
    rep, freq, pres = (np.array(x, dtype=np.float32) for x in ([1.2, 1.0, 1.1, 1.3], [0.01, 0.03, 0.0, 0.02], [0.02, 0.0, 0.01, 0.0]))
    ids, bias = rng.integers(0, V, size=(nB, 5)).astype(np.int32), rng.normal(0, 0.1, (nB, 5)).astype(np.float32)
    allowed = rng.random((nB, 1, V)) < 0.7
    if ruled:
        ref, margins = zip(*(ruled_greedy(ot, prompts[b], N, *(float(x[b]) for x in (rep, freq, pres)), ids[b], bias[b], allowed[b, 0]) for b in range(nB)))
    else:
        ref, margins = zip(*(ruled_greedy(ot, prompts[b], N, 1.0, 0.0, 0.0, [], [], np.ones(V, dtype=bool)) for b in range(nB)))
    assert min(margins) > 2 * helpers.LOGIT_TOL["fp32"]
    # proposals by absolute position, three of four right
    truth = np.zeros((nB, L_max), dtype=np.int32)
    for b in range(nB):
        truth[b, lens[b]:lens[b] + N] = ref[b]
    table = si.make_proposal_table(truth, 0.75, V, seed)

    gpu = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    me = Caller(B, desc, w, nB, L_max, page, seed)
    seq = torch.zeros((nB, L_max), dtype=torch.int32, device=DEV)
    for b in range(nB):
        seq[b, :lens[b]] = torch.tensor(prompts[b], dtype=torch.int32)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    # all prompts but their last token in one ragged pass
    first = [m - 1 for m in lens]
    start = torch.tensor(np.concatenate([[0], np.cumsum(first)]), dtype=torch.int32, device=DEV)
    me.forward(torch.cat([seq[b, :first[b]] for b in range(nB)]), B.PagedBatch(me.table, n - 1, sum(first), row_start=start))
    rules = B.LogitRules(tokens=seq, prompt_len=n.clone(), length=n, repetition=gpu(rep), frequency=gpu(freq), presence=gpu(pres), bias_ids=gpu(ids),
                         bias=gpu(bias), mask=bits(allowed).to(DEV)) if ruled else B.LogitRules()
    length = n + s
    batch = B.PagedBatch(me.table, length, nB * (s + 1))
    out, accepted = [[] for _ in range(nB)], 0
    while min(len(o) for o in out) < N:
        nh = n.tolist()
        props = gpu(np.stack([table[b, nh[b]:nh[b] + s] for b in range(nB)])) if s else None
        rows = torch.stack([seq[b, nh[b] - 1] for b in range(nB)])[:, None]
        logits = me.forward(torch.cat([rows, props], dim=1).flatten() if s else rows.flatten(), batch).view(nB, s + 1, V)
        acc, emitted = B.spec_greedy_accept(B.spec_process_logits(logits, rules, props, out=logits), props)
        for b, l in enumerate(acc.tolist()):
            new = emitted[b, :l + 1].tolist()[:N - len(out[b])]  # a sequence that has all its tokens stands still
            seq[b, nh[b]:nh[b] + len(new)] = torch.tensor(new, dtype=torch.int32)
            n[b] += len(new)
            out[b] += new
            accepted += l
        length.copy_(n + s)
    assert out == [list(r) for r in ref]
    assert s == 0 or accepted > 0

    # a context of the library under the same rules
    ctx = B.Context(desc, w, None, None, dtype, nB, max(s, 1), L_max, N, B.PROPOSALS_EXTERNAL)
    if ruled:
        ctx.spec_set_logit_rules(B.LogitRules(repetition=gpu(rep), frequency=gpu(freq), presence=gpu(pres), bias_ids=gpu(ids), bias=gpu(bias),
                                              mask=bits(allowed).to(DEV)))
    ctx.spec_set_proposal_table(table)
    ctx.spec_reset_ragged(prompts)
    ctx.spec_round(s, N)
    assert ctx.spec_read_output()[0] == out
