"""spec_process_logits against its rules in 64 bits, and spec_set_logit_rules inside a context against the oracle's logits under the same rules."""
import math

import numpy as np
import pytest
import torch

import helpers
import synth_inputs as si
from logit_reference import apply_rules, bits, ruled_greedy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(nB, s, V, L, n_bias, mask_rows, dtype, seed, pad=0):
    rng = np.random.default_rng(seed)
    c = dict(tokens=rng.integers(-2, V + 2, size=(nB, L)).astype(np.int32), length=rng.integers(0, L + 1, size=nB).astype(np.int32),
             proposals=rng.integers(0, V, size=(nB, s)).astype(np.int32), rep=rng.uniform(0.8, 1.6, nB).astype(np.float32),
             freq=rng.uniform(-0.5, 1, nB).astype(np.float32), pres=rng.uniform(-0.5, 1, nB).astype(np.float32),
             bias_ids=rng.integers(-1, V + 1, size=(nB, n_bias)).astype(np.int32), bias=rng.normal(0, 5, (nB, n_bias)).astype(np.float32),
             allowed=rng.random((nB, mask_rows, V)) < 0.5)
    c["length"][-1], c["prompt"] = L, (c["length"] * rng.random(nB)).astype(np.int32)
    if s:  # tokens that come again, among the proposals too
        c["proposals"][:, -1] = c["proposals"][:, 0]
        c["tokens"][:, L // 2:] = c["proposals"][:, :1]
    if n_bias:
        c["bias_ids"][:, -1] = c["bias_ids"][:, 0]
    if mask_rows:
        c["allowed"][0, 0] = False  # a row that allows nothing
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((nB, s + 1, V + pad), generator=g) * 3).to(dtype)
    x[0, 0, : min(4, V)] = torch.tensor([math.inf, -math.inf, math.nan, 0.0])[: min(4, V)].to(dtype)
    c["logits"] = x
    return c


CASES = [(1, 0, 1, 1, 1, 1), (2, 3, 37, 9, 2, 4), (3, 1, 1000, 100, 5, 1), (2, 15, 4099, 700, 300, 16), (1, 0, 32000, 500, 8, 1), (5, 8, 50272, 3000, 32, 9),
         (33, 3, 32000, 64, 0, 0), (40, 2, 151936, 5000, 3, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "B%d_s%d_V%d" % c[:3])
def test_rules_match_their_definition(case, dtype):
    from paper_2310_18813_amd import binding as B
    nB, s, V, L, n_bias, mask_rows = case
    pad = 0 if V % 4 else 4 * (V % 8 == 0)  # padded rows, 16-byte loads or single ones
    c = make(*case, dtype, seed=V + s, pad=pad)
    gpu = lambda a: torch.from_numpy(a).to(DEV)
    rules = B.LogitRules(tokens=gpu(c["tokens"]), prompt_len=gpu(c["prompt"]), length=gpu(c["length"]), repetition=gpu(c["rep"]),
                         frequency=gpu(c["freq"]), presence=gpu(c["pres"]), bias_ids=gpu(c["bias_ids"]) if n_bias else None,
                         bias=gpu(c["bias"]) if n_bias else None, mask=bits(c["allowed"]).to(DEV) if mask_rows else None)
    x = c["logits"].to(DEV)[:, :, :V]
    got = B.spec_process_logits(x, rules, gpu(c["proposals"]) if s else None).cpu().double().numpy()
    for b in sorted({0, 1 % nB, nB - 1}):
        for j in range(s + 1):
            allowed = c["allowed"][b, j % mask_rows] if mask_rows else np.ones(V, dtype=bool)
            with np.errstate(invalid="ignore"):
                want, err = apply_rules(c["logits"][b, j, :V].double().numpy(), j, c["tokens"][b, :c["length"][b]], c["prompt"][b], c["proposals"][b],
                                        *(float(c[k][b]) for k in ("rep", "freq", "pres")), c["bias_ids"][b], c["bias"][b].astype(np.float64), allowed)
                odd = ~np.isfinite(want)
                assert np.array_equal(got[b, j][odd], want[odd], equal_nan=True), (b, j)
                assert (np.abs(got[b, j] - want)[~odd] <= err[~odd]).all(), (b, j)


def test_each_rule_alone_and_in_place():
    from paper_2310_18813_amd import binding as B
    c = make(3, 2, 1000, 50, 4, 3, torch.float32, seed=2)
    gpu = lambda a: torch.from_numpy(a).to(DEV)
    one = dict(rep=1.0, freq=0.0, pres=0.0)
    seen = dict(tokens=gpu(c["tokens"]), prompt_len=gpu(c["prompt"]), length=gpu(c["length"]))
    for kw, use in ((dict(), set()), (dict(repetition=gpu(c["rep"]), **seen), {"rep"}), (dict(frequency=gpu(c["freq"]), **seen), {"freq"}),
                    (dict(presence=gpu(c["pres"]), **seen), {"pres"}), (dict(bias_ids=gpu(c["bias_ids"]), bias=gpu(c["bias"])), {"bias"}),
                    (dict(mask=bits(c["allowed"]).to(DEV)), {"mask"}), (dict(frequency=gpu(c["freq"])), {"proposals"})):
        x = c["logits"].to(DEV).clone()
        props = gpu(c["proposals"]) if use & {"rep", "freq", "pres", "proposals"} else None
        assert B.spec_process_logits(x, B.LogitRules(**kw), props, out=x) is x
        got = x.cpu().double().numpy()
        for b in range(3):
            for j in range(3):
                k = {n: float(c[n][b]) if n in use or n == "freq" and "proposals" in use else one[n] for n in one}
                toks = c["tokens"][b, :c["length"][b]] if "tokens" in kw else []
                with np.errstate(invalid="ignore"):
                    want, err = apply_rules(c["logits"][b, j].double().numpy(), j, toks, c["prompt"][b], c["proposals"][b] if props is not None else [],
                                            k["rep"], k["freq"], k["pres"], c["bias_ids"][b] if "bias" in use else [],
                                            c["bias"][b].astype(np.float64) if "bias" in use else [],
                                            c["allowed"][b, j] if "mask" in use else np.ones(1000, dtype=bool))
                    odd = ~np.isfinite(want)
                    assert np.array_equal(got[b, j][odd], want[odd], equal_nan=True) and (np.abs(got[b, j] - want)[~odd] <= err[~odd]).all(), (use, b, j)


def test_captured_call_follows_its_tensors():
    from paper_2310_18813_amd import binding as B
    c = make(4, 2, 5000, 60, 4, 1, torch.float32, seed=3)
    gpu = lambda a: torch.from_numpy(a).to(DEV)
    t = {k: gpu(c[k]) for k in ("tokens", "prompt", "length", "rep", "bias_ids", "bias", "proposals")}
    rules = B.LogitRules(tokens=t["tokens"], prompt_len=t["prompt"], length=t["length"], repetition=t["rep"], bias_ids=t["bias_ids"], bias=t["bias"],
                         mask=bits(c["allowed"]).to(DEV))
    x, out = c["logits"].to(DEV), torch.empty((4, 3, 5000), device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        B.spec_process_logits(x, rules, t["proposals"], out=out)
    for k in range(4):
        t["length"].fill_(15 * k)
        t["tokens"].add_(k)
        t["bias"].normal_()
        x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.spec_process_logits(x, rules, t["proposals"])), k


# ---------------------------------------------------------------- inside a context
def tiny(nB, s_max, P, N, mode, L_extra=4):
    from oracle import oracle as om
    from paper_2310_18813_amd import binding as B
    dtype, seed, tdesc, ddesc = si.CONFIGS["tiny_fp32"]
    orc = om.Oracle("f64")
    ot, od, wt, wd = helpers.build_pair(orc, tdesc, ddesc, dtype, seed, DEV)
    L = P + N + s_max + L_extra
    ctx = B.Context(tdesc, wt, ddesc, wd, dtype, nB, s_max, L, N, mode)
    return ot, ctx, si.make_prompts(nB, P, tdesc["vocab"], seed), tdesc["vocab"], L


@pytest.mark.parametrize("s", [0, 1, 4])
@pytest.mark.parametrize("draft", [False, True])
def test_rounds_of_a_context_follow_the_rules(s, draft):
    from paper_2310_18813_amd import binding as B
    nB, P, N = 3, 12, 20
    ot, ctx, prompts, V, L = tiny(nB, 4, P, N, B.PROPOSALS_DRAFT if draft else B.PROPOSALS_EXTERNAL)
    rng = np.random.default_rng(5)
    rep, freq, pres = np.array([1.0, 1.3, 1.1]), np.array([0.0, 0.02, 0.05]), np.array([0.0, 0.03, 0.0])
    ids, bias = rng.integers(0, V, size=(nB, 6)), rng.normal(0, 0.1, (nB, 6)).astype(np.float32)
    allowed = rng.random((nB, 1, V)) < 0.6
    ref, margins = zip(*(ruled_greedy(ot, prompts[b], N, float(np.float32(rep[b])), float(np.float32(freq[b])), float(np.float32(pres[b])), ids[b], bias[b],
                                      allowed[b, 0]) for b in range(nB)))
    assert min(margins) > 2 * helpers.LOGIT_TOL["fp32"]  # no decision that fp32 could take otherwise
    f32 = lambda a: torch.tensor(a, dtype=torch.float32, device=DEV)
    rules = B.LogitRules(repetition=f32(rep), frequency=f32(freq), presence=f32(pres), bias_ids=torch.tensor(ids, dtype=torch.int32, device=DEV),
                         bias=f32(bias), mask=bits(allowed).to(DEV))
    ctx.spec_set_logit_rules(rules)
    if not draft:  # three of four proposals are what the rules give
        ctx.spec_set_proposal_table(si.make_proposal_table(helpers.truth_table(np.array(ref), P, L), 0.75, V, 3))
    ctx.spec_reset(prompts)
    ctx.spec_round(s, N)
    out, hist = ctx.spec_read_output()
    assert out == [list(r) for r in ref]
    assert draft or s == 0 or sum(hist[1:]) > 0
    # without rules the context is what it was
    ctx.spec_set_logit_rules(None)
    ctx.spec_reset(prompts)
    ctx.spec_round(0, N)
    out, _ = ctx.spec_read_output()
    assert out[0] == [int(t) for t in ot.greedy(prompts[0], N)]


def test_sampling_in_a_context_takes_the_processed_logits():
    from paper_2310_18813_amd import binding as B
    nB, P, N, s = 4, 10, 8, 3
    _, ctx, prompts, V, L = tiny(nB, s, P, N, B.PROPOSALS_EXTERNAL)
    g = torch.Generator(device=DEV).manual_seed(1)
    u = torch.rand((nB, L, 3), generator=g, device=DEV)
    rng = np.random.default_rng(6)
    allowed = rng.random((nB, s + 1, V)) < 0.3
    rules = B.LogitRules(repetition=torch.full((nB,), 1.5, device=DEV), mask=bits(allowed).to(DEV))
    table = rng.integers(0, V, size=(nB, L)).astype(np.int32)
    ctx.spec_set_proposal_table(table)
    raw = None
    for on in (False, True):
        ctx.spec_set_logit_rules(rules if on else None)
        tl, _ = ctx.spec_set_sampling(0.7, u)
        ctx.spec_reset(prompts)
        ctx.spec_round(s, 1)
        if not on:
            raw = tl.clone().view(nB, s + 1, V)
    # the same rules on the raw logits, as a caller with its own model would apply them
    seq = torch.tensor(prompts, dtype=torch.int32, device=DEV)
    n = torch.full((nB,), P, dtype=torch.int32, device=DEV)
    props = torch.tensor(table[:, P:P + s].copy(), device=DEV)
    alone = B.LogitRules(tokens=seq, prompt_len=n, length=n, repetition=rules.tensors[3], mask=rules.tensors[8])
    want = B.spec_process_logits(raw, alone, props)
    assert torch.equal(tl.view(nB, s + 1, V), want)
    _, acc, emitted = B.spec_sample_accept(want, None, props, u[:, P:P + s + 1].contiguous(), 0.7)
    out, _ = ctx.spec_read_output()
    for b in range(nB):
        k = int(acc[b]) + 1
        assert out[b] == emitted[b, :k].tolist()
        assert all(allowed[b, j, t] for j, t in enumerate(out[b]))


def test_rules_of_a_context_are_refused_where_they_cannot_hold():
    from paper_2310_18813_amd import binding as B
    nB, s = 2, 2
    _, ctx, prompts, V, L = tiny(nB, s, 8, 8, B.PROPOSALS_EXTERNAL)
    toks = torch.zeros((nB, 4), dtype=torch.int32, device=DEV)
    n = torch.zeros(nB, dtype=torch.int32, device=DEV)
    with pytest.raises(B.SpecError) as e:
        ctx.spec_set_logit_rules(B.LogitRules(tokens=toks, length=n))
    assert e.value.code == B.ERR_INVALID_ARG and "the context's own" in str(e.value)
    words = (V + 31) // 32
    with pytest.raises(B.SpecError) as e:
        ctx.spec_set_logit_rules(B.LogitRules(mask=torch.zeros((nB, 2, words), dtype=torch.int32, device=DEV)))
    assert e.value.code == B.ERR_INVALID_ARG and "mask_rows" in str(e.value)
    rules = B.LogitRules(repetition=torch.ones(nB, device=DEV))
    rc = B.lib.spec_set_logit_rules(ctx.h, B.C.byref(rules.desc), None)
    assert rc == B.ERR_INVALID_ARG  # greedy rounds need the buffer
    u = torch.rand((nB, L, 3), device=DEV)
    ctx.spec_set_proposal_table(np.zeros((nB, L), dtype=np.int32))
    ctx.spec_set_sampling(1.0, u)
    assert B.lib.spec_set_logit_rules(ctx.h, B.C.byref(rules.desc), None) == B.OK
    ctx.spec_reset(prompts)
    ctx.spec_round(s, 1)
    ctx.spec_set_sampling(1.0, None)
    for call in (lambda: ctx.spec_round(s, 1), lambda: ctx.spec_verify_step(0)):
        with pytest.raises(B.SpecError) as e:
            call()
        assert e.value.code == B.ERR_STATE and "no buffer" in str(e.value)
    ctx.spec_set_logit_rules(None)
    ctx.spec_verify_step(0)
    with pytest.raises(B.SpecError) as e:
        ctx.spec_set_logit_rules(rules)
    assert e.value.code == B.ERR_STATE
    ctx.spec_accept_commit(0)
