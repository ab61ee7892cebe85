"""The rules on logits in 64 bits, row by row."""
import math

import numpy as np
import torch


def apply_rules(x, j, tokens, prompt, proposals, rep, freq, pres, bias_ids, bias, allowed):
    """One row in float64 -> (values, |error| bound of fp32 arithmetic: a product or quotient, a product and a sum of the penalties, two sums,
    2^-24 of their size each)."""
    V = x.shape[0]
    c = np.zeros(V)
    for t in list(tokens[prompt:]) + list(proposals[:j]):
        if 0 <= t < V:
            c[t] += 1
    seen = c > 0
    for t in tokens[:prompt]:
        if 0 <= t < V:
            seen[t] = True
    z1 = np.where(seen, np.where(x > 0, x / rep, x * rep), x)
    pen = freq * c + np.where(c > 0, pres, 0.0)
    add = np.zeros(V)
    for t, v in zip(bias_ids, bias):
        if 0 <= t < V:
            add[t] = v
    z = z1 - pen + add
    with np.errstate(invalid="ignore"):
        err = 2.0 ** -24 * (np.abs(z1) + 2 * np.abs(pen) + np.abs(z1 - pen) + np.abs(z)) * 1.01
    return np.where(allowed, z, -np.inf), err


def bits(allowed):
    """[..][V] truth values -> [..][ceil(V / 32)] int32"""
    V = allowed.shape[-1]
    pad = np.zeros(allowed.shape[:-1] + ((V + 31) // 32 * 32,), dtype=np.uint8)
    pad[..., :V] = allowed
    return torch.from_numpy(np.packbits(pad, axis=-1, bitorder="little").view(np.int32))


def ruled_greedy(ot, prompt, n, rep, freq, pres, ids, bias, allowed):
    """Greedy continuation under the rules from the oracle's logits in 64 bits, with the least margin of a decision."""
    seq, P, margin = [int(t) for t in prompt], len(prompt), math.inf
    for _ in range(n):
        lg = ot.forward(ot.cache(len(seq) + 1), seq, 0)[-1]
        z, _ = apply_rules(np.asarray(lg, dtype=np.float64), 0, seq, P, [], rep, freq, pres, ids, bias, allowed)
        top = np.sort(z)[-2:]
        margin = min(margin, top[1] - top[0])
        seq.append(int(z.argmax()))
    return seq[P:], margin
