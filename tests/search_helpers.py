"""Weights under which a token's logits hang on what attention reads, and how far two bf16 pipelines may be apart on them.

The generated matrices, N(0, 0.02), with wq and wk twice and wv and wo four times as large: attention's share of a hidden state is then as large as
the rest, where it is a few percent otherwise.  With its operands rounded to bf16 (norms, queries, keys, values, probabilities, attention outputs,
gated products) the oracle's logits move by up to 6.5e-3 of a row's largest on these shapes, with 8-bit pools by up to 2.1e-2 (a rounding in front may
move a key or value to the next code, 2^-3 away).  Two such pipelines are apart by twice that; half as much again is left for a larger
sample of rows."""
import dataclasses

import numpy as np
import torch

from harness import workload as W
from harness.runner import Stage
from oracle import ends_oracle as E
from oracle import stage_oracle as O
from stage_helpers import oracle_layers, oracle_shape

SCALES = {"wq": 2.0, "wk": 2.0, "wv": 4.0, "wo": 4.0}
LOGITS_TOL, LOGITS_TOL_8BIT = 2e-2, 6.3e-2
VOCAB = 512
# shape, lengths of the prompts, beams, new tokens, end token, scales of 8-bit pools
SEARCHES = [("tiny", [5], 4, 20, -1, None), ("tiny_gqa", [40, 16, 33], 3, 36, -1, None), ("tiny_gqa", [24, 7], 8, 18, 13, (0.05, 0.04)),
            ("tiny_h128", [64, 65], 5, 17, -1, None), ("tiny_mqa", [60], 2, 10, 7, None), ("tiny", [1, 2, 3], 1, 12, -1, None)]


class AttentiveStage(Stage):
    def load_weights(self, dtype=torch.bfloat16):
        super().load_weights(dtype)
        for l in range(self.shape.n_layers):
            for name, factor in SCALES.items():
                w = (W.weight(self.shape, self.layer_offset + l, name, device="cuda", dtype=dtype) * factor).contiguous()
                self.tdp.tdp_stage_set_weight(self.h, l, self.tdp.WEIGHT_IDS[name], w, self.tdp.BF16, self.tdp.DEVICE, *w.shape)


class AttentiveOracle:
    """The same model in 64 bits: hidden states and caches of tokens, and the logits behind a last token and given caches."""

    def __init__(self, shape, kv_scales=None):
        self.shape = dataclasses.replace(oracle_shape(shape), kv_scales=kv_scales)
        self.layers = [dataclasses.replace(w, **{n: getattr(w, n) * f for n, f in SCALES.items()}) for w in oracle_layers(shape, device="cpu")]
        self.table, self.head = (W.ends_weight(shape, n, VOCAB).double().numpy() for n in ("embedding", "lm_head"))
        self.gain, self.eps = W.ends_weight(shape, "final_norm", VOCAB, dtype=torch.float32).double().numpy(), shape.rms_eps

    def caches(self, tokens):
        return O.stage_forward(E.embed(tokens, self.table), None, self.layers, self.shape)[1]

    def logits(self, token, caches):
        h = E.embed([token], self.table)
        for w, (k, v) in zip(self.layers, caches):
            h, _, _ = O.layer_forward(h, k, v, w, self.shape)
        return E.final_logits(h, self.gain, self.head, self.eps)[0]


def histories(prompts, selections):
    """What every row of every step continues: [step][row] -> tokens, None for a row that continues nothing.  selections: (parent, token) of every
    step, [groups][beams] each."""
    steps = [[list(p) for p in prompts]]
    for parent, token in selections:
        before = steps[-1]
        steps.append([None if p < 0 or before[p] is None else before[p] + [int(t)] for p, t in zip(np.ravel(parent), np.ravel(token))])
    return steps
