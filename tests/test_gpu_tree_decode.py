"""The example that runs the operators of a step together: drafted trees give the tokens of one token a step, and its logits are the oracle's for the
weights that the codes stand for."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import atts_oracle as O
from oracle import step_oracle as S
from synth import ModelConfig, make_weights
from util import announce, weights_to_numpy

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_trees_decode_what_single_tokens_do():
    import tree_decode as E
    announce("tree decode")
    plain, trees = E.main()
    assert plain == trees and all(len(t) == 24 for t in plain)


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-4), ("bf16", 6e-2)])       # of the scoring pass: 32 bits, and bf16 activations through two layers
def test_logits_against_the_oracle(dtype, tol):
    import tree_decode as E
    cfg = ModelConfig(2, 256, 4, 2, 64, 512, 768, dtype)
    w = make_weights(cfg, seed=5, device="cuda")
    model = E.TreeDecoder(cfg, w, 2, capacity=120)
    host = weights_to_numpy(w)
    for name, key in (("wqkv", "qkv"), ("wo", "o"), ("w_gate_up", "gate_up"), ("w_down", "down")):
        for l, layer in enumerate(model.layers):
            q = layer[key]
            host[name][l] = S.dequantize(q.codes.cpu().numpy(), q.scales.float().cpu().numpy(), q.zeros.cpu().numpy()).astype(np.float32)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, cfg.vocab, n).tolist() for n in (70, 3)]
    trees = [rng.integers(0, cfg.vocab, n).tolist() for n in (7, 2)]
    parents = [[-1, 0, 1, 0, -1, 4, 4], [-1, -1]]
    announce("tree step against the oracle", dtype)
    model.step(prompts, [list(range(-1, len(p) - 1)) for p in prompts])
    model.keep([list(range(len(p))) for p in prompts])
    got, r = model.step(trees, parents).cpu().numpy(), 0
    for prompt, tree, up in zip(prompts, trees, parents):
        for i in range(len(tree)):
            ids = np.array(prompt + [tree[j] for j in reversed(S.path(up, i))], dtype=np.int32)
            hidden = O.rmsnorm(O.decoder_hidden(host, cfg, ids), host["final_norm"], cfg.rms_eps)[-1]
            assert np.abs(got[r] - hidden @ host["lm_head"].astype(np.float64).T).max() <= tol
            r += 1
