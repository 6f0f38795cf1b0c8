"""The example that trains the vocabulary projection under a grammar and decodes from its 4-bit weights, at a small size."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "grammar_head.py")
    spec = importlib.util.spec_from_file_location("grammar_head", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_learns_and_decodes_admitted_tokens():
    """The loss falls, every token decoded is admitted by its state, and a state's learned token comes back from 4 bits."""
    g = _example()
    s = g.prepare(V=2000, D=128, rows=300)
    weight, losses = g.train(s, steps=25)
    assert losses[-1] < 0.2 * losses[0]
    masks = torch.arange(s["state_mask"].shape[0], device="cuda", dtype=torch.int32)
    admitted = g.cz.cfgzip_expand_mask(g.cz.cfgzip_class_masks(s["state_mask"], s["C"], masks), s["C"], s["c"])
    trained = set(s["states"].tolist())
    for token, logits, states in g.serve(s, weight, steps=6, batch=20):
        for b in range(20):
            q, t = int(states[b]), int(token[b])
            if not 0 < q < admitted.shape[0] or int(s["best"][q]) < 0:
                continue
            assert int(admitted[q, t // 32]) >> (t % 32) & 1
            if q in trained:
                assert t == int(s["best"][q])
