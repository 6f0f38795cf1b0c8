"""A vocabulary projection learned under a grammar, then kept in 4 bits and decoded with under the same grammar.

    python examples/grammar_head.py

The grammar is a byte automaton; the vocabulary's classes and the masks of its states come from the library as for any decode
loop.  A row's hidden state stands for the automaton state that the row is in (random, fixed: only the projection learns).

  training   masks of the rows' states -> loss over the admitted tokens and its gradients -> a step on the weights
  serving    weights to 4 bits once; per step: masks of the rows' states -> masked logits -> the best token -> next states
"""

from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2605_29986_amd as cz  # noqa: E402
import synthetic_inputs as si  # noqa: E402


def live_states(table: np.ndarray, accepting: np.ndarray) -> np.ndarray:
    """uint8 [S]: states from which an accepting one can be reached (state 0 rejects)."""
    live = accepting.astype(bool)
    while True:
        more = live | live[table].any(1)
        more[0] = False
        if (more == live).all():
            return live.astype(np.uint8)
        live = more


def prepare(V: int, D: int, rows: int, seed: int = 0):
    """Classes and state masks of a small grammar, hidden states of its states, and a training batch."""
    cfg = si.make_config(1, V=V)
    vocab, table, S = cfg["vocab"], cfg["table"], cfg["S"]
    rng = np.random.default_rng(seed)
    accepting = rng.random(S) < 0.5
    accepting[0] = False
    tok_bytes, tok_off = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (vocab.tok_bytes, vocab.tok_off))
    tab = torch.from_numpy(table).cuda()
    sig, h = cz.cfgzip_signatures(tok_bytes, tok_off, tab)
    c, r, C, _ = cz.cfgzip_build_classes(tok_bytes, tok_off, tab, sig, h)
    rep_bytes, rep_off = cz.cfgzip_representative_vocabulary(tok_bytes, tok_off, r.contiguous())
    sig_rep, _ = cz.cfgzip_signatures(rep_bytes[:max(int(rep_off[-1]), 1)].contiguous(), rep_off, tab, want_hash=False)
    state_mask = cz.cfgzip_state_masks(sig_rep, torch.from_numpy(live_states(table, accepting)).cuda())
    gen = torch.Generator(device="cuda").manual_seed(seed)
    of_state = torch.randn((S, D), device="cuda", generator=gen).bfloat16()
    states = torch.randint(1, S, (rows,), device="cuda", generator=gen).int()
    cls_bits = cz.cfgzip_class_masks(state_mask, C, states)
    # what is to be learned: one of a state's admitted tokens, the same for all rows in that state; no target where there is none
    admitted = cz.cfgzip_apply_mask(torch.rand((S, V), device="cuda", generator=gen),
                                    cz.cfgzip_class_masks(state_mask, C, torch.arange(S, device="cuda", dtype=torch.int32)),
                                    class_of_token=c, C=C)
    best = torch.where(admitted.amax(1) > -torch.inf, admitted.argmax(1), -1).int()
    return {"c": c, "C": C, "sig_rep": sig_rep, "state_mask": state_mask, "of_state": of_state, "states": states, "cls_bits": cls_bits,
            "target": best[states.long()], "best": best, "V": V, "D": D}


def train(s, steps: int, rate: float = 40.0):
    """(weight, mean loss of every step)"""
    gen = torch.Generator(device="cuda").manual_seed(1)
    master = torch.randn((s["V"], s["D"]), device="cuda", generator=gen) * (0.5 / s["D"] ** 0.5)
    hidden = s["of_state"][s["states"].long()]
    masks = {"bits": s["cls_bits"], "class_of_token": s["c"], "C": s["C"]}
    learned = s["target"] >= 0
    grad_loss = learned.float() / learned.sum().clamp(min=1)
    losses = []
    for _ in range(steps):
        weight = master.bfloat16()
        loss, lse = cz.cfgzip_head_loss(hidden, weight, s["target"], **masks)
        _, grad = cz.cfgzip_head_loss_grad(hidden, weight, s["target"], lse, grad_loss, want_hidden=False, **masks)
        master -= rate / s["D"] * grad.float()
        losses.append((loss * grad_loss).sum())
    return master.bfloat16(), torch.stack(losses).tolist()


def serve(s, weight, steps: int, batch: int):
    """Greedy decoding with the weights in 4 bits; (tokens, the masked logits of every step, the states in front of it)"""
    codes, scales = cz.cfgzip_mx4_quantize(weight)
    states = s["states"][:batch].clone()
    out = []
    for _ in range(steps):
        cls_bits = cz.cfgzip_class_masks(s["state_mask"], s["C"], states)
        logits = cz.cfgzip_mx4_logits(s["of_state"][states.long()], codes, scales, bits=cls_bits, class_of_token=s["c"], C=s["C"])
        token = logits.argmax(1).int()
        out.append((token, logits, states.clone()))
        cz.cfgzip_advance_states(s["sig_rep"], s["c"], token, states)
    return out


def main() -> None:
    s = prepare(V=4096, D=256, rows=512)
    weight, losses = train(s, steps=30)
    print("mean loss over the admitted tokens: first step %.3f, last %.3f" % (losses[0], losses[-1]))
    right = total = 0
    for token, logits, states in serve(s, weight, steps=8, batch=16):
        there = s["best"][states.long()] >= 0
        right += int((token == s["best"][states.long()])[there].sum())
        total += int(there.sum())
        assert torch.isfinite(logits.gather(1, token.long()[:, None]))[there].all()
    print("greedy tokens from 4-bit weights that are the learned ones: %d of %d" % (right, total))


if __name__ == "__main__":
    main()
