#!/usr/bin/env python3
"""A training step of the package's operators, its memory estimated beside it.

A residual MLP policy (embedding, blocks of two linear layers, vocabulary head) takes steps of the clipped policy
loss with Newton-Schulz updates.  Every tensor that a step takes and gives back is written down as the profiler would (time,
address, bytes); the package's estimate of these events (pairing, orchestration, replay through the caching
allocator's model) stands beside what the device's allocator saw.

    python examples/policy_step.py [--hidden 2048 --layers 24 --vocab 50304 --tokens 8192 --steps 3]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import paper_2510_21048_amd as xm
from paper_2510_21048_amd.binding import XMEM_CAT_OTHER, XMEM_CAT_PARAMETER

BF = torch.bfloat16


class Ledger:
    """What was taken and given back, in order, as raw allocator events."""

    def __init__(self):
        self.raw, self.category = [], []

    def _add(self, t, sign, category):
        self.raw.append((len(self.raw), t.data_ptr(), sign * t.untyped_storage().nbytes()))
        self.category.append(category)

    def take(self, *tensors, category=XMEM_CAT_OTHER):
        for t in tensors:
            if t is not None and t.numel():
                self._add(t, 1, category)
        return tensors[0] if len(tensors) == 1 else tensors

    def give(self, *tensors):
        for t in tensors:
            if t is not None and t.numel():
                self._add(t, -1, XMEM_CAT_OTHER)

    def estimate(self):
        """Peak allocated and peak reserved bytes of these events."""
        dev = torch.device("cuda")
        on = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
        raw = np.array(self.raw, dtype=xm.RAW_EVENT_DTYPE)
        off, none = on(np.array([0, len(raw)], np.int64)), on(np.array([0, 0], np.int64))
        blocks, block_off, _, _ = xm.lifecycles(on(raw.view(np.uint8)), off, on(np.array(self.category, np.int32)))
        no_marks = torch.empty(0, dtype=torch.int64, device=dev)
        words, word_off, _ = xm.orchestrate(blocks, block_off, no_marks, none, no_marks, none)
        out, _ = xm.replay(words[: int(word_off[-1])], word_off, xm.params(xm.XMEM_PRESET_PYTORCH_LIKE))
        got = xm.to_numpy(out)[0]
        return int(got["peak_allocated"]), int(got["peak_reserved"])


class Policy:
    def __init__(self, hidden, layers, vocab, tokens, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *s: (torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5).to(BF)
        self.table = new(vocab, hidden) * hidden ** 0.5
        self.up, self.down, self.head = new(layers, 4 * hidden, hidden), new(layers, hidden, 4 * hidden) * 0.1, new(vocab, hidden) * 0.1
        self.up_b, self.down_b = torch.zeros(layers, 4 * hidden, device="cuda"), torch.zeros(layers, hidden, device="cuda")
        self.grads = [torch.empty_like(w) for w in (self.up, self.down)]
        self.momenta = [torch.zeros(w.shape, device="cuda") for w in (self.up, self.down, self.head)]
        # one workspace for every call of a step: its size is known from the shapes
        m, h = tokens, hidden
        self.workspace = torch.empty(max(
            xm.xmem_linear_forward_workspace_bytes(m, 4 * h, h, h, h), xm.xmem_linear_forward_workspace_bytes(m, h, 4 * h, 4 * h, 4 * h),
            xm.xmem_linear_forward_workspace_bytes(m, vocab, h, h, h),
            xm.xmem_linear_backward_workspace_bytes(m, 4 * h, h, 4 * h, h, h, xm.ACTIVATIONS["gelu"]),
            xm.xmem_linear_backward_workspace_bytes(m, h, 4 * h, h, 4 * h, 4 * h, 0),
            xm.xmem_linear_backward_workspace_bytes(m, vocab, h, vocab, h, h, 0), xm.xmem_policy_loss_workspace_bytes(m, vocab),
            *(xm.xmem_muon_update_workspace_bytes(*s) for s in ((layers, 4 * h, h), (layers, h, 4 * h), (1, vocab, h)))),
            dtype=torch.uint8, device="cuda")

    def state(self):
        return [self.table, self.up, self.down, self.head, self.up_b, self.down_b, *self.grads, *self.momenta, self.workspace]

    def forward(self, ids, led):
        """Logits, and what the backward pass needs of each block."""
        h, kept = led.take(self.table[ids]), []
        for i in range(len(self.up)):
            mid, z = led.take(*xm.linear_forward(h, self.up[i], self.up_b[i], activation="gelu", save_z=True, workspace=self.workspace))
            out = led.take(xm.linear_forward(mid, self.down[i], self.down_b[i], residual=h, workspace=self.workspace)[0])
            kept.append((h, mid, z))
            h = out
        return led.take(xm.linear_forward(h, self.head, workspace=self.workspace)[0]), h, kept

    def logp(self, ids, tokens):
        led = Ledger()
        return xm.token_logp(self.forward(ids, led)[0], tokens)

    def step(self, ids, tokens, weights, old_logp, advantages, ref_logp, led, lr=0.02, kl_coef=0.02):
        logits, h, kept = self.forward(ids, led)
        stats, logp, dlogits = xm.policy_loss(logits, tokens, weights, old_logp, advantages, ref_logp, clip_high=0.28, kl_coef=kl_coef,
                                              in_place=True, workspace=self.workspace)
        led.take(stats, logp)
        dh, dhead, _ = xm.linear_backward(dlogits, h, self.head, need_db=False, workspace=self.workspace)
        led.take(dh, dhead)
        led.give(logits, h)
        del logits, dlogits, h
        for i in reversed(range(len(kept))):
            h, mid, z = kept.pop()
            dmid, dw, db = led.take(*xm.linear_backward(dh, mid, self.down[i], workspace=self.workspace))
            self.grads[1][i].copy_(dw)
            self.down_b[i].add_(db, alpha=-lr)
            led.give(mid, dw, db)
            del mid, dw, db
            dprev, dw, db = led.take(*xm.linear_backward(dmid, h, self.up[i], z, "gelu", workspace=self.workspace))
            self.grads[0][i].copy_(dw)
            self.up_b[i].add_(db, alpha=-lr)
            dprev.add_(dh)  # the residual's gradient
            led.give(dmid, dh, h, z, dw, db)
            dh = dprev
            del dprev, dmid, h, z, dw, db
        led.give(dh)
        del dh
        for w, grad, momentum in zip((self.up, self.down, self.head), (*self.grads, dhead), self.momenta):
            scale = max(1.0, w.shape[-2] / w.shape[-1]) ** 0.5
            update = led.take(xm.muon_update(grad, momentum, scale=scale, workspace=self.workspace))
            w.add_(update, alpha=-lr)
            led.give(update)
            del update
        led.give(dhead, logp)
        return stats


def train(hidden=256, layers=4, vocab=1024, tokens=512, steps=4, seed=0):
    """Returns a dict: the loss of each step, the log-probability that tokens of positive (and of negative) advantage gained, and
    the estimated and measured peaks in bytes."""
    policy = Policy(hidden, layers, vocab, tokens, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    ids = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    sampled = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    advantages = torch.randn(tokens, generator=g, device="cuda")
    kept = torch.arange(tokens, device="cuda") >= tokens // 8  # the prompt
    weights = kept.float() / kept.sum()
    old = policy.logp(ids, sampled)
    batch = [ids, sampled, weights, old, advantages, old.clone()]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()

    led = Ledger()
    held = policy.state() + batch
    led.take(*held, category=XMEM_CAT_PARAMETER)
    up512 = lambda t: -(-t.untyped_storage().nbytes() // 512) * 512
    beside = torch.cuda.memory_allocated() - sum(up512(t) for t in held)  # what else lives on the device
    torch.cuda.reset_peak_memory_stats()
    stats = [policy.step(*batch, led) for _ in range(steps)]
    torch.cuda.synchronize()
    measured = torch.cuda.max_memory_allocated() - beside, torch.cuda.max_memory_reserved()
    losses = [s.cpu().tolist() for s in stats]
    gained = policy.logp(ids, sampled) - old
    up, down = (float(gained[kept & side].mean()) for side in (advantages > 0, advantages < 0))
    estimated = led.estimate()
    return {"loss": [s[0] for s in losses], "clipped": [s[3] for s in losses], "gained": (up, down), "events": len(led.raw),
            "estimated": estimated, "measured": measured}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("hidden", 1024), ("layers", 12), ("vocab", 50304), ("tokens", 4096), ("steps", 4)):
        ap.add_argument("--" + name, type=int, default=default)
    got = train(**vars(ap.parse_args()))
    for i, (loss, clipped) in enumerate(zip(got["loss"], got["clipped"])):
        print(f"step {i}: loss {loss:+.5f}, clipped {100 * clipped:.1f}%")
    print("log-probability gained: %+.3f where the advantage is positive, %+.3f where it is negative" % got["gained"])
    for what, a, b in zip(("allocated", "reserved"), got["estimated"], got["measured"]):
        print(f"peak {what}: estimated {a / 2**20:.1f} MiB from {got['events']} events, measured {b / 2**20:.1f} MiB")


if __name__ == "__main__":
    main()
