#!/usr/bin/env python3
"""A training step of the package's operators, its memory estimated beside it.

A residual MLP policy (embedding, blocks of two linear layers, vocabulary head) takes steps of the clipped policy
loss with Newton-Schulz updates; with --normed its blocks stand between norms, the embedding learns too and all gradients are
clipped together.  Every tensor that a step takes and gives back is written down as the profiler would (time,
address, bytes); the package's estimate of these events (pairing, orchestration, replay through the caching
allocator's model) stands beside what the device's allocator saw.

    python examples/policy_step.py [--hidden 2048 --layers 24 --vocab 50304 --tokens 8192 --steps 3] [--normed]
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


class NormedPolicy(Policy):
    """Blocks between norms: x <- x + scale norm(block(norm(x))), norms of the root mean square."""

    def __init__(self, hidden, layers, vocab, tokens, seed=0):
        super().__init__(hidden, layers, vocab, tokens, seed)
        one = lambda *s: torch.ones(*s, device="cuda")
        # each block's scale, the norm after it and the one before the next (the head); the norm before the first block
        self.scale, self.post, self.pre, self.first = 0.5 * one(layers, hidden), one(layers, hidden), one(layers, hidden), one(hidden)
        need = max(xm.xmem_residual_norm_backward_workspace_bytes(tokens, hidden, xm.XMEM_BF16), xm.xmem_clip_grad_norm_workspace_bytes(),
                   xm.xmem_embedding_backward_workspace_bytes(tokens, vocab, hidden))
        if need > self.workspace.numel():
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")

    def vectors(self):
        return [self.scale, self.post, self.pre, self.first, self.up_b, self.down_b]

    def state(self):
        return super().state() + [self.scale, self.post, self.pre, self.first]

    def how(self, i):
        return dict(scale=self.scale[i], post="rms", post_weight=self.post[i], pre="rms", pre_weight=self.pre[i])

    def forward(self, ids, led):
        x = led.take(xm.embedding_forward(self.table, ids))
        _, y, stats = xm.residual_norm_forward(x, pre_weight=self.first, save_stats=True)
        led.take(y, stats)
        kept = [(x, stats)]
        for i in range(len(self.up)):
            mid, z = led.take(*xm.linear_forward(y, self.up[i], self.up_b[i], activation="gelu", save_z=True, workspace=self.workspace))
            out = led.take(xm.linear_forward(mid, self.down[i], self.down_b[i], workspace=self.workspace)[0])
            x, y_next, stats = led.take(*xm.residual_norm_forward(x, out, save_stats=True, **self.how(i)))
            kept.append((y, mid, z, out, x, stats))
            y = y_next
        return led.take(xm.linear_forward(y, self.head, workspace=self.workspace)[0]), y, kept

    def gradients(self, ids, tokens, weights, old_logp, advantages, ref_logp, led, kl_coef=0.02):
        """Stats and log-probabilities of the loss, and the gradients of (table, up, down, head, *vectors())."""
        logits, y, kept = self.forward(ids, led)
        stats, logp, dlogits = xm.policy_loss(logits, tokens, weights, old_logp, advantages, ref_logp, clip_high=0.28, kl_coef=kl_coef,
                                              in_place=True, workspace=self.workspace)
        led.take(stats, logp)
        dy, dhead, _ = xm.linear_backward(dlogits, y, self.head, need_db=False, workspace=self.workspace)
        led.take(dy, dhead)
        led.give(logits, y)
        del logits, dlogits, y
        vectors = [led.take(torch.empty_like(v)) for v in self.vectors()]
        dscale, dpost, dpre, dfirst, dup_b, ddown_b = vectors
        dx = None
        for i in reversed(range(len(self.up))):
            y, mid, z, out, x, saved = kept.pop()
            dx_next, dout, _, *sums = xm.residual_norm_backward(dy, dx, x, saved, out, in_place=dx is not None, workspace=self.workspace, **self.how(i))
            led.take(*(t for t in (None if dx is not None else dx_next, dout, *sums) if t is not None))
            dscale[i], dpost[i], dpre[i] = sums[0], sums[1], sums[3]
            led.give(dy, out, x, saved, *sums)
            dx = dx_next
            del dx_next, sums, out, x, saved, dy
            dmid, dw, db = led.take(*xm.linear_backward(dout, mid, self.down[i], workspace=self.workspace))
            self.grads[1][i].copy_(dw)
            ddown_b[i] = db
            led.give(dout, mid, dw, db)
            del dout, mid, dw, db
            dy, dw, db = led.take(*xm.linear_backward(dmid, y, self.up[i], z, "gelu", workspace=self.workspace))
            self.grads[0][i].copy_(dw)
            dup_b[i] = db
            led.give(dmid, y, z, dw, db)
            del dmid, y, z, dw, db
        x, saved = kept.pop()
        made = dx is None
        dx, _, _, _, _, _, dw, _ = xm.residual_norm_backward(dy, dx, x, saved, pre_weight=self.first, in_place=not made, workspace=self.workspace)
        led.take(*((dx, dw) if made else (dw,)))
        dfirst.copy_(dw)
        led.give(dy, x, saved, dw)
        del dy, x, saved, dw
        dtable = led.take(xm.embedding_backward(dx, ids, len(self.table), workspace=self.workspace))
        led.give(dx)
        return stats, logp, [dtable, *self.grads, dhead, *vectors]

    def step(self, ids, tokens, weights, old_logp, advantages, ref_logp, led, lr=0.02, kl_coef=0.02, max_norm=1.0):
        stats, logp, grads = self.gradients(ids, tokens, weights, old_logp, advantages, ref_logp, led, kl_coef)
        norm = led.take(xm.clip_grad_norm(grads, max_norm, workspace=self.workspace))
        dtable, dup, ddown, dhead, *vectors = grads
        for w, grad, momentum in zip((self.up, self.down, self.head), (dup, ddown, dhead), self.momenta):
            scale = max(1.0, w.shape[-2] / w.shape[-1]) ** 0.5
            update = led.take(xm.muon_update(grad, momentum, scale=scale, workspace=self.workspace))
            w.add_(update, alpha=-lr)
            led.give(update)
            del update
        for w, grad in zip((self.table, *self.vectors()), (dtable, *vectors)):
            w.add_(grad, alpha=-lr)
        led.give(dtable, dhead, logp, norm, *vectors)
        return stats


def train(hidden=256, layers=4, vocab=1024, tokens=512, steps=4, seed=0, normed=False):
    """Returns a dict: the loss of each step, the log-probability that tokens of positive (and of negative) advantage gained, and
    the estimated and measured peaks in bytes."""
    policy = (NormedPolicy if normed else Policy)(hidden, layers, vocab, tokens, seed)
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
    ap.add_argument("--normed", action="store_true")
    got = train(**vars(ap.parse_args()))
    for i, (loss, clipped) in enumerate(zip(got["loss"], got["clipped"])):
        print(f"step {i}: loss {loss:+.5f}, clipped {100 * clipped:.1f}%")
    print("log-probability gained: %+.3f where the advantage is positive, %+.3f where it is negative" % got["gained"])
    for what, a, b in zip(("allocated", "reserved"), got["estimated"], got["measured"]):
        print(f"peak {what}: estimated {a / 2**20:.1f} MiB from {got['events']} events, measured {b / 2**20:.1f} MiB")


if __name__ == "__main__":
    main()
