"""A VLM's prefix beside the rolling expert: the prompt of a fleet goes through a
small random-init decoder whose keys and values live in a ContextCache, each
robot decodes a few tokens (a subtask, say), the prefix shrinks to a budget by
the attention mass that its tokens drew, and what stays becomes the context of
the rolling step.

    python examples/vlm_prefix.py [--robots 4] [--prompt 200] [--decode 8] [--keep 96]

The decoder's attention shape is the expert's (its layers, heads and head dim),
as the expert reads the VLM's keys and values layer by layer."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import synth  # noqa: E402
from paper_2609_34170_gb300 import ContextCache, RollingSession  # noqa: E402


class Decoder:
    """Pre-norm attention and MLP layers, weights ~ N(0, 1 / fan-in); rotary
    positions are left out: the cache holds whatever keys it is given."""

    def __init__(self, layers, width, hq, hkv, hd, vocab, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.hq, self.hkv, self.hd = hq, hkv, hd

        def w(*shape):
            return (torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[0])).to(torch.bfloat16)

        self.embed = w(vocab, width) * math.sqrt(vocab)
        self.layers = [dict(qkv=w(width, (hq + 2 * hkv) * hd), o=w(hq * hd, width), up=w(width, 2 * width), down=w(2 * width, width))
                       for _ in range(layers)]

    @staticmethod
    def norm(x):
        return torch.nn.functional.rms_norm(x, x.shape[-1:])

    def run(self, cache, tokens, starts, counts, causal, mass):
        """tokens [B, n] at positions starts[b] .. of each robot, counts[b] of them
        real; returns the last real token's logits.  mass[l]: increased by layer
        l's attention mass."""
        x = self.embed[tokens]
        lengths = starts + counts
        for index, w in enumerate(self.layers):
            qkv = (self.norm(x) @ w["qkv"]).unflatten(-1, (self.hq + 2 * self.hkv, self.hd))
            # columns of one projection, as they are
            q, k, v = qkv[:, :, :self.hq], qkv[:, :, self.hq:self.hq + self.hkv], qkv[:, :, self.hq + self.hkv:]
            cache.append(index, k, v, starts, counts)
            att = cache.attend(index, q, lengths, counts, causal=causal, mass=mass[index], add_mass=True)
            x = x + att.flatten(2) @ w["o"]
            x = x + torch.nn.functional.silu(self.norm(x) @ w["up"]) @ w["down"]
        last = (counts - 1).clamp(min=0).long()
        return self.norm(x[torch.arange(len(x), device=x.device), last]) @ self.embed.t()


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("robots", 4), ("prompt", 200), ("decode", 8), ("keep", 96), ("layers", 4), ("width", 256)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    cfg = synth.ExpertConfig(layers=a.layers, width=a.width, n_q_heads=8, n_kv_heads=1, head_dim=64, mlp_dim=4 * a.width, slots=10,
                             action_dim=7, prefix=a.keep, fop_tokens=0, batch=a.robots, dtype="bf16")
    room = a.prompt + a.decode
    model = Decoder(cfg.layers, cfg.width, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, vocab=512)
    shape = dict(layers=cfg.layers, n_q_heads=cfg.n_q_heads, n_kv_heads=cfg.n_kv_heads, head_dim=cfg.head_dim, max_batch=a.robots)
    cache = ContextCache(**shape, max_tokens=room, max_queries=a.prompt)
    small = ContextCache(**shape, max_tokens=a.keep)
    mass = torch.zeros((cfg.layers, a.robots, cfg.n_kv_heads, room), device="cuda")

    # prompts of different lengths: every token of one sees every other
    g = torch.Generator("cuda").manual_seed(1)
    tokens = torch.randint(0, 512, (a.robots, a.prompt), generator=g, device="cuda")
    counts = torch.tensor([a.prompt - 7 * b % (a.prompt // 2) for b in range(a.robots)], dtype=torch.int32, device="cuda")
    starts = torch.zeros_like(counts)
    nxt = model.run(cache, tokens, starts, counts, causal=False, mass=mass).argmax(-1)
    # decoded tokens see what came before them
    lengths, one = counts.clone(), torch.ones_like(counts)
    said = []
    for _ in range(a.decode):
        said.append(nxt)
        nxt = model.run(cache, nxt[:, None], lengths, one, causal=True, mass=mass).argmax(-1)
        lengths += one

    # the prefix down to its budget, layer by layer, and into the expert's context
    ks, vs, kept = [], [], []
    for layer in range(cfg.layers):
        new_lengths, index, _ = cache.evict(layer, small, layer, lengths, mass[layer], a.keep, sinks=4, recent=a.decode)
        k, v = small.read(layer, a.robots, a.keep, lengths=new_lengths)
        ks.append(k)
        vs.append(v)
        kept.append(index)
    session = RollingSession(cfg, synth.make_weights(cfg))
    session.reset(synth.robot_seeds(7, a.robots))
    length = int(new_lengths.min())   # the same for all where every prompt is longer than the budget
    k, v = (torch.stack(x)[:, :, :, :length].contiguous() for x in (ks, vs))
    session.set_context(k, v, length)
    released = session.step(synth.staggered_times(cfg.slots), None, synth.make_delta(a.robots, 2, cfg.slots)).clone()
    torch.cuda.synchronize()
    held = cfg.layers * a.robots * cfg.n_kv_heads * room * 2 * (cfg.head_dim + 1 / 16)
    print(f"{a.robots} robots, prompts of {counts.tolist()} tokens, {a.decode} decoded; {held / 2 ** 20:.2f} MiB held in 8 bits; "
          f"{length} tokens per robot stay; released action 0: {[round(x, 3) for x in released[0].tolist()]}")
    return dict(tokens=torch.stack(said, 1), kept=kept, lengths=lengths, context=(k, v), released=released, mass=mass, cfg=cfg)


if __name__ == "__main__":
    main()
