#!/usr/bin/env python3
"""A user's events, encoded: non-pooled lookup -> layer norm -> causal attention with a learned bias by distance, trained with the library's own
backward passes and row-wise AdaGrad, then served one event at a time from a cache.

Every event has an id; its table row holds a query, a key and a value for each head, side by side.  The rows of a batch's sequences lie one
after the other, as the lookup leaves them, and are only ever addressed as column blocks of that one matrix.  The toy task: the output
at an event is to match a fixed random direction of the previous event's id, which takes attending one event back.

    python examples/event_encoder.py [--steps 60] [--users 256] [--io bf16]
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2508_03854_amd import TBE


class EventEncoder:
    def __init__(self, ids: int, heads: int = 2, dim: int = 32, buckets: int = 16, far: int = 64, io: torch.dtype = torch.float32, seed: int = 0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.heads, self.dim, self.io, self.width = heads, dim, io, 3 * heads * dim
        self.tbe = TBE([ids], [self.width])
        self.tables = torch.empty(ids * self.width, device="cuda").uniform_(-0.1, 0.1, generator=g)
        self.state = torch.zeros(ids, device="cuda")
        self.weight, self.norm_bias = torch.ones(self.width, device="cuda"), torch.zeros(self.width, device="cuda")
        self.bias = torch.zeros(heads, buckets, device="cuda")
        # nearest distances one bucket each, further ones by their logarithm
        d = torch.arange(-far, far + 1).abs()
        near = buckets // 2
        log = near + (torch.log(d.clamp(min=1) / near) / math.log(far / near) * (buckets - near)).long()
        self.bucket_map = torch.where(d < near, d, log.clamp(max=buckets - 1)).to(torch.int32).cuda()

    def rows(self, ids: torch.Tensor) -> torch.Tensor:
        """The events' table rows, [events, width]."""
        out = torch.empty(ids.numel() * self.width, dtype=self.io, device="cuda")
        self.tbe.lookup_seq(self.tables, ids, torch.tensor([0, ids.numel()], dtype=ids.dtype, device="cuda"), out)
        return out.view(-1, self.width)

    def blocks(self, x: torch.Tensor):
        """Query, key and value of every event and head: column blocks of one matrix."""
        return x.view(-1, 3 * self.heads, self.dim).split(self.heads, 1)

    def forward(self, ids: torch.Tensor, offsets: torch.Tensor) -> dict:
        x = self.rows(ids)
        y, mean, rstd = self.tbe.layer_norm(x, self.weight, self.norm_bias)
        q, k, v = self.blocks(y)
        ws = self.tbe.alloc_attention_workspace(offsets.numel() - 1, len(x), len(x), self.heads, self.heads, self.dim, buckets=self.bias.shape[1])
        out, lse = self.tbe.attention(q, k, v, offsets, offsets, ws, bias=self.bias, bucket_map=self.bucket_map)
        return {"x": x, "y": y, "mean": mean, "rstd": rstd, "out": out, "lse": lse}

    def gradients(self, f: dict, grad_out: torch.Tensor, offsets: torch.Tensor):
        """Of the rows, the norm's weight and bias, and the table of biases."""
        q, k, v = self.blocks(f["y"])
        n = len(f["x"])
        grad_y = torch.empty_like(f["y"])
        gq, gk, gv = self.blocks(grad_y)
        ws = self.tbe.alloc_attention_workspace(offsets.numel() - 1, n, n, self.heads, self.heads, self.dim, buckets=self.bias.shape[1], backward=True)
        grad_bias = self.tbe.attention_backward(grad_out, q, k, v, f["out"], f["lse"], offsets, offsets, ws, bias=self.bias,
                                                bucket_map=self.bucket_map, grad_q=gq, grad_k=gk, grad_v=gv)[3]
        grad_x, grad_weight, grad_norm_bias = self.tbe.layer_norm_backward(grad_y, f["x"], self.weight, f["mean"], f["rstd"],
                                                                           self.tbe.alloc_layer_norm_workspace(n, self.width))
        return grad_x, grad_weight, grad_norm_bias, grad_bias

    def train_step(self, ids: torch.Tensor, offsets: torch.Tensor, target: torch.Tensor, lr: float = 0.05) -> torch.Tensor:
        f = self.forward(ids, offsets)
        diff = f["out"].float() - target
        grad = (2.0 / ids.numel() * diff).to(self.io)
        gx, gw, gn, gb = self.gradients(f, grad, offsets)
        for p, g in ((self.weight, gw), (self.norm_bias, gn), (self.bias, gb)):
            p -= lr * g
        one = torch.tensor([0, ids.numel()], dtype=ids.dtype, device="cuda")
        self.tbe.backward_seq_rowwise_adagrad(gx.view(-1), ids, one, self.tables, self.state, self.tbe.alloc_workspace(1, ids.numel()), lr=lr, eps=1e-8)
        return diff.square().sum(2).mean()

    def serve_step(self, ids: torch.Tensor, cache: dict) -> torch.Tensor:
        """One new event per user against the cached keys and values of the earlier ones; the cache, which has room, gets the new ones."""
        y, _, _ = self.tbe.layer_norm(self.rows(ids), self.weight, self.norm_bias, stats=False)
        q, k, v = self.blocks(y)
        at = cache["starts"][:-1] + cache["lengths"]
        cache["k"][at], cache["v"][at] = k, v
        cache["lengths"] += 1
        return self.tbe.attention(q, cache["k"], cache["v"], cache["one_each"], cache["starts"], cache["workspace"], k_lengths=cache["lengths"],
                                  bias=self.bias, bucket_map=self.bucket_map, stats=False)[0]

    def new_cache(self, users: int, room: int) -> dict:
        shape = (users * room, self.heads, self.dim)
        return {"k": torch.zeros(shape, dtype=self.io, device="cuda"), "v": torch.zeros(shape, dtype=self.io, device="cuda"),
                "starts": torch.arange(users + 1, device="cuda") * room, "lengths": torch.zeros(users, dtype=torch.int64, device="cuda"),
                "one_each": torch.arange(users + 1, device="cuda"),
                "workspace": self.tbe.alloc_attention_workspace(users, users, users * room, self.heads, self.heads, self.dim, buckets=self.bias.shape[1])}


def batch(users: int, ids: int, seed: int):
    """Sequences of very different lengths, and for every event its target: a direction of the event before."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n = torch.exp(2.0 + torch.randn(users, generator=g, device="cuda")).round().clamp(1, 200).long()
    offsets = torch.cat([n.new_zeros(1), n.cumsum(0)])
    events = torch.randint(0, ids, (int(offsets[-1]),), generator=g, device="cuda")
    before = torch.where(torch.isin(torch.arange(events.numel(), device="cuda"), offsets[:-1]), events, events.roll(1))
    return events, offsets, before


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--users", type=int, default=256)
    ap.add_argument("--ids", type=int, default=500)
    ap.add_argument("--io", choices=("f32", "f16", "bf16"), default="f32")
    args = ap.parse_args(argv)
    enc = EventEncoder(args.ids, io={"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[args.io])
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    directions = torch.randn(args.ids, enc.heads, enc.dim, generator=g, device="cuda") * 0.5
    losses = []
    for step in range(args.steps):
        ids, offsets, before = batch(args.users, args.ids, step % 8)
        losses.append(float(enc.train_step(ids, offsets, directions[before])))
        if step % 10 == 0 or step == args.steps - 1:
            print(f"step {step}: {ids.numel()} events, loss {losses[-1]:.4f}", flush=True)
    # whole sequences, and the same events one at a time
    users, events = 8, 20
    ids = torch.randint(0, args.ids, (users * events,), generator=g, device="cuda")
    offsets = torch.arange(users + 1, device="cuda") * events
    whole = enc.forward(ids, offsets)["out"]
    cache, worst = enc.new_cache(users, events + 4), 0.0
    for t in range(events):
        out = enc.serve_step(ids[offsets[:-1] + t], cache)
        worst = max(worst, float((out.float() - whole[offsets[:-1] + t].float()).abs().max()))
    print(f"served {events} events for each of {users} users: at most {worst:.2e} from the whole sequences", flush=True)
    return losses, worst


if __name__ == "__main__":
    main()
