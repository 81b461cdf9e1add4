"""Early-exit decoding with weights in 8 bits, the 4-bit cache and sampled tokens: a whole step is one graph.

A small decoder (random weights) with one exit in the middle.  The projections and both heads are products with weights held in 8 bits;
tokens are chosen by temperature, top-k and top-p from given random numbers, and the confidence that comes with a token decides
whether its request leaves at the exit.  Lengths, tokens and waiting hidden states live on the GPU and are updated in place, so that a
step is captured once and then replayed: nothing is read back until the end.

    python examples/f8_decode.py [--steps 32] [--seqs 6] [--threshold 0.02] [--eager]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2312_04916_amd as ee  # noqa: E402

LAYERS, EXIT, D, HEADS, KV_HEADS, HD, FF, VOCAB = 4, 2, 256, 8, 2, 64, 704, 1000
CAP = 3  # tokens of a request that may wait for the deeper layers; one more goes through whatever its confidence
TOP_K, TOP_P = 50, 0.9


class Decoder:
    def __init__(self, seed=0):
        g = torch.Generator(device="cuda:0").manual_seed(seed)

        def w(*shape):
            return (torch.randn(*shape, device="cuda:0", generator=g) / math.sqrt(shape[-1])).to(torch.bfloat16)

        self.embed = w(VOCAB, D) * 16
        self.qkv = [ee.F8Weight(w((HEADS + 2 * KV_HEADS) * HD, D)) for _ in range(LAYERS)]
        self.o = [ee.F8Weight(w(D, HEADS * HD)) for _ in range(LAYERS)]
        self.gate_up = [ee.F8Weight(w(FF, D), up=w(FF, D)) for _ in range(LAYERS)]
        self.down = [ee.F8Weight(w(D, FF)) for _ in range(LAYERS)]
        self.exit_head, self.head = ee.F8Weight(w(VOCAB, D) * 2), ee.F8Weight(w(VOCAB, D) * 2)
        self.freq = 10000.0 ** (-torch.arange(HD // 2, device="cuda:0") / (HD // 2))

    @staticmethod
    def norm(x):
        x = x.float()
        return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).to(torch.bfloat16)

    def rotate(self, x, positions):
        a = positions.clamp_min(0)[:, None].float() * self.freq
        c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
        lo, hi = x.float().chunk(2, -1)
        return torch.cat([lo * c - hi * s, hi * c + lo * s], -1).to(torch.bfloat16)

    def layers(self, cache, which, x):
        """Rows of the latest plan through these layers."""
        n = x.shape[0]
        pos = cache.positions[:n]
        for i in which:
            qkv = self.qkv[i].matmul(self.norm(x)).view(n, HEADS + 2 * KV_HEADS, HD)
            cache.append(i, self.rotate(qkv[:, HEADS:HEADS + KV_HEADS], pos), qkv[:, HEADS + KV_HEADS:])
            a = cache.attend(i, self.rotate(qkv[:, :HEADS], pos))
            x = self.o[i].matmul(a.view(n, HEADS * HD), add=x)
            x = self.down[i].matmul(self.gate_up[i].matmul(self.norm(x)), add=x)
        return x

    def choose(self, head, x, u, temperature):
        """-> tokens, confidences."""
        z = head.matmul(self.norm(x), dtype=torch.float32)
        token, _, confidence = ee.sample(z, u, temperature=temperature, top_k=TOP_K, top_p=TOP_P, scores=True)
        return token, confidence


class Batch:
    """Requests on their way: all that a step reads and writes stays at its place."""

    def __init__(self, model, prompts, temperature, steps, threshold, seed=0, block=32):
        self.model, self.threshold, self.temperature = model, threshold, temperature  # (temperature: one per request; 0 takes the likeliest)
        self.n = n = len(prompts)
        lens = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda:0")
        n_blocks = sum(-(-(len(p) + steps + 1) // block) for p in prompts)
        total = sum(len(p) for p in prompts)
        self.cache = ee.Kv4Cache(LAYERS, HEADS, KV_HEADS, HD, block, n_blocks, n, max(len(p) for p in prompts) + steps + 1, max(total, n * (CAP + 1)))
        self.u = torch.rand(steps + 1, 2, n, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(seed))
        self.ids, self.at = torch.arange(n, device="cuda:0"), torch.zeros(1, dtype=torch.int64, device="cuda:0")
        zero = torch.zeros_like(lens)
        self.cache.plan(zero, zero, lens, total)
        x = model.layers(self.cache, range(LAYERS), model.embed[torch.cat(prompts)])
        last = x[self.cache.row_start[1:n + 1].long() - 1]
        self.token = model.choose(model.head, last, self.u[steps, 0], temperature)[0]
        self.held, self.deep = lens.clone(), lens.clone()  # positions whose K and V the first layers have, and all layers
        self.waiting = torch.zeros(n, CAP + 1, D, dtype=torch.bfloat16, device="cuda:0")  # hidden states at the exit, by position
        self.out = torch.zeros(steps, n, dtype=torch.int32, device="cuda:0")
        self.left = torch.zeros(n, dtype=torch.int32, device="cuda:0")

    def deeper(self, start, end):
        """What waits at positions [start, end) through the deeper layers.  There is room for as many rows as there can be; the rest
        belong to no request."""
        rows = self.n * (CAP + 1)
        self.cache.plan(end, start, end, rows, CAP + 1)
        seq, pos = self.cache.row_seq[:rows].long().clamp_min(0), self.cache.positions[:rows].long().clamp_min(0)
        return self.model.layers(self.cache, range(EXIT, LAYERS), self.waiting[seq, pos % (CAP + 1)])

    def step(self):
        model, cache, n = self.model, self.cache, self.n
        u = self.u.index_select(0, self.at)[0]
        self.out.index_copy_(0, self.at, self.token[None])
        self.at += 1
        end = self.held + 1
        cache.plan(self.held, self.held, end, n, 1)
        x = model.layers(cache, range(EXIT), model.embed[self.token.long()])
        self.waiting[self.ids, self.held.long() % (CAP + 1)] = x
        early, confidence = model.choose(model.exit_head, x, u[0], self.temperature)
        leaves = (confidence >= self.threshold) & (end - self.deep <= CAP)
        y = self.deeper(torch.where(leaves, end, self.deep), end)
        last = (cache.row_start[1:n + 1].long() - 1).clamp_min(0)
        token, _ = model.choose(model.head, y[last], u[1], self.temperature)
        self.token.copy_(torch.where(leaves, early, token))
        self.left += leaves
        self.deep.copy_(torch.where(leaves, self.deep, end))
        self.held.copy_(end)

    def finish(self):
        """Whoever still waits goes through, so that every layer holds every position."""
        self.deeper(self.deep, self.held)
        return self.out.T, self.left


def generate(model, prompts, temperature, steps, threshold, captured=True, seed=0):
    """-> tokens [requests][steps], how many left early per request, the batch."""
    batch = Batch(model, prompts, temperature, steps, threshold, seed)
    if captured and steps > 2:
        batch.step()  # (once eagerly: what is set up at the first call is not captured)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            batch.step()
        for _ in range(steps - 1):
            graph.replay()
    else:
        for _ in range(steps):
            batch.step()
    tokens, left = batch.finish()
    return tokens, left, batch


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--seqs", type=int, default=6)
    ap.add_argument("--threshold", type=float, default=0.02)
    ap.add_argument("--eager", action="store_true")
    args = ap.parse_args()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, VOCAB, (5 + 11 * i,), generator=g).cuda() for i in range(args.seqs)]
    temperature = torch.linspace(0, 1.2, args.seqs).cuda()
    tokens, left, batch = generate(Decoder(), prompts, temperature, args.steps, args.threshold, not args.eager)
    for i in range(args.seqs):
        print(f"request {i}: prompt {len(prompts[i])}, temperature {float(temperature[i]):.2f}, {int(left[i])} of {args.steps} tokens left at layer "
              f"{EXIT}: {tokens[i, :12].tolist()} ...")
    batch.cache.close()


if __name__ == "__main__":
    main()
