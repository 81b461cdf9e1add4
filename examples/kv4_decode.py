"""Early-exit decoding of a batch over the 4-bit cache, with every length on the GPU.

A small decoder (random weights, rotary positions, heads that share K and V) with one exit in the middle.  A step runs the layers up
to the exit for each request's new token.  Requests whose token is confident enough leave there; the K and V that the deeper
layers lack for it are filled in later, when a token of the same request goes through (KV recomputation).  Which requests
leave, how many rows the deeper layers get and where they go is decided on the GPU: the host enqueues the same calls at every
step and reads nothing back until the end.

    python examples/kv4_decode.py [--steps 32] [--seqs 6] [--threshold 0.02]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2312_04916_amd as ee  # noqa: E402

LAYERS, EXIT, D, HEADS, KV_HEADS, HD, VOCAB = 4, 2, 256, 8, 2, 64, 512
CAP = 4  # tokens of a request that may wait for the deeper layers; one more goes through whatever its confidence


class Decoder:
    def __init__(self, seed=0):
        g = torch.Generator(device="cuda:0").manual_seed(seed)

        def w(*shape):
            return (torch.randn(*shape, device="cuda:0", generator=g) / math.sqrt(shape[-1])).to(torch.bfloat16)

        self.embed = w(VOCAB, D) * 16
        self.qkv = [w((HEADS + 2 * KV_HEADS) * HD, D) for _ in range(LAYERS)]
        self.o = [w(D, HEADS * HD) for _ in range(LAYERS)]
        self.up = [w(4 * D, D) for _ in range(LAYERS)]
        self.down = [w(D, 4 * D) for _ in range(LAYERS)]
        self.head = w(VOCAB, D) * 2
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
            qkv = (self.norm(x) @ self.qkv[i].T).view(n, HEADS + 2 * KV_HEADS, HD)
            q = self.rotate(qkv[:, :HEADS], pos)
            cache.append(i, self.rotate(qkv[:, HEADS:HEADS + KV_HEADS], pos), qkv[:, HEADS + KV_HEADS:])
            x = x + cache.attend(i, q).view(n, HEADS * HD) @ self.o[i].T
            x = x + torch.nn.functional.silu(self.norm(x) @ self.up[i].T) @ self.down[i].T
        return x

    def logits(self, x):
        return self.norm(x).float() @ self.head.float().T


def generate(model, prompts, steps, threshold, block=32):
    """-> tokens [requests][steps], how many left early per request, the cache."""
    n = len(prompts)
    lens = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda:0")
    most = max(len(p) for p in prompts) + steps + 1
    n_blocks = sum(-(-(len(p) + steps + 1) // block) for p in prompts)
    total = sum(len(p) for p in prompts)
    cache = ee.Kv4Cache(LAYERS, HEADS, KV_HEADS, HD, block, n_blocks, n, most, max(total, n * (CAP + 1)))
    zero = torch.zeros_like(lens)
    ids = torch.arange(n, device="cuda:0")

    # prompts: every position through every layer
    cache.plan(zero, zero, lens, total)
    x = model.layers(cache, range(LAYERS), model.embed[torch.cat(prompts)])
    token = model.logits(x[cache.row_start[1:n + 1].long() - 1]).argmax(-1)

    held = lens.clone()   # positions whose K and V the first layers have
    deep = lens.clone()   # ... and all layers
    waiting = torch.zeros(n, CAP + 1, D, dtype=torch.bfloat16, device="cuda:0")  # hidden states at the exit, by position
    out, left = [], torch.zeros(n, dtype=torch.int32, device="cuda:0")
    for _ in range(steps):
        out.append(token)
        end = held + 1
        cache.plan(held, held, end, n, 1)
        x = model.layers(cache, range(EXIT), model.embed[token])
        waiting[ids, held.long() % (CAP + 1)] = x
        probability, early = torch.softmax(model.logits(x), -1).max(-1)
        leaves = (probability >= threshold) & (end - deep <= CAP)
        # the others' rows: what waits, and the new one.  There is room for as many as there can be; the rest belong to no request.
        start = torch.where(leaves, end, deep)
        cache.plan(end, start, end, n * (CAP + 1), CAP + 1)
        rows = n * (CAP + 1)
        seq, pos = cache.row_seq[:rows].long().clamp_min(0), cache.positions[:rows].long().clamp_min(0)
        y = model.layers(cache, range(EXIT, LAYERS), waiting[seq, pos % (CAP + 1)])
        last = (cache.row_start[1:n + 1].long() - 1).clamp_min(0)
        token = torch.where(leaves, early, model.logits(y[last]).argmax(-1))
        left += leaves.int()
        deep = torch.where(leaves, deep, end)
        held = end
    # whoever still waits goes through, so that every layer holds every position
    cache.plan(held, deep, held, n * (CAP + 1), CAP + 1)
    seq, pos = cache.row_seq[:rows].long().clamp_min(0), cache.positions[:rows].long().clamp_min(0)
    model.layers(cache, range(EXIT, LAYERS), waiting[seq, pos % (CAP + 1)])
    return torch.stack(out, 1), left, cache


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--seqs", type=int, default=6)
    ap.add_argument("--threshold", type=float, default=0.02)
    args = ap.parse_args()
    model = Decoder()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, VOCAB, (5 + 11 * i,), generator=g).cuda() for i in range(args.seqs)]
    tokens, left, cache = generate(model, prompts, args.steps, args.threshold)
    for i in range(args.seqs):
        print(f"request {i}: prompt {len(prompts[i])}, {int(left[i])} of {args.steps} tokens left at layer {EXIT}: {tokens[i, :12].tolist()} ...")
    held = 2 * LAYERS * KV_HEADS * HD * sum(len(p) + args.steps for p in prompts)
    print(f"cache: {held * 17 // 32} bytes hold what bf16 would in {held * 2}; {int(cache.n_free)} blocks free")
    cache.close()


if __name__ == "__main__":
    main()
