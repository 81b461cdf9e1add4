"""The example that decodes over the 4-bit cache (examples/kv4_decode.py): whatever leaves early, the cache ends up holding what one
pass over the same tokens leaves in it, for every layer and position, and without exits the tokens are those of full passes."""
import importlib.util
import os

import pytest
import torch

import paper_2312_04916_amd as ee

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("kv4_decode", os.path.join(ROOT, "examples", "kv4_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def whole_pass(ex, model, sequences, block=32):
    """Every position of the sequences through every layer at once -> hidden states, the cache."""
    n, lens = len(sequences), [len(s) for s in sequences]
    cache = ee.Kv4Cache(ex.LAYERS, ex.HEADS, ex.KV_HEADS, ex.HD, block, sum(-(-a // block) for a in lens), n, max(lens), sum(lens))
    zero = torch.zeros(n, dtype=torch.int32, device="cuda:0")
    cache.plan(zero, zero, torch.tensor(lens, dtype=torch.int32, device="cuda:0"), sum(lens))
    return model.layers(cache, range(ex.LAYERS), model.embed[torch.cat(sequences)]), cache


@pytest.mark.parametrize("threshold", [1.1, 0.0, 0.02])
def test_the_cache_holds_what_one_pass_leaves(threshold):
    ex = load()
    model = ex.Decoder()
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(0, ex.VOCAB, (k,), generator=g).cuda() for k in (1, 7, 30, 64)]
    steps = 14
    tokens, left, cache = ex.generate(model, prompts, steps, threshold)
    if threshold > 1:
        assert not left.any()
    elif threshold == 0:
        assert (left == steps - steps // (ex.CAP + 1)).all()  # one in CAP + 1 goes through
    sequences = [torch.cat([p, t]) for p, t in zip(prompts, tokens)]
    _, want = whole_pass(ex, model, sequences)
    for i, s in enumerate(sequences):
        p = torch.arange(len(s), device="cuda:0")
        at, at_w = (c.table[i, p // 32].long() * 32 + p % 32 for c in (cache, want))
        for layer in range(ex.LAYERS):
            for got, ref in zip(cache.read(layer, at), want.read(layer, at_w)):
                # the projections' products may be summed in another order for another number of rows, which moves a value by
                # bf16 steps, and near the middle between two levels the level: all but a few agree, and none by more than
                # half of its group's largest
                d = (got.float() - ref.float()).abs()
                assert (d > 0).float().mean() < 0.25, (i, layer, (d > 0).float().mean())
                top = ref.float().abs().view(*ref.shape[:-1], -1, 32).amax(-1, keepdim=True).expand(-1, -1, -1, 32).reshape(ref.shape)
                assert (d <= 0.5 * top + 1e-6).all(), (i, layer)
    if threshold > 1:
        # greedy choice of the whole pass at each generated position, wherever its two best are apart
        hidden, _ = whole_pass(ex, model, sequences)
        at = 0
        for p, t in zip(prompts, tokens):
            z = model.logits(hidden[at + len(p) - 1:at + len(p) + steps - 1])
            best, arg = z.topk(2, -1)
            apart = best[:, 0] - best[:, 1] > 0.25 * z.std()
            assert apart.any() and (arg[apart, 0] == t[apart]).all()
            at += len(p) + steps
    cache.close()
    want.close()
