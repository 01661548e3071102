"""The operators for prompts and drafts together, as a small model uses them, against the same model without a cache."""
import importlib.util
import os

import pytest
import torch

import paper_2608_12573_b200 as profk
from paper_2608_12573_b200 import _build

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    _build.build()
    profk.lib()
    spec = importlib.util.spec_from_file_location("prompted_generation", os.path.join(ROOT, "examples", "prompted_generation.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _wide(model):
    """The model's logits in 64 bits, from formulas of this file's own."""
    def logits(sequence):
        x = model.embed.double()[sequence]
        t, half = len(sequence), model.frequencies.numel()
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), torch.arange(t, device="cuda").double()[:, None] * model.frequencies)[:, None]

        def turned(a):
            pairs = a[..., :2 * half].unflatten(-1, (half, 2)) if model.interleaved else a[..., :2 * half].unflatten(-1, (2, half)).transpose(-1, -2)
            w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            return torch.cat([(w if model.interleaved else w.transpose(-1, -2)).flatten(-2), a[..., 2 * half:]], -1)

        for n in range(model.layers):
            joint = (x @ model.qkv[n].double().t()).unflatten(-1, (-1, model.dim))
            q, k, v = joint.split([model.heads, model.kv_heads, model.kv_heads], 1)
            q, k = turned(q).unflatten(1, (model.kv_heads, -1)), turned(k)
            z = torch.einsum("tkgd,skd->kgts", q, k) * model.dim ** -0.5
            p = torch.softmax(z.masked_fill(torch.ones(t, t, dtype=torch.bool, device="cuda").triu(1), float("-inf")), -1)
            x = x + torch.einsum("kgts,skd->tkgd", p, v).reshape(t, -1) @ model.o[n].double().t()
        return x @ model.unembed.double().t()
    return logits


# Activations are rounded to bf16 six times a layer (2^-9 relative each) and the logits, of some units, once: with two layers a
# logit may be off by a few times 2^-8 of values around 10.
NEAR = 0.25


@pytest.mark.parametrize("lengths,part,page,interleaved", [([1], 64, 16, False), ([5, 130, 64, 1], 64, 16, False), ([40, 3], 7, 5, True), ([300, 17], 1000, 32, True)])
def test_prompts_in_parts_give_the_model_s_logits(example, lengths, part, page, interleaved):
    model = example.Decoder(1009, interleaved=interleaved, seed=len(lengths))
    g = torch.Generator()
    g.manual_seed(part)
    prompts = [torch.randint(0, 1009, (n,), generator=g).tolist() for n in lengths]
    with torch.no_grad():
        cache = example.Cache(model, len(prompts), max(lengths) + 3, page)
        got = example.read_prompts(model, prompts, cache, part)
        for i, p in enumerate(prompts):
            assert (got[i].double() - _wide(model)(torch.tensor(p, device="cuda"))[-1]).abs().max() < NEAR
    assert int(cache.missing) == 0 and cache.lengths.tolist() == lengths


def test_generation(example):
    model = example.Decoder(1009, seed=3)
    g = torch.Generator()
    g.manual_seed(1)
    prompts = [torch.randint(0, 1009, (n,), generator=g).tolist() for n in (20, 3, 77)]
    allowed = torch.arange(1009) % 3 != 0
    words = torch.zeros(32, dtype=torch.int64)
    words.scatter_add_(0, torch.arange(1009) // 32, allowed.long() << (torch.arange(1009) % 32))
    mask = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).cuda()
    repetition, presence, steps = 1.5, 0.5, 9
    with torch.no_grad():
        tokens, lengths, cache, seen = example.generate(model, prompts, steps, part=16, repetition=repetition, presence=presence, mask=mask)
        for i, p in enumerate(prompts):
            sequence = tokens[i, :int(lengths[i])]
            assert sequence[:len(p)].tolist() == p and len(sequence) == len(p) + steps
            raw = _wide(model)(sequence)
            for s in range(steps):
                held = sequence[:len(p) + s]
                want = raw[len(p) + s - 1].clone()
                once = torch.unique(held)
                want[once] = torch.where(want[once] > 0, want[once] / repetition, want[once] * repetition)
                want[torch.unique(held[len(p):])] -= presence
                want[~allowed.cuda()] = float("-inf")
                got = seen[s, i].double()
                assert torch.equal(torch.isneginf(got), torch.isneginf(want))
                assert (got - want)[allowed.cuda()].abs().max() < NEAR * repetition
                assert int(sequence[len(p) + s]) == int(torch.argmax(got))          # (ties go to the lowest token)


def test_drafts_are_checked_as_single_tokens_are(example):
    """The logits behind several drafted tokens at once are those of the same tokens one by one, and leave the cache as it was."""
    model = example.Decoder(1009, seed=5)
    prompts = [[1, 2, 3, 4, 5], list(range(100, 161))]
    drafts = torch.tensor([[9, 8, 7, 6], [11, 12, 13, 14]], device="cuda")
    with torch.no_grad():
        cache = example.Cache(model, 2, 70)
        example.read_prompts(model, prompts, cache, 32)
        held, pool = cache.lengths.clone(), cache.pool.clone()
        together = example.check_drafts(model, cache, drafts)
        again = example.Cache(model, 2, 70)
        again.pool.copy_(pool)
        again.tables, again.lengths = cache.tables, held
        for t in range(4):
            again.lengths = again.lengths + 1
            one = model.logits(model.hidden(drafts[:, t].contiguous(), again.pool, again.tables, again.lengths))
            assert (one.float() - together[:, t].float()).abs().max() < NEAR
            for i, p in enumerate(prompts):
                want = _wide(model)(torch.tensor(p + drafts[i, :t + 1].tolist(), device="cuda"))[-1]
                assert (together[i, t].double() - want).abs().max() < NEAR
        assert torch.equal(cache.lengths, held)


def test_the_training_form_has_the_cache_s_logits_and_the_formula_s_gradients(example):
    model = example.Decoder(211, layers=1, heads=4, kv_heads=2, dim=32, seed=7, dtype=torch.float32)
    sequences = torch.randint(0, 211, (3, 20), generator=torch.Generator().manual_seed(2)).cuda()
    with torch.no_grad():
        for s in sequences:
            assert (model.dense_logits(s[None])[0].double() - _wide(model)(s)).abs().max() < 1e-3
    weights = [model.qkv[0], model.o[0], model.unembed, model.embed]
    for w in weights:
        w.requires_grad_(True)
    loss = model.loss(sequences)
    grads = torch.autograd.grad(loss, weights)
    wide = _wide(model)
    plain = -torch.stack([torch.log_softmax(wide(s[:-1]), -1).gather(1, s[1:, None]) for s in sequences]).mean()
    # 32-bit sums of a few hundred products of order one: 2^-24 * 2^9 relative, and the loss likewise
    assert abs(float(loss.detach()) - float(plain.detach())) < 1e-4
    for got, want in zip(grads, torch.autograd.grad(plain, weights)):
        assert (got.double() - want).norm() < 1e-4 * want.norm()


def test_the_example_runs(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["prompted_generation.py", "--prompts", "2", "--steps", "3", "--vocab", "503"])
    example.main()
    assert capsys.readouterr().out.count("prompt of") == 2
