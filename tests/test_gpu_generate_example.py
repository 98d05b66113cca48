"""The generation example: the operators together against a plain fp32 decoder, and tokens generated in bubbles."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from examples import generate_in_bubbles as example      # noqa: E402


def _rotate(x, cos, sin):
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain(model, tokens):
    """Logits behind the last of `tokens` (the prompt included), fp32 throughout, one sequence."""
    n = tokens.shape[0]
    x = model.embed[tokens].float()
    half = model.head_dim // 2
    cos, sin = model.rotary[:n, None, :half], model.rotary[:n, None, half:]
    norm = lambda y: y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-5)
    hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
    for layer in model.layers:
        qkv = (norm(x) @ layer["qkv"].float().t()).view(n, model.qkv_heads, model.head_dim)
        q, k, v = qkv.split([model.q_heads, model.kv_heads, model.kv_heads], 1)
        q, k = _rotate(q, cos, sin), _rotate(k, cos, sin)
        out = []
        for h in range(model.q_heads):
            g = h // (model.q_heads // model.kv_heads)
            s = (q[:, h] @ k[:, g].t()) / math.sqrt(model.head_dim)
            out.append(torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ v[:, g])
        x = x + torch.cat(out, 1) @ layer["out"].float().t()
        x = x + torch.nn.functional.gelu(norm(x) @ layer["up"].float().t()) @ layer["down"].float().t()
    return (norm(x) @ model.unembed.float().t())[-1]


def test_steps_follow_a_plain_decoder():
    model = example.Decoder(batch=256, prompt=256, new=20, seed=3)
    model.prefill()
    worst = 0.0
    for i in range(20):                                 # (a page ends inside)
        before = model.tokens.clone()
        current = model.current.clone()
        model.step()
        torch.cuda.synchronize()
        if i not in (0, 1, 15, 16, 19):
            continue
        for b in (0, 77, 255):
            tokens = torch.cat([model.prompt, model.first[b:b + 1], before[:i, b].long()])
            assert tokens[-1] == current[b]
            want, got = _plain(model, tokens), model.logits[b].float()
            # activations are rounded to 8 significant bits some ten times a layer: each 2^-9 of their size, 2 layers
            worst = max(worst, float((got - want).norm() / want.norm()))
            assert worst <= 2 * 10 * 2.0 ** -9
    assert int(model.done) == 20 and int((model.tokens < 0).sum()) == 0


def test_a_replayed_step_is_the_step():
    model = example.Decoder(new=12, seed=4)
    model.prefill()
    for _ in range(12):
        model.step()
    torch.cuda.synchronize()
    want = model.tokens.clone()
    assert len(set(want[:, 0].tolist())) > 1
    model.reset()
    model.capture()
    for _ in range(2):                                  # replays, twice over, other work between them
        model.reset()
        for i in range(12):
            model.graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(model.tokens[:i + 1], want[:i + 1]), i


def test_tokens_generated_in_bubbles_are_those_generated_outside():
    model = example.Decoder(new=24, seed=5)
    model.prefill()
    model.capture()
    want, step_ns = example.standalone(model)
    got, progress, bubble_ns = example.harvest(model, step_ns, epochs=10)
    assert progress.steps == 24 and progress.runs_completed == 1 and progress.work_units_done == 24 * model.batch
    assert bubble_ns > 0
    assert torch.equal(got, want)
