"""The example that runs the cache's calls together: with room for everything it answers as attention over all tokens, cut it stays near."""
import importlib.util
import os

import pytest
import torch

from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "bounded_cache.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("bounded_cache", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


SIZE = dict(batch=2, heads=4, heads_kv=2, dim=64, prompt=150, chunk=60, tokens=20, slack=8, grid=4)


def full_attention(example, s):
    """The same draws, turned by the oracle, through a softmax over every token so far."""
    g = torch.Generator(device="cuda").manual_seed(0)
    pairs = s["dim"] // 2
    sections = (pairs // 4, pairs * 3 // 8, pairs - pairs // 4 - pairs * 3 // 8)
    inv = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().numpy()
    ks, vs, want = [], [], []
    steps = [(b, min(s["chunk"], s["prompt"] - b)) for b in range(0, s["prompt"], s["chunk"])] + [(s["prompt"] + t, 1) for t in range(s["tokens"])]
    for first, n in steps:
        q, k, v = (torch.randn(s["batch"], h, n, s["dim"], generator=g, device="cuda").bfloat16() for h in (s["heads"], s["heads_kv"], s["heads_kv"]))
        pos = example.positions(first, n, s["grid"]).expand(s["batch"], -1, -1).cpu().numpy()
        turn = lambda x: torch.from_numpy(co.rotary(x.double().cpu().numpy(), pos, inv, sections))
        ks.append(turn(k))
        vs.append(v.double().cpu())
        if first + n >= s["prompt"]:
            group = s["heads"] // s["heads_kv"]
            key, val = (torch.cat(x, 2).repeat_interleave(group, 1) for x in (ks, vs))
            p = torch.softmax(turn(q)[:, :, -1:] @ key.transpose(2, 3) * s["dim"] ** -0.5, -1)
            want.append(p @ val)
    return torch.cat(want, 2)


def test_with_room_for_everything(example):
    out, lens, kept = example.serve(budget=400, **SIZE)
    assert lens.tolist() == [170, 170]
    assert kept[0, 1, :150].tolist() == list(range(150)) and (kept[:, :, 150:] == -1).all()
    want = full_attention(example, SIZE)
    got = out.double().cpu()
    # keys and queries are rounded to bf16 after their turn: scores within 2^-8 of about |q||k| / sqrt(D), so outputs within a few 2^-8
    assert torch.all((got - want).abs() <= 3e-2 + 2.0 ** -7 * want.abs())
    assert float((got - want).norm() / want.norm()) <= 1e-2


def test_cut_to_a_budget(example):
    out, lens, kept = example.serve(budget=64, **SIZE)
    assert bool(torch.isfinite(out).all()) and int(lens.max()) <= 64 + SIZE["slack"]
    assert kept.shape == (2, 2, 64) and (kept[:, :, 1:] > kept[:, :, :-1]).all() and kept[..., :4].tolist() == [[[0, 1, 2, 3]] * 2] * 2
    again, _, _ = example.serve(budget=64, **SIZE)
    assert torch.equal(out, again)
