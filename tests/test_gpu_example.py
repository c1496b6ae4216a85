"""The example that serves a small model with the 4-bit cache: the same tokens
all at once and one by one, and what is left in the cache at the end."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("serve_4bit_cache", os.path.join(ROOT, "examples", "serve_4bit_cache.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_serving_run(example):
    import torch
    model, cache, text, said, live = example.run(layers=2, prompts=(150, 37), tokens=9, continuations=3)
    assert [t.shape[0] for t in text] == [159, 46] and [len(s) for s in said] == [10] * 3
    # left: the first prompt (159 tokens, three pages, the last one its own again) and a
    # continuation of it (its own third page)
    assert cache.length.tolist() == [159, 0, 168, 0, 0, 0, 0, 0]
    assert live == 4 and sorted(cache.refs.tolist(), reverse=True)[:5] == [2, 2, 1, 1, 0]
    assert cache.refs[:4].min().item() >= 1 and not cache.refs[4:].any().item()


def test_all_at_once_and_one_by_one(example):
    """The logits of a prompt given at once and token by token: the same cache
    contents up to fp16 roundings in front of the rounding to 4 bits, so nearly
    the same direction."""
    import torch
    from paper_2609_09240_gb300 import tq
    model = example.Model(layers=2)
    tokens = torch.randint(0, 8192, (40,), device="cuda")
    cache = tq.Kv4Cache.empty(2, 8, model.kv_heads, model.dim, slots=2, max_pages=4)
    whole = model.step(cache, example.int32([0]), example.int32([40]), tokens, 40)
    for t in range(40):
        single = model.step(cache, example.int32([1]), example.int32([1]), tokens[t:t + 1], 1)
    cache.check()
    assert torch.isfinite(whole).all() and torch.isfinite(single).all()
    assert float(torch.nn.functional.cosine_similarity(whole, single).item()) > 0.99
