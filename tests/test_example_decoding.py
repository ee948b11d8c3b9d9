"""The example of speculative decoding over the 4-bit cache writes the target's text, with and without eviction."""

import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "speculative_decoding.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("speculative_decoding", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def check_text(r, prompt):
    """The text after the prompt is the chain of successors."""
    assert int(r.length.max()) < r.text.shape[1]
    for b, n in enumerate(r.length.tolist()):
        assert torch.equal(r.text[b, prompt:n], r.target.after[r.text[b, prompt - 1:n - 1]])


def test_text_and_cache_without_eviction(example):
    r = example.run(B=3, prompt=130, rounds=8, slots=512, seed=1)
    check_text(r, 130)
    assert r.evictions == 0 and r.accepted.float().mean() > 2
    assert torch.equal(r.ctx_len + 1, r.length) and torch.equal(r.ctx_len, 130 + r.accepted.sum(0))
    # the cache holds the text's keys and values, in the order of the text: what writing them one after the other gives
    n, B = int(r.ctx_len.max()), 3
    _, k, v = r.target.qkv(r.text[:, :n])
    same = example.KVCache(r.cache.n_kv_heads, r.cache.head_dim, num_pages=r.cache.pages.shape[0])
    same.write(k, v, r.table, torch.zeros_like(r.ctx_len), count=r.ctx_len.to(torch.int32))
    got, want = ([torch.zeros((B, n, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2))
    r.cache.read(r.table, r.ctx_len, *got)
    same.read(r.table, r.ctx_len, *want)
    # (a tree's rows and a text's may come from products of different shapes: a last bit may move a code by one place)
    for g, w in zip(got, want):
        assert torch.equal(g[:, :130], w[:, :130])
        assert (g != w).float().mean() < 0.02


def test_text_with_eviction_and_window(example):
    r = example.run(B=5, prompt=300, rounds=24, seed=2)
    check_text(r, 300)
    assert r.evictions >= 1 and int(r.cached.max()) <= 512
    r = example.run(B=2, prompt=300, rounds=4, window=100, seed=3)
    check_text(r, 300)
