"""Calls on logits that the other tests do not make."""

import pytest
import torch

from paper_2606_01813_amd import adjust_logits, distill, distill_grad, verify_tree
from tests import _logits_ref as ref
from tests.test_logits_checks import rec  # noqa: F401  (a fixture)

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
I32 = torch.int32


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", [BF, F16, F32])
def test_a_tree_of_its_root_alone(dtype, in_place):
    """cap = 0: count's nodes are none, and the root's row is adjusted as every tree's is."""
    B, V = 3, 700
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.randn((B, 1, V), generator=gen, device="cuda") * 3).to(dtype)
    kw = dict(history=torch.randint(V, (B, 40), generator=gen, device="cuda", dtype=I32), repetition=torch.full((B,), 1.5, device="cuda"),
              frequency=torch.full((B,), 0.25, device="cuda"), token_ids=torch.zeros((B, 0), dtype=I32, device="cuda"),
              parent=torch.zeros((B, 0), dtype=I32, device="cuda"), count=torch.tensor([0, -3, 7], dtype=I32, device="cuda"))
    want, tol = ref.adjust(ref.f64(x), dtype, **kw)
    y = x.clone()
    out = adjust_logits(y, y if in_place else torch.full_like(x, 9.0), **kw)
    assert bool((abs(ref.f64(out) - want) <= tol).all())
    acc, index, tokens = (torch.full(s, 9, dtype=I32, device="cuda") for s in ((B,), (B, 1), (B, 1)))
    verify_tree(x, kw["token_ids"], kw["parent"], kw["count"], acc, index, tokens)
    assert acc.tolist() == [1] * B and index.flatten().tolist() == [0] * B
    assert tokens.flatten().tolist() == x[:, 0].float().argmax(-1).tolist()


def test_a_tree_of_its_root_alone_has_no_count(rec):  # noqa: F811
    """Empty arrays have no address: the library would take the call for one without a tree, whose rows are `count`."""
    x, none, n = torch.zeros((2, 1, 70), dtype=BF), torch.zeros((2, 0), dtype=I32), torch.zeros(2, dtype=I32)
    adjust_logits(x, x, token_ids=none, parent=none, count=n)
    adjust_logits(x, x, count=n)
    (_, (with_tree, _)), (_, (without, _)) = rec.calls
    assert n.data_ptr() not in with_tree and n.data_ptr() in without
    with pytest.raises(TypeError):
        adjust_logits(x, x, token_ids=none, parent=none, count=n.long())


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,V", [(1, 3, 50), (1, 3, 20000), (70, 9, 3000), (40, 15, 70000)])
@pytest.mark.parametrize("dtype", [BF, F16, F32])
def test_no_nan_is_chosen_signalling_or_quiet(B, T, V, dtype):
    """NaNs of every kind, next to the largest logit, before it and after it."""
    from paper_2606_01813_amd import verify_workspace
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((B, T, V), generator=gen, device="cuda").to(dtype)
    at = torch.randint(V - 2, (B, T), generator=gen, device="cuda") + 1
    x.scatter_(2, at[..., None], 50.0)
    bits = {BF: (torch.int16, [0x7f81, -0x7f, 0x7fc0, -0x40, 0x7fbf]), F16: (torch.int16, [0x7c01, -0x3ff, 0x7e00, -0x200, 0x7dff]),
            F32: (torch.int32, [0x7f800001, -0x7fffff, 0x7fc00000, -0x400000, 0x7fbfffff])}[dtype]
    nan = torch.tensor(bits[1], dtype=bits[0], device="cuda").view(dtype)
    assert bool(torch.isnan(nan).all())
    raw = x.view(bits[0])
    for i in range(5):
        raw[:, :, i::11] = bits[1][i]
    raw.scatter_(2, at[..., None] + 1, bits[1][0])
    raw.scatter_(2, at[..., None] - 1, bits[1][0])
    x.scatter_(2, at[..., None], 50.0)
    none = torch.full((B, T - 1), -1, dtype=I32, device="cuda")
    tok = torch.zeros((B, T - 1), dtype=I32, device="cuda")
    count = torch.zeros(B, dtype=I32, device="cuda")
    for ws in (None, verify_workspace(x)):
        acc, index, tokens = (torch.full(s, 9, dtype=I32, device="cuda") for s in ((B,), (B, 1), (B, 1)))
        verify_tree(x, tok, none, count, acc, index, tokens, workspace=ws)
        assert tokens[:, 0].tolist() == at[:, 0].tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [400000, 1 << 20])
def test_a_graph_of_rows_that_take_much_lds(V):
    """Past some vocabulary a launch has to say how much LDS it takes, in a captured call too."""
    B, K = 70, 4
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((B, 1, V), generator=gen, device="cuda").to(BF)
    ids = torch.randint(V, (B, 1, K), generator=gen, device="cuda", dtype=I32)
    target = torch.randn((B, 1, K), generator=gen, device="cuda")
    loss, stats, grad, grad2 = torch.zeros((B, 1), device="cuda"), torch.zeros((B, 1, 3), device="cuda"), torch.zeros_like(x), torch.zeros_like(x)

    def call():
        distill(x, ids, target, loss, grad=grad, stats=stats)
        distill_grad(x, ids, target, stats, grad2)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        for t in (loss, stats, grad, grad2):
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (loss, stats, grad, grad2)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(g, t) for g, t in zip(got, (loss, stats, grad, grad2)))
        assert bool(torch.isfinite(loss).all()) and bool((loss > 0).all())
