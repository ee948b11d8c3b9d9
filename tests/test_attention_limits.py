"""Windows as long as the sequence or far longer, up to the largest the argument takes (GPU): they hide nothing."""

import pytest
import torch

from tests import _attention_ref as ref
from tests.test_attention import BF, F16, Filled, attend_cache, cache_rows, check, i32, i64, make, windowed

pytestmark = pytest.mark.gpu
LARGE = [2 ** 31 - 1, 2 ** 31 - 64, 2 ** 30]

KEYS = [
    # T, S, q_len, k_len
    (100, 100, None, None),                               # a last tile that is not full
    (16, 100, None, None),
    (8, 100, None, None),                                 # few rows: tiles of 32 keys
    (130, 130, None, None),
    (40, 30, [40, 20], [30, 5]),                          # more queries than keys: the first are before position 0
    (150, 70, [150, 100], [70, 65]),
]


@pytest.mark.parametrize("causal", [True, False], ids=["chain", "block"])
@pytest.mark.parametrize("case", KEYS, ids=[f"{c[0]}-{c[1]}" for c in KEYS])
def test_windows_past_every_key(case, causal):
    T, S, q_len, k_len = case
    q, k, v = make((2, T, 4, 64), BF, 1), make((2, S, 2, 64), BF, 2), make((2, S, 2, 64), BF, 3)
    ql, kl = q_len or [T] * 2, k_len or [S] * 2
    lens = (q_len and i32(q_len), k_len and i32(k_len))
    rows = list(ref.window_reference(q, k, v, 0, 0, causal, 0.125, ql, kl))
    for window in LARGE:
        for sinks in (0, 3, 2 ** 31 - 1):
            for workspace in (True, False):
                out, lse = windowed(q, k, v, *lens, window, sinks, causal, workspace=workspace)
                check(rows, out, lse, untouched=7.0)


@pytest.mark.parametrize("causal", [True, False], ids=["chain", "block"])
@pytest.mark.parametrize("T,S", [(100, 100), (7, 100), (40, 30)])
def test_windows_around_the_length(T, S, causal):
    q, k, v = make((1, T, 2, 128), F16, 1), make((1, S, 2, 128), F16, 2), make((1, S, 2, 128), F16, 3)
    for window in (S - 2, S - 1, S, S + 1, S + T):
        rows = ref.window_reference(q, k, v, window, 0, causal, 128 ** -0.5, [T], [S])
        check(rows, *windowed(q, k, v, None, None, window, 0, causal))


@pytest.mark.parametrize("T", [20, 100, 200])
@pytest.mark.parametrize("order", ["chain", "block"])
def test_windows_past_every_key_of_a_cache(order, T):
    f = Filled(2, 2, 64, [190, 3], BF)
    q, k, v = make((2, T, 4, 64), BF, 5), make((2, T, 2, 64), BF, 6), make((2, T, 2, 64), BF, 7)
    reach = 64 * f.table.shape[1] + T                     # positions are below it
    for window in LARGE + [reach, reach - 1, 189 + T, 100 + T]:
        rows = cache_rows(f, q, k, v, order, None, window, 2)
        for workspace in (True, False):
            out, lse = attend_cache(f, q, k, v, order, None, window, 2, workspace=workspace)
            check(rows, out, lse)


@pytest.mark.parametrize("T", [3, 100])
def test_scores_through_windows_past_every_key(T):
    f = Filled(2, 2, 64, [190, 3], BF)
    q, k, v = make((2, T, 4, 64), BF, 5), make((2, T, 2, 64), BF, 6), make((2, T, 2, 64), BF, 7)
    _, lse = attend_cache(f, q, k, v, "chain", None, 0, 0)
    old = torch.rand((2, 2, f.table.shape[1] * 64), generator=torch.Generator().manual_seed(1)).cuda()
    want = torch.zeros_like(old)
    f.cache.score(q, f.table, i64(f.ctx), lse, old, want)
    for window in LARGE:
        got = torch.zeros_like(old)
        f.cache.score(q, f.table, i64(f.ctx), lse, old, got, window=window, sinks=1)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("T", [3, 40])
def test_scales_and_inputs_that_cancel(T):
    """Powers of two moved between the scale and the inputs change nothing, as far as the products stay finite."""
    q, k, v = make((1, T, 4, 64), BF, 1), make((1, 200, 2, 64), BF, 2), make((1, 200, 2, 64), BF, 3)
    want, wl = windowed(q, k, v, None, None, 0, 0, True, scale=0.125)
    check(ref.window_reference(q, k, v, 0, 0, True, 0.125, [T], [200]), want, wl)
    for up in (20, 50, 57, -40):
        out, lse = windowed(q * 2.0 ** up, k * 2.0 ** up, v, None, None, 0, 0, True, scale=0.125 * 2.0 ** (-2 * up))
        assert torch.equal(out, want) and torch.equal(lse, wl), up


def test_a_scale_of_zero_weighs_all_keys_alike():
    """... whatever their products are."""
    q, k, v = (make((1, 20, 2, 64), BF, s) for s in (1, 2, 3))
    for up in (0, 50):
        rows = list(ref.window_reference(q, k, v, 0, 0, True, 0.0, [20], [20]))
        check(rows, *windowed(q * 2.0 ** up, k * 2.0 ** up, v, None, None, 0, 0, True, scale=0.0))
