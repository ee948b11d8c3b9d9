"""Eviction writes no array that it reads, and none twice: such calls are refused before anything is enqueued (CPU)."""

import ctypes

import pytest

from paper_2606_01813_amd import _lib
from tests.test_attention_checks import INVALID, _c_cache

WRITTEN = ("new_scores", "new_len", "kept", "workspace", "pages")


def sizes():
    """Bytes of the arrays of a call for 2 sequences of 2 kv heads.  (No device is touched: every call is refused.)"""
    need = _lib.lib().caddtree_evict_workspace_bytes(ctypes.byref(_c_cache()), 2, 300, 20000)
    return dict(page_table=2 * 300 * 4, ctx_len=16, scores=4 * 20000 * 4, new_table=2 * 3 * 4, new_scores=4 * 192 * 4, new_len=16,
                kept=4 * 150 * 4, workspace=need, pages=9 * 2 * 68 * 64)


def apart():
    at, end = {}, 1 << 20
    for n, size in sizes().items():
        at[n] = end
        end += (size + 4095) // 4096 * 4096 + 4096
    return at


PAIRS = [(w, o) for w in WRITTEN for o in ("page_table", "ctx_len", "scores", "new_table") + WRITTEN if o != w]


def call(**at):
    """The status of an eviction with its arrays apart but for these."""
    at = dict(apart(), **at)
    c, lib = _c_cache(pages=at["pages"]), _lib.lib()
    status = lib.caddtree_cache_evict(
        ctypes.byref(c), 2, at["page_table"], 300, at["ctx_len"], at["scores"], 20000, 150, 4, 9, at["new_table"], 3,
        at["new_scores"], 192, at["new_len"], at["kept"], at["workspace"], sizes()["workspace"], None)
    return status, lib.caddtree_last_error().decode()


@pytest.mark.parametrize("written,other", PAIRS, ids=["-".join(p) for p in PAIRS])
def test_a_written_array_is_no_other(written, other):
    at, size = apart(), sizes()
    for place in (at[other], at[other] + size[other] - 4, at[other] + 4 - size[written]):
        step = 256 if written in ("workspace", "pages") else 4
        # a place of the written array's alignment that still reaches into the other
        place = place // step * step if place >= at[other] else -(-place // step) * step
        if place >= at[other] + size[other] or place + size[written] <= at[other]:
            continue
        status, message = call(**{written: place})
        assert status == INVALID and message.endswith(" overlap"), (place, message)
        assert written in {n.replace("the cache's ", "") for n in message.removesuffix(" overlap").split(" and ")}, message


def test_new_pages_are_of_another_table():
    status, message = call(new_table=apart()["page_table"])
    assert status == INVALID and "new_table" in message
