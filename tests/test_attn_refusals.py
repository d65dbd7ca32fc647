"""CPU-only: calls of the attention library that are refused before anything is launched (the pointers are never followed)."""
import pytest

import paper_2206_14148_amd as A
from paper_2206_14148_amd import attn

GB = 10 ** 9
D = 64


def meet(rows, heads, ld, hs):
    at = [i * ld + h * hs for i in range(rows) for h in range(heads)]
    at.sort()
    return any(b - a < D for a, b in zip(at, at[1:]))


@pytest.mark.parametrize("rows,heads,ld,hs", [
    (2, 2, 64, 64), (5, 2, 64, 256), (5, 3, 64, 192), (3, 4, 192, 64), (4, 2, 128, 192 + 32), (7, 5, 320, 256 + 64), (100, 16, 1000, 3000),
    (1000, 2, 64, 64 * 999), (9, 3, 64, 64 * 3), (3, 2, 100, 150), (1 << 20, 2, 64, 1 << 25), (65, 65, 65, 64)])
def test_outputs_whose_heads_lie_on_each_others_rows(rows, heads, ld, hs):
    if rows < 2000:
        assert meet(rows, heads, ld, hs)
    lib, bad = attn._load(), A.KNN_ERR_INVALID_ARG
    fine, out = attn.RowsStruct(0x1000, 1 << 20, D), attn.RowsStruct(0x1000, ld, hs)
    heads_first = attn.RowsStruct(0x1000, D, 1 << 40)
    o = attn.OptionsStruct(dtype=0, causal=1, scale=0.1, cap=0.0, docs=1)
    ws, limit = (0x1000, 1 << 50), 1 << 50
    assert lib.attn_apply(fine, fine, fine, rows, 5, heads, heads, D, o, limit, *ws, out, None, None) == bad
    for which in range(3):
        grads = [heads_first, heads_first, heads_first]
        grads[which] = out
        n, m = (rows, 5) if which == 0 else (5, rows)
        assert lib.attn_grad(fine, fine, fine, fine, 0x1000, fine, n, m, heads, heads, D, o, limit, *ws, *grads, None) == bad
    cache = attn.CacheStruct(0x1000, 0x1000, 0x1000, 0x1000, 10, heads, D, 16, 0)
    if rows < 65536:
        assert lib.attn_cache_apply(cache, 0, fine, 1, rows, heads, 0x1000, 4, 0x1000, 0.1, 0.0, None, limit, *ws, out, None) == bad
    assert lib.attn_cache_apply(cache, 0, fine, rows, 1, heads, 0x1000, 4, 0x1000, 0.1, 0.0, None, limit, *ws, out, None) == bad


def test_appends_of_more_heads_than_a_cache_can_be_read_with():
    lib, rows = attn._load(), attn.RowsStruct(0x1000, 1 << 30, D)
    for heads in (65536, 1 << 27):
        cache = attn.CacheStruct(0x1000, 0x1000, 0x1000, 0x1000, 10, heads, D, 16, 0)
        assert lib.attn_cache_append(cache, 0, rows, rows, 1, 0x1000, None) == A.KNN_ERR_UNSUPPORTED
