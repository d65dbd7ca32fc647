"""CPU-only: the attention library's symbols, plans and refusals (no GPU call is made)."""
import ctypes
import os
import re

import pytest

import paper_2206_14148_amd as A
from paper_2206_14148_amd import attn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GB = 10 ** 9


def test_the_header_and_the_library_agree_on_the_symbols():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "attn.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(attn_[a-z0-9_]+)\s*\(", text))
    assert names == set(A.ATTN_SYMBOLS)
    raw = ctypes.CDLL(A.library_path())
    for name in names:
        getattr(raw, name)


def up(v):
    return (v + 255) // 256 * 256


@pytest.mark.parametrize("n,m,hq,hkv,d", [(1, 1, 1, 1, 1), (3, 50_021, 16, 2, 128), (8192, 8192, 32, 8, 128),
                                         (100, 100_000, 4, 4, 64), (0, 5, 2, 1, 64), (5, 0, 2, 1, 64), (7, 1 << 30, 1, 1, 8)])
def test_plans_stay_under_their_limit_and_count_what_they_keep(n, m, hq, hkv, d):
    for limit in (0, 10 ** 4, 10 ** 6, GB, 1 << 40):
        p = A.attn_plan(n, m, hq, hkv, d, limit)
        assert p.workspace_bytes <= limit and p.min_limit_bytes == 0
        assert p.workspace_bytes == (up(p.n_splits * n * hq * (d + 2) * 4) if p.n_splits > 1 else 0)
        assert p.n_splits == 1 or m // p.n_splits >= 64
        least = up(8 * n * hq)
        if limit < least:
            with pytest.raises(A.KnnError) as e:
                A.attn_grad_plan(n, m, hq, hkv, d, limit)
            assert e.value.status == A.KNN_ERR_MEM_LIMIT_TOO_SMALL and e.value.min_limit_bytes == least
            continue
        g = A.attn_grad_plan(n, m, hq, hkv, d, limit)
        assert g.min_limit_bytes == least and 1 <= g.n_splits <= 256
        parts = [up(s * size * d * 4) if s > 1 else 0 for s, size in ((g.n_splits, 2 * m * hkv), (g.row_splits, n * hq))]
        assert g.workspace_bytes == least + sum(parts) <= limit and 1 <= g.row_splits <= 256


def test_shapes_that_are_refused():
    for plan in (A.attn_plan, A.attn_grad_plan):
        for shape in [(-1, 5, 1, 1, 8), (5, -1, 1, 1, 8), (5, 5, 0, 1, 8), (5, 5, 1, 0, 8), (5, 5, 3, 2, 8), (5, 5, 1, 2, 8),
                      (5, 5, 1, 1, 0)]:
            with pytest.raises(A.KnnError) as e:
                plan(*shape, GB)
            assert e.value.status == A.KNN_ERR_INVALID_ARG
        for shape in [(5, 5, 1, 1, 129), ((1 << 30) + 1, 5, 1, 1, 8), (5, (1 << 30) + 1, 1, 1, 8), (5, 5, 65536, 1, 8)]:
            with pytest.raises(A.KnnError) as e:
                plan(*shape, 1 << 60)
            assert e.value.status == A.KNN_ERR_UNSUPPORTED


def options(**other):
    o = attn.OptionsStruct(dtype=0, causal=1, scale=0.1, cap=0.0, docs=1)
    for k, v in other.items():
        setattr(o, k, v)
    return o


def call(o=None, n=4, m=4, hq=2, hkv=1, d=64, ws=0x1000, ws_bytes=1 << 30, limit=GB, lse=0x1000, grad=False, **rows):
    """Every call here is refused before anything is launched: the pointers are never followed."""
    lib = attn._load()
    t = {name: attn.RowsStruct(0x1000, 128, 64) for name in ("q", "k", "v", "out", "g", "dq", "dk", "dv")}
    t.update(rows)
    o = options() if o is None else o
    if grad:
        return lib.attn_grad(t["q"], t["k"], t["v"], t["out"], lse, t["g"], n, m, hq, hkv, d, o, limit, ws, ws_bytes,
                             t["dq"], t["dk"], t["dv"], None)
    return lib.attn_apply(t["q"], t["k"], t["v"], n, m, hq, hkv, d, o, limit, ws, ws_bytes, t["out"], lse, None)


def test_calls_that_are_refused():
    bad = [dict(dtype=2), dict(dtype=-1), dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
           dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(starts=0x1000),
           dict(k_starts=0x1000), dict(docs=2), dict(starts=0x1000, k_starts=0x1000, docs=0),
           dict(starts=0x1000, k_starts=0x1000, docs=1 << 31)]
    bad += [dict(scale=1e-30), dict(scale=1e30), dict(cap=1e-30), dict(cap=1e30)]
    null, backward = attn.RowsStruct(None, 128, 64), attn.RowsStruct(0x1000, -1, 64)
    for grad in (False, True):
        for o in bad:
            assert call(options(**o), grad=grad) == A.KNN_ERR_INVALID_ARG, o
        for name in ("q", "k", "v", "out") + (("g", "dq", "dk", "dv") if grad else ()):
            assert call(grad=grad, **{name: null}) == A.KNN_ERR_INVALID_ARG
            assert call(grad=grad, **{name: backward}) == A.KNN_ERR_INVALID_ARG
        assert call(d=129, grad=grad) == A.KNN_ERR_UNSUPPORTED
        for name in ("dq", "dk", "dv") if grad else ("out",):  # outputs whose rows or heads lie on each other
            heads = 1 if name in ("dk", "dv") else 2
            assert call(grad=grad, **{name: attn.RowsStruct(0x1000, 63, 64)}) == A.KNN_ERR_INVALID_ARG
            assert heads == 1 or call(grad=grad, **{name: attn.RowsStruct(0x1000, 128, 0)}) == A.KNN_ERR_INVALID_ARG
    # few rows, many keys: parts in the workspace
    assert call(m=100_000, ws=None) == A.KNN_ERR_INVALID_ARG
    assert call(m=100_000, ws=0x1001) == A.KNN_ERR_INVALID_ARG
    assert call(m=100_000, ws_bytes=10) == A.KNN_ERR_WORKSPACE_TOO_SMALL
    assert call(grad=True, lse=None) == A.KNN_ERR_INVALID_ARG
    assert call(grad=True, ws=None) == A.KNN_ERR_INVALID_ARG
    assert call(grad=True, ws_bytes=0) == A.KNN_ERR_WORKSPACE_TOO_SMALL
    assert call(grad=True, limit=0) == A.KNN_ERR_MEM_LIMIT_TOO_SMALL
    lib = attn._load()
    assert lib.attn_plan(4, 4, 2, 1, 64, GB, None) == A.KNN_ERR_INVALID_ARG
    assert lib.attn_apply(None, None, None, 4, 4, 2, 1, 64, options(), GB, None, 0, None, None, None) == A.KNN_ERR_INVALID_ARG
    assert lib.attn_apply(None, None, None, 4, 4, 2, 1, 64, None, GB, None, 0, None, None, None) == A.KNN_ERR_INVALID_ARG


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    torch = pytest.importorskip("torch")
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(A.KnnError) as e:
        A.attn_apply(q, q, q, GB)
    assert e.value.status == A.KNN_ERR_INVALID_ARG


def test_the_formulas_gradients_against_differences():
    """attn_formulas.py, which the kernels are held to: its gradients against central differences of its own O."""
    torch = pytest.importorskip("torch")
    from attn_formulas import attention

    gen = torch.Generator().manual_seed(3)
    n, m, hq, hkv, d = 11, 17, 2, 1, 5
    Q, K, V, dO = (torch.randn(r, h, d, generator=gen, dtype=torch.float64) for r, h in
                   ((n, hq), (m, hkv), (m, hkv), (n, hq)))
    o = dict(causal=True, cap=2.0, slopes=[0.3, 0.1], starts=[0, 4, 11], k_starts=[0, 2, 17], prefix=[1, 5])
    r = attention(Q, K, V, dO, **o)
    for which, name in enumerate(("dQ", "dK", "dV")):
        for _ in range(3):
            way = torch.randn((Q, K, V)[which].shape, generator=gen, dtype=torch.float64)
            step, value = 1e-5, []
            for side in (step, -step):
                data = [Q, K, V]
                data[which] = data[which] + side * way
                value.append(float((attention(*data, **o)["O"] * dO).sum()))
            want = float((r[name] * way).sum())
            # step^2 of a third derivative, and 2^-53 of sums of 110 terms over 2e-5
            assert abs((value[0] - value[1]) / (2 * step) - want) < 1e-7 * (1 + abs(want))


# ---- the cache ------------------------------------------------------------------------------

@pytest.mark.parametrize("batch,nq,hq,hkv,d,longest", [(1, 1, 8, 1, 128, 200_000), (64, 1, 32, 8, 128, 8192), (0, 1, 1, 1, 64, 100),
                                                      (4, 3, 8, 4, 64, 512), (1, 1, 1, 1, 1, 0), (1, 1, 1, 1, 8, 1 << 30)])
def test_cache_plans_stay_under_their_limit(batch, nq, hq, hkv, d, longest):
    for limit in (0, 10 ** 4, 10 ** 6, GB):
        p = A.attn_cache_plan(batch, nq, hq, hkv, d, longest, limit)
        assert p.workspace_bytes <= limit and p.range_tokens % 256 == 0 and p.range_tokens > 0
        assert p.n_ranges == max(1, -(-longest // p.range_tokens))
        assert p.workspace_bytes == (up(p.n_ranges * batch * nq * hq * (d + 2) * 4) if p.n_ranges > 1 else 0)


def test_cache_shapes_that_are_refused():
    for shape in [(-1, 1, 1, 1, 8, 5), (1, 0, 1, 1, 8, 5), (1, 1, 3, 2, 8, 5), (1, 1, 1, 1, 0, 5), (1, 1, 1, 1, 8, -1)]:
        with pytest.raises(A.KnnError) as e:
            A.attn_cache_plan(*shape, GB)
        assert e.value.status == A.KNN_ERR_INVALID_ARG
    for shape in [(1, 1, 1, 1, 129, 5), (1, 1, 1, 1, 8, (1 << 30) + 1), ((1 << 30) + 1, 1, 1, 1, 8, 5), (1, 65536, 1, 1, 8, 5)]:
        with pytest.raises(A.KnnError) as e:
            A.attn_cache_plan(*shape, GB)
        assert e.value.status == A.KNN_ERR_UNSUPPORTED
    assert [attn._load().attn_cache_row(d) for d in (0, 1, 64, 65, 128, 129, -3)] == [0, 64, 64, 128, 128, 0, 0]
    assert A.AttnCache.blocks_within(GB, 8, 128, 64) == GB // (8 * (2 * 64 * 128 + 8))


def cache(**other):
    c = attn.CacheStruct(0x1000, 0x1000, 0x1000, 0x1000, 10, 2, 64, 16, 0)
    for k, v in other.items():
        setattr(c, k, v)
    return c


def test_cache_calls_that_are_refused():
    """Refused before anything is launched."""
    lib, bad = attn._load(), A.KNN_ERR_INVALID_ARG
    rows, null = attn.RowsStruct(0x1000, 128, 64), attn.RowsStruct(None, 128, 64)

    def append(c=None, dtype=0, k=rows, v=rows, count=3, slots=0x1000):
        return lib.attn_cache_append(cache() if c is None else c, dtype, k, v, count, slots, None)

    def apply(c=None, dtype=0, q=rows, batch=2, nq=1, hq=4, table=0x1000, width=100, lengths=0x1000, scale=0.1, cap=0.0,
              limit=GB, ws=0x1000, ws_bytes=1 << 30, out=rows):
        return lib.attn_cache_apply(cache() if c is None else c, dtype, q, batch, nq, hq, table, width, lengths, scale, cap,
                                    None, limit, ws, ws_bytes, out, None)

    for other in [dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=0x1008), dict(v=0x1004), dict(blocks=-1),
                  dict(hkv=0), dict(d=0), dict(d=129), dict(block=8), dict(block=48), dict(block=512), dict(code=2), dict(code=-1)]:
        assert append(cache(**other)) == bad and apply(cache(**other)) == bad, other
    assert append(dtype=2) == bad and append(k=null) == bad and append(v=null) == bad and append(count=-1) == bad
    assert append(slots=None) == bad and lib.attn_cache_append(None, 0, rows, rows, 1, 0x1000, None) == bad
    assert append(count=1 << 31) == A.KNN_ERR_UNSUPPORTED
    assert apply(dtype=2) == bad and apply(q=null) == bad and apply(out=null) == bad and apply(table=None) == bad
    assert apply(lengths=None) == bad and apply(scale=0.0) == bad and apply(scale=float("nan")) == bad and apply(cap=-1.0) == bad
    assert apply(hq=3) == bad and apply(nq=0) == bad and apply(batch=-1) == bad and apply(width=-1) == bad
    assert apply(width=1 << 28) == A.KNN_ERR_UNSUPPORTED and append(count=1 << 27) == A.KNN_ERR_UNSUPPORTED
    assert apply(out=attn.RowsStruct(0x1000, 128, 63)) == bad and apply(out=attn.RowsStruct(0x1000, 0, 64)) == bad
    assert apply(scale=1e30) == bad and apply(cap=1e-30) == bad
    assert apply(ws=None) == bad and apply(ws=0x1010) == bad and apply(ws_bytes=8) == A.KNN_ERR_WORKSPACE_TOO_SMALL

    def tables(lengths=0x1000, news=0x1000, batch=2, table=0x1000, width=4, block=16, free=0x1000, n_free=3, starts=0x1000,
               slots=0x1000, n_slots=5, used=0x1000):
        return lib.attn_cache_map(lengths, news, batch, table, width, block, free, n_free, starts, slots, n_slots, used, None)

    for other in [dict(lengths=None), dict(news=None), dict(table=None), dict(free=None), dict(starts=None), dict(slots=None),
                  dict(used=None), dict(batch=-1), dict(width=-1), dict(n_free=-1), dict(n_slots=-1), dict(block=0), dict(block=24)]:
        assert tables(**other) == bad, other
    assert tables(batch=16385) == A.KNN_ERR_UNSUPPORTED and tables(width=1 << 27) == A.KNN_ERR_UNSUPPORTED


def test_the_definition_of_an_append_on_a_case_worked_by_hand():
    torch = pytest.importorskip("torch")
    from attn_formulas import append

    k, v = torch.zeros(2, 1, 16, 64, dtype=torch.float64), torch.zeros(2, 1, 64, 16, dtype=torch.float64)
    s = torch.zeros(2, 1)
    x = torch.zeros(2, 1, 3, dtype=torch.bfloat16)
    x[0, 0], x[1, 0] = torch.tensor([127.0, -1.5, 0.5]), torch.tensor([254.0, 3.0, -2.0])
    k, v, ks, vs = append(k, v, s, s, x[:1], x[:1], [0], 3, 16, "int8")
    assert ks[0, 0] == 1.0 and k[0, 0, 0, :4].tolist() == [127.0, -2.0, 0.0, 0.0]
    k, v, ks, vs = append(k, v, ks, vs, x[1:], x[1:], [1], 3, 16, "int8")
    assert ks[0, 0] == 2.0  # 127 / 2 = 63.5 to 64, -2 / 2 = -1; 3 / 2 to 2
    assert k[0, 0, :2, :3].tolist() == [[64.0, -1.0, 0.0], [127.0, 2.0, -1.0]]
    assert v[0, 0, :3, 1].tolist() == [127.0, 2.0, -1.0]
