"""Attention and its gradient against their formulas in 64 bits (attn_formulas.py, whose bounds count the
documented roundings): sizes from one row up, every kind of mask, shared heads, odd widths and strides."""
import math

import pytest

import paper_2206_14148_amd as A

torch = pytest.importorskip("torch")
from attn_formulas import attention, compare  # noqa: E402

pytestmark = pytest.mark.gpu
GB = 10 ** 9
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def make(n, m, hq, hkv, d, dtype, seed, size=1.0):
    gen = torch.Generator().manual_seed(seed)
    q, g = (torch.randn(n, hq, d, generator=gen) * s for s in (size, 1.0))
    k, v = (torch.randn(m, hkv, d, generator=gen) for _ in range(2))
    return tuple(t.to(TYPES[dtype]).cuda() for t in (q, k, v, g))


def words(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def check(Q, K, V, dO, limit=GB, **o):
    device = dict(o)
    for name in ("starts", "k_starts", "prefix"):
        if name in o:
            device[name] = words(o[name])
    if o.get("slopes") is not None:
        device["slopes"] = torch.tensor(o["slopes"], dtype=torch.float32, device="cuda")
        o["slopes"] = device["slopes"].tolist()
    O, lse = A.attn_apply(Q, K, V, limit, **device)
    grads = A.attn_grad(Q, K, V, O, lse, dO, limit, **device)
    torch.cuda.synchronize()
    r = attention(Q, K, V, dO, **o)
    share = [compare(name, got, r) for name, got in zip(("O", "lse", "dQ", "dK", "dV"), (O, lse) + tuple(grads))]
    return O, lse, grads, share


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,m,hq,hkv,d", [
    (1, 1, 1, 1, 64), (1, 300, 2, 1, 128), (3, 64, 2, 2, 64), (65, 129, 4, 2, 96), (128, 128, 1, 1, 128),
    (129, 64, 2, 1, 64), (200, 333, 3, 1, 128), (333, 200, 2, 2, 80), (257, 257, 6, 2, 72), (31, 33, 2, 2, 1),
    (70, 90, 2, 1, 5), (64, 500, 2, 2, 100), (300, 300, 4, 4, 32), (40, 130, 8, 1, 120)])
def test_against_the_formulas(n, m, hq, hkv, d, causal, dtype):
    check(*make(n, m, hq, hkv, d, dtype, n + m + d), causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("options", [
    {"cap": 5.0}, {"cap": 30.0, "causal": True}, {"slopes": [0.5, 0.0, 0.03, 0.25], "causal": True},
    {"slopes": [0.5, 0.25, 0.0625, 0.01], "cap": 20.0}, {"scale": 0.3, "causal": True}])
def test_caps_slopes_and_scales(options, d, dtype):
    check(*make(150, 211, 4, 2, d, dtype, 7, 3.0), **options)


DOCUMENTS = [
    # ragged, some empty, some one row long
    dict(n=301, m=301, starts=[0, 0, 1, 70, 200, 200, 301]),
    # as many documents as a tile has rows and more
    dict(n=150, m=150, starts=list(range(151))),
    # rows before the first and behind the last belong to none
    dict(n=260, m=260, starts=[5, 40, 41, 190]),
    # keys of other lengths: fewer keys than rows (with causal the first rows see none), none at all, many
    dict(n=200, m=310, starts=[0, 60, 90, 90, 160, 200], k_starts=[0, 20, 20, 33, 301, 310]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("which", range(len(DOCUMENTS)))
@pytest.mark.parametrize("causal,prefixed", [(False, False), (True, False), (True, True)])
def test_documents(which, causal, prefixed, dtype):
    case = dict(DOCUMENTS[which])
    n, m = case.pop("n"), case.pop("m")
    if prefixed:
        k = case.get("k_starts", case["starts"])
        case["prefix"] = [(7 * c) % (k[c + 1] - k[c] + 3) for c in range(len(k) - 1)]
    check(*make(n, m, 4, 2, 64, dtype, which), causal=causal, **case)


def test_rows_and_keys_outside_the_documents_are_left_as_they_were():
    n, starts = 260, [5, 40, 41, 190]
    Q, K, V, dO = make(n, n, 2, 1, 64, "bf16", 3)
    # not read either: NaN there changes nothing
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[starts[0]:starts[-1]] = False
    clean = A.attn_apply(Q, K, V, GB, causal=True, starts=words(starts))
    cleang = A.attn_grad(Q, K, V, *clean, dO, GB, causal=True, starts=words(starts))
    for t in (Q, K, V, dO):
        t[outside] = float("nan")
    O, lse = torch.full_like(Q, 3.0), torch.full((2, n), 3.0, device="cuda")
    g = [torch.full_like(t, 3.0) for t in (Q, K, V)]
    A.attn_apply(Q, K, V, GB, causal=True, starts=words(starts), out=(O, lse))
    A.attn_grad(Q, K, V, O, lse, dO, GB, causal=True, starts=words(starts), out=g)
    for got, want in zip([O, lse.T] + g, [clean[0], clean[1].T] + list(cleang)):
        assert (got[outside] == 3.0).all()
        assert torch.equal(got[~outside], want[~outside])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_work_split_along_the_keys_and_over_the_heads(dtype):
    for n, m, hq, hkv, d, o in [(1, 5000, 2, 1, 128, {}), (7, 4097, 4, 2, 64, {"causal": True, "cap": 20.0}),
                                (3, 2100, 2, 2, 80, {"slopes": [0.01, 0.002], "causal": True}),
                                (9, 1500, 2, 1, 33, {"starts": [1, 4, 9], "k_starts": [10, 400, 1490]})]:
        assert A.attn_plan(n, m, hq, hkv, d, GB).n_splits > 1 and A.attn_plan(n, m, hq, hkv, d, 0).n_splits == 1
        data = make(n, m, hq, hkv, d, dtype, m)
        check(*data, **dict(o))
        device = {k: words(v) if k.endswith("starts") else torch.tensor(v, device="cuda") if k == "slopes" else v
                  for k, v in o.items()}
        O, lse = A.attn_apply(*data[:3], 0, **device)  # no room for parts
        r = attention(*data[:3], None, **o)
        compare("O", O, r)
        compare("lse", lse, r)
    # parts of the gradient by keys begin and end within a head's rows
    assert A.attn_grad_plan(300, 300, 8, 1, 64, GB).n_splits > 8 and A.attn_grad_plan(700, 300, 3, 1, 64, GB).n_splits > 3
    data = make(300, 300, 8, 1, 64, dtype, 5)
    check(*data, causal=True)
    check(*make(700, 300, 3, 1, 64, dtype, 6), starts=[0, 100, 333, 690], k_starts=[0, 10, 200, 299])
    least = A.attn_grad_plan(300, 300, 8, 1, 64, GB).min_limit_bytes
    assert A.attn_grad_plan(300, 300, 8, 1, 64, least).n_splits == 1
    check(*data, causal=True, limit=least)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_dq_from_ranges_of_the_keys(dtype):
    for n, m, hq, hkv, d, o in [(1, 5000, 2, 1, 128, {}), (7, 4097, 4, 2, 64, {"causal": True, "cap": 20.0}),
                                (140, 2100, 2, 2, 80, {"slopes": [0.01, 0.002], "causal": True}),
                                (9, 1500, 2, 1, 33, {"starts": [1, 4, 9], "k_starts": [10, 400, 1490]})]:
        plan = A.attn_grad_plan(n, m, hq, hkv, d, GB)
        assert plan.row_splits > 1 and A.attn_grad_plan(n, m, hq, hkv, d, plan.min_limit_bytes).row_splits == 1
        data = make(n, m, hq, hkv, d, dtype, m)
        check(*data, **dict(o))
        check(*data, limit=plan.min_limit_bytes, **dict(o))
    # a key that is not finite makes the dQ of who sees it NaN, whichever range it lies in, and no other's
    Q, K, V, dO = make(6, 3000, 2, 1, 64, dtype, 3)
    assert A.attn_grad_plan(6, 3000, 2, 1, 64, GB).row_splits > 1
    K[2995] = math.nan
    O, lse = A.attn_apply(Q, K, V, GB, causal=True)
    got = torch.isnan(A.attn_grad(Q, K, V, O, lse, dO, GB, causal=True)[0])
    assert got[1:].all() and not got[0].any()


def test_no_rows_and_no_keys():
    Q, K, V, dO = make(5, 4, 2, 1, 64, "bf16", 1)
    O, lse = A.attn_apply(Q[:0], K, V, GB)
    assert O.shape == (0, 2, 64) and lse.shape == (2, 0)
    dQ, dK, dV = A.attn_grad(Q[:0], K, V, O, lse, dO[:0], GB)
    assert dQ.shape == (0, 2, 64) and not dK.any() and not dV.any()
    O, lse = A.attn_apply(Q, K[:0], V[:0], GB)
    assert not O.any() and (lse == -math.inf).all()
    dQ, dK, dV = A.attn_grad(Q, K[:0], V[:0], O, lse, dO, GB)
    assert not dQ.any() and dK.shape == (0, 1, 64)


@pytest.mark.parametrize("how", ["columns", "heads_first", "odd", "shared"])
@pytest.mark.parametrize("d", [64, 100, 128])
def test_strides_and_alignments(how, d):
    n, m, hq, hkv = 75, 140, 4, 2
    Q, K, V, dO = make(n, m, hq, hkv, d, "bf16", 9)

    def moved(t):
        if how == "columns":  # parts of a wider row, as one projection gives them
            wide = torch.zeros(t.shape[0], t.shape[1] + 1, t.shape[2] + 24, dtype=t.dtype, device="cuda")
            view = wide[:, 1:, 16:16 + d]
        elif how == "heads_first":
            view = torch.zeros(t.shape[1], t.shape[0], t.shape[2], dtype=t.dtype, device="cuda").transpose(0, 1)
        elif how == "odd":
            view = torch.zeros(t.shape[0], t.shape[1], t.shape[2] + 3, dtype=t.dtype, device="cuda")[:, :, 1:1 + d]
        else:  # one head for all, by a stride of zero
            return t[:, :1].contiguous().expand(t.shape) if t.shape[1] == hkv else t
        view.copy_(t)
        return view

    data = [moved(t) for t in (Q, K, V, dO)]
    O, lse, grads, _ = check(*data, causal=True)
    if how == "shared":
        return
    out = [moved(t) for t in (O, *grads)]
    for t in out:
        t.fill_(7.0)
    lse2 = torch.empty_like(lse)
    A.attn_apply(*data[:3], GB, causal=True, out=(out[0], lse2))
    A.attn_grad(*data[:3], out[0], lse2, data[3], GB, causal=True, out=out[1:])
    for a, b in zip([*out, lse2], [O, *grads, lse]):
        assert torch.equal(a, b)
    base = out[0]._base
    if base is not None and how != "heads_first":  # nothing beside the views
        touched = torch.ones_like(base, dtype=torch.bool)
        torch.as_strided(touched, out[0].shape, out[0].stride(), out[0].storage_offset()).fill_(False)
        assert not base[touched].any()


@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_finite_reaches_who_sees_it_and_no_others(d):
    n, starts = 200, [0, 90, 200]
    Q, K, V, dO = make(n, n, 2, 2, d, "bf16", 4)
    o = dict(causal=True, starts=words(starts))
    O0, lse0 = A.attn_apply(Q, K, V, GB, **o)
    g0 = A.attn_grad(Q, K, V, O0, lse0, dO, GB, **o)
    nan, inf = float("nan"), float("inf")
    # V: row 50 in document 0, row 120 in document 1
    W = V.clone()
    W[50, 0, 3], W[120, 0, 5], W[130, 0, 5], W[150, 1, 7] = inf, -inf, inf, nan
    O, lse = A.attn_apply(Q, K, W, GB, **o)
    assert torch.equal(lse, lse0)
    want = O0.clone()
    want[50:90, 0, 3] = inf
    want[120:, 0, 5] = -inf
    want[130:, 0, 5] = nan
    want[150:, 1, 7] = nan
    assert torch.equal(torch.isnan(O), torch.isnan(want))
    fine = ~torch.isnan(want)
    assert torch.equal(O[fine], want[fine])
    # K: a row that sees it has a NaN or infinite score
    W = K.clone()
    W[60, 1, 0] = nan
    O, lse = A.attn_apply(Q, W, V, GB, **o)
    assert torch.isnan(O[60:90, 1]).all() and torch.isnan(lse[1, 60:90]).all()
    keep = torch.ones(n, 2, dtype=torch.bool, device="cuda")
    keep[60:90, 1] = False
    assert torch.equal(O[keep], O0[keep]) and torch.equal(lse.T[keep], lse0.T[keep])
    dQ, dK, dV = A.attn_grad(Q, W, V, O, lse, dO, GB, **o)
    assert torch.equal(dQ[keep], g0[0][keep]) and not torch.isfinite(dQ[60:90, 1]).any()
    # every key up to 89 of that head is seen by a row that is NaN, the second document by none
    for t, t0 in ((dK, g0[1]), (dV, g0[2])):
        assert not torch.isfinite(t[:90, 1]).any()
        assert torch.equal(t[90:], t0[90:]) and torch.equal(t[:, 0], t0[:, 0])
    # Q and dO: the row itself, and the keys that it sees
    for which in (0, 3):
        data = [Q.clone(), K, V, dO.clone()]
        data[which][100, 0, 1] = nan
        O, lse = A.attn_apply(*data[:3], GB, **o)
        dQ, dK, dV = A.attn_grad(*data[:3], O, lse, data[3], GB, **o)
        keep = torch.ones(n, 2, dtype=torch.bool, device="cuda")
        keep[100, 0] = False
        assert torch.equal(dQ[keep], g0[0][keep]) and not torch.isfinite(dQ[100, 0]).any()
        keep[90:101, 0] = False
        for t, t0 in ((dK, g0[1]), (dV, g0[2])):
            assert torch.equal(t[keep], t0[keep])
            assert not torch.isfinite(t[90:101, 0]).any()


def test_lowest_and_large_values():
    # scores far apart, and all of a row at the type's lowest: finite results
    for dtype in ("bf16", "f16"):
        Q, K, V, dO = make(70, 90, 2, 1, 64, dtype, 6)
        check(Q * 30, K, V, dO, causal=True)
        low = torch.finfo(TYPES[dtype]).min if dtype == "f16" else -1e30
        K2 = torch.zeros_like(K)
        K2[:, :, 0] = low
        Q2 = torch.zeros_like(Q)
        Q2[:, :, 0] = 1.0
        O, lse = A.attn_apply(Q2, K2, V, GB)  # equal scores: the mean
        assert torch.isfinite(lse).all()
        mean = V.float().mean(0)
        u = torch.finfo(TYPES[dtype]).eps / 2
        most = 2 * u * V.float().abs().mean(0) + u * mean.abs()
        assert ((O.float() - mean).abs() <= most + 1e-6).all()


def test_same_bits_other_streams_and_captured_graphs():
    Q, K, V, dO = make(300, 300, 4, 2, 128, "bf16", 8)
    o = dict(causal=True, starts=words([0, 120, 300]))

    def step():
        O, lse = A.attn_apply(Q, K, V, GB, **o)
        return (O, lse) + tuple(A.attn_grad(Q, K, V, O, lse, dO, GB, **o))

    want = step()
    for t, w in zip(step(), want):
        assert torch.equal(t, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    for t, w in zip(other, want):
        assert torch.equal(t, w)
    # two graphs, one workspace: each makes all that it reads
    ws = torch.empty(max(A.attn_grad_plan(300, 300, 4, 2, 128, GB).workspace_bytes,
                         A.attn_plan(7, 3000, 4, 2, 128, GB).workspace_bytes), dtype=torch.uint8, device="cuda")
    q2, k2, v2, _ = make(7, 3000, 4, 2, 128, "bf16", 9)
    few = A.attn_apply(q2, k2, v2, GB)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        O, lse = A.attn_apply(Q, K, V, GB, workspace=ws, **o)
        got = (O, lse) + tuple(A.attn_grad(Q, K, V, O, lse, dO, GB, workspace=ws, **o))
    with torch.cuda.graph(graphs[1]):
        got_few = A.attn_apply(q2, k2, v2, GB, workspace=ws)
    for _ in range(3):
        for t in got + got_few:
            t.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for t, w in zip(got + got_few, want + few):
            assert torch.equal(t, w)
        ws.fill_(255)


def test_rows_far_apart_in_memory():
    """Offsets beyond 32 bits: rows of a very wide matrix, at both ways of reading them, and rows very far apart."""
    d, hq, hkv = 64, 2, 1
    big = torch.zeros(1 << 32, dtype=torch.int8, device="cuda").view(torch.bfloat16)  # 2^31 entries
    big = torch.cat([big, big[: 1 << 27]])
    for n, ld, shift in ((50_000, 44_000, 0), (50_000, 44_000, 1), (17, 1 << 27, 0)):
        base = torch.as_strided(big, (n, hkv, d), (ld, d, 1), shift)
        small = make(40, n, hq, hkv, d, "bf16", 3)
        base.copy_(small[1])
        starts, k_starts = [0, 40], [max(0, n - 300), n]
        o = dict(causal=True, starts=words(starts), k_starts=words(k_starts))
        want = A.attn_apply(*small[:3], GB, **o)
        got = A.attn_apply(small[0], base, small[2], GB, **o)
        for g, w in zip(got, want):
            assert torch.equal(g, w)
        grads = A.attn_grad(*small[:3], *want, small[3], GB, **o)
        out = [torch.empty_like(small[0]), base, torch.empty_like(small[2])]
        got = A.attn_grad(*small[:3], *want, small[3], GB, out=out, **o)
        assert torch.equal(got[0], grads[0])
        for g, w in zip(got[1:], grads[1:]):
            assert torch.equal(g[k_starts[0]:], w[k_starts[0]:])
        base.zero_()


def test_gpu_refusals():
    Q, K, V, dO = make(8, 9, 4, 2, 64, "bf16", 2)

    def refused(f):
        with pytest.raises(A.KnnError) as e:
            f()
        assert e.value.status == A.KNN_ERR_INVALID_ARG, e.value

    refused(lambda: A.attn_apply(Q, K.half(), V, GB))
    refused(lambda: A.attn_apply(Q.float(), K.float(), V.float(), GB))
    refused(lambda: A.attn_apply(Q, K, V[:5], GB))
    refused(lambda: A.attn_apply(Q[0], K, V, GB))
    refused(lambda: A.attn_apply(Q[:, :, ::2], K[:, :, ::2], V[:, :, ::2], GB))
    refused(lambda: A.attn_apply(Q, K.cpu(), V, GB))
    refused(lambda: A.attn_apply(Q[:, :3], K, V, GB))
    refused(lambda: A.attn_apply(Q, K, V, GB, slopes=torch.ones(3, device="cuda")))
    refused(lambda: A.attn_apply(Q, K, V, GB, slopes=torch.ones(4)))
    refused(lambda: A.attn_apply(Q, K, V, GB, starts=words([0, 8]).long()))
    refused(lambda: A.attn_apply(Q, K, V, GB, starts=words([0, 8]), k_starts=words([0, 4, 9])))
    refused(lambda: A.attn_apply(Q, K, V, GB, k_starts=words([0, 9])))
    refused(lambda: A.attn_apply(Q, K, V, GB, starts=words([0])))
    refused(lambda: A.attn_apply(Q, K, V, GB, prefix=words([1, 2])))
    refused(lambda: A.attn_apply(Q, K, V, GB, scale=0.0))
    refused(lambda: A.attn_apply(Q, K, V, GB, cap=-1.0))
    lse = torch.empty(4, 8, device="cuda")
    refused(lambda: A.attn_apply(Q, K, V, GB, out=(torch.empty_like(Q)[:, :1].expand(Q.shape), lse)))
    refused(lambda: A.attn_apply(Q, K, V, GB, out=(torch.empty_like(Q), lse.T)))
    refused(lambda: A.attn_apply(Q, K, V, GB, workspace=torch.empty(10, device="cuda")))
    refused(lambda: A.attn_grad(Q, K, V, Q, lse.double(), dO, GB))
    refused(lambda: A.attn_grad(Q, K, V, Q, lse, dO[:4], GB))
    with pytest.raises(A.KnnError) as e:
        A.attn_grad(Q, K, V, Q, lse, dO, 10)
    assert e.value.status == A.KNN_ERR_MEM_LIMIT_TOO_SMALL and e.value.min_limit_bytes == 256
    with pytest.raises(A.KnnError) as e:
        A.attn_grad(Q, K, V, Q, lse, dO, GB, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == A.KNN_ERR_WORKSPACE_TOO_SMALL
