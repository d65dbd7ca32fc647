"""Attention over the whole range of what it accepts: entries that are not finite, caps of every size, gradients and
weights of every magnitude, on each way of reading rows and with the work in parts.  Values and bounds: attn_bounds.py."""
import pytest

import paper_2206_14148_amd as A

torch = pytest.importorskip("torch")
import attn_formulas as F  # noqa: E402
from attn_bounds import STEP32, attention, compare  # noqa: E402
from test_attn_cache_gpu import check_append, check_map, filled, values  # noqa: E402

pytestmark = pytest.mark.gpu
GB = 10 ** 9
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")
NAMES = ("O", "lse", "dQ", "dK", "dV")


def make(n, m, hq, hkv, d, dtype, seed, sizes=(1.0, 1.0, 1.0, 1.0)):
    gen = torch.Generator().manual_seed(seed)
    shapes = ((n, hq), (m, hkv), (m, hkv), (n, hq))
    return [(torch.randn(r, h, d, generator=gen) * s).to(TYPES[dtype]).cuda() for (r, h), s in zip(shapes, sizes)]


def words(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def odd(t):
    """The same rows where they cannot be read 16 bytes at a time."""
    view = torch.zeros(t.shape[0], t.shape[1], t.shape[2] + 3, dtype=t.dtype, device="cuda")[:, :, 1:1 + t.shape[2]]
    view.copy_(t)
    return view


def check(Q, K, V, dO, limit=GB, names=NAMES, **o):
    device = {k: words(v) if k in ("starts", "k_starts", "prefix") else torch.tensor(v, device="cuda") if k == "slopes" else v
              for k, v in o.items()}
    O, lse = A.attn_apply(Q, K, V, limit, **device)
    got = (O, lse) + (tuple(A.attn_grad(Q, K, V, O, lse, dO, limit, **device)) if names == NAMES else ())
    torch.cuda.synchronize()
    r = attention(Q, K, V, dO if names == NAMES else None, **o)
    return got, r, [compare(name, t, r) for name, t in zip(names, got)]


# ---- entries that are not finite ------------------------------------------------------------

@pytest.mark.parametrize("reading", ["16 bytes", "entries"])
@pytest.mark.parametrize("cap", [0.0, 20.0, 1e5])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128), ("bf16", 96)])
def test_infinities_reach_the_gradients_of_who_meets_them(dtype, d, cap, reading):
    """An infinity in Q, K, V or dO, of either sign: not finite where it is met, whatever the scores come to, and
    nothing changed for the others."""
    starts = [0, 90, 200]
    o = dict(causal=True, cap=cap, starts=starts)
    clean = make(200, 200, 4, 2, d, dtype, 4)
    clean[0][60:90, :, 0] = clean[0][60:90, :, 0].abs() + 0.5  # one sign: K = -infinity hides that key from all of them
    moved = odd if reading == "entries" else lambda t: t
    clean = [moved(t) for t in clean]
    first, _, _ = check(*clean, **o)
    for which, row, head in ((0, 100, 1), (1, 60, 1), (2, 150, 0), (3, 30, 2)):
        for value in (INF, -INF, float("nan")):
            data = [t.clone() if reading == "16 bytes" else odd(t) for t in clean]
            data[which][row, head, 0] = value
            got, r, _ = check(*data, **o)
            # whoever does not meet it has the same bits
            document = (0, 90) if row < 90 else (90, 200)
            heads = range(4) if which in (0, 3) else (2 * head, 2 * head + 1)
            heads = [head] if which in (0, 3) else list(heads)
            kv = heads[0] // 2
            q_met, k_met = torch.zeros(200, 4, dtype=torch.bool), torch.zeros(200, 2, dtype=torch.bool)
            for h in heads:
                q_met[(row if which in (0, 3) else row):(row + 1 if which in (0, 3) else document[1]), h] = True
            k_met[document[0]:document[1], kv] = True
            for name, a, b, met in zip(NAMES, got, first, (q_met, q_met.T, q_met, k_met, k_met)):
                same = (a == b) | (torch.isnan(a) & torch.isnan(b))
                same = same.cpu() if name == "lse" else same.all(2).cpu()
                assert (same | met).all(), (which, value, name)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_infinities_where_the_work_is_in_parts(dtype, cap):
    n, m, d = 6, 3000, 64
    plan, grad = A.attn_plan(n, m, 2, 1, d, GB), A.attn_grad_plan(n, m, 2, 1, d, GB)
    assert plan.n_splits > 1 and grad.row_splits > 1
    for which, row in ((1, 2997), (1, 40), (2, 2998), (2, 1500), (0, 3), (3, 2)):
        for value in (INF, -INF):
            data = make(n, m, 2, 1, d, dtype, 5)
            data[0][:, :, 1] = data[0][:, :, 1].abs() + 0.25
            data[which][row, 0, 1] = value
            check(*data, causal=True, cap=cap)
    # the gradient by keys in parts: many rows, few keys
    assert A.attn_grad_plan(700, 130, 2, 1, d, GB).n_splits > 1
    for which, row in ((0, 600), (3, 17), (1, 100)):
        data = make(700, 130, 2, 1, d, dtype, 6)
        data[which][row, 0, 1] = -INF
        check(*data, cap=cap)


@pytest.mark.parametrize("reading", ["16 bytes", "entries"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinities_of_v_behind_small_weights(dtype, reading):
    """Scores 20, 60 and 200 apart: a weight that rounds to nothing still carries an infinity or a NaN."""
    for n, m in ((5, 100), (3, 3000)):
        for away in (20.0, 60.0, 200.0):
            Q, K, V, _ = make(n, m, 2, 1, 64, dtype, 7)
            Q.zero_(), K.zero_()
            Q[:, :, 0] = 8.0
            K[:, :, 0] = -away
            K[7, :, 0] = 0.0
            K2 = K.roll(m - 10, 0)  # what outweighs them before them, and far behind them
            for value in (INF, -INF, float("nan")):
                W = V.clone()
                W[m - 30, 0, 5] = value
                W[11, 0, 9] = value
                check(Q, K2, W, None, names=NAMES[:2])
                if reading == "entries":
                    check(odd(Q), odd(K), odd(W), None, names=NAMES[:2])
                else:
                    check(Q, K, W, None, names=NAMES[:2])


def test_rows_whose_scores_are_all_minus_infinity():
    """They count as rows that see no key, with an infinity of their own as well."""
    for which in (0, 1):
        data = make(70, 50, 2, 1, 64, "bf16", 8)
        data[0][:, :, 0] = data[0][:, :, 0].abs() + 0.5
        data[1][:, :, 0] = -data[1][:, :, 0].abs() - 0.5
        if which:
            data[1][:, 0, 0] = -INF
        else:
            data[0][33, 1, 0] = INF
        got, r, _ = check(*data)
        lost = r["lse"] == -INF
        assert lost.any() and (got[2].cpu()[lost.T] == 0).all() and (got[0].cpu()[lost.T] == 0).all()


# ---- caps -----------------------------------------------------------------------------------

CAPS = [0.5, 64.0, 65.0, 300.0, 1e4, 1e6, 1e9, 2.0 ** 60]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("cap", CAPS)
def test_caps_of_every_size(cap, dtype):
    for d, size in ((64, 1.0), (128, 3.0), (80, 40.0)):
        check(*make(150, 211, 4, 2, d, dtype, 7, (size, 1.0, 1.0, 1.0)), cap=cap, causal=d == 128)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("cap", CAPS)
def test_caps_of_every_size_over_the_cache(cap, code):
    d, hq, hkv, block, lengths = 64, 4, 2, 16, [5, 130, 700]
    gen = torch.Generator().manual_seed(3)
    cache = A.AttnCache.empty(60, hkv, d, block, code)
    K, V = (torch.randn(sum(lengths), hkv, d, generator=gen).half().cuda() for _ in range(2))
    table = torch.zeros(3, 44, dtype=torch.int32, device="cuda")
    slots = A.attn_cache_map(words(lengths), words(lengths), table, torch.arange(60, dtype=torch.int32, device="cuda"), block,
                             sum(lengths))[2]
    A.attn_cache_append(cache, K, V, slots)
    Q = (6 * torch.randn(3, 2, hq, d, generator=gen)).half().cuda()
    got = A.attn_cache_apply(Q, cache, table, words(lengths), GB, cap=cap).double().cpu()
    k, v = cache.k.cpu().float().double(), cache.v.cpu().float().double()
    scales = cache.k_scale.cpu(), cache.v_scale.cpu()
    O, most = F.cache_attention(Q, k, v, *scales, table.tolist(), lengths, d, block, cap=cap)
    if cap > 64:  # the bound without a cap, whose scores these are or smaller ones; 16 steps more of a score
        _, most = F.cache_attention(Q, k, v, *scales, table.tolist(), lengths, d, block)
        score = d ** -0.5 * float(Q.abs().double().sum(3).max()) * float((k.abs().amax((2, 3)) * scales[0]).max())
        most = most + 4 * 16 * STEP32 * score * float((v.abs().amax((2, 3)) * scales[1]).max())
    assert ((got - O).abs() <= most).all(), ((got - O).abs() / most).max()


# ---- magnitudes -----------------------------------------------------------------------------

@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3, 1e-4])
def test_gradients_of_small_ones_in_f16(size):
    """dO of a mean loss: ds is some size / m."""
    check(*make(16, 4096, 2, 1, 128, "f16", 11, (1.0, 1.0, 1.0, size)))
    check(*make(300, 2000, 2, 2, 64, "f16", 12, (1.0, 1.0, 1.0, size)), cap=30.0, starts=[0, 100, 300], k_starts=[0, 1500, 2000])
    # larger K and Q, so that what comes out is not small itself
    check(*make(40, 3000, 2, 1, 64, "f16", 13, (0.05, 20.0, 1.0, size)))


def test_gradients_of_large_ones_in_f16():
    """<dO, V> beyond the largest f16, gradients well within it."""
    for causal in (False, True):
        got, _, _ = check(*make(300, 300, 4, 2, 64, "f16", 14, (0.01, 0.01, 100.0, 1000.0)), causal=causal)
        assert all(torch.isfinite(t).all() for t in got)
    # rows of very different magnitudes, in either order
    for turn in (False, True):
        data = make(200, 260, 2, 1, 64, "f16", 15)
        steps = torch.logspace(-6, 3, 200, device="cuda")[:, None, None]
        data[3] = (data[3].float() * (steps.flip(0) if turn else steps)).half()
        check(*data)


def test_gradients_beside_documents_of_other_magnitudes_in_f16():
    """What a row does not see, and rows that do not see a key, have no influence on how its ds is rounded."""
    starts = [0, 37, 64, 150, 300]
    Q, K, V, dO = make(300, 300, 4, 2, 64, "f16", 19)
    V[37:64] *= 1000.0
    dO[64:150] *= 1e-3
    dO[170:200] = 0.0
    V[150:] *= 1e-2
    for causal in (False, True):
        first, _, _ = check(Q, K, V, dO, causal=causal, starts=starts)
        # other values in the other documents: the same bits
        data = [t.clone() for t in (Q, K, V, dO)]
        for t in data:
            t[:64] *= 30.0
            t[150:] *= 1e-2
        again, _, _ = check(*data, causal=causal, starts=starts)
        for a, b in zip(first, again):
            a, b = (t.T if t.dim() == 2 else t for t in (a, b))
            assert torch.equal(a[64:150], b[64:150])


def test_dv_of_many_keys_in_f16():
    """Weights of 4e-6 each, far below f16's normal numbers."""
    check(*make(4, 1 << 18, 1, 1, 64, "f16", 16, (0.1, 1.0, 1.0, 100.0)))


@pytest.mark.parametrize("limit", [GB, 0])
def test_many_small_weights_beside_a_large_one_in_f16(limit):
    """One key of weight 1 and value 0, 60000 of weight 2^-24.5 and value 1: what they add up to counts."""
    m = 60_000
    Q, K, V, _ = make(2, m, 1, 1, 64, "f16", 17)
    Q.zero_(), K.zero_()
    Q[:, :, 0], K[:, :, 0] = 8.0, -17.0
    V.fill_(1.0)
    K[777], V[777] = 0.0, 0.0
    check(Q, K, V, None, limit=limit, names=NAMES[:2])


def test_values_near_the_largest_number():
    """Sums of weights that are not yet divided by their total, of values whose mean is finite."""
    for n, m in ((70, 300), (2, 4000)):
        Q, K, V, _ = make(n, m, 2, 1, 64, "bf16", 18)
        V = (1e38 * (1 + 0.5 * torch.tanh(V.float()))).bfloat16()
        got, _, _ = check(Q, K, V, None, names=NAMES[:2])
        assert torch.isfinite(got[0]).all()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_cache_blocks_of_very_different_scales(code):
    """A block of small values that has nearly all weight beside one of large values that has none."""
    d, hq, block = 64, 2, 16
    cache = A.AttnCache.empty(4, 1, d, block, code)
    gen = torch.Generator().manual_seed(5)
    K, V = torch.ones(64, 1, d), torch.randn(64, 1, d, generator=gen)
    K[16:32] = -1.0
    V[:16] *= 1e-3
    V[16:32] *= 1e4
    V[32:] *= 1e-3
    A.attn_cache_append(cache, K.bfloat16().cuda(), V.bfloat16().cuda(), torch.arange(64, device="cuda"))
    for size in (1.5, 2.5):
        Q = torch.full((1, 1, hq, d), size, dtype=torch.bfloat16, device="cuda")
        got = A.attn_cache_apply(Q, cache, words([[0, 1, 2, 3]]), words([64]), GB).double().cpu()
        k, v = cache.k.cpu().float().double(), cache.v.cpu().float().double()
        O, _ = F.cache_attention(Q, k, v, cache.k_scale.cpu(), cache.v_scale.cpu(), [[0, 1, 2, 3]], [64], d, block)
        vv = (v[:, 0] * cache.v_scale.cpu().double()[:, :, None]).transpose(1, 2).reshape(64, d)
        u = size * d ** -0.5 * (k[:, 0] * cache.k_scale.cpu().double()[:, :, None]).sum(2).view(64)
        P = torch.softmax(u, 0)
        err = STEP32 * (d + 24) * float(u.abs().max())
        # weights in f16, a step of 2^-24 at the least, 2^14 times as large, in units of the largest scale
        most = (2.0 ** -11 + 4 * err) * (P @ vv.abs()) + 2.0 ** -39 * 127 * float(cache.v_scale.max()) * 64 + 2.0 ** -9 * O.abs()
        assert ((got - O).abs() <= 1.01 * most).all(), ((got - O).abs() / most).max()


# ---- appends whose rows do not all have a place ---------------------------------------------

@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("block", [16, 32, 64, 256])
def test_rows_without_a_place_within_a_run_are_passed_over(block, code):
    """-1, and slots behind the cache, before, within and behind the rows of a block: few and very many; what stands in those
    rows does not count for the scale."""
    d, hkv, blocks = 64, 2, 7
    gen = torch.Generator().manual_seed(block)
    for gaps in ((1,), (2, 1, 70), (300, 1, 2500), (64, 63, 65, 5000), (1, 1, 1, 1, 1, 1)):
        slots, gap = [], 0
        for b, begin, count in ((5, 0, block // 2 + 3), (2, 3, 4), (6, block - 1, 1), (0, 0, block), (3, 1, 1), (1, 0, 1)):
            for t in range(count):
                if t in (0, 1, 2, count - 1):
                    slots += [(-1, blocks * block, 1 << 40, -7)[gap % 4]] * gaps[gap % len(gaps)]
                    gap += 1
                slots.append(b * block + begin + t)
        slots += [slots[-1]] + [-1] * gaps[-1]  # one given twice, then the rest of a padded step
        cache = filled(blocks, hkv, d, block, code, 3)
        K, V = (torch.randn(len(slots), hkv, d, generator=gen).half() for _ in range(2))
        lost = torch.tensor([not 0 <= s < blocks * block for s in slots])
        K[lost], V[lost] = 3000.0, -3000.0
        check_append(cache, K.cuda(), V.cuda(), slots, d, block, code)
    before = [t.clone() for t in values(cache)]
    A.attn_cache_append(cache, K.cuda(), V.cuda(), torch.full((len(slots),), -1, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(before, values(cache)))


def test_outputs_whose_heads_lie_between_each_others_rows():
    """Strides in no order that nevertheless keep every entry apart."""
    for n, hq, ld, hs in ((2, 2, 128, 192), (3, 2, 192, 64), (2, 3, 320, 128), (40, 2, 64, 64 * 40), (5, 4, 256, 64)):
        Q, K, V, dO = make(n, 90, hq, hq, 64, "bf16", n)
        want = A.attn_apply(Q, K, V, GB)
        grad = A.attn_grad(Q, K, V, *want, dO, GB)
        views = [torch.as_strided(torch.zeros(20_000, dtype=torch.bfloat16, device="cuda"), (n, hq, 64), (ld, hs, 1)) for _ in range(2)]
        A.attn_apply(Q, K, V, GB, out=(views[0], torch.empty_like(want[1])))
        A.attn_grad(Q, K, V, *want, dO, GB, out=(views[1], *(torch.empty_like(t) for t in grad[1:])))
        assert torch.equal(views[0], want[0]) and torch.equal(views[1], grad[0])


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_an_odd_number_of_ranges_of_odd_rows(code):
    """Three ranges of three heads of 37: what is kept of a range begins anywhere."""
    d, hq, block, length = 37, 3, 16, 2090
    plan = A.attn_cache_plan(1, 1, hq, 1, d, 2096, GB)
    assert plan.n_ranges % 2 == 1 and plan.n_ranges > 1
    cache = filled(131, 1, d, block, code, 6)
    table = torch.arange(131, dtype=torch.int32, device="cuda").flip(0).contiguous()[None]
    gen = torch.Generator().manual_seed(2)
    for batch in (1, 3):
        Q = torch.randn(batch, 1, hq, d, generator=gen).half().cuda()
        lengths = [length, 700, 1][:batch]
        got = A.attn_cache_apply(Q, cache, table.expand(batch, -1).contiguous(), words(lengths), GB).double().cpu()
        O, most = F.cache_attention(Q, *values(cache), table.tolist() * batch, lengths, d, block)
        assert ((got - O).abs() <= most).all()


def test_maps_of_the_largest_batches():
    """Their sums need more than 48 and more than 64 KiB of LDS."""
    for batch in (6200, 16384):
        lengths = [(37 * i) % 120 for i in range(batch)]
        news = [(11 * i) % (n + 1) for i, n in enumerate(lengths)]
        check_map(lengths, news, 8, 16, batch * 2, seed=batch)
    with pytest.raises(A.KnnError) as e:
        A.attn_cache_map(words([1]), words([1]), words([[0]]), words([0]), 16, -1)
    assert e.value.status == A.KNN_ERR_INVALID_ARG
