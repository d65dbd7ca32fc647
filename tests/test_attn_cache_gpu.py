"""The cache of 8-bit blocks: its tables and slots, what an append writes and attention over it, against their
definitions (attn_formulas.py).  Whole numbers, codes and scales have to be equal."""
import random

import pytest

import paper_2206_14148_amd as A

torch = pytest.importorskip("torch")
import attn_formulas as F  # noqa: E402

pytestmark = pytest.mark.gpu
GB = 10 ** 9
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def words(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


# ---- tables and slots -----------------------------------------------------------------------

def check_map(lengths, news, width, block, n_free, more=3, seed=0):
    rng = random.Random(seed)
    blocks = list(range(len(lengths) * width + n_free))
    rng.shuffle(blocks)
    table = [[-7] * width for _ in lengths]
    for i, (length, new) in enumerate(zip(lengths, news)):
        length = min(max(length, 0), width * block)
        for b in range(-(-(length - min(max(new, 0), length)) // block)):
            table[i][b] = blocks.pop()
    free = blocks[:n_free]
    n_slots = max(0, sum(max(0, min(n, 1 << 20)) for n in news) + more)
    want = F.cache_map(lengths, news, table, free, block, n_slots)
    args = (words(lengths), words(news), words(table).view(len(lengths), width), words(free))
    for _ in range(2):  # calling again writes the same
        got = A.attn_cache_map(*args, block, n_slots)
        torch.cuda.synchronize()
        assert got[0].tolist() == want[0] and got[1].tolist() == want[1]
        assert got[2].tolist() == want[2] and got[3].tolist() == [want[3]]
    return got


@pytest.mark.parametrize("block", [16, 64, 256])
@pytest.mark.parametrize("batch", [1, 2, 63, 513, 1500])
def test_map(batch, block):
    rng = random.Random(batch + block)
    width = 6
    lengths = [rng.choice([0, 1, block, block + 1, width * block, rng.randint(0, width * block)]) for _ in range(batch)]
    news = [rng.choice([0, 1, n, rng.randint(0, n)]) for n in lengths]
    check_map(lengths, news, width, block, batch * width, seed=batch)
    check_map(lengths, news, width, block, batch // 2, more=-2 if sum(news) > 2 else 0)  # too few blocks, too few slots


def test_map_edges():
    check_map([], [], 4, 16, 3)
    check_map([5], [5], 1, 16, 1, more=0)
    check_map([0, 0], [0, 0], 2, 16, 0)
    # lengths that do not fit are taken as the nearest that do
    check_map([100, -5, 20, 7], [100, 3, -2, 9], 2, 16, 10)
    # sums beyond 32 bits are cut, and nothing is written outside
    big = 1 << 24
    table = torch.full((200, 1 << 16), -1, dtype=torch.int32, device="cuda")
    lengths = torch.full((200,), big, dtype=torch.int32, device="cuda")
    got = A.attn_cache_map(lengths, lengths, table, words([4]), 256, 10)
    torch.cuda.synchronize()
    step = (1 << 16) * 256
    assert got[1].tolist() == [min(i * step, 2 ** 31 - 1) for i in range(201)]
    assert got[2].tolist() == [4 * 256 + t for t in range(10)] and got[3].tolist() == [200 << 16]


# ---- appends --------------------------------------------------------------------------------

def filled(blocks, hkv, d, block, code, seed):
    gen = torch.Generator().manual_seed(seed)
    cache = A.AttnCache.empty(blocks, hkv, d, block, code)
    for t, turned in ((cache.k, False), (cache.v, True)):
        x = (torch.randn(blocks, hkv, block, d, generator=gen) * F.MOST[code] / 3).clamp(-F.MOST[code], F.MOST[code])
        x = x.round().to(torch.int8) if code == "int8" else x.to(torch.float8_e4m3fn)
        whole = torch.zeros(blocks, hkv, block, t.shape[2] if turned else t.shape[3], dtype=torch.uint8)
        whole[..., :d] = x.view(torch.uint8)
        whole = whole.transpose(2, 3).contiguous() if turned else whole
        t.view(torch.uint8).copy_(whole)
    for s in (cache.k_scale, cache.v_scale):
        s.copy_(0.005 + 0.01 * torch.rand(blocks, hkv, generator=gen))
    return cache


def values(cache):
    return [t.cpu().float().double() for t in (cache.k, cache.v)] + [t.cpu() for t in (cache.k_scale, cache.v_scale)]


def check_append(cache, K, V, slots, d, block, code):
    before = values(cache)
    want = F.append(*before, K, V, slots, d, block, code)
    A.attn_cache_append(cache, K, V, words(slots, torch.int64))
    torch.cuda.synchronize()
    got = values(cache)
    for name, g, w in zip(("k_scale", "v_scale", "k", "v"), got[2:] + got[:2], want[2:] + want[:2]):
        assert torch.equal(g, w), (name, int((g != w).sum()), g[g != w][:4], w[g != w][:4])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("block,d,hkv", [(16, 64, 2), (16, 128, 1), (32, 80, 3), (64, 128, 2), (64, 5, 1), (256, 100, 1)])
def test_append(block, d, hkv, code, dtype):
    gen = torch.Generator().manual_seed(block + d)
    cache = filled(9, hkv, d, block, code, d)

    def rows(n, size):
        x = torch.randn(n, hkv, d, generator=gen) * size * torch.rand(n, 1, 1, generator=gen)
        return x.to(TYPES[dtype]).cuda()

    # one new row in several blocks: begun anew, grown, not grown, the last of its block; one without a place
    slots = [3 * block, 5 * block + 7, -1, 0 * block + block - 1, 7 * block + 2, 9 * block, 2 * block + 1]
    for size in (0.01, 1.0, 300.0):
        check_append(cache, rows(7, size), rows(7, size), slots, d, block, code)
    # runs: the rest of a block and whole ones, then part of the next
    slots = [4 * block + t for t in range(block - 3, block)] + [6 * block + t for t in range(block)] + \
        [1 * block + t for t in range(block // 2 + 1)]
    check_append(cache, rows(len(slots), 2.0), rows(len(slots), 5.0), slots, d, block, code)
    # a run out of order with a slot given twice: the last counts
    slots = [8 * block + t for t in (4, 2, 9, 4, 3)]
    check_append(cache, rows(5, 1.0), rows(5, 1.0), slots, d, block, code)
    check_append(cache, rows(0, 1.0), rows(0, 1.0), [], d, block, code)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_append_of_zeros_tiny_and_not_finite_values(code):
    d, block = 64, 16
    cache = filled(4, 1, d, block, code, 1)
    K = torch.zeros(4, 1, d, dtype=torch.bfloat16)
    K[1, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 2.0])
    K[2, 0, :3] = torch.tensor([1e-39, -3e-39, 1e-40])
    K[3, 0, :] = float("nan")
    K = K.cuda()
    check_append(cache, K, -K, [0, 2 * block, 1 * block, 3 * block], d, block, code)
    check_append(cache, K, -K, [1, 2 * block + 1, 1 * block + 1, 3 * block + 3], d, block, code)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_append_rounds_quotients_of_real_numbers(code):
    """Every pair of a bf16 value and a scale of a bf16 value: ties and their neighbours among them."""
    d, block = 128, 16
    x = torch.arange(1, 256, dtype=torch.float32) / 64
    for most in (1.0, 1.2734375, 127 / 64, 3.5, 3.984375):
        use = x[x <= most].to(torch.bfloat16)
        use = torch.cat([use, torch.full(((-len(use)) % d,), 0.25, dtype=torch.bfloat16)]).view(-1, 1, d)
        use[0, 0, 0] = most
        cache = A.AttnCache.empty(3, 1, d, block, code)
        slots = [block + t for t in range(len(use))]
        check_append(cache, use.cuda(), (use * 3).cuda(), slots, d, block, code)


def test_append_strides():
    d, block, hkv = 128, 32, 2
    gen = torch.Generator().manual_seed(5)
    wide = torch.randn(6, 2 * hkv, d + 8, generator=gen).bfloat16().cuda()
    for view in (lambda t, x: t[:, x * hkv:(x + 1) * hkv, 8:], lambda t, x: t[:, x::2, 3:3 + d]):
        cache = filled(4, hkv, d, block, "int8", 2)
        check_append(cache, view(wide, 0), view(wide, 1), [32, 33, 34, 64 + 31, 96, 97], d, block, "int8")


# ---- attention over the cache ---------------------------------------------------------------

def check_apply(Q, cache, table, lengths, d, block, limit=GB, **o):
    device = dict(o)
    if o.get("slopes") is not None:
        device["slopes"] = torch.tensor(o["slopes"], device="cuda")
        o["slopes"] = device["slopes"].tolist()
    got = A.attn_cache_apply(Q, cache, words(table).view(Q.shape[0], -1), words(lengths), limit, **device)
    torch.cuda.synchronize()
    want, most = F.cache_attention(Q, *values(cache), table, lengths, d, block, **o)
    off = (got.double().cpu() - want).abs()
    assert (off <= most).all(), (int((off > most).sum()), off.max(), (off / most).max())
    return got


def tables(lengths, block, blocks, width, seed):
    rng = random.Random(seed)
    order = list(range(blocks))
    rng.shuffle(order)
    return [[order.pop() if b < -(-n // block) else -1 for b in range(width)] for n in lengths]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("block", [16, 32, 64, 256])
@pytest.mark.parametrize("d,hq,hkv,nq", [(64, 2, 2, 1), (128, 8, 1, 1), (128, 8, 2, 3), (80, 6, 1, 4), (128, 40, 1, 1),
                                        (37, 3, 1, 2)])
def test_cache_apply(d, hq, hkv, nq, block, code, dtype):
    lengths = [0, 1, 2, nq, block - 1, block, block + 1, 63, 64, 65, 300, 517]
    width = -(-max(lengths) // block)
    blocks = sum(-(-n // block) for n in lengths) + 1
    cache = filled(blocks, hkv, d, block, code, d + block)
    gen = torch.Generator().manual_seed(d)
    Q = torch.randn(len(lengths), nq, hq, d, generator=gen).to(TYPES[dtype]).cuda()
    table = tables(lengths, block, blocks, width, 3)
    check_apply(Q, cache, table, lengths, d, block)
    check_apply(3 * Q, cache, table, lengths, d, block, cap=5.0, slopes=[0.5 / (h + 1) for h in range(hq)])


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_cache_apply_long_and_split(code):
    d, hq, hkv, block = 128, 8, 2, 16
    lengths = [9001, 5, 4096]
    width = 9200 // block
    blocks = sum(-(-n // block) for n in lengths)
    cache = filled(blocks, hkv, d, block, code, 2)
    Q = torch.randn(3, 1, hq, d, generator=torch.Generator().manual_seed(1)).half().cuda()
    table = tables(lengths, block, blocks, width, 4)
    plan = A.attn_cache_plan(3, 1, hq, hkv, d, width * block, GB)
    assert plan.n_ranges > 1 and plan.workspace_bytes > 0
    one = A.attn_cache_plan(3, 1, hq, hkv, d, width * block, 0)
    assert one.n_ranges == 1 and one.workspace_bytes == 0
    for limit in (GB, 0):
        check_apply(Q, cache, table, lengths, d, block, limit=limit, slopes=[0.01 * h for h in range(hq)])


def test_cache_apply_what_it_does_not_see():
    d, hq, hkv, block = 64, 4, 2, 32
    for code in ("int8", "e4m3"):
        lengths = [70, 33, 0, 200]
        width = 7
        table = tables(lengths, block, 13, width, 1)
        cache = filled(13, hkv, d, block, code, 7)
        Q = torch.randn(4, 2, hq, d, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
        # table entries that are no block: their tokens are not seen
        table[3][1], table[3][4], table[1][0] = -1, 13, 1 << 30
        want = check_apply(Q, cache, table, lengths, d, block)
        # lengths beyond the table, and below zero, are taken as the nearest that fits
        long = [row[:3] for row in table]
        check_apply(Q, cache, long, [1000, -3, 96, 97], d, block)
        # what lies behind the last token, and in blocks that no request has, is not looked at: NaN codes and scales
        used = {b for i, row in enumerate(table) for b in row[:-(-lengths[i] // block)] if 0 <= b < 13}
        for b in range(13):
            if b not in used:
                cache.k.view(torch.uint8)[b], cache.v.view(torch.uint8)[b] = 0x7f, 0xff
                cache.k_scale[b], cache.v_scale[b] = float("nan"), float("inf")
        for i, n in enumerate(lengths):
            b = table[i][(n - 1) // block] if n else -1
            if 0 <= b < 13 and n % block:
                cache.k.view(torch.uint8)[b, :, n % block:] = 0x7f
                cache.v.view(torch.uint8)[b, :, :, n % block:] = 0xff
        got = A.attn_cache_apply(Q, cache, words(table), words(lengths), GB)
        assert torch.equal(got, want)


def test_cache_apply_strides_streams_and_graphs():
    d, hq, hkv, block = 100, 4, 1, 16
    lengths = [40, 900, 17]
    blocks = sum(-(-n // block) for n in lengths)
    cache = filled(blocks, hkv, d, block, "int8", 3)
    table = tables(lengths, block, blocks, 900 // block + 1, 1)
    Q = torch.randn(3, 2, hq + 2, d + 4, generator=torch.Generator().manual_seed(2)).half().cuda()
    view = Q[:, :, 1:1 + hq, 4:]
    want = check_apply(view.contiguous(), cache, table, lengths, d, block)
    out = torch.full_like(Q, 9.0)
    got = A.attn_cache_apply(view, cache, words(table), words(lengths), GB, out=out[:, :, 1:1 + hq, 4:])
    assert torch.equal(got, want)
    out[:, :, 1:1 + hq, 4:] = 9.0
    assert (out == 9.0).all()
    t, n = words(table), words(lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = A.attn_cache_apply(view, cache, t, n, GB)
    side.synchronize()
    assert torch.equal(other, want)


def test_a_service_step_by_step_and_as_a_graph():
    """Prompts and then tokens: tables, slots, appends and attention as a service runs them, the step as one graph that is
    replayed with other lengths; every step against the formulas on the codes that the definition gives."""
    d, hq, hkv, block, width, batch = 64, 4, 2, 16, 12, 3
    gen = torch.Generator().manual_seed(11)
    cache = A.AttnCache.empty(40, hkv, d, block, "int8")
    codes = values(cache)
    free = list(range(40))
    random.Random(3).shuffle(free)
    lengths = [37, 16, 90]
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")

    def rows(n, heads):
        return torch.randn(n, heads, d, generator=gen).half().cuda()

    # the prompts
    total = sum(lengths)
    K, V = rows(total, hkv), rows(total, hkv)
    want = F.cache_map(lengths, lengths, table.tolist(), free, block, total)
    _, starts, slots, used = A.attn_cache_map(words(lengths), words(lengths), table, words(free), block, total)
    assert table.tolist() == want[0] and slots.tolist() == want[2]
    A.attn_cache_append(cache, K, V, slots)
    codes = F.append(*codes, K, V, want[2], d, block, "int8")
    for g, w in zip(values(cache), codes):
        assert torch.equal(g, w)
    free = free[want[3]:]
    # a step: one token each; captured once, replayed as the requests grow
    n, one = words(lengths), words([1] * batch)
    bank = torch.full((40,), -1, dtype=torch.int32, device="cuda")
    k1, v1, q1 = rows(batch, hkv), rows(batch, hkv), torch.zeros(batch, 1, hq, d, dtype=torch.half, device="cuda")
    ws = torch.empty(max(A.attn_cache_plan(batch, 1, hq, hkv, d, width * block, GB).workspace_bytes, 256), dtype=torch.uint8,
                     device="cuda")

    def step():
        _, _, at, used = A.attn_cache_map(n, one, table, bank, block, batch)
        A.attn_cache_append(cache, k1, v1, at)
        return A.attn_cache_apply(q1, cache, table, n, GB, workspace=ws, cap=30.0), used

    graph = None
    for t in range(20):
        lengths = [x + 1 for x in lengths]
        before = table.tolist()
        n.copy_(words(lengths))
        bank[:len(free)] = words(free)
        k1.copy_(rows(batch, hkv)), v1.copy_(rows(batch, hkv))
        q1.copy_(rows(batch, hq).view(batch, 1, hq, d))
        if t < 2:
            got, used = step()
        elif t == 2:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got, used = step()
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        want = F.cache_map(lengths, [1] * batch, before, free, block, batch)
        assert table.tolist() == want[0] and used.tolist() == [want[3]]
        codes = F.append(*codes, k1, v1, want[2], d, block, "int8")
        for g, w in zip(values(cache), codes):
            assert torch.equal(g, w)
        O, most = F.cache_attention(q1, *codes, want[0], lengths, d, block, cap=30.0)
        assert ((got.double().cpu() - O).abs() <= most).all()
        free = free[want[3]:]


def test_a_cache_beyond_32_bits():
    """Blocks whose codes lie more than 2^32 bytes into the cache."""
    d, hq, hkv, block, blocks = 128, 8, 8, 64, 66_000
    big = A.AttnCache.empty(blocks, hkv, d, block, "int8")
    assert big.k.numel() > 1 << 32
    gen = torch.Generator().manual_seed(1)
    K, V = (torch.randn(130, hkv, d, generator=gen).half().cuda() for _ in range(2))
    small = A.AttnCache.empty(3, hkv, d, block, "int8")
    A.attn_cache_append(small, K, V, torch.arange(130, device="cuda"))
    A.attn_cache_append(big, K, V, torch.arange(130, device="cuda") + (blocks - 3) * block)
    for a, b in ((small.k, big.k), (small.v, big.v), (small.k_scale, big.k_scale), (small.v_scale, big.v_scale)):
        assert torch.equal(a, b[-3:]) and not b[:4].any()
    Q = torch.randn(1, 1, hq, d, generator=gen).half().cuda()
    want = A.attn_cache_apply(Q, small, words([[0, 1, 2]]), words([130]), GB)
    got = A.attn_cache_apply(Q, big, words([[blocks - 3, blocks - 2, blocks - 1]]), words([130]), GB)
    assert torch.equal(got, want)


def test_gpu_refusals():
    cache = A.AttnCache.empty(4, 2, 64, 16, "int8")
    K = torch.zeros(3, 2, 64, dtype=torch.half, device="cuda")
    slots = torch.arange(3, device="cuda")
    Q = torch.zeros(2, 1, 4, 64, dtype=torch.half, device="cuda")
    table, lengths = words([[0], [1]]), words([3, 2])

    def refused(f):
        with pytest.raises(A.KnnError) as e:
            f()
        assert e.value.status == A.KNN_ERR_INVALID_ARG, e.value

    refused(lambda: A.attn_cache_append(cache, K.float(), K.float(), slots))
    refused(lambda: A.attn_cache_append(cache, K, K[:2], slots))
    refused(lambda: A.attn_cache_append(cache, K, K, slots.int()))
    refused(lambda: A.attn_cache_append(cache, K, K, slots[:2]))
    refused(lambda: A.attn_cache_append(cache, K[:, :1], K[:, :1], slots))
    refused(lambda: A.attn_cache_append(A.AttnCache(cache.k, cache.k, cache.k_scale, cache.v_scale, 64), K, K, slots))
    refused(lambda: A.attn_cache_append(A.AttnCache(cache.k.float(), cache.v, cache.k_scale, cache.v_scale, 64), K, K, slots))
    refused(lambda: A.attn_cache_append(A.AttnCache(cache.k, cache.v, cache.k_scale.half(), cache.v_scale, 64), K, K, slots))
    refused(lambda: A.attn_cache_append(A.AttnCache(cache.k, cache.v, cache.k_scale, cache.v_scale, 65), K, K, slots))
    refused(lambda: A.attn_cache_apply(Q, cache, table.long(), lengths, GB))
    refused(lambda: A.attn_cache_apply(Q, cache, table[:1], lengths, GB))
    refused(lambda: A.attn_cache_apply(Q, cache, table, lengths[:1], GB))
    refused(lambda: A.attn_cache_apply(Q[0], cache, table, lengths, GB))
    refused(lambda: A.attn_cache_apply(Q[:, :, :3], cache, table, lengths, GB))
    refused(lambda: A.attn_cache_apply(Q, cache, table, lengths, GB, slopes=torch.ones(3, device="cuda")))
    refused(lambda: A.attn_cache_apply(Q, cache, table, lengths, GB, out=Q.float()))
    refused(lambda: A.attn_cache_apply(Q, cache, table, lengths, GB, scale=-1.0))
    refused(lambda: A.attn_cache_map(lengths.cpu(), lengths, table, lengths, 16, 4))
    refused(lambda: A.attn_cache_map(lengths, lengths[:1], table, lengths, 16, 4))
    refused(lambda: A.attn_cache_map(lengths, lengths, table, lengths.long(), 16, 4))
    refused(lambda: A.attn_cache_map(lengths, lengths, table, lengths, 17, 4))
