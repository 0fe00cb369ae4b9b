"""Writing into pages, key weights, eviction, and a run of all of them together."""
import math

import pytest
import torch

import paper_2602_05853_amd as rr
from cache_util import U32, attend, check_rows, fill_pages, positions, sees
from test_gpu_paged_attention import check, make, query

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,d,layout", [(torch.bfloat16, 128, "phld"), (torch.bfloat16, 8, "plhd"), (torch.float32, 80, "phld")])
@pytest.mark.parametrize("T,page", [(1, 16), (5, 48), (130, 64)])
@pytest.mark.parametrize("weighted", [False, True])
def test_write(dtype, d, layout, T, page, weighted):
    """Ragged counts, starts inside pages; everything else stays as it was."""
    lengths = [200, T, 0, 131, 3]
    cache = make(lengths, 3, d, page, dtype, weight=True, layout=layout)
    count = torch.tensor([T, T, T, max(0, T - 4), 0], dtype=torch.int32, device=DEV)
    cache.table[0, 1] = -1
    K = torch.randn(5, T, 3, d, device=DEV).to(dtype).transpose(1, 2)
    V = torch.randn(5, T, 3, d, device=DEV).to(dtype).transpose(1, 2)
    first = torch.rand(5, 3, T, device=DEV) if weighted else None
    want = [x.clone() for x in (cache.K, cache.V, cache.weight)]
    for b, n in enumerate(lengths):
        c = int(count[b])
        for t in range(c):
            pos = n - c + t
            e = int(cache.table[b, pos // page]) if pos >= 0 else -1
            if e < 0:
                continue
            want[0][e, :, pos % page], want[1][e, :, pos % page] = K[b, :, t], V[b, :, t]
            want[2][e, :, pos % page] = first[b, :, t] if weighted else 0.0
    for _ in range(2):                                        # a second time changes nothing
        rr.rr_paged_write(cache, K, V, count, first)
        for got, w in zip((cache.K, cache.V, cache.weight), want):
            assert torch.equal(got, w)


def test_write_holds_counts_and_lengths():
    cache = make([40, 40], 1, 64)
    before = cache.K.clone()
    cache.length.copy_(torch.tensor([-3, 10 ** 9], dtype=torch.int32))
    K = torch.ones(2, 1, 4, 64, dtype=torch.bfloat16, device=DEV)
    rr.rr_paged_write(cache, K, K, torch.tensor([9, -1], dtype=torch.int32, device=DEV))
    assert torch.equal(before, cache.K)


def test_write_a_prompt_without_weights():
    cache = make([1000], 2, 128, 64)
    K = torch.randn(1, 2, 1000, 128, device=DEV).to(torch.bfloat16)
    rr.rr_paged_write(cache, K, K * 2)
    for kv in range(2):
        assert torch.equal(positions(cache, 0, 1000, kv, "K")[0], K[0, kv])
        assert torch.equal(positions(cache, 0, 1000, kv, "V")[0], K[0, kv] * 2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 128), (3, 1, 64), (2, 2, 80), (7, 1, 256), (2, 1, 8), (2, 1, 200)])
@pytest.mark.parametrize("L,Lq", [(1, 1), (33, 33), (300, 300), (300, 17), (513, 1), (129, 128)])
def test_key_weights(dtype, Hq, Hkv, d, L, Lq):
    g = torch.Generator(device=DEV).manual_seed(L + d)
    Q = (torch.randn(2, Hq, Lq, d, generator=g, device=DEV) * 2).to(dtype)
    K = torch.randn(2, Hkv, L, d, generator=g, device=DEV).to(dtype)
    seen = sees(torch.arange(L - Lq, L, device=DEV), L, 0, 0)
    G = Hq // Hkv
    lse = torch.empty(2, Hq, Lq, device=DEV)
    want = torch.zeros(2, Hkv, L, dtype=torch.float64, device=DEV)
    slack = torch.zeros_like(want)
    for b in range(2):
        for h in range(Hq):
            _, l, p, _, delta = attend(Q[b, h], K[b, h // G], K[b, h // G], seen)
            lse[b, h] = l
            if h == 0 and Lq > 2:                             # a row without a key gives nothing
                lse[b, h, 2] = -math.inf
                p[2] = 0
            want[b, h // G] += p.sum(0)
            # the score, the given lse's rounding and that of its product with log2(e), exp2
            slack[b, h // G] += ((delta[:, None] + 4 * U32 * l.abs()[:, None] + 8 * U32) * p).sum(0)
    got = rr.rr_key_weights(Q, K, lse)
    tol = slack * 1.01 + (G * Lq + 8) * U32 * want + 1e-30
    err = (got.double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("L,Lq,Hq,Hkv,batch", [(3000, 3000, 6, 2, 1), (5000, 40, 8, 2, 1), (2000, 700, 3, 1, 2), (700, 256, 2, 1, 1), (700, 288, 2, 1, 1)])
def test_key_weights_of_longer_contexts(L, Lq, Hq, Hkv, batch):
    """Tiles of keys shared by several workgroups, and one workgroup to a tile; every row gives one to its keys in all."""
    g = torch.Generator(device=DEV).manual_seed(L)
    Q = (torch.randn(batch, Hq, Lq, 128, generator=g, device=DEV) * 2).to(torch.bfloat16)
    K = torch.randn(batch, Hkv, L, 128, generator=g, device=DEV).to(torch.bfloat16)
    seen = sees(torch.arange(L - Lq, L, device=DEV), L, 0, 0)
    lse = torch.empty(batch, Hq, Lq, device=DEV)
    want = torch.zeros(batch, Hkv, L, dtype=torch.float64, device=DEV)
    slack = torch.zeros_like(want)
    for b in range(batch):
        for h in range(Hq):
            _, l, p, _, delta = attend(Q[b, h], K[b, h * Hkv // Hq], K[b, h * Hkv // Hq], seen)
            lse[b, h] = l
            want[b, h * Hkv // Hq] += p.sum(0)
            slack[b, h * Hkv // Hq] += ((delta[:, None] + 4 * U32 * l.abs()[:, None] + 8 * U32) * p).sum(0)
    n = rr.rr_key_weights_workspace_bytes(Q, K)
    got = rr.rr_key_weights(Q, K, lse, workspace=torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device=DEV))
    G = Hq // Hkv
    tol = slack * 1.01 + (G * Lq + 8) * U32 * want + 1e-30
    assert ((got.double() - want).abs() <= tol).all()
    assert torch.equal(got, rr.rr_key_weights(Q, K, lse))


def test_key_weights_of_rows_in_wider_tensors():
    big = torch.full((1, 150, 4, 80), math.nan, dtype=torch.bfloat16, device=DEV)
    Q, K = big[:, 10:60, 0:2, 8:72].transpose(1, 2), big[:, 20:120, 2:3, 8:72].transpose(1, 2)
    Q.copy_(torch.randn(Q.shape, device=DEV))
    K.copy_(torch.randn(K.shape, device=DEV))
    lse = torch.empty(1, 2, 50, device=DEV)
    rr.rr_window_attn(Q, K, K, 1000, 0, lse=lse)
    out = torch.full((1, 1, 100), math.nan, device=DEV)
    assert rr.rr_key_weights(Q, K, lse, out=out) is out
    assert abs(float(out.sum()) - 100.0) < 1e-3               # every row gives one


def evict_reference(cache, keep, sinks, recent):
    """Kept positions of every sequence and head, by sorting."""
    out = []
    for b, n in enumerate(cache.length.tolist()):
        n = min(max(n, 0), cache.table.shape[1] * cache.K.shape[2])
        for kv in range(cache.K.shape[1]):
            w, good = positions(cache, b, n, kv, "weight")
            w, good = w.tolist(), good.tolist()
            if n <= keep:
                out.append(list(range(n)))
                continue
            def rank(j):
                value = math.inf if math.isnan(w[j]) else w[j]
                return (not good[j], not math.isnan(w[j]), -value, j)
            middle = sorted(range(sinks, n - recent), key=rank)[:keep - sinks - recent]
            out.append(sorted(list(range(sinks)) + middle + list(range(n - recent, n))))
    return out


def evict(cache, keep, sinks, recent):
    b, (pages, Hkv, page, d) = cache.table.shape[0], cache.K.shape
    used = set(cache.table[cache.table >= 0].tolist())
    width = -(-keep // page)
    fresh = torch.arange(pages, pages + b * width, dtype=torch.int32)[torch.randperm(b * width)].reshape(b, width)
    grown = rr.PagedCache(*(torch.cat([x, torch.full((b * width,) + x.shape[1:], 5.0, dtype=x.dtype, device=DEV)]) for x in (cache.K, cache.V)),
                          cache.table, cache.length, torch.cat([cache.weight, torch.full((b * width, Hkv, page), 5.0, device=DEV)]))
    before = [x.clone() for x in (grown.K, grown.V, grown.weight)]
    want = evict_reference(grown, keep, sinks, recent)
    new, kept = rr.rr_cache_evict(grown, fresh.to(DEV), keep, sinks, recent)
    assert used and new.K is grown.K
    lengths = grown.length.tolist()
    for i in range(b):
        n = min(max(lengths[i], 0), cache.table.shape[1] * page)
        assert int(new.length[i]) == min(n, keep)
        for kv in range(Hkv):
            w = want[i * Hkv + kv]
            assert kept[i, kv].tolist() == w + [-1] * (keep - len(w)), (i, kv)
            pos, r = torch.tensor(w, dtype=torch.int64, device=DEV), torch.arange(len(w), device=DEV)
            s, t = grown.table[i].long()[pos // page], fresh[i].long().to(DEV)[r // page]
            good = (s >= 0) & (s < grown.K.shape[0])
            pos, r, s, t = pos[good], r[good], s[good], t[good]
            for x in before:
                x[t, kv, r % page] = x[s, kv, pos % page]
    for got, w in zip((grown.K, grown.V, grown.weight), before):
        assert torch.equal(got.view(torch.int32 if got.dtype == torch.float32 else torch.int16),
                           w.view(torch.int32 if w.dtype == torch.float32 else torch.int16))
    return new, kept


@pytest.mark.parametrize("dtype,d,page,layout", [(torch.bfloat16, 128, 16, "phld"), (torch.float32, 40, 48, "plhd"), (torch.bfloat16, 64, 128, "phld")])
@pytest.mark.parametrize("keep,sinks,recent", [(64, 4, 16), (1, 0, 0), (1, 1, 0), (1, 0, 1), (100, 0, 100), (100, 60, 40), (37, 0, 0), (200, 3, 5)])
def test_evict(dtype, d, page, layout, keep, sinks, recent):
    evict(make([300, 64, 65, 0, 1, 38, 201], 2, d, page, dtype, weight=True, layout=layout), keep, sinks, recent)


def test_evict_equal_and_special_weights():
    cache = make([500, 500, 500, 500], 2, 64, weight=True)
    w = cache.weight
    w.copy_(torch.randint(0, 4, w.shape, device=DEV).float())               # many equal ones
    pages = cache.table[1, :31].long()
    w[pages] = 0.0
    w[pages[3]] = -0.0                                                      # both zeros are equal
    pages = cache.table[2, :31].long()
    w[pages[4], :, 3] = math.nan
    w[pages[5], :, 1] = math.inf
    w[pages[6]] = -math.inf
    w[pages[7]] = 1e-42                                                     # a denormal is more than zero
    cache.table[3, 7] = -1
    w[cache.table[3, :7].long()] = -math.inf
    evict(cache, 120, 3, 10)


@pytest.mark.parametrize("n,keep", [(5000, 2500), (1024, 1023), (1025, 1024), (2048, 7), (40000, 20000)])
def test_evict_longer(n, keep):
    evict(make([n], 1, 8, 64, weight=True), keep, min(4, keep), keep // 4)


@pytest.mark.parametrize("keep,sinks,recent", [(20000, 4, 3000), (24999, 0, 0), (5, 2, 3), (1, 0, 0), (8192, 8000, 192), (30000, 5, 9)])
def test_evict_caches_of_more_positions_than_lds_holds(keep, sinks, recent):
    """Sequences of several chunks of 8192 next to short ones, equal weights across chunk borders, a page that is none."""
    cache = make([25000, 8192, 300, 0, 40961], 2, 8, 48, weight=True)
    w = cache.weight
    w[cache.table[4, :].clamp(min=0).long()] = torch.randint(0, 3, (cache.table.shape[1], 2, 48), device=DEV).float()
    w[cache.table[0, 3].long()] = math.nan
    cache.table[4, 200] = -1
    evict(cache, keep, sinks, recent)


def test_evict_into_its_own_length():
    cache = make([300, 20], 1, 64, weight=True)
    cache.K = torch.cat([cache.K, cache.K])
    cache.V = torch.cat([cache.V, cache.V])
    cache.weight = torch.cat([cache.weight, cache.weight])
    n = cache.K.shape[0] // 2
    table = torch.arange(n, n + 10, dtype=torch.int32, device=DEV).reshape(2, 5)
    new, _ = rr.rr_cache_evict(cache, table, 80, 1, 8, length=cache.length)
    assert new.length is cache.length and cache.length.tolist() == [80, 20]


def test_a_captured_prompt_and_step():
    """Key weights, a write with them, a step's write and its attention in one graph, replayed on new inputs; two workspaces shared."""
    g = torch.Generator(device=DEV).manual_seed(8)
    cache = make([500], 2, 128, 16, weight=True)
    Q, K = torch.empty(1, 8, 500, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 2, 500, 128, dtype=torch.bfloat16, device=DEV)
    lse, first = torch.empty(1, 8, 500, device=DEV), torch.empty(1, 2, 500, device=DEV)
    q, O = torch.empty(1, 8, 1, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 8, 1, 128, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(max(rr.rr_key_weights_workspace_bytes(Q, K), rr.rr_paged_workspace_bytes(q, cache, accumulate=True)), dtype=torch.uint8, device=DEV)

    def fill():
        for x in (Q, K, q):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        rr.rr_window_attn(Q, K, K, 500, 0, lse=lse)

    def work():
        rr.rr_key_weights(Q, K, lse, out=first, workspace=ws)
        rr.rr_paged_write(cache, K, K, weight=first)
        rr.rr_paged_attn(q, cache, accumulate=True, O=O, workspace=ws)
    fill()
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(4):
        fill()
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone(), first.clone(), cache.weight.clone()
        work()
        assert torch.equal(got[0], O) and torch.equal(got[1], first) and torch.equal(got[2], cache.weight)
        assert abs(float(first.sum()) - 8 * 500) < 0.1


def test_evict_captured():
    cache = make([700, 90], 2, 64, weight=True, spare=30)
    used = set(cache.table.flatten().tolist())
    free = [e for e in range(cache.K.shape[0]) if e not in used][:16]
    table = torch.tensor(free, dtype=torch.int32, device=DEV).reshape(2, 8)
    length, kept = torch.empty(2, dtype=torch.int32, device=DEV), torch.empty(2, 2, 128, dtype=torch.int32, device=DEV)
    rr.rr_cache_evict(cache, table, 128, 4, 30, length=length, kept=kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rr.rr_cache_evict(cache, table, 128, 4, 30, length=length, kept=kept)
    for _ in range(3):
        cache.weight.copy_(torch.rand(cache.weight.shape, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        want = evict_reference(cache, 128, 4, 30)
        assert [[j for j in k if j >= 0] for k in kept.reshape(4, 128).tolist()] == want


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_a_served_sequence(dtype, d):
    """Two prompts of different lengths: their attention, their keys' weights, into the pages, steps of one token with weights
    kept, an eviction, and more steps; every step against 64 bits."""
    Hq, Hkv, page, keep = 8, 2, 16, 100
    lengths, steps = [150, 97], 6
    g = torch.Generator(device=DEV).manual_seed(4)
    cache = rr.PagedCache.allocate(64, page, Hkv, d, 2, 12, DEV, dtype, weight=True)
    fill_pages(cache, torch.randperm(40, generator=torch.Generator().manual_seed(1)).int(), [n + 2 * steps for n in lengths])
    cache.length.zero_()

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV).to(dtype)
    # the prompts, padded to one tensor: rows behind a prompt are written nowhere
    T = max(lengths)
    Q, K, V = normal(2, Hq, T, d) * 2, normal(2, Hkv, T, d), normal(2, Hkv, T, d)
    first = torch.full((2, Hkv, T), 77.0, device=DEV)
    for b, n in enumerate(lengths):
        q, k, v = (x[b:b + 1, :, :n] for x in (Q, K, V))
        lse = torch.empty(1, Hq, n, device=DEV)
        O = rr.rr_window_attn(q, k, v, n, 0, lse=lse)
        seen = sees(torch.arange(n, device=DEV), n, 0, 0)
        for h in range(Hq):
            check_rows(O[0, h], lse[0, h], q[0, h], k[0, h // 4], v[0, h // 4], seen, dtype == torch.bfloat16)
        first[b, :, :n] = rr.rr_key_weights(q, k, lse)[0]
    count = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    cache.length.copy_(count)
    rr.rr_paged_write(cache, K, V, count, first)

    def step():
        cache.length.add_(1)
        rr.rr_paged_write(cache, normal(2, Hkv, 1, d), normal(2, Hkv, 1, d))
        q, before, lse = normal(2, Hq, 1, d) * 2, cache.weight.clone(), torch.empty(2, Hq, 1, device=DEV)
        O = rr.rr_paged_attn(q, cache, accumulate=True, lse=lse)
        check(cache, q, O, lse, before=before)
        return q
    for _ in range(steps):
        step()
    total = [float(sum(positions(cache, b, n + steps, kv, "weight")[0].sum() for kv in range(Hkv))) for b, n in enumerate(lengths)]
    assert all(abs(t - Hq * (n + steps)) < 1e-2 for t, n in zip(total, lengths))     # every query gave one per head
    want = evict_reference(cache, keep, 4, 32)
    table = torch.full((2, 12), -1, dtype=torch.int32, device=DEV)
    table[:, :8] = torch.arange(40, 56, dtype=torch.int32, device=DEV).reshape(2, 8)
    source = [positions(cache, b, lengths[b] + steps, kv, "K")[0] for b in range(2) for kv in range(Hkv)]
    cache, kept = rr.rr_cache_evict(cache, table, keep, 4, 32)
    for i in range(4):
        assert kept[i // 2, i % 2].tolist() == want[i]
        assert torch.equal(positions(cache, i // 2, keep, i % 2, "K")[0], source[i][want[i]])
    for _ in range(steps):
        step()
    assert cache.length.tolist() == [keep + steps] * 2
