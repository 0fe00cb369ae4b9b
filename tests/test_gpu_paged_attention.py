"""Attention over a paged cache against 64 bits: types, head layouts, pages, lengths, windows, weights, and where it can go wrong."""
import math

import pytest
import torch

import paper_2602_05853_amd as rr
from cache_util import U32, attend, check_rows, fill_pages, positions, sees

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(lengths, Hkv=2, d=128, page=16, dtype=torch.bfloat16, weight=False, seed=0, spare=3, layout="phld"):
    g = torch.Generator(device=DEV).manual_seed(seed)
    width = max(1, max(-(-n // page) for n in lengths)) + 1
    pages = sum(-(-n // page) for n in lengths) + spare
    cache = rr.PagedCache.allocate(pages, page, Hkv, d, len(lengths), width, DEV, dtype, weight)
    if layout == "plhd":
        cache.K, cache.V = (torch.empty(pages, page, Hkv, d, dtype=dtype, device=DEV).transpose(1, 2) for _ in range(2))
    cache.K.copy_(torch.randn(cache.K.shape, generator=g, device=DEV))
    cache.V.copy_(torch.randn(cache.V.shape, generator=g, device=DEV))
    if weight:
        cache.weight.copy_(torch.rand(cache.weight.shape, generator=g, device=DEV))
    fill_pages(cache, torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int(), lengths)
    return cache


def query(cache, Hq, T=1, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(cache.table.shape[0], Hq, T, cache.K.shape[3], generator=g, device=DEV) * 2).to(cache.K.dtype)


def check(cache, Q, O, lse, window=0, sinks=0, before=None):
    b, Hq, T, _ = Q.shape
    Hkv, page = cache.K.shape[1], cache.K.shape[2]
    G = Hq // Hkv
    want = None if before is None else before.double().clone()
    slack = None if before is None else torch.zeros_like(want)
    for i, n in enumerate(cache.length.tolist()):
        n = min(max(n, 0), cache.table.shape[1] * page)
        pos = torch.arange(n - T, n, device=DEV)
        for kv in range(Hkv):
            K, good = positions(cache, i, n, kv, "K")
            V, _ = positions(cache, i, n, kv, "V")
            seen = (sees(pos, n, window, sinks) & good).repeat(G, 1)
            h = slice(kv * G, kv * G + G)
            p, delta, m = check_rows(O[i, h].reshape(G * T, -1), lse[i, h].reshape(-1), Q[i, h].reshape(G * T, -1), K, V, seen,
                                     what=(i, kv, n))
            if want is not None and n:
                t = torch.arange(n, device=DEV)[good]
                at = cache.table[i].long()[t // page], kv, t % page
                want[at] += p.sum(0)[good]
                slack[at] = ((2 * delta[:, None] + (m + 24) * U32 + 4 * U32 * lse[i, h].reshape(-1, 1).abs().clamp(max=1e4)) * p).sum(0)[good]
    if want is not None:
        # G T terms are added, and their sum once to what was there
        tol = slack * 1.01 + (G * T + 2) * U32 * want.abs()
        err = (cache.weight.double() - want).abs()
        assert (err <= tol).all(), float((err - tol).max())


def run(cache, Hq, T=1, window=0, sinks=0, accumulate=False, **kw):
    Q = query(cache, Hq, T)
    lse = torch.full((Q.shape[0], Hq, T), 7.0, device=DEV)
    before = cache.weight.clone() if accumulate else None
    n = rr.rr_paged_workspace_bytes(Q, cache, window, sinks, accumulate)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)             # NaN, whatever it is read as
    O = rr.rr_paged_attn(Q, cache, window, sinks, accumulate, lse=lse, workspace=ws, **kw)
    check(cache, Q, O, lse, window, sinks, before)
    return Q, O, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (4, 4, 64), (6, 3, 80), (2, 1, 8), (4, 1, 40), (4, 2, 256), (3, 1, 200), (2, 2, 16)])
def test_types_heads_and_widths(dtype, Hq, Hkv, d):
    run(make([1, 0, 130, 777, 16], Hkv, d, dtype=dtype, weight=True), Hq, accumulate=True)


@pytest.mark.parametrize("Hq,Hkv,T", [(17, 1, 1), (32, 1, 1), (40, 1, 1), (8, 2, 5), (28, 4, 3), (4, 4, 9), (70, 2, 1)])
@pytest.mark.parametrize("d", [128, 64])
def test_more_rows_than_a_tile(Hq, Hkv, T, d):
    """Rows of several tiles of 16 or 32, steps of more positions than a sequence has."""
    run(make([2, 300, 0, 1025], Hkv, d, weight=True), Hq, T, accumulate=True)
    run(make([2, 300, 0, 1025], Hkv, d), Hq, T, window=140, sinks=3)


@pytest.mark.parametrize("page", [16, 32, 48, 64, 112, 128, 256])
@pytest.mark.parametrize("layout", ["phld", "plhd"])
def test_pages(page, layout):
    """Pages that end inside a tile, a block or behind both, in both orders of heads and slots."""
    run(make([page - 1, page, page + 1, 5 * page + 7, 1], page=page, layout=layout, weight=True), 8, accumulate=True)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (127, 0), (128, 128), (129, 200), (100000, 5), (300, 100000), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_windows(window, sinks, dtype):
    run(make([1, 128, 129, 255, 256, 1000, 0, 640], dtype=dtype, weight=True), 4, window=window, sinks=sinks, accumulate=True)


def test_many_sequences():
    """More sequences than a workgroup has threads, most of them empty or short."""
    g = torch.Generator().manual_seed(3)
    lengths = [int(n) for n in torch.randint(0, 40, (700,), generator=g)]
    lengths[5], lengths[650] = 2000, 900
    lengths[200:300] = [0] * 100
    run(make(lengths, 1, 64, weight=True), 2, accumulate=True)


@pytest.mark.parametrize("batch", [63, 64, 65, 256, 257])
@pytest.mark.parametrize("d,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_numbers_of_sequences(batch, d, dtype):
    """Around what a wave's lanes and a workgroup's threads hold; one long sequence last, so that the short ones share."""
    run(make([(7 * i) % 33 for i in range(batch - 1)] + [1500], 1, d, dtype=dtype, weight=True), 2, accumulate=True)


def test_memory_that_a_call_allocates_belongs_to_its_stream():
    cache = make([3000, 100], 2, 128, weight=True)
    Q = query(cache, 8)
    want = rr.rr_paged_attn(Q, cache)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = []
    for _ in range(8):
        got.append(rr.rr_paged_attn(Q, cache, stream=s))
        torch.full((1 << 20,), math.nan, device=DEV)                         # what the current stream frees and fills is not the call's
    s.synchronize()
    assert all(torch.equal(want, g) for g in got)


def test_a_workspace_with_gaps_is_refused():
    cache = make([3000], 2, 128)
    Q = query(cache, 8)
    ws = torch.empty(2 * rr.rr_paged_workspace_bytes(Q, cache), dtype=torch.uint8, device=DEV)
    with pytest.raises(rr.RRError):
        rr.rr_paged_attn(Q, cache, workspace=ws[::2])


def test_all_empty():
    cache = make([0, 0], weight=True)
    run(cache, 4, accumulate=True)


def test_uneven_lengths_share_a_launch():
    run(make([30000, 1, 17, 4097, 12000], 2, 128, page=64, weight=True), 8, accumulate=True)


def test_lengths_out_of_range_are_held():
    cache = make([64, 100, 33], weight=True)
    cap = cache.table.shape[1] * 16
    cache.length.copy_(torch.tensor([-5, 10 ** 9, 33], dtype=torch.int32))
    cache.table[1, -1] = cache.table[1, 0]
    assert cap >= 100
    run(cache, 4)


def test_entries_that_are_no_page():
    cache = make([200, 300, 64], weight=True)
    cache.table[0, 3] = -1
    cache.table[1, 0] = cache.K.shape[0]
    cache.table[1, 18] = 2 ** 31 - 1
    cache.table[2] = -7
    run(cache, 4, accumulate=True)
    run(cache, 4, window=20, sinks=20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_nobody_sees_may_hold_anything(dtype):
    """Infinities and NaN behind the end, in unseen pages, and between sinks and window."""
    cache = make([300, 77], dtype=dtype, weight=True)
    own = set(cache.table[cache.table >= 0].tolist())
    for e in range(cache.K.shape[0]):
        if e not in own:
            cache.K[e], cache.V[e] = math.nan, math.inf
    for b, n in ((0, 300), (1, 77)):
        e = int(cache.table[b, n // 16])
        cache.K[e, :, n % 16:], cache.V[e, :, n % 16:] = math.inf, math.nan
    e = int(cache.table[0, 5])                                              # positions 80 .. 95
    cache.V[e] = math.nan
    cache.K[e, :, :8] = math.nan
    cache.K[e, :, 8:] = math.inf
    run(cache, 4, window=64, sinks=10, accumulate=True)


def test_infinite_values_that_are_seen():
    cache = make([100], Hkv=1, d=64)
    cache.V[int(cache.table[0, 2]), 0, 3, 5] = math.inf
    Q = query(cache, 2)
    O = rr.rr_paged_attn(Q, cache)
    assert (O[..., 5] == math.inf).all()
    O[..., 5] = 0
    assert O.isfinite().all()


def test_large_scores():
    """Scores of thousands: one key takes everything."""
    cache = make([500], Hkv=1, d=128, dtype=torch.float32)
    cache.K.mul_(300.0)
    Q, O, lse = run(cache, 2)
    assert O.isfinite().all() and lse.abs().max() > 1000


def test_strided_queries_and_kept_outputs():
    cache = make([64, 200], 2, 64)
    big = torch.randn(2, 3, 4, 96, device=DEV).to(torch.bfloat16)
    Q = big.transpose(1, 2)[:, :, 1:2, :64]                                  # [2, 4, 1, 64], row stride 4 * 96
    out = torch.full((2, 3, 4, 96), 3.0, dtype=torch.bfloat16, device=DEV)
    O = out.transpose(1, 2)[:, :, 1:2, :64]
    lse = torch.empty(2, 4, 1, device=DEV)
    assert rr.rr_paged_attn(Q, cache, O=O, lse=lse) is O
    check(cache, Q, O, lse)
    O.fill_(3.0)
    assert (out == 3.0).all()                                                # nothing beside the rows was written


def test_max_length_and_default_workspace():
    cache = make([50, 40], 2, 128, page=64)
    Q = query(cache, 8)
    a = rr.rr_paged_attn(Q, cache)
    assert torch.equal(a, rr.rr_paged_attn(Q, cache, max_length=64))
    # lengths are held to it
    cut = rr.rr_paged_attn(Q, cache, max_length=45)
    cache.length.clamp_(max=45)
    assert torch.equal(cut, rr.rr_paged_attn(Q, cache, max_length=45))


def test_pages_shared_by_sequences():
    cache = make([160, 200], 2, 128)
    cache.table[1, :10] = cache.table[0, :10]
    run(cache, 4)


def test_equal_calls_give_equal_bits_on_any_stream():
    cache = make([5000, 30, 900], 2, 128, weight=True)
    Q = query(cache, 8)
    w0 = cache.weight.clone()
    a = rr.rr_paged_attn(Q, cache, accumulate=True)
    wa = cache.weight.clone()
    cache.weight.copy_(w0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = rr.rr_paged_attn(Q, cache, accumulate=True, stream=s, workspace=torch.empty(1 << 26, dtype=torch.uint8, device=DEV))
    s.synchronize()
    assert torch.equal(a, b) and torch.equal(wa, cache.weight)


def test_captured_steps():
    """Two captured steps that share a workspace, replayed with eager work in between and lengths that grow."""
    cache = make([900, 64, 333], 2, 128, weight=True)
    cache.table[1, 4:6] = torch.tensor([cache.K.shape[0] - 1, cache.K.shape[0] - 2], dtype=torch.int32)
    own = cache.table[[0, 2]].flatten().tolist()
    free = [e for e in range(cache.K.shape[0]) if e not in own and e not in cache.table[1, :4].tolist()]
    cache.table[1, 4:6] = torch.tensor(free[:2], dtype=torch.int32, device=DEV)
    Q, Q2 = query(cache, 8), query(cache, 8, seed=9)
    ws = torch.empty(rr.rr_paged_workspace_bytes(Q, cache, accumulate=True), dtype=torch.uint8, device=DEV)
    O, O2 = torch.empty_like(Q), torch.empty_like(Q)
    lse = torch.empty(3, 8, 1, device=DEV)
    rr.rr_paged_attn(Q, cache, accumulate=True, O=O, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rr.rr_paged_attn(Q, cache, accumulate=True, O=O, lse=lse, workspace=ws)
        rr.rr_paged_attn(Q2, cache, window=100, sinks=4, O=O2, workspace=ws)
    for step in range(4):
        cache.length[1] += 5
        before = cache.weight.clone()
        graph.replay()
        torch.cuda.synchronize()
        check(cache, Q, O, lse, before=before)
        cache.weight.copy_(before)
        assert torch.equal(O2, rr.rr_paged_attn(Q2, cache, window=100, sinks=4))
        assert torch.equal(O, rr.rr_paged_attn(Q, cache))


def test_long_cache_past_32_bit_offsets():
    """A pool of more than 2^31 elements, whose last pages a sequence uses."""
    page, Hkv, d = 128, 8, 128
    pages = 2 ** 31 // (page * Hkv * d) + 40
    pool = torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device=DEV)
    other = torch.empty_like(pool)
    cache = rr.PagedCache(pool, other, torch.tensor([[pages - 1, 0, pages - 2, pages - 3]], dtype=torch.int32, device=DEV),
                          torch.tensor([450], dtype=torch.int32, device=DEV))
    for e in (pages - 1, 0, pages - 2, pages - 3):
        pool[e] = torch.randn(Hkv, page, d, device=DEV).to(torch.bfloat16)
        other[e] = torch.randn(Hkv, page, d, device=DEV).to(torch.bfloat16)
    run(cache, 32)


def test_reference_of_a_row_by_hand():
    """One key: O is its value, lse its score."""
    cache = make([1], Hkv=1, d=64, dtype=torch.float32)
    Q, O, lse = run(cache, 1)
    K, _ = positions(cache, 0, 1, 0, "K")
    V, _ = positions(cache, 0, 1, 0, "V")
    assert torch.equal(O[0, 0], V)
    ref = attend(Q[0, 0], K, V, torch.ones(1, 1, dtype=torch.bool, device=DEV))
    assert abs(float(lse) - float(ref[1])) <= float(ref[4]) + 8 * U32 * abs(float(ref[1]))


def test_empty_sequences_between():
    """Workgroups whose shares cross hundreds of empty sequences, in batches of one wave's lanes and of more."""
    for batch in (60, 900):
        lengths = [0] * batch
        for b, n in ((0, 130), (1, 700), (batch // 2, 5), (batch - 2, 1300), (batch - 1, 257)):
            lengths[b] = n
        run(make(lengths, 3, 64, weight=True), 6, accumulate=True)
