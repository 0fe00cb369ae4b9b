"""Attention with a sliding window and sinks against 64 bits."""
import math

import pytest
import torch

import paper_2602_05853_amd as rr
from cache_util import check_rows, sees

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(L, Lq, Hq=4, Hkv=2, d=128, dtype=torch.bfloat16, batch=1, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = [(torch.randn(batch, h, n, d, generator=g, device=DEV) * by).to(dtype) for h, n, by in ((Hq, Lq, 2.0), (Hkv, L, 1.0), (Hkv, L, 1.0))]
    return t


def matrix_kernel(Q, K):
    """Whether a call without packed sequences runs on the kernel that rounds probabilities to bf16."""
    (b, Hq, Lq, d), L = Q.shape, K.shape[2]
    return Q.dtype == torch.bfloat16 and d == 128 and b * Hq * ((L - 1) // 128 - (L - Lq) // 128 + 1) > 128


def check(Q, K, V, O, lse, window, sinks, start=None, rounded_p=None, rows=None, entries=None):
    (b, Hq, Lq, d), (Hkv, L) = Q.shape, K.shape[1:3]
    G = Hq // Hkv
    pos = torch.arange(L - Lq, L, device=DEV)
    rows = torch.arange(Lq, device=DEV) if rows is None else rows
    seen = sees(pos[rows], L, window, sinks, 0 if start is None else start[rows])
    rounded = matrix_kernel(Q, K) if rounded_p is None else rounded_p
    for i in range(b) if entries is None else entries:
        for h in range(Hq):
            check_rows(O[i, h, rows], None if lse is None else lse[i, h, rows], Q[i, h, rows], K[i, h // G], V[i, h // G], seen, rounded,
                       what=(i, h))


def run(L, Lq, window, sinks, **kw):
    Q, K, V = make(L, Lq, **kw)
    lse = torch.full(Q.shape[:3], 5.0, device=DEV)
    O = rr.rr_window_attn(Q, K, V, window, sinks, lse=lse)
    check(Q, K, V, O, lse, window, sinks)
    return Q, K, V, O, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [8, 40, 64, 80, 96, 128, 168, 256])
def test_types_and_widths(dtype, d):
    run(333, 333, 50, 3, d=d, dtype=dtype)
    run(333, 100, 200, 17, d=d, dtype=dtype, Hq=3, Hkv=1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,Lq", [(1, 1), (2, 2), (127, 127), (128, 128), (129, 129), (1000, 1000), (1000, 1), (1000, 129), (700, 333), (640, 256)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (17, 0), (64, 70), (128, 0), (129, 4), (300, 128), (256, 260), (100000, 0), (90, 100000)])
def test_lengths_windows_and_sinks(d, L, Lq, window, sinks):
    run(L, Lq, window, sinks, d=d)


@pytest.mark.parametrize("L,Lq", [(1, 1), (127, 127), (128, 128), (129, 129), (1000, 1000), (1000, 20), (1000, 129), (700, 333), (640, 256)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (17, 0), (64, 70), (128, 0), (129, 4), (300, 128), (256, 260), (513, 64), (100000, 0), (90, 100000)])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (14, 2)])
def test_matrix_kernel(Hq, Hkv, L, Lq, window, sinks):
    """bf16, d = 128, on more than 128 query blocks: the first and the last entry of a batch that has as many."""
    batch = 128 // (Hq * ((L - 1) // 128 - (L - Lq) // 128 + 1)) + 1
    Q, K, V = make(L, Lq, Hq=Hq, Hkv=Hkv, batch=batch)
    assert matrix_kernel(Q, K)
    lse = torch.full(Q.shape[:3], 5.0, device=DEV)
    O = rr.rr_window_attn(Q, K, V, window, sinks, lse=lse)
    check(Q, K, V, O, lse, window, sinks, entries=[0, batch - 1])


def test_matrix_kernel_of_values_that_nobody_sees_and_one_that_is_infinite():
    Q, K, V = make(900, 40, batch=65)
    window, sinks = 60, 5
    gap = slice(sinks, 900 - 40 - window + 1)
    K[:, :, gap], V[:, :, gap] = math.nan, math.inf
    lse = torch.empty(Q.shape[:3], device=DEV)
    O = rr.rr_window_attn(Q, K, V, window, sinks, lse=lse)
    assert matrix_kernel(Q, K)
    check(Q, K, V, O, lse, window, sinks, entries=[0, 64])
    Q, K, V = make(600, 600, Hq=2, Hkv=1, batch=14)
    assert matrix_kernel(Q, K)
    V[3, 0, 200, 7] = math.inf
    O = rr.rr_window_attn(Q, K, V, 100, 0)
    assert (O[3, :, 200:300, 7] == math.inf).all()
    O[3, :, 128:384, 7] = 0
    assert O.isfinite().all()


def test_matrix_kernel_strides_and_what_lies_beside():
    g = torch.Generator(device=DEV).manual_seed(2)

    def inside(n, heads, fill):
        big = torch.full((10, n + 2, heads + 1, 144), fill, dtype=torch.bfloat16, device=DEV)
        return big, big[:, 1:n + 1, :heads, 8:136].transpose(1, 2)
    bigs, views = zip(*(inside(n, h, math.nan) for n, h in ((200, 8), (300, 2), (300, 2))))
    for v in views:
        v.copy_(torch.randn(v.shape, generator=g, device=DEV))
    Q, K, V = views
    assert matrix_kernel(Q, K)
    out, O = inside(200, 8, 3.0)
    lse = torch.empty(Q.shape[:3], device=DEV)
    rr.rr_window_attn(Q, K, V, 77, 9, O=O, lse=lse)
    check(Q, K, V, O, lse, 77, 9, entries=[0, 9])
    O.fill_(3.0)
    assert (out == 3.0).all()


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128)])
def test_a_window_over_everything_is_dense(dtype, d):
    Q, K, V, O, lse = run(500, 500, 2 ** 31 - 1, 2 ** 31 - 1, dtype=dtype, d=d)
    B = 64 if d * 128 > 8192 else 128
    want = torch.empty_like(lse)
    dense = rr.rr_dense_attn(Q, K, V, B, lse=want)
    assert (O.float() - dense.float()).abs().max() <= 0.05 and (lse - want).abs().max() <= 1e-4


@pytest.mark.parametrize("L,window,sinks", [(4096, 1024, 4), (5000, 1111, 130), (3000, 128 * 9, 256), (2048, 640, 0)])
def test_longer_prompts(L, window, sinks):
    Q, K, V = make(L, L, Hq=8, Hkv=2)
    lse = torch.empty(Q.shape[:3], device=DEV)
    O = rr.rr_window_attn(Q, K, V, window, sinks, lse=lse)
    check(Q, K, V, O, lse, window, sinks)


@pytest.mark.parametrize("dtype,d,B", [(torch.bfloat16, 128, 128), (torch.bfloat16, 128, 64), (torch.bfloat16, 64, 48), (torch.float32, 80, 16)])
@pytest.mark.parametrize("window,sinks", [(20, 0), (100, 5), (300, 200), (10000, 0)])
def test_packed_sequences(dtype, d, B, window, sinks):
    blocks = [3, 1, 1, 7, 2, 4]
    L = B * sum(blocks) - 9
    Q, K, V = make(L, L, d=d, dtype=dtype, batch=2, Hq=8)
    sf = rr.packed_seq_first(blocks, DEV)
    lse = torch.empty(Q.shape[:3], device=DEV)
    O = rr.rr_window_attn(Q, K, V, window, sinks, lse=lse, seq_first=sf, B=B)
    start = (sf.long() * B).repeat_interleave(B)[:L]
    check(Q, K, V, O, lse, window, sinks, start=start, rounded_p=d == 128 and B == 128 and dtype == torch.bfloat16)


@pytest.mark.parametrize("dtype,d,Hq,Hkv", [(torch.bfloat16, 128, 8, 2), (torch.bfloat16, 128, 32, 1), (torch.bfloat16, 64, 6, 3), (torch.float32, 80, 4, 1)])
@pytest.mark.parametrize("L,Lq", [(1, 1), (1000, 1), (5000, 1), (3000, 4)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (200, 4), (1025, 130), (100000, 0)])
def test_steps_with_a_workspace(dtype, d, Hq, Hkv, L, Lq, window, sinks):
    Q, K, V = make(L, Lq, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, batch=2)
    n = rr.rr_window_workspace_bytes(Q, K, window, sinks)
    step = Hq // Hkv * Lq <= 32
    assert n == 0 or step
    ws = torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device=DEV)
    lse = torch.empty(Q.shape[:3], device=DEV)
    O = rr.rr_window_attn(Q, K, V, window, sinks, lse=lse, workspace=ws)
    check(Q, K, V, O, lse, window, sinks, rounded_p=False if step else None)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
def test_strides_and_what_lies_beside(dtype, d):
    """[batch, L, heads, d] tensors inside wider ones: reads stay in them, writes too."""
    L, Lq, H = 300, 200, 4
    g = torch.Generator(device=DEV).manual_seed(2)

    def inside(n, heads, fill):
        big = torch.full((2, n + 2, heads + 1, d + 16), fill, dtype=dtype, device=DEV)
        return big, big[:, 1:n + 1, :heads, 8:8 + d].transpose(1, 2)
    bigs, views = zip(*(inside(n, h, math.nan) for n, h in ((Lq, H), (L, 2), (L, 2))))
    for v in views:
        v.copy_(torch.randn(v.shape, generator=g, device=DEV))
    Q, K, V = views
    out, O = inside(Lq, H, 3.0)
    lse = torch.empty(Q.shape[:3], device=DEV)
    rr.rr_window_attn(Q, K, V, 77, 9, O=O, lse=lse)
    check(Q, K, V, O, lse, 77, 9)
    O.fill_(3.0)
    assert (out == 3.0).all()


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
def test_values_that_nobody_sees(dtype, d):
    """Keys between the sinks and the windows of the step's queries."""
    Q, K, V = make(900, 40, d=d, dtype=dtype)
    window, sinks = 60, 5
    K[:, :, sinks:900 - 40 - window + 1], V[:, :, sinks:900 - 40 - window + 1] = math.nan, math.inf
    lse = torch.empty(Q.shape[:3], device=DEV)
    O = rr.rr_window_attn(Q, K, V, window, sinks, lse=lse)
    check(Q, K, V, O, lse, window, sinks)


def test_one_infinite_value_reaches_the_rows_that_see_it():
    Q, K, V = make(600, 600, Hq=2, Hkv=1)
    V[0, 0, 200, 7] = math.inf
    O = rr.rr_window_attn(Q, K, V, 100, 0)
    assert (O[0, :, 200:300, 7] == math.inf).all()
    rest = O.clone()
    rest[0, :, 128:384, 7] = 0                                # tiles of queries that hold a row which sees it
    assert rest.isfinite().all()


def test_captured_and_replayed():
    Q, K, V = make(700, 700, Hq=24, Hkv=2)                    # 144 query blocks: the matrix kernel
    assert matrix_kernel(Q, K)
    step = Q[:, :, -1:].contiguous()
    ws = torch.empty(rr.rr_window_workspace_bytes(step, K, 300, 4), dtype=torch.uint8, device=DEV)
    O, S = torch.empty_like(Q), torch.empty_like(step)
    rr.rr_window_attn(Q, K, V, 300, 4, O=O)
    rr.rr_window_attn(step, K, V, 300, 4, O=S, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rr.rr_window_attn(Q, K, V, 300, 4, O=O)
        rr.rr_window_attn(step, K, V, 300, 4, O=S, workspace=ws)
    for k in range(4):
        Q.mul_(-1.0)
        step.mul_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, rr.rr_window_attn(Q, K, V, 300, 4))
        assert torch.equal(S, rr.rr_window_attn(step, K, V, 300, 4, workspace=ws))


def test_batch_on_another_stream():
    Q, K, V = make(400, 400, batch=12)
    assert matrix_kernel(Q, K)
    want = rr.rr_window_attn(Q, K, V, 128, 4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = rr.rr_window_attn(Q, K, V, 128, 4, stream=s)
    s.synchronize()
    assert torch.equal(want, got)
