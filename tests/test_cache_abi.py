"""Host side of window attention, the paged cache, key weights and eviction: arguments that are refused before any launch, sizes
of workspaces, and the layout of the struct."""
import ctypes as C
import os

import pytest
import torch

import paper_2602_05853_amd as rr
from paper_2602_05853_amd import binding as bd

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rr_attn.h")
FAKE = 0x1000


def shape(L=4096, Lq=1, Hq=32, Hkv=8, d=128, dtype=bd.RR_BF16, batch=2, page=64):
    return bd.rr_shape(batch, L, Hq, Hkv, d, dtype, Hq * Lq * d, Lq * d, d, Hkv * page * d, page * d, d, Lq)


def pages(page=64, num=200, width=64, **kw):
    f = dict(K=FAKE, V=FAKE, weight=FAKE, table=FAKE, length=FAKE)
    f.update(kw)
    return bd.rr_paged_cache(f["K"], f["V"], f["weight"], f["table"], f["length"], page, num, width)


def test_struct_layout(tmp_path):
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rr_attn.h"\nint main(void) { printf("%zu %zu %zu %zu %u\\n", '
                   'sizeof(rr_paged_cache), offsetof(rr_paged_cache, weight), offsetof(rr_paged_cache, page), '
                   'offsetof(rr_paged_cache, width), RR_FLAG_ACCUMULATE); return 0; }\n')
    exe = tmp_path / "layout"
    subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)], check=True)
    got = list(map(int, subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()))
    c = bd.rr_paged_cache
    assert got == [C.sizeof(c), c.weight.offset, c.page.offset, c.width.offset, bd.RR_FLAG_ACCUMULATE]


def attn(s=None, c=None, Q=FAKE, window=0, sinks=0, flags=0, O=FAKE, ws=FAKE * 16, n=1 << 40):
    return bd.lib.rr_paged_attn(C.byref(s or shape()), Q, C.byref(c or pages()), window, sinks, flags, O, None, ws, n, None)


def test_paged_attention_refusals():
    assert attn(ws=None) == bd.RR_ERR_WORKSPACE and attn(n=100) == bd.RR_ERR_WORKSPACE and attn(ws=FAKE * 16 + 64) == bd.RR_ERR_WORKSPACE
    assert attn(Q=None) == bd.RR_ERR_NULL and attn(O=None) == bd.RR_ERR_NULL
    for name in ("K", "V", "table", "length"):
        assert attn(c=pages(**{name: None})) == bd.RR_ERR_NULL
    assert attn(c=pages(weight=FAKE + 4), flags=1) == bd.RR_ERR_SHAPE
    assert attn(c=pages(weight=None), flags=1) == bd.RR_ERR_NULL and attn(c=pages(weight=None), ws=None) == bd.RR_ERR_WORKSPACE
    assert bd.lib.rr_paged_attn(C.byref(shape()), FAKE, None, 0, 0, 0, FAKE, None, FAKE * 16, 1 << 40, None) == bd.RR_ERR_NULL
    assert bd.lib.rr_paged_attn(None, FAKE, C.byref(pages()), 0, 0, 0, FAKE, None, FAKE * 16, 1 << 40, None) == bd.RR_ERR_NULL
    assert attn(window=-1) == bd.RR_ERR_PARAM and attn(sinks=-1) == bd.RR_ERR_PARAM and attn(flags=2) == bd.RR_ERR_PARAM
    for page in (0, 8, 24, 100, -16):
        assert attn(c=pages(page=page)) == bd.RR_ERR_SHAPE
    assert attn(c=pages(num=0)) == bd.RR_ERR_SHAPE and attn(c=pages(width=0)) == bd.RR_ERR_SHAPE
    assert attn(c=pages(width=63)) == bd.RR_ERR_SHAPE                        # the table does not hold L positions
    assert attn(s=shape(L=4, Lq=5)) == bd.RR_ERR_SHAPE                       # more rows than positions
    assert attn(s=shape(d=12)) == bd.RR_ERR_SHAPE and attn(s=shape(Hq=30)) == bd.RR_ERR_SHAPE and attn(s=shape(dtype=3)) == bd.RR_ERR_DTYPE
    assert attn(Q=FAKE + 2) == bd.RR_ERR_SHAPE and attn(c=pages(K=FAKE + 8)) == bd.RR_ERR_SHAPE
    s = shape()
    s.q_stride_h = 0                                                         # outputs that would lie on each other
    assert attn(s=s) == bd.RR_ERR_SHAPE
    s = shape()
    s.kv_stride_l = 130
    assert attn(s=s) == bd.RR_ERR_SHAPE
    s = shape(L=(1 << 30) + 1)
    assert attn(s=s, c=pages(page=1 << 20, width=1 << 20)) == bd.RR_ERR_SHAPE
    # more blocks than a launch's 32-bit sums hold
    s = shape(L=1 << 30, batch=300)
    assert attn(s=s, c=pages(page=1 << 20, width=1 << 10)) == bd.RR_ERR_SHAPE


def workspace(s, c=None, window=0, sinks=0, flags=0):
    return bd.lib.rr_paged_workspace_bytes(C.byref(s), C.byref(c or pages(K=None, V=None, table=None, length=None, weight=None)), window, sinks, flags)


def test_paged_workspace():
    assert workspace(shape()) > 0 and workspace(shape(), flags=4) == 0 and workspace(shape(), window=-1) == 0
    assert workspace(shape(d=12)) == 0 and workspace(shape(), pages(page=10)) == 0
    # with weights: one fp32 score per row and position more, and a sum per row
    more = workspace(shape(), flags=1) - workspace(shape())
    assert more == 2 * 8 * 32 * 4 * 128 * 4 + 2 * 32 * 4
    # a window bounds it
    assert workspace(shape(), window=64, flags=1) < workspace(shape(), flags=1)


@pytest.mark.parametrize("window", [1, 2, 127, 128, 129, 130, 255, 256, 257, 1000])
@pytest.mark.parametrize("sinks", [0, 1, 128, 129, 400])
def test_workspace_covers_every_length(window, sinks):
    """The scores of a call are as many as the blocks that a length visits, and some lengths visit more than longer ones."""
    s = shape(L=2048, Hq=4, Hkv=1, batch=1, Lq=2)
    room = (workspace(s, window=window, sinks=sinks, flags=1) - workspace(s, window=window, sinks=sinks) - 256) // (8 * 128 * 4)
    for n in range(1, 2049):
        seen = set()
        for i in range(max(0, n - 2), n):
            seen |= set(range(max(0, i - window + 1) // 128, i // 128 + 1)) | set(range(0, (min(sinks, i + 1) + 127) // 128))
        assert len(seen) <= room, n


def test_window_refusals():
    def call(s=None, Q=FAKE, K=FAKE, V=FAKE, window=100, sinks=0, sf=None, B=128, O=FAKE, ws=None, n=0):
        return bd.lib.rr_window_attn(C.byref(s or shape()), Q, K, V, window, sinks, sf, B, O, None, ws, n, None)
    assert call(Q=None) == bd.RR_ERR_NULL and call(K=None) == bd.RR_ERR_NULL and call(V=None) == bd.RR_ERR_NULL and call(O=None) == bd.RR_ERR_NULL
    assert call(window=0) == bd.RR_ERR_PARAM and call(window=-4) == bd.RR_ERR_PARAM and call(sinks=-1) == bd.RR_ERR_PARAM
    assert call(Q=FAKE + 4) == bd.RR_ERR_SHAPE and call(V=FAKE + 8) == bd.RR_ERR_SHAPE and call(O=FAKE + 8) == bd.RR_ERR_SHAPE
    assert call(s=shape(d=300)) == bd.RR_ERR_SHAPE and call(s=shape(dtype=9)) == bd.RR_ERR_DTYPE and call(s=shape(Lq=5000)) == bd.RR_ERR_SHAPE
    assert call(sf=FAKE) == bd.RR_ERR_PARAM                                  # packed sequences and a step
    for B in (0, 8, 24, 144, -16):
        assert call(s=shape(Lq=4096), sf=FAKE, B=B) == bd.RR_ERR_SHAPE
    # a workspace counts where the call takes one
    assert call(window=1000, ws=FAKE * 16, n=16) == bd.RR_ERR_WORKSPACE and call(window=1000, ws=FAKE * 16 + 8, n=1 << 40) == bd.RR_ERR_WORKSPACE

    def room(s, window=100):
        return bd.lib.rr_window_workspace_bytes(C.byref(s), window, 0)
    assert room(shape(), 1000) > 0 and room(shape(Lq=8), 1000) > 0 and room(shape()) == 0 and room(shape(Lq=9)) == 0 and room(shape(Lq=17, Hq=8)) == 0
    assert room(shape(), 0) == 0 and room(shape(d=9)) == 0


def test_write_weights_and_evict_refusals():
    def write(s=None, c=None, K=FAKE, V=FAKE, weight=None):
        return bd.lib.rr_paged_write(C.byref(s or shape()), C.byref(c or pages()), K, V, None, weight, None)
    assert write(K=None) == bd.RR_ERR_NULL and write(V=None) == bd.RR_ERR_NULL and write(c=pages(K=None)) == bd.RR_ERR_NULL
    assert write(c=pages(weight=None), weight=FAKE) == bd.RR_ERR_NULL
    assert write(K=FAKE + 2) == bd.RR_ERR_SHAPE and write(s=shape(batch=70000)) == bd.RR_ERR_SHAPE

    def evict(s=None, c=None, keep=100, sinks=4, recent=10, to=FAKE, width=2, length=FAKE, kept=FAKE, ws=None, n=0):
        return bd.lib.rr_cache_evict(C.byref(s or shape()), C.byref(c or pages()), keep, sinks, recent, to, width, length, kept, ws, n, None)
    long, wide = shape(L=30000), pages(width=500)
    assert bd.lib.rr_cache_evict_workspace_bytes(C.byref(shape()), C.byref(pages())) == 0
    need = bd.lib.rr_cache_evict_workspace_bytes(C.byref(long), C.byref(wide))
    assert need >= 3 * 16 * 2048 * 4
    for ws, n in ((None, 1 << 40), (FAKE * 16, need - 1), (FAKE * 16 + 64, 1 << 40)):
        assert evict(s=long, c=wide, ws=ws, n=n) == bd.RR_ERR_WORKSPACE
    assert evict(c=pages(weight=FAKE + 4)) == bd.RR_ERR_SHAPE
    assert evict(c=pages(weight=None)) == bd.RR_ERR_NULL and evict(to=None) == bd.RR_ERR_NULL and evict(length=None) == bd.RR_ERR_NULL
    assert evict(kept=None) == bd.RR_ERR_NULL
    assert evict(keep=0) == bd.RR_ERR_PARAM and evict(sinks=-1) == bd.RR_ERR_PARAM and evict(recent=-1) == bd.RR_ERR_PARAM
    assert evict(sinks=60, recent=41) == bd.RR_ERR_PARAM and evict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1) == bd.RR_ERR_PARAM
    assert evict(width=1) == bd.RR_ERR_SHAPE and evict(width=0) == bd.RR_ERR_SHAPE and evict(s=shape(batch=70000)) == bd.RR_ERR_SHAPE

    def weights(s=None, Q=FAKE, K=FAKE, lse=FAKE, out=FAKE, ws=FAKE * 16, n=1 << 40):
        return bd.lib.rr_key_weights(C.byref(s or shape(Lq=512)), Q, K, lse, out, ws, n, None)
    assert bd.lib.rr_key_weights_workspace_bytes(C.byref(shape(Lq=512))) > 0 == bd.lib.rr_key_weights_workspace_bytes(C.byref(shape(Lq=1)))
    assert weights(ws=None) == bd.RR_ERR_WORKSPACE and weights(n=64) == bd.RR_ERR_WORKSPACE and weights(ws=FAKE * 16 + 16) == bd.RR_ERR_WORKSPACE
    assert weights(Q=None) == bd.RR_ERR_NULL and weights(lse=None) == bd.RR_ERR_NULL and weights(out=None) == bd.RR_ERR_NULL
    assert weights(K=FAKE + 2) == bd.RR_ERR_SHAPE and weights(s=shape(batch=70000)) == bd.RR_ERR_SHAPE


def refused(status, f, *a, **kw):
    with pytest.raises(rr.RRError) as e:
        f(*a, **kw)
    assert e.value.status == status


def test_binding_refusals():
    """Wrong tensors never reach the library; neither do tensors that are not on a GPU."""
    def cache(**kw):
        c = rr.PagedCache.allocate(8, 16, 2, 64, 3, 4, "cpu", weight=True)
        for k, v in kw.items():
            setattr(c, k, v)
        return c
    Q = torch.zeros(3, 4, 1, 64, dtype=torch.bfloat16)
    refused(bd.RR_ERR_PARAM, rr.rr_paged_attn, Q, cache())                   # on the CPU
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q[:2], cache())
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q[..., :32], cache())
    refused(bd.RR_ERR_DTYPE, rr.rr_paged_attn, Q.float(), cache())
    refused(bd.RR_ERR_DTYPE, rr.rr_paged_attn, Q, cache(table=torch.zeros(3, 4, dtype=torch.int64)))
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q, cache(table=torch.zeros(4, 3, dtype=torch.int32).T))
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q, cache(length=torch.zeros(2, dtype=torch.int32)))
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q, cache(weight=torch.zeros(8, 2, 17)))
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q, cache(V=torch.zeros(8, 2, 16, 32, dtype=torch.bfloat16)))
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q, cache(), O=torch.zeros(3, 4, 2, 64, dtype=torch.bfloat16))
    refused(bd.RR_ERR_DTYPE, rr.rr_paged_attn, Q, cache(), lse=torch.zeros(3, 4, 1, dtype=torch.float64))
    new = torch.zeros(3, 2, 5, 64, dtype=torch.bfloat16)
    refused(bd.RR_ERR_PARAM, rr.rr_paged_write, cache(), new, new)
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_write, cache(), new[:, :1], new[:, :1])
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_write, cache(), new, new[:, :, :4])
    refused(bd.RR_ERR_DTYPE, rr.rr_paged_write, cache(), new, new, torch.zeros(3))
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_write, cache(), new, new, None, torch.zeros(3, 2, 4))
    table = torch.zeros(3, 2, dtype=torch.int32)
    refused(bd.RR_ERR_PARAM, rr.rr_cache_evict, cache(), table, 20)
    refused(bd.RR_ERR_PARAM, rr.rr_cache_evict, cache(), table, 0)
    refused(bd.RR_ERR_SHAPE, rr.rr_cache_evict, cache(), table[:2], 20)
    refused(bd.RR_ERR_DTYPE, rr.rr_cache_evict, cache(), table.long(), 20)
    q, k = torch.zeros(1, 4, 8, 64), torch.zeros(1, 2, 8, 64)
    refused(bd.RR_ERR_PARAM, rr.rr_window_attn, q, k, k, 4)
    refused(bd.RR_ERR_DTYPE, rr.rr_window_attn, q, k.bfloat16(), k, 4)
    refused(bd.RR_ERR_SHAPE, rr.rr_window_attn, q, k, k[:, :, :7], 4)
    refused(bd.RR_ERR_SHAPE, rr.rr_window_attn, q, k, k, 4, lse=torch.zeros(1, 4, 7))
    refused(bd.RR_ERR_PARAM, rr.rr_window_attn, q, k, k, 4, seq_first=torch.zeros(3, dtype=torch.int32))
    refused(bd.RR_ERR_PARAM, rr.rr_key_weights, q, k, torch.zeros(1, 4, 8))
    refused(bd.RR_ERR_SHAPE, rr.rr_key_weights, q, k, torch.zeros(1, 4, 9))
    refused(bd.RR_ERR_SHAPE, rr.rr_window_attn, q[:, :, :0], k, k, 4)        # no queries
    refused(bd.RR_ERR_SHAPE, rr.rr_key_weights, q[:, :, :0], k, torch.zeros(1, 4, 0))
    refused(bd.RR_ERR_SHAPE, rr.rr_paged_attn, Q[:, :, :0], cache())


def test_numbers_that_32_bits_do_not_hold():
    """ctypes would take their low bits."""
    q, k = torch.zeros(1, 4, 8, 64), torch.zeros(1, 2, 8, 64)
    c = rr.PagedCache.allocate(8, 16, 2, 64, 3, 4, "cpu", weight=True)
    Q = torch.zeros(3, 4, 1, 64, dtype=torch.bfloat16)
    for big in (2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1):
        refused(bd.RR_ERR_PARAM, rr.rr_window_attn, q, k, k, big)
        refused(bd.RR_ERR_PARAM, rr.rr_window_attn, q, k, k, 4, big)
        refused(bd.RR_ERR_PARAM, rr.rr_window_workspace_bytes, q, k, big)
        refused(bd.RR_ERR_PARAM, rr.rr_paged_attn, Q, c, big)
        refused(bd.RR_ERR_PARAM, rr.rr_paged_attn, Q, c, 0, big)
        refused(bd.RR_ERR_PARAM, rr.rr_paged_attn, Q, c, max_length=big)
        refused(bd.RR_ERR_PARAM, rr.rr_paged_workspace_bytes, Q, c, big)
        refused(bd.RR_ERR_PARAM, rr.rr_cache_evict, c, torch.zeros(3, 2, dtype=torch.int32), big)
        refused(bd.RR_ERR_PARAM, rr.rr_cache_evict, c, torch.zeros(3, 2, dtype=torch.int32), 20, big)


def test_a_cache_follows_its_tensors():
    """The struct of a cache is that of the tensors it has now, and no part of a copy."""
    import copy
    c = rr.PagedCache.allocate(8, 16, 2, 64, 3, 4, "cpu", weight=True)
    s = c.c_struct()
    assert (s.K, s.weight, s.page, s.num_pages, s.width) == (c.K.data_ptr(), c.weight.data_ptr(), 16, 8, 4) and c.c_struct() is s
    c.table = torch.zeros(3, 5, dtype=torch.int32)
    assert c.c_struct().width == 5 and c.c_struct().table == c.table.data_ptr()
    c.weight = None
    assert c.c_struct().weight is None
    c.K.data, c.V.data = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16)
    assert c.c_struct().num_pages == 9 and c.c_struct().K == c.K.data_ptr()
    d = copy.deepcopy(c)
    assert d.c_struct().K == d.K.data_ptr() != c.K.data_ptr()
    c.length = torch.zeros(3)
    refused(bd.RR_ERR_DTYPE, c.c_struct)


def test_names_of_the_package():
    """Every exported entry point is reachable from the package, also after a reload."""
    import importlib
    for name in ("rr_window_attn", "rr_window_workspace_bytes", "PagedCache", "rr_paged_attn", "rr_paged_workspace_bytes", "rr_paged_write",
                 "rr_key_weights", "rr_key_weights_workspace_bytes", "rr_cache_evict", "rr_cache_evict_workspace_bytes"):
        assert getattr(rr, name) is getattr(bd, name)
    importlib.reload(rr)
    assert "rr_paged_attn" not in vars(rr) and rr.rr_paged_attn is bd.rr_paged_attn and "rr_paged_attn" in vars(rr)
    with pytest.raises(AttributeError):
        rr.rr_no_such_name
