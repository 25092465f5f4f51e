"""Block-sparse attention on the host (no GPU): query blocks, completed blocks, refusals."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest

import sparse_ref as R
import test_asm_hazards as H
from paper_2608_26523_amd import binding as B
from paper_2608_26523_amd import build as BLD

GOOD = 1 << 20  # an aligned address that no refused call reads


@pytest.mark.parametrize("size", [1, 2, 7, 64, 128])
@pytest.mark.parametrize("lens,prefix,start", [([1], [0], [0]), ([0, 5, 0, 130, 64], [9, 0, 3, 1000, 63], [0, 64, 0, 128, 640]), ([], [], [])])
def test_query_blocks(lens, prefix, start, size):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(int)
    got = B.vpp_query_blocks(cu, start, prefix, size, 64)
    want = R.query_blocks(cu.tolist(), prefix, size)
    assert [tuple(int(g[f]) for f in ("row0", "rows", "segment", "pos0")) for g in got] == want
    assert [int(g["kv_start"]) for g in got] == [start[w[2]] for w in want]


@pytest.mark.parametrize("cu,start,prefix,size,block", [
    ([1, 2], [0], [0], 1, 64), ([0, 5, 3], [0, 0], [0, 0], 1, 64), ([0, 5], [-64], [0], 1, 64), ([0, 5], [0], [-1], 1, 64),
    ([0, 5], [32], [0], 1, 64), ([0, 5], [64], [0], 1, 128), ([0, 5], [0], [0], 0, 64), ([0, 5], [0], [0], 129, 64),
    ([0, 5], [0], [0], 1, 96), ([0, 5], [0], [2 ** 31], 1, 64), ([0, 5], [2 ** 31 - 256], [0], 1, 64),
    ([0, 5], [0], [2 ** 63 - 1], 1, 64), ([0, 5], [2 ** 63 - 64], [2 ** 62], 1, 64)])
def test_query_block_refusals(cu, start, prefix, size, block):
    with pytest.raises(B.VppError):
        B.vpp_query_blocks(cu, start, prefix, size, block)


def test_query_blocks_are_counted_past_the_capacity():
    cu, z = np.array([0, 10], dtype=np.int32), np.zeros(1, dtype=np.int64)
    n = ctypes.c_int32(0)
    buf = np.zeros(4, dtype=B.QUERY_BLOCK_DTYPE)
    args = (1, cu.ctypes.data, z.ctypes.data, z.ctypes.data, 3, 64)
    assert B.load().vpp_query_blocks(*args, None, 0, ctypes.byref(n)) == 0 and n.value == 4
    assert B.load().vpp_query_blocks(*args, buf.ctypes.data, 2, ctypes.byref(n)) == 0 and n.value == 4
    assert buf["rows"].tolist() == [3, 3, 0, 0]
    assert B.load().vpp_query_blocks(*args, None, 2, ctypes.byref(n)) == B.VPP_ERR_INVALID_ARG
    assert B.load().vpp_query_blocks(*args, None, 0, None) == B.VPP_ERR_INVALID_ARG


@pytest.mark.parametrize("block,page", [(64, 64), (64, 256), (128, 128), (256, 1024)])
def test_completed_blocks(block, page):
    """Chunk by chunk every block is completed once, by the chunk that holds its last row."""
    rng = np.random.default_rng(block + page)
    table = rng.permutation(64).reshape(2, 32).astype(np.int32)
    start, at = [block, 0], [0, 0]
    seen = []
    for _ in range(12):
        n = rng.integers(0, 300, size=2)
        cu = np.concatenate([[0], np.cumsum(n)])
        got = B.vpp_completed_blocks(cu, start, at, table, page, block).tolist()
        want = []
        for s in range(2):
            for b in range(at[s] + n[s] + 1):
                if at[s] < (b + 1) * block <= at[s] + n[s]:
                    row = start[s] + b * block
                    want.append(int(table[s, row // page]) * (page // block) + row % page // block)
            at[s] += int(n[s])
        assert got == want
        seen += got
    assert len(seen) == len(set(seen)) == sum(a // block for a in at)


def test_completed_block_refusals():
    table = np.zeros((1, 2), dtype=np.int32)
    for cu, start, prefix, page, block in [([0, 200], [0], [0], 64, 64), ([0, 64], [0], [0], 64, 128), ([0, 64], [0], [0], 96, 64),
                                           ([0, 64], [32], [0], 64, 64), ([0, 64], [0], [-1], 64, 64), ([0, -1], [0], [0], 64, 64),
                                           ([0, 64], [0], [2 ** 40], 64, 64)]:
        with pytest.raises(B.VppError):
            B.vpp_completed_blocks(cu, start, prefix, table, page, block)
    with pytest.raises(B.VppError):
        B.vpp_completed_blocks([0, 64], [0], [0], table - 1, 64, 64)


def _cfg(**over):
    a = dict(num_q_heads=8, num_kv_heads=2, head_dim_qk=128, head_dim_v=128, softmax_scale=0.0, block_size=64, query_block=16,
             max_blocks=8, sink_blocks=1, local_blocks=2)
    a.update(over)
    return B.BlockConfig(**a)


@pytest.mark.parametrize("bad,status", [
    (dict(num_q_heads=0), 1), (dict(num_kv_heads=0), 1), (dict(num_q_heads=7), 1), (dict(num_q_heads=258), 1),
    (dict(head_dim_qk=96), 2), (dict(head_dim_v=64), 2), (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=math.nan), 1),
    (dict(softmax_scale=math.inf), 1), (dict(block_size=32), 1), (dict(block_size=512), 1), (dict(block_size=96), 1),
    (dict(query_block=0), 1), (dict(query_block=129), 1), (dict(max_blocks=0), 1), (dict(max_blocks=2049), 1),
    (dict(max_blocks=3), 1), (dict(max_blocks=4, query_block=66), 1), (dict(sink_blocks=-1), 1), (dict(local_blocks=0), 1),
    (dict(sink_blocks=2 ** 31 - 1), 1), (dict(local_blocks=2 ** 31 - 1, sink_blocks=2 ** 31 - 1), 1)])
def test_config_refusals(bad, status):
    n = ctypes.c_size_t(0)
    assert B.load().vpp_block_attn_workspace(ctypes.byref(_cfg(**bad)), 1, 1, ctypes.byref(n)) == status
    assert _summarize(cfg=_cfg(**bad)) == status and _select(cfg=_cfg(**bad)) == status and _run(cfg=_cfg(**bad)) == status


def test_smallest_lists():
    n = ctypes.c_size_t(0)
    for ok in (dict(max_blocks=4), dict(max_blocks=4, query_block=65), dict(max_blocks=1, query_block=1, sink_blocks=0, local_blocks=1)):
        assert B.load().vpp_block_attn_workspace(ctypes.byref(_cfg(**ok)), 1, 1, ctypes.byref(n)) == 0
    for args in ((-1, 1), (1, -1)):
        assert B.load().vpp_block_attn_workspace(ctypes.byref(_cfg()), *args, ctypes.byref(n)) == B.VPP_ERR_INVALID_ARG
    assert B.load().vpp_block_attn_workspace(ctypes.byref(_cfg()), 1, 1, None) == B.VPP_ERR_INVALID_ARG


def _summarize(cfg=None, k=GOOD, ks=(16384, 256, 128), page=64, pages=9, ids=GOOD, n=3, sums=GOOD):
    return B.load().vpp_block_summarize_paged(ctypes.byref(cfg or _cfg()), k, *ks, page, pages, ids, n, sums, None)


@pytest.mark.parametrize("bad", [
    dict(k=0), dict(k=GOOD + 8), dict(ids=0), dict(ids=GOOD + 4), dict(sums=0), dict(sums=GOOD + 8), dict(n=-1), dict(page=32),
    dict(page=96), dict(pages=0), dict(ks=(16384, 100, 128)), dict(ks=(16384, 64, 128)), dict(ks=(16384, 256, 64)),
    dict(ks=(16380, 256, 128)), dict(ks=(0, 256, 128)), dict(cfg=_cfg(block_size=128))])
def test_summarize_refusals(bad):
    assert _summarize(**bad) == B.VPP_ERR_INVALID_ARG


def _select(cfg=None, qb=GOOD, n=4, q=GOOD, qs=(1024, 128), tokens=64, sums=GOOD, page=64, pages=9, bt=GOOD, bts=16, segs=2, per_row=16,
            most=1024, blocks=GOOD, ws=GOOD, wsb=1 << 40):
    return B.load().vpp_block_select_paged(ctypes.byref(cfg or _cfg()), qb, n, q, *qs, tokens, sums, page, pages, bt, bts, segs, per_row, most,
                                           blocks, ws, wsb, None)


@pytest.mark.parametrize("bad,status", [
    (dict(qb=0), 1), (dict(qb=GOOD + 4), 1), (dict(n=-1), 1), (dict(q=0), 1), (dict(q=GOOD + 8), 1), (dict(qs=(1020, 128)), 1),
    (dict(qs=(1024, 64)), 1), (dict(qs=(64, 128)), 1), (dict(tokens=-1), 1), (dict(sums=0), 1), (dict(sums=GOOD + 2), 1), (dict(page=32), 1),
    (dict(pages=0), 1), (dict(bt=0), 1), (dict(bt=GOOD + 2), 1), (dict(bts=-1), 1), (dict(segs=0), 1), (dict(per_row=0), 1), (dict(most=-1), 1),
    (dict(blocks=0), 1), (dict(blocks=GOOD + 2), 1), (dict(most=32768 * 64 + 1), 2), (dict(ws=0), 3), (dict(ws=GOOD + 64), 3),
    (dict(wsb=4 * 2 * 16 * 4 - 1), 3)])
def test_select_refusals(bad, status):
    assert _select(**bad) == status


def test_select_workspace():
    def need(n, most, **over):
        return B.vpp_block_select_workspace(_cfg(**over), n, most)
    assert need(4, 1024) == 4 * 2 * 16 * 4 and need(0, 1024) == 0 and need(4, 8 * 64) == 0 and need(4, 8 * 64 + 1) == 4 * 2 * 9 * 4
    big = need(1 << 20, 1 << 20)
    assert 255 << 20 < big <= 256 << 20  # a slab, however many query blocks
    assert need(1 << 20, 1 << 21, num_q_heads=128, num_kv_heads=128) == 64 * 128 * 32768 * 4
    for args in ((-1, 64), (1, -1), (1, 32768 * 64 + 1)):
        with pytest.raises(B.VppError):
            need(*args)


def _run(cfg=None, qb=GOOD, n=4, q=GOOD, qs=(1024, 128), tokens=64, k=GOOD, ks=(16384, 256, 128), v=GOOD, vs=(16384, 256, 128), page=64,
         pages=9, bt=GOOD, bts=16, segs=2, per_row=16, blocks=GOOD, out=GOOD, os_=(1024, 128), lse=GOOD, lses=64, ws=GOOD, wsb=1 << 40):
    return B.load().vpp_block_attn_run_paged(ctypes.byref(cfg or _cfg()), qb, n, q, *qs, tokens, k, *ks, v, *vs, page, pages, bt, bts, segs,
                                             per_row, blocks, out, *os_, lse, lses, ws, wsb, None)


@pytest.mark.parametrize("bad", [
    dict(qb=0), dict(qb=GOOD + 8), dict(n=-1), dict(q=0), dict(q=GOOD + 4), dict(qs=(1024, 100)), dict(qs=(1024, 64)), dict(tokens=-1),
    dict(k=0), dict(k=GOOD + 4), dict(v=0), dict(v=GOOD + 4), dict(ks=(16384, 64, 128)), dict(ks=(16384, 1 << 24, 128)), dict(ks=(0, 256, 128)),
    dict(vs=(16384, 256, 64)), dict(vs=(16384, 1 << 24, 128)), dict(page=32), dict(page=1 << 21), dict(pages=0), dict(bt=0), dict(bts=-1),
    dict(segs=0), dict(per_row=0), dict(blocks=0), dict(blocks=GOOD + 1), dict(out=0), dict(out=GOOD + 4), dict(os_=(1024, 0)),
    dict(os_=(1024, 64)), dict(os_=(512, 128)), dict(os_=(128, 128)), dict(lse=GOOD + 2), dict(lses=63)])
def test_run_refusals(bad):
    assert _run(**bad) == B.VPP_ERR_INVALID_ARG


def test_run_workspace():
    """Few workgroups split their lists; the parts need a workspace."""
    one = _cfg(query_block=1, max_blocks=64, num_q_heads=32, num_kv_heads=8)
    need = B.vpp_block_attn_workspace(one, 1, 1)
    assert need == 16 * 1 * 32 * 129 * 4 and B.vpp_block_attn_workspace(one, 1 << 16, 1 << 16) == 0
    for ws, wsb in ((0, need), (GOOD, need - 1), (GOOD + 128, need)):
        assert _run(cfg=one, n=1, tokens=1, qs=(4096, 128), os_=(4096, 128), ks=(65536, 1024, 128), vs=(65536, 1024, 128), ws=ws,
                    wsb=wsb) == B.VPP_ERR_WORKSPACE


def test_calls_of_nothing():
    assert _summarize(n=0) == 0 and _select(n=0) == 0 and _run(n=0) == 0 and _select(tokens=0) == 0 and _run(tokens=0) == 0
    lib = B.load()
    assert lib.vpp_block_summarize_paged(None, GOOD, 8, 8, 8, 64, 1, GOOD, 1, GOOD, None) == B.VPP_ERR_INVALID_ARG


def test_wrapper_refusals_without_a_gpu():
    from paper_2608_26523_amd.sparse import BlockSparseAttention
    for bad in (dict(max_blocks=0), dict(max_blocks=8, block_size=32), dict(max_blocks=8, query_block=0)):
        with pytest.raises(B.VppError):
            BlockSparseAttention(8, 2, 128, 128, **bad)
    with pytest.raises(ValueError):
        BlockSparseAttention(8, 2, 128, 128, max_blocks=8, device="cpu")


# -- the plain implementations themselves -------------------------------------------------------------
def test_reference_grid_and_rotation():
    x = np.array([[0.5, 1.0, -3.0, 0.01], [0.0, 0.0, 0.0, 0.0], [2.0 ** 70, 1.0, -2.0 ** 55, np.nan]])
    g = R.grid(x)
    assert g[0].tolist() == [0.5, 1.0, -3.0, 0.015625] and not g[1].any()
    assert g[2].tolist() == [2.0 ** 60, 0.0, -2.0 ** 55, 0.0]
    y, _ = R.rotated(np.array([[[1.0, 0.0, 0.0, 0.0]]]), [1], [math.pi / 2, 0.0], 0, False)
    assert np.allclose(y[0, 0], [0, 0, 1, 0], atol=1e-15)
    y, _ = R.rotated(np.array([[[1.0, 0.0, 2.0, 0.0]]]), [3], [math.pi / 2, 0.0], 0, True, scale=2.0, inverse=True)
    assert np.allclose(y[0, 0], [0, 2, 4, 0], atol=1e-14)


def test_scalar_alu_asm_declares_scc():
    for path in BLD.MORE_SRCS:
        for template, clobbers in H._asm_statements(open(path).read()):
            ops = [ln.split()[0] for ln in template.replace("\\n", "\n").replace("\\t", "").splitlines() if ln.strip()]
            assert "scc" in clobbers or not any(H.SCC_WRITE.match(op) for op in ops), template


@pytest.mark.skipif(not os.path.exists(BLD.hipcc()), reason="hipcc not installed")
def test_device_code_keeps_scc_and_uses_no_scratch(tmp_path):
    """No SCC value is read across a copy that writes it; and no spill to memory, whose loads the copies' counted
    waits would take for copies."""
    out = str(tmp_path / "attn.s")
    base = [BLD.hipcc()] + [f for f in BLD.HIPCC_FLAGS if f not in ("-shared", "-Wall")] + ["-I", BLD.INCLUDE]
    src = next(p for p in BLD.MORE_SRCS if p.endswith("vpp_block_attn.hip"))
    log = subprocess.run(base + ["--cuda-device-only", "-S", "-o", out, src], capture_output=True, text=True, timeout=600)
    assert log.returncode == 0, log.stderr[-2000:]
    text = open(out).read()
    assert "buffer_load_dwordx4" in text and ";;#ASMSTART" in text
    assert H._scan(text) == []
    sizes = re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text)
    assert len(sizes) == 14 and set(sizes) == {"0"}
