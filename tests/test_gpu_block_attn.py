"""Block summaries, selection and attention against 64-bit results (GPU).

Summaries and lists are exact by definition and compared bit for bit; the attention's bounds are
elementwise (tests/sparse_ref.py): the roundings of P and of the result to bf16 and fp32 sums.
"""
import math

import numpy as np
import pytest
import torch

import sparse_ref as R

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _attn(hq, hkv, dqk, dv, most, **kw):
    from paper_2608_26523_amd.sparse import BlockSparseAttention
    return BlockSparseAttention(hq, hkv, dqk, dv, max_blocks=most, **kw)


def _bf16(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)


# -- summaries ----------------------------------------------------------------------------------
@pytest.mark.parametrize("hkv,d,block,page,pages", [
    (1, 64, 64, 64, 3), (8, 128, 64, 256, 5), (3, 192, 128, 128, 4), (5, 128, 256, 512, 3), (16, 192, 64, 128, 9), (2, 64, 256, 256, 2)])
@pytest.mark.parametrize("strided", [False, True])
def test_summaries(hkv, d, block, page, pages, strided):
    print("case:", hkv, d, block, page, pages, strided, flush=True)
    rng = np.random.default_rng(d + block)
    k = _bf16(rng, pages, page, hkv + 1, d + 8)[:, :, 1:, 8:] if strided else _bf16(rng, pages, page, hkv, d)
    # blocks of one size, of one sign, of nothing but zeros
    k[0, :block] = k[0, :block].abs()
    k[1, :block] = 0
    k[1, :block, 0, 0] = 1e-30
    k = k.to(DEV) if not strided else k._base.to(DEV)[:, :, 1:, 8:]
    attn = _attn(hkv, hkv, d, 64 if d == 64 else 128, 8, block_size=block)
    sums = attn.new_summaries(pages, page)
    sums.fill_(7)
    per = page // block
    total = pages * per
    ids = rng.permutation(total)[:max(1, total - 2)]
    listed = np.concatenate([ids, ids[:1], [-1, total, 1 << 40]])  # one twice, three outside
    got = attn.summarize(k, torch.as_tensor(listed, device=DEV), sums)
    assert got is sums
    torch.cuda.synchronize()
    want = np.full((pages, per, hkv, d), 7.0)
    kf = R.f64(k)
    for i in ids:
        for h in range(hkv):
            want[i // per, i % per, h] = R.summary(kf[i // per, i % per * block:(i % per + 1) * block, h])
    assert np.array_equal(R.f64(sums), want)


def test_summaries_of_extreme_keys():
    rng = np.random.default_rng(1)
    k = _bf16(rng, 6, 64, 2, 128)
    k[0, 3, 0, 5] = math.inf
    k[0, 4, 0, 6] = -math.inf
    k[0, 5, 0, 7] = math.nan
    k[0, 5:7, 0, 8] = torch.tensor([math.inf, -math.inf])
    k[1] *= 2.0 ** 100                       # past the largest value of a grid
    k[2] *= 2.0 ** -80                       # below its smallest step
    k[3, :, :, ::2] *= 2.0 ** -20            # far apart
    k[4] = 2.0                               # largest on a power of two
    k[4, :, :, 1] = 2.0 - 2.0 ** -7          # next to it
    k[5] = torch.finfo(torch.bfloat16).max
    attn = _attn(2, 2, 128, 128, 8)
    sums = attn.new_summaries(6, 64)
    attn.summarize(k.to(DEV), torch.arange(6, device=DEV), sums)
    torch.cuda.synchronize()
    kf = R.f64(k)
    want = np.stack([[[R.summary(kf[p, :, h]) for h in range(2)]] for p in range(6)])
    assert np.array_equal(R.f64(sums), want)
    assert np.all(np.isfinite(want)) and want[0, 0, 0, 5] == 2.0 ** 60 and want[0, 0, 0, 7] == 0


# -- selection ----------------------------------------------------------------------------------
SEGS = [
    ([(0, 1)], "one token"),
    ([(5000, 1), (63, 1), (64, 1), (0, 1), (777, 1), (4095, 1)], "single tokens"),
    ([(3000, 37), (0, 0), (130, 70), (0, 200)], "packed, one empty"),
    ([(10000, 130)], "long"),
]
HEADS = [(1, 1, 64, 64), (4, 2, 128, 128), (3, 1, 128, 128), (8, 2, 192, 128), (10, 2, 64, 64), (16, 2, 128, 128),
         (16, 1, 128, 128), (24, 1, 192, 128), (3, 3, 192, 128)]


def _chunk(segs, block, kv_pages, page, seed):
    lens, prefix = [n for _, n in segs], [p for p, _ in segs]
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(int).tolist()
    rng = np.random.default_rng(seed)
    start = [int(rng.integers(0, kv_pages + 1)) * block for _ in segs]
    return cu, prefix, start, [s + p + n for s, p, n in zip(start, prefix, lens)], rng


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("segs", range(len(SEGS)))
@pytest.mark.parametrize("size,block,page,most,sink,local", [
    (1, 64, 64, 8, 1, 1), (1, 128, 256, 5, 0, 3), (2, 64, 128, 12, 2, 1), (3, 64, 64, 6, 0, 1), (16, 64, 64, 20, 1, 2),
    (64, 256, 256, 4, 1, 1), (100, 64, 128, 9, 0, 2), (128, 64, 64, 70, 1, 4)])
def test_selection(heads, segs, size, block, page, most, sink, local):
    hq, hkv, d, dv = heads
    segs = SEGS[segs][0]
    if hq * size > 700 and sum(n for _, n in segs) > 150:
        size = 32
    print("case:", heads, segs, size, block, page, most, sink, local, flush=True)
    cu, prefix, start, rows, rng = _chunk(segs, block, 2, page, hq + size + page)
    per = page // block
    table, (_,) = R.paged(rng, rows, page, (1,))
    pages = int(table.max()) + 1
    # few different values, so that scores repeat: of equal ones the lowest blocks are chosen
    sums = torch.from_numpy(rng.integers(-2, 3, size=(pages, per, hkv, d)) * (rng.random((pages, per, hkv, d)) < 0.05)).to(torch.bfloat16)
    if size == 1:
        sums = torch.from_numpy(R.grid(rng.standard_normal((pages, per, hkv, d)))).to(torch.bfloat16)
    q = _bf16(rng, cu[-1], hq, d)
    q[::3] = q[::3].round()
    attn = _attn(hq, hkv, d, dv, most, block_size=block, query_block=size, sink_blocks=sink, local_blocks=local)
    n = attn.plan(cu, start, prefix)
    got = attn.select(q.to(DEV), sums.to(DEV), torch.as_tensor(table, device=DEV))
    torch.cuda.synchronize()
    want = R.selected(R.f64(q), R.f64(sums), table, cu, start, prefix, hkv=hkv, block=block, size=size, most=most,
                      sink=sink, local=local)
    assert got.shape == (n, hkv, most)
    assert np.array_equal(got.cpu().numpy(), want)


def test_selection_of_extreme_queries():
    rng = np.random.default_rng(3)
    cu, prefix, start, rows, rng = _chunk([(2000, 12)], 64, 0, 64, 3)
    table, (_,) = R.paged(rng, rows, 64, (1,))
    sums = torch.from_numpy(R.grid(rng.standard_normal((int(table.max()) + 1, 1, 1, 128)) * 2.0 ** 40)).to(torch.bfloat16)
    q = _bf16(rng, 12, 2, 128)
    q[0, 0, 3], q[1, 0, 3], q[2] = math.inf, -math.inf, math.nan
    q[3] *= 2.0 ** 110
    q[4] *= 2.0 ** -100
    q[5] = 0
    q[6, :, 1:] *= 2.0 ** -12
    attn = _attn(2, 1, 128, 128, 6)
    attn.plan(cu, start, prefix)
    got = attn.select(q.to(DEV), sums.to(DEV), torch.as_tensor(table, device=DEV))
    want = R.selected(R.f64(q), R.f64(sums), table, cu, start, prefix, hkv=1, block=64, size=1, most=6, sink=1, local=1)
    assert np.array_equal(got.cpu().numpy(), want)


def test_selection_among_many_blocks():
    """As many blocks as one selection takes; two segments in one launch, lists of thousands."""
    rng = np.random.default_rng(4)
    rows, page = 32768 * 64, 4096
    cu, prefix, start = [0, 2, 5], [rows - 2, 700000], [0, 0]
    per = page // 64
    table = np.stack([rng.permutation(rows // page), rng.permutation(rows // page)]).astype(np.int32)
    sums = torch.from_numpy(R.grid(rng.standard_normal((rows // page, per, 1, 64)))).to(torch.bfloat16)
    q = _bf16(rng, 5, 4, 64)
    for most in (2048, 9):
        attn = _attn(4, 1, 64, 64, most, local_blocks=3)
        attn.plan(cu, start, prefix)
        got = attn.select(q.to(DEV), sums.to(DEV), torch.as_tensor(table, device=DEV))
        want = R.selected(R.f64(q), R.f64(sums), table, cu, start, prefix, hkv=1, block=64, size=1, most=most, sink=1, local=3)
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("heads,size,tokens", [
    ((64, 64, 64, 64), 1, 600), ((32, 16, 64, 64), 1, 1100), ((32, 8, 128, 128), 1, 1100), ((24, 8, 64, 64), 1, 1100),
    ((64, 8, 64, 64), 1, 600), ((64, 4, 128, 128), 1, 600), ((64, 4, 192, 128), 1, 1100), ((64, 4, 128, 128), 2, 600),
    ((64, 4, 192, 128), 3, 700), ((16, 16, 192, 128), 64, 4200), ((16, 8, 64, 64), 100, 8000), ((32, 8, 192, 128), 1, 1100)])
def test_selection_of_many_query_blocks(heads, size, tokens):
    """Launches whose workgroups hold several query blocks, across the boundaries of segments."""
    hq, hkv, d, dv = heads
    print("case:", heads, size, tokens, flush=True)
    cut = [tokens // 3 + 1, 5, tokens - tokens // 3 - 6]
    cu, prefix, start, rows, rng = _chunk([(1500, cut[0]), (2000, cut[1]), (700, cut[2])], 64, 2, 128, tokens)
    table, (_,) = R.paged(rng, rows, 128, (1,))
    sums = torch.from_numpy(R.grid(rng.standard_normal((int(table.max()) + 1, 2, hkv, d)))).to(torch.bfloat16)
    q = _bf16(rng, cu[-1], hq, d)
    attn = _attn(hq, hkv, d, dv, 9, query_block=size, local_blocks=2)
    attn.plan(cu, start, prefix)
    got = attn.select(q.to(DEV), sums.to(DEV), torch.as_tensor(table, device=DEV))
    torch.cuda.synchronize()
    want = R.selected(R.f64(q), R.f64(sums), table, cu, start, prefix, hkv=hkv, block=64, size=size, most=9, sink=1, local=2)
    assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("heads,size", [((32, 1, 64, 64), 16), ((16, 2, 192, 128), 64), ((24, 2, 128, 128), 32),
                                        ((8, 4, 192, 128), 64)])
@pytest.mark.parametrize("prefix", [2500, 4200])
def test_selection_of_query_blocks_of_many_rows(heads, size, prefix):
    """128 to 512 rows a query block, those above 128 in several passes whose maxima meet in memory; half of the blocks
    are chosen, so that the last one's score decides too."""
    hq, hkv, d, dv = heads
    rng = np.random.default_rng(prefix + size)
    tokens, most = 20 * size + 3, prefix // 128
    cu, start, rows = [0, tokens], [0], [prefix + tokens]
    table, (_,) = R.paged(rng, rows, 128, (1,))
    sums = torch.from_numpy(R.grid(rng.standard_normal((int(table.max()) + 1, 2, hkv, d)))).to(torch.bfloat16)
    q = _bf16(rng, tokens, hq, d)
    attn = _attn(hq, hkv, d, dv, most, query_block=size)
    attn.plan(cu, start, [prefix])
    want = R.selected(R.f64(q), R.f64(sums), table, cu, start, [prefix], hkv=hkv, block=64, size=size, most=most, sink=1, local=1)
    for _ in range(3):
        got = attn.select(q.to(DEV), sums.to(DEV), torch.as_tensor(table, device=DEV))
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("prefix", [31000, 40000, 100000, 130000, 300000, 600000])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("tokens,hkv", [(3, 1), (9, 8)])
def test_selection_of_each_number_of_blocks(prefix, ties, tokens, hkv):
    """Keys of one wave, of several, of a workgroup; scores that repeat past the end of a list."""
    rng = np.random.default_rng(prefix)
    rows, page = prefix + tokens, 1024
    table = rng.permutation(-(-rows // page)).astype(np.int32)[None]
    shape = (table.shape[1], page // 64, hkv, 64)
    sums = rng.integers(-1, 2, size=shape) * (rng.random(shape) < 0.02) if ties else R.grid(rng.standard_normal(shape))
    sums = torch.from_numpy(sums.astype(np.float64)).to(torch.bfloat16)
    q = _bf16(rng, tokens, hkv * 2, 64)
    if ties:
        q = q.sign()
    for most in (5, 64, 300):
        attn = _attn(hkv * 2, hkv, 64, 64, most, local_blocks=2)
        attn.plan([0, tokens], [0], [prefix])
        got = attn.select(q.to(DEV), sums.to(DEV), torch.as_tensor(table, device=DEV))
        want = R.selected(R.f64(q), R.f64(sums), table, [0, tokens], [0], [prefix], hkv=hkv, block=64, size=1, most=most, sink=1, local=2)
        assert np.array_equal(got.cpu().numpy(), want)


def test_selection_slab_by_slab():
    """More scores than the workspace holds: 128 heads, 16384 blocks, 64 query blocks a slab."""
    rng = np.random.default_rng(5)
    hkv, page, prefix, tokens = 128, 4096, 16384 * 64 - 200, 130
    pages = -(-(prefix + tokens) // page)
    table = rng.permutation(pages).astype(np.int32)[None]
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    sums = torch.randint(-127, 128, (pages, page // 64, hkv, 64), generator=g, device=DEV).to(torch.bfloat16)
    q = _bf16(rng, tokens, hkv, 64)
    attn = _attn(hkv, hkv, 64, 64, 12)
    attn.plan([0, tokens], [0], [prefix])
    assert attn.select_bytes < tokens * hkv * 16384 * 4
    got = attn.select(q.to(DEV), sums, torch.as_tensor(table, device=DEV)).cpu().numpy()
    at = torch.as_tensor(table[0].astype(np.int64), device=DEV)
    keys = sums[at].flatten(0, 1).double()  # [blocks, hkv, 64]
    for t in (0, 63, 64, 100, 129):
        f = (prefix + t) // 64
        score = (keys[1:f] * torch.from_numpy(R.grid(R.f64(q[t]))).to(DEV)).sum(-1).T.cpu().numpy()  # whole multiples: exact
        for h in range(0, hkv, 37):
            order = np.lexsort((np.arange(f - 1), -score[h]))[:10] + 1
            assert got[t, h].tolist() == sorted(order.tolist() + [0, f]), (t, h)


# -- attention ----------------------------------------------------------------------------------
def _lists(rng, cu, prefix, hkv, block, size, most):
    """Random lists: ascending with their own last block, then holes, repeats, blocks of the future
    and of nowhere, and one that is empty."""
    qb = R.query_blocks(cu, prefix, size)
    out = np.full((len(qb), hkv, most), -1, dtype=np.int32)
    for n, (r0, rows, s, pos) in enumerate(qb):
        c = (pos + rows - 1) // block
        for h in range(hkv):
            got = sorted(set(rng.integers(0, c + 1, size=most - 1).tolist()) | {c})[-most:]
            if (n + h) % 3 == 1:
                got = rng.permutation(got).tolist()
                got[0] = rng.choice([-1, c + 1, 2 ** 31 - 1, got[-1], -2 ** 31])
            if (n + h) % 7 == 6:
                got = [-1] * (most - 1) + [c]
            if (n + h) % 11 == 10:
                got = []
            out[n, h, :len(got)] = got
    return out


def _check(got, lse, want, wlse, bound, lbound, what=""):
    off = np.abs(R.f64(got) - want) - bound
    assert np.all(off <= 0), "%s out: %g past the bound" % (what, off.max())
    lse = R.f64(lse)
    assert np.array_equal(np.isneginf(lse), np.isneginf(wlse)), what
    fine = ~np.isneginf(wlse)
    off = np.abs(lse[fine] - wlse[fine]) - lbound[fine]
    assert off.size == 0 or np.all(off <= 0), "%s lse: %g past the bound" % (what, off.max())


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("segs", range(len(SEGS)))
@pytest.mark.parametrize("size,block,page,most", [(1, 64, 64, 5), (1, 128, 256, 4), (2, 64, 128, 13), (3, 64, 64, 1 + 1),
                                                  (16, 64, 64, 9), (64, 256, 256, 3), (100, 64, 128, 6)])
def test_attention(heads, segs, size, block, page, most):
    hq, hkv, d, dv = heads
    segs = SEGS[segs][0]
    print("case:", heads, segs, size, block, page, most, flush=True)
    cu, prefix, start, rows, rng = _chunk(segs, block, 2, page, hq * 7 + size)
    table, (k, v) = R.paged(rng, rows, page, (hkv, d), (hkv, dv))
    q = _bf16(rng, cu[-1], hq, d)
    lists = _lists(rng, cu, prefix, hkv, block, size, most)
    scale = 0.0 if size != 2 else 0.31
    attn = _attn(hq, hkv, d, dv, most, block_size=block, query_block=size, sink_blocks=0, softmax_scale=scale)
    attn.plan(cu, start, prefix)
    lse = torch.full((hq, cu[-1] + 3), 7.0, device=DEV)
    out, same = attn.run_paged(q.to(DEV), k.to(DEV), v.to(DEV), torch.as_tensor(table, device=DEV), torch.as_tensor(lists, device=DEV), lse=lse)
    torch.cuda.synchronize()
    assert same is lse and torch.all(lse[:, cu[-1]:] == 7)
    want = R.attended(R.f64(q), R.f64(k), R.f64(v), table, lists, cu, start, prefix, block=block, size=size, scale=scale or None)
    _check(out, lse[:, :cu[-1]], *want)


@pytest.mark.parametrize("heads,size,tokens", [
    ((16, 16, 64, 64), 1, 560), ((32, 8, 64, 64), 1, 560), ((24, 8, 64, 64), 1, 700), ((64, 4, 128, 128), 1, 300),
    ((16, 8, 128, 128), 2, 1100), ((16, 16, 192, 128), 1, 530), ((40, 8, 64, 64), 1, 300)])
@pytest.mark.parametrize("tidy", [True, False])
def test_attention_of_query_blocks_that_share_workgroups(heads, size, tokens, tidy):
    """Tokens whose common blocks are read once: lists that ascend, of several requests in a workgroup, and
    among them lists that do not; and infinite values in blocks that only some of them list."""
    hq, hkv, d, dv = heads
    print("case:", heads, size, tokens, tidy, flush=True)
    cu, prefix, start, rows, rng = _chunk([(700, tokens // 2 + 3), (300, 7), (64, tokens - tokens // 2 - 10)], 64, 2, 128, tokens + hq)
    table, (k, v) = R.paged(rng, rows, 128, (hkv, d), (hkv, dv))
    q = _bf16(rng, cu[-1], hq, d)
    qb = R.query_blocks(cu, prefix, size)
    lists = np.full((len(qb), hkv, 6), -1, dtype=np.int32)
    for n, (r0, nr, s, pos) in enumerate(qb):
        c = (pos + nr - 1) // 64
        for h in range(hkv):
            got = sorted(set(rng.integers(0, c + 1, size=5).tolist()) | {c})
            lists[n, h, :len(got)] = got
    if not tidy:
        messy = _lists(rng, cu, prefix, hkv, 64, size, 6)
        lists[::23] = messy[::23]
    attn = _attn(hq, hkv, d, dv, 6, query_block=size, sink_blocks=0)
    attn.plan(cu, start, prefix)
    run = lambda: attn.run_paged(*[x.to(DEV) for x in (q, k, v, torch.as_tensor(table), torch.as_tensor(lists))],  # noqa: E731
                                 lse=torch.empty(hq, cu[-1], device=DEV))
    out, lse = run()
    again, _ = run()
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    _check(out, lse, *R.attended(R.f64(q), R.f64(k), R.f64(v), table, lists, cu, start, prefix, block=64, size=size))
    if hq * tokens > 10000:
        return
    # block 5 of the first request becomes infinite in one column: its readers', and nobody else's
    j = start[0] + 5 * 64 + 3
    v[table[0][j // 128], j % 128, :, 9] = math.inf
    wild, _ = run()
    torch.cuda.synchronize()
    want = out.clone()
    for n, (r0, nr, s, pos) in enumerate(qb):
        if s == 0:
            for h in range(hkv):
                if 5 in lists[n, h]:
                    want[r0:r0 + nr, h * (hq // hkv):(h + 1) * (hq // hkv), 9] = math.inf
    assert torch.equal(wild, want)


def _random_run(seed, hq=8, hkv=2, d=128, dv=128, segs=((700, 50), (64, 3), (0, 129)), size=16, block=64, page=64, most=7):
    cu, prefix, start, rows, rng = _chunk(segs, block, 2, page, seed)
    table, (k, v) = R.paged(rng, rows, page, (hkv, d), (hkv, dv))
    q = _bf16(rng, cu[-1], hq, d)
    lists = _lists(rng, cu, prefix, hkv, block, size, most)
    attn = _attn(hq, hkv, d, dv, most, block_size=block, query_block=size, sink_blocks=0)
    return attn, (cu, start, prefix), rows, table, k, v, q, lists


@pytest.mark.parametrize("size", [1, 4, 16, 64])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
def test_what_a_token_does_not_see_does_not_reach_it(size, dims):
    """Infinities and NaN in keys and values behind each token, in rows that the cache has not got yet, and
    in pages of nobody; the tokens that do see them get them."""
    attn, plan, rows, table, k, v, q, lists = _random_run(8 + size, d=dims[0], dv=dims[1], size=size)
    cu, start, prefix = plan
    kf, vf = R.f64(k), R.f64(v)
    want = R.attended(R.f64(q), kf, vf, table, lists, cu, start, prefix, block=64, size=size)
    page = k.shape[1]
    used = np.zeros(k.shape[:2], dtype=bool)
    for s in range(len(prefix)):
        j = np.arange(start[s], rows[s])
        used[table[s][j // page], j % page] = True
    k[torch.from_numpy(~used)] = math.nan
    v[torch.from_numpy(~used)] = math.inf
    # the third token from the end of each segment, and all behind it, see wild values
    first = np.array(cu[1:]) - np.array(cu[:-1]) - 3
    wild_rows = np.zeros(cu[-1], dtype=bool)
    for s in range(len(prefix)):
        if first[s] < 1:
            continue
        for t, (x, y) in zip(range(first[s], first[s] + 3), [(math.nan, 1.0), (math.inf, math.nan), (-math.inf, math.inf)]):
            j = start[s] + prefix[s] + t
            at = table[s][j // page], j % page
            v[at[0], at[1], :, 5] = x
            v[at[0], at[1], :, 17] = y
        wild_rows[cu[s] + first[s]:cu[s + 1]] = True
    attn.plan(*plan)
    out, lse = attn.run_paged(q.to(DEV), k.to(DEV), v.to(DEV), torch.as_tensor(table, device=DEV), torch.as_tensor(lists, device=DEV),
                              lse=torch.empty(q.shape[1], cu[-1], device=DEV))
    torch.cuda.synchronize()
    sane = ~wild_rows
    assert np.any(sane) and np.any(wild_rows)
    _check(out[torch.from_numpy(sane).to(DEV)], lse[:, torch.from_numpy(sane).to(DEV)], want[0][sane], want[1][:, sane], want[2][sane], want[3][:, sane])
    # the others: as 64 bits have it, value by value
    with np.errstate(invalid="ignore"):
        wild = R.attended(R.f64(q), kf, R.f64(v), table, lists, cu, start, prefix, block=64, size=size)[0][wild_rows]
    got = R.f64(out)[wild_rows]
    assert np.array_equal(np.isnan(got), np.isnan(wild))
    fine = ~np.isnan(wild)
    assert np.array_equal(np.isinf(got[fine]), np.isinf(wild[fine])) and np.array_equal(np.sign(got[fine & np.isinf(wild)]), np.sign(wild[fine & np.isinf(wild)]))
    assert np.any(np.isnan(wild))


@pytest.mark.parametrize("size", [1, 16, 64])
def test_infinite_values_reach_the_tokens_that_see_them(size):
    """One infinite value of each sign: its column is infinite from its token on, all else as without it."""
    attn, plan, rows, table, k, v, q, lists = _random_run(77, segs=((130, 40),), size=size)
    cu, start, prefix = plan
    qb = R.query_blocks(cu, prefix, size)
    lists[:] = -1
    for n, (r0, nr, s, pos) in enumerate(qb):
        c = (pos + nr - 1) // 64
        lists[n, :, :c + 1] = np.arange(c + 1)
    args = lambda: [x.to(DEV) for x in (q, k, v, torch.as_tensor(table), torch.as_tensor(lists))]  # noqa: E731
    attn.plan(*plan)
    want, _ = attn.run_paged(*args())
    for t, col, x in ((11, 3, math.inf), (20, 90, -math.inf)):
        j = start[0] + prefix[0] + t
        v[table[0][j // 64], j % 64, :, col] = x
    got, _ = attn.run_paged(*args())
    torch.cuda.synchronize()
    want[11:, :, 3], want[20:, :, 90] = math.inf, -math.inf
    assert torch.equal(got, want)


def test_keys_that_are_infinite_or_nan():
    """A visible NaN key makes its rows NaN and no others; a key of -infinite score counts for nothing."""
    attn, plan, rows, table, k, v, q, lists = _random_run(21, size=16)
    cu, start, prefix = plan
    lists[:] = -1
    for n, (r0, nr, s, pos) in enumerate(R.query_blocks(cu, prefix, 16)):
        c = (pos + nr - 1) // 64
        lists[n, :, :min(c + 1, 7)] = np.arange(c + 1)[-7:]
    q = q.abs()
    j = start[0] + prefix[0] + 20
    k[table[0][j // 64], j % 64, 0] = math.nan          # of token 20 of the first segment
    j = start[2] + 40
    k[table[2][j // 64], j % 64, 0] = -math.inf
    attn.plan(*plan)
    out, lse = attn.run_paged(q.to(DEV), k.to(DEV), v.to(DEV), torch.as_tensor(table, device=DEV), torch.as_tensor(lists, device=DEV),
                              lse=torch.empty(q.shape[1], cu[-1], device=DEV))
    torch.cuda.synchronize()
    bad = np.zeros((cu[-1], 8), dtype=bool)
    bad[20:cu[1], :4] = True
    assert np.array_equal(np.isnan(R.f64(out)).any(-1), bad) and np.array_equal(np.isnan(R.f64(lse)).T, bad)
    kf = R.f64(k)
    kf[np.isnan(kf)] = 0
    kf[np.isneginf(kf)] = -1e6  # exp of its scores is 0 in 64 bits too
    want = R.attended(R.f64(q), kf, R.f64(v), table, lists, cu, start, prefix, block=64, size=16)
    rows3 = slice(cu[2], cu[3])
    assert np.all(np.abs(R.f64(out)[rows3] - want[0][rows3]) <= R.HALF_BF16 * 3 * (1 + np.abs(want[0][rows3])) * 3)


@pytest.mark.parametrize("size", [1, 16])
def test_strides_streams_and_rows_of_nobody(size):
    attn, plan, rows, table, k, v, q, lists = _random_run(5, size=size)
    cu = plan[0]
    hq, d = q.shape[1:]
    attn.plan(*plan)
    args = [x.to(DEV) for x in (q, k, v, torch.as_tensor(table), torch.as_tensor(lists))]
    out, lse = attn.run_paged(*args, lse=torch.empty(hq, cu[-1], device=DEV))
    # queries and results with heads outermost and gaps, caches inside larger ones, a padded table
    q2 = torch.zeros(hq, cu[-1] + 4, d + 8, dtype=torch.bfloat16, device=DEV).transpose(0, 1)[..., :d]
    q2[:cu[-1]] = args[0]
    k2 = torch.zeros(k.shape[0] + 1, k.shape[1], 5, d + 16, dtype=torch.bfloat16, device=DEV)[1:, :, 2:4, 8:8 + d]
    v2 = torch.zeros(k.shape[0], 2, k.shape[1], v.shape[3], dtype=torch.bfloat16, device=DEV).transpose(1, 2)  # heads before rows
    k2.copy_(args[1]), v2.copy_(args[2])
    t2 = torch.zeros(table.shape[0] + 2, table.shape[1] + 5, dtype=torch.int32, device=DEV)[:, :table.shape[1]]
    t2[:table.shape[0]] = args[3]
    wide = torch.full((cu[-1] + 4, hq + 1, v.shape[3] + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    l2 = torch.full((hq, cu[-1] + 9), 7.0, device=DEV)
    got, _ = attn.run_paged(q2, k2, v2, t2, args[4], out=wide[:, :hq, :v.shape[3]], lse=l2, stream=side)
    again, none = attn.run_paged(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert none is None and torch.equal(again, out)
    assert torch.equal(got[:cu[-1]], out) and torch.equal(l2[:, :cu[-1]], lse)
    assert torch.all(wide[cu[-1]:] == 7) and torch.all(wide[:, hq:] == 7) and torch.all(wide[..., v.shape[3]:] == 7)
    assert torch.all(l2[:, cu[-1]:] == 7)


def test_no_query_blocks_and_unplanned():
    attn = _attn(4, 2, 64, 64, 4)
    q, k, table = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(1, 64, 2, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 1, dtype=torch.int32, device=DEV)
    with pytest.raises(RuntimeError):
        attn.select(q, attn.new_summaries(1, 64), table)
    assert attn.plan([0, 0, 0], [0, 0], [7, 0]) == 0
    blocks = attn.select(q, attn.new_summaries(1, 64), table)
    assert blocks.shape == (0, 2, 4)
    out, lse = attn.run_paged(q, k, k, table, blocks)
    assert out.shape == (0, 4, 64) and lse is None
    attn.summarize(k, torch.zeros(0, dtype=torch.int64, device=DEV), attn.new_summaries(1, 64))
    torch.cuda.synchronize()


def test_bad_device_values_stay_in_bounds():
    """Pages, query blocks and lists that point nowhere: refused on the device, neighbours as they were."""
    attn, plan, rows, table, k, v, q, lists = _random_run(9, size=16)
    cu, start, prefix = plan
    attn.plan(*plan)
    args = [x.to(DEV) for x in (q, k, v)]
    good, _ = attn.run_paged(*args, torch.as_tensor(table, device=DEV), torch.as_tensor(lists, device=DEV))
    wild = table.copy()
    wild[1] = [2 ** 31 - 1, -5, 12345][:1] * table.shape[1]
    got, _ = attn.run_paged(*args, torch.as_tensor(wild, device=DEV), torch.as_tensor(lists, device=DEV))
    torch.cuda.synchronize()
    keep = torch.tensor([r for r in range(cu[-1]) if not cu[1] <= r < cu[2]], device=DEV)
    assert torch.equal(got[keep], good[keep]) and torch.all(torch.isfinite(got.float()))
    # query blocks: rows past the chunk, before it, of no segment, of no position
    qb = attn._qb.view(-1, 8)
    n = attn.num_query_blocks
    for i, bad in enumerate([(cu[-1], 16, 0, 0, 0), (-1, 4, 0, 0, 0), (0, -3, 0, 0, 0), (0, 4, 99, 0, 0), (0, 4, 0, -1, 0)]):
        if i < n:
            qb[i, :5] = torch.tensor(bad, dtype=torch.int32)
    out = torch.full((cu[-1], 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    attn.run_paged(*args, torch.as_tensor(table, device=DEV), torch.as_tensor(lists, device=DEV), out=out)
    blocks = attn.select(args[0], attn.new_summaries(k.shape[0], 64), torch.as_tensor(table, device=DEV))
    torch.cuda.synchronize()
    rows_left = [(a, b) for i, (a, b, _, _) in enumerate(R.query_blocks(cu, prefix, 16)) if i >= 5]
    for a, b in rows_left:
        assert torch.equal(out[a:a + b], good[a:a + b])
    left = set(r for a, b in rows_left for r in range(a, a + b))
    gone = torch.tensor([r for r in range(cu[-1]) if r not in left], device=DEV)
    assert torch.all(out[gone] == 7) and torch.all(blocks[:min(5, n)] == -1)


def test_far_offsets_in_a_large_cache():
    """Keys and values past 2^31 elements of their pools."""
    hkv, d, page = 8, 128, 256
    pages = 9000
    attn = _attn(8, 8, d, d, 4, block_size=256, local_blocks=1)
    k = torch.zeros(pages, page, hkv, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    table = np.array([[8999, 0, 8500, 3, 8700]], dtype=np.int32)
    for p in table[0]:
        k[p] = torch.randn(page, hkv, d, generator=g, device=DEV).bfloat16()
        v[p] = torch.randn(page, hkv, d, generator=g, device=DEV).bfloat16()
    q = torch.randn(1, 8, d, generator=g, device=DEV).bfloat16()
    cu, start, prefix = [0, 1], [0], [5 * 256 - 1]
    attn.plan(cu, start, prefix)
    sums = attn.new_summaries(pages, page)
    attn.summarize(k, attn.completed(cu, start, [0], table, page), sums)
    attn.summarize(k, torch.as_tensor(table[0].astype(np.int64), device=DEV), sums)
    blocks = attn.select(q, sums, torch.as_tensor(table, device=DEV))
    out, lse = attn.run_paged(q, k, v, torch.as_tensor(table, device=DEV), blocks, lse=torch.empty(8, 1, device=DEV))
    torch.cuda.synchronize()
    at = np.argsort(table[0])
    small = np.empty(5, dtype=np.int32)
    small[at] = np.arange(5)
    few = torch.as_tensor(table[0][at].astype(np.int64), device=DEV)
    kf, vf, sf = R.f64(k[few]), R.f64(v[few]), R.f64(sums[few])
    for i in range(5):
        assert np.array_equal(sf[i, 0, 0], R.summary(kf[i, :, 0]))
    want = R.selected(R.f64(q), sf, small[None], cu, start, prefix, hkv=8, block=256, size=1, most=4, sink=1, local=1)
    assert np.array_equal(blocks.cpu().numpy(), want)
    _check(out, lse, *R.attended(R.f64(q), kf, vf, small[None], want, cu, start, prefix, block=256, size=1))


@pytest.mark.parametrize("heads,size", [((4, 2, 64, 64), 1), ((1, 1, 192, 128), 64), ((32, 1, 128, 128), 1), ((16, 1, 192, 128), 8), ((2, 2, 128, 128), 16)])
@pytest.mark.parametrize("block", [64, 256])
def test_longest_lists(heads, size, block):
    """2048 entries a list, a few of them blocks: the most LDS that a launch takes."""
    hq, hkv, d, dv = heads
    rng = np.random.default_rng(hq + size)
    cu, prefix, start, rows, rng = _chunk([(3000, size + 1), (100, 3)], block, 1, 256, 9)
    table, (k, v) = R.paged(rng, rows, 256, (hkv, d), (hkv, dv))
    q = _bf16(rng, cu[-1], hq, d)
    qb = R.query_blocks(cu, prefix, size)
    lists = np.full((len(qb), hkv, 2048), -1, dtype=np.int32)
    for n, (r0, nr, s, pos) in enumerate(qb):
        c = (pos + nr - 1) // block
        got = rng.permutation(c + 1)
        lists[n, :, rng.permutation(2048)[:len(got)]] = got[:, None]
    attn = _attn(hq, hkv, d, dv, 2048, block_size=block, query_block=size)
    attn.plan(cu, start, prefix)
    out, lse = attn.run_paged(*[x.to(DEV) for x in (q, k, v, torch.as_tensor(table), torch.as_tensor(lists))], lse=torch.empty(hq, cu[-1], device=DEV))
    torch.cuda.synchronize()
    _check(out, lse, *R.attended(R.f64(q), R.f64(k), R.f64(v), table, lists, cu, start, prefix, block=block, size=size))


# -- together -----------------------------------------------------------------------------------
def _layer(hq, hkv, d, dv, page, segs, seed, size=16, most=6, **kw):
    """A layer's state for requests whose prefixes are in the cache already."""
    from paper_2608_26523_amd.rotary import Rotary
    cu, prefix, start, rows, rng = _chunk(segs, 64, 0, page, seed)
    table, (k, v) = R.paged(rng, rows, page, (hkv, d), (hkv, dv))
    attn = _attn(hq, hkv, d, dv, most, query_block=size, **kw)
    mla = d == 192
    rot = Rotary(d, rotary_dim=64 if mla else d, offset=128 if mla else 0, layout="interleaved" if mla else "half")
    sums = attn.new_summaries(k.shape[0], page)
    k, v = k.to(DEV), v.to(DEV)
    before = attn.completed([0] + np.cumsum([p for p, _ in segs]).tolist(), start, [0] * len(segs), table, page)
    attn.summarize(k, before, sums)
    new = [_bf16(rng, cu[-1], n, w).to(DEV) for n, w in ((hq, d), (hkv, d), (hkv, dv))]
    return attn, rot, (cu, start, prefix), table, k, v, sums, new


def _step(attn, rot, plan, table, k, v, sums, new, slots, pos, done, dev_table, q, blocks, out, lse):
    rot.append_paged(new[0], new[1], new[2], k, v, slots, pos, q_out=q)
    attn.summarize(k, done, sums)
    attn.select(q, sums, dev_table, blocks=blocks)
    attn.run_paged(q, k, v, dev_table, blocks, out=out, lse=lse)


@pytest.mark.parametrize("heads", [(8, 2, 128, 128), (3, 3, 192, 128), (16, 1, 64, 64)])
@pytest.mark.parametrize("size,segs", [(1, [(1500, 1), (63, 1), (127, 1)]), (1, [(1000, 70), (60, 9)]), (16, [(1111, 100), (0, 200)])])
def test_a_layer_step(heads, size, segs):
    """Append with rotation, summaries, selection and attention, as a layer calls them, against the same in
    64 bits from the rotated keys that the cache holds."""
    from paper_2608_26523_amd import binding as B
    hq, hkv, d, dv = heads
    page = 128
    print("case:", heads, size, segs, flush=True)
    attn, rot, plan, table, k, v, sums, new = _layer(hq, hkv, d, dv, page, segs, 7 + size, size=size)
    cu, start, prefix = plan
    pos = np.concatenate([np.arange(p, p + n) for p, n in segs])
    slots = torch.as_tensor(B.vpp_paged_slot_mapping(cu, start, prefix, table, page), device=DEV)
    dev_table = torch.as_tensor(table, device=DEV)
    n = attn.plan(*plan)
    q, out = torch.empty_like(new[0]), torch.empty(cu[-1], hq, dv, dtype=torch.bfloat16, device=DEV)
    blocks, lse = torch.empty(n, hkv, 6, dtype=torch.int32, device=DEV), torch.empty(hq, cu[-1], device=DEV)
    done = attn.completed(cu, start, prefix, table, page)
    _step(attn, rot, plan, table, k, v, sums, new, slots, torch.as_tensor(pos, device=DEV), done, dev_table, q, blocks, out, lse)
    torch.cuda.synchronize()
    want, mag = R.rotated(R.f64(new[0]), pos, rot.freq, rot.cfg.offset, bool(rot.cfg.interleaved))
    assert np.all(np.abs(R.f64(q) - want) <= R.rotation_bound(want, mag))
    kf, sf = R.f64(k), R.f64(sums)
    for s, (p, m) in enumerate(segs):
        for b in range((p + m) // 64):
            at = table[s][b * 64 // page], b * 64 % page
            for h in range(hkv):
                assert np.array_equal(sf[at[0], at[1] // 64, h], R.summary(kf[at[0], at[1]:at[1] + 64, h]))
    lists = R.selected(R.f64(q), sf, table, cu, start, prefix, hkv=hkv, block=64, size=size, most=6, sink=1, local=1)
    assert np.array_equal(blocks.cpu().numpy(), lists)
    _check(out, lse, *R.attended(R.f64(q), kf, R.f64(v), table, lists, cu, start, prefix, block=64, size=size))


@pytest.mark.parametrize("heads", [(8, 2, 128, 128), (4, 4, 64, 64), (2, 2, 192, 128)])
def test_lists_of_all_blocks_give_dense_attention(heads):
    from paper_2608_26523_amd.attention import ChunkAttention
    hq, hkv, d, dv = heads
    segs = [(900, 130), (0, 64), (250, 1)]
    attn, rot, plan, table, k, v, sums, new = _layer(hq, hkv, d, dv, 64, segs, 31, size=32, most=40)
    dense = ChunkAttention(hq, hkv, d, dv, max_chunk_tokens=plan[0][-1], max_kv_len=4096)
    dense.plan(*plan)
    attn.plan(*plan)
    dev_table = torch.as_tensor(table, device=DEV)
    lse, l2 = torch.empty(hq, plan[0][-1], device=DEV), torch.empty(hq, plan[0][-1], device=DEV)
    want, _ = dense.run_paged(new[0], k, v, dev_table, lse=lse)
    blocks = attn.select(new[0], sums, dev_table)
    got, _ = attn.run_paged(new[0], k, v, dev_table, blocks, lse=l2)
    torch.cuda.synchronize()
    bound = R.attended(R.f64(new[0]), R.f64(k), R.f64(v), table, blocks.cpu().numpy(), *plan, block=64, size=32)
    _check(got, l2, *bound)
    _check(want, lse, *bound)


def test_a_captured_layer_step_and_its_replays():
    """Two graphs of one object, replayed with new inputs between eager runs."""
    from paper_2608_26523_amd import binding as B
    hq, hkv, d, dv, page = 8, 2, 128, 128, 64
    segs = [(1500, 1), (127, 1), (700, 1), (64, 1)]
    attn, rot, plan, table, k, v, sums, new = _layer(hq, hkv, d, dv, page, segs, 41, size=1, most=9)
    cu, start, prefix = plan
    slots = torch.as_tensor(B.vpp_paged_slot_mapping(cu, start, prefix, table, page), device=DEV)
    pos = torch.as_tensor([p for p, _ in segs], device=DEV)
    dev_table = torch.as_tensor(table, device=DEV)
    attn.plan(*plan)
    done = attn.completed(cu, start, prefix, table, page)

    def buffers():
        return (torch.empty_like(new[0]), torch.empty(4, hkv, 9, dtype=torch.int32, device=DEV),
                torch.empty(4, hq, dv, dtype=torch.bfloat16, device=DEV), torch.empty(hq, 4, device=DEV))
    sets = [buffers(), buffers(), buffers()]
    run = lambda b: _step(attn, rot, plan, table, k, v, sums, new, slots, pos, done, dev_table, *b)  # noqa: E731
    run(sets[2])
    torch.cuda.synchronize()
    graphs = []
    for b in sets[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(b)
    for i in range(3):
        for x in new:
            x.copy_(_bf16(np.random.default_rng(i), *x.shape))
        for b in sets:
            for x in b:
                x.zero_()
        graphs[0].replay()
        graphs[1].replay()
        run(sets[2])
        torch.cuda.synchronize()
        for b in sets[:2]:
            assert all(torch.equal(x, y) for x, y in zip(b, sets[2]))
        assert bool(sets[2][2].float().abs().sum() > 0)


def test_planning_is_refused_within_a_capture():
    attn = _attn(4, 2, 64, 64, 4)
    attn.plan([0, 5], [0], [70])
    q, sums = _bf16(np.random.default_rng(1), 5, 4, 64).to(DEV), attn.new_summaries(2, 64)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    blocks = attn.select(q, sums, table)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: attn.plan([0, 5], [0], [70]), lambda: attn.completed([0, 5], [0], [70], [[1, 0]], 64)):
            with pytest.raises(RuntimeError, match="before the capture"):
                call()
        attn.select(q, sums, table, blocks)
    before = blocks.clone()
    blocks.fill_(7)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(blocks, before)


def test_a_chunk_that_completes_no_block():
    attn = _attn(4, 2, 64, 64, 4)
    done = attn.completed([0, 5], [0], [70], np.array([[1, 0]], dtype=np.int32), 64)
    assert done.numel() == 0 and done.is_cuda and done.dtype == torch.int64
    sums = attn.new_summaries(2, 64)
    attn.summarize(torch.ones(2, 64, 2, 64, dtype=torch.bfloat16, device=DEV), done, sums)
    assert not sums.any()
