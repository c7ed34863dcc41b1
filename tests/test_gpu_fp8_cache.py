"""The 8-bit base cache on the GPU: what the producer writes and what the read back returns, bit for bit against the
fp64 oracle (oracle/fp8_cache.py).  Nothing here has a tolerance but C (bf16 results of fp32 sums)."""
import numpy as np
import pytest
import torch

from oracle import fp8_cache as o
from paper_2604_06370_amd import runtime as rt

pytestmark = pytest.mark.gpu
PS, D, THETA = 16, 128, 500000.0


def _rows(rng, n, hkv, kind):
    x = rng.standard_normal((n, hkv, D))
    if kind == "wide":  # every magnitude of bf16, subnormals to the largest
        x = x * np.exp2(rng.uniform(-140, 126, size=(n, hkv, 1))) * np.exp2(rng.uniform(-12, 0, size=(n, hkv, D)))
    elif kind == "odd":  # zeros, infinities, NaN, the largest, ties
        x[0] = 0.0
        if n > 1:
            x[1, :, 5], x[1, :, 70] = np.inf, np.nan
        if n > 2:
            x[2] = -3.3895313892515355e38
        if n > 3:
            x[3] = np.inf
        if n > 4:
            x[4] = 1e-38
        if n > 5:
            x[5] = (np.arange(D) - 64) / 16 * 7
            x[5, :, 0] = 448.0
        if n > 6:
            x[6, :, ::3] = -0.0
    return torch.from_numpy(x).to(torch.bfloat16)


def _same(got, want):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


def _table(rng, pages, pool_pages):
    return rng.permutation(pool_pages)[:pages].astype(np.int32)


def _cos_sin(pos, cos, sin):
    """Rows of a table for positions `pos`, in fp64."""
    p, i = np.asarray(pos)[:, None], np.arange(D // 2)[None]
    at = (p // 16) * 1024 + (i // 16) * 256 + (p % 16 + 16 * (i % 16 // 4)) * 4 + i % 4
    return [t.cpu().double().numpy().reshape(-1)[at] for t in (cos, sin)]


@pytest.mark.parametrize("hkv", [1, 2, 3, 8])
@pytest.mark.parametrize("pos0,n", [(0, 1), (0, 16), (5, 1), (15, 2), (3, 7), (7, 41), (16, 33), (30, 4)])
@pytest.mark.parametrize("kind", ["plain", "wide", "odd"])
def test_write_and_read_back(hkv, pos0, n, kind):
    rng = np.random.default_rng(hkv * 1000 + pos0 * 50 + n)
    k, v = _rows(rng, n, hkv, kind), _rows(rng, n, hkv, kind)
    pages = (pos0 + n + PS - 1) // PS
    bt = _table(rng, pages, pages + 3)
    before = rng.integers(0, 256, size=(pages + 3, o.page_bytes(hkv)), dtype=np.uint8)
    want = before.copy()
    for j in range(n):
        o.write(want, bt[(pos0 + j) // PS], (pos0 + j) % PS, k[j].double().numpy(), v[j].double().numpy())
    pool, btd = torch.from_numpy(before).cuda(), torch.from_numpy(bt).cuda()
    rt.produce_tokens_fp8([(btd, None, None, pos0, n, 0)], None, k.cuda(), v.cuda(), None, pool, None, hkv, D, 0, PS)
    got = pool.cpu().numpy()
    # a NaN's sign is not fixed: compare the values of the written slots, and every other byte as it was
    sel = np.zeros_like(want, dtype=bool)
    i = np.arange(D)
    for j in range(n):
        pg, s = bt[(pos0 + j) // PS], (pos0 + j) % PS
        for h in range(hkv):
            sel[pg, h * 4096 + o.k_byte(s, i)] = sel[pg, h * 4096 + 2048 + o.v_byte(s, i)] = True
    same = (got == want) | (sel & ((got & 127) == 127) & ((want & 127) == 127))
    assert same.all(), np.argwhere(~same)[:5]
    ko, vo = (torch.full((n + 2, hkv, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rt.gather_tokens_fp8([(btd, pos0, n, 1)], pool, ko, vo, hkv, D, PS)
    _same(ko[1:-1], o.nearest(k.double().numpy()))
    _same(vo[1:-1], o.nearest(v.double().numpy()))
    assert (ko[[0, -1]] == 7).all() and (vo[[0, -1]] == 7).all()  # rows outside the ranges stay


def test_nothing_to_write_or_read():
    pool = torch.full((3, o.page_bytes(2)), 77, dtype=torch.uint8, device="cuda")
    bt = torch.zeros(2, dtype=torch.int32, device="cuda")
    none, x = torch.empty(0, 2, D, dtype=torch.bfloat16, device="cuda"), torch.ones(4, 2, D, dtype=torch.bfloat16, device="cuda")
    for k in (none, x):
        rt.produce_tokens_fp8([(bt, None, None, 3, 0, 0), (None, None, None, 0, 0, 0)], None, k, k, None, pool, None, 2, D, 0, PS)
        rt.produce_tokens_fp8([], None, k, k, None, pool, None, 2, D, 0, PS)
        rt.gather_tokens_fp8([(bt, 3, 0, 0)], pool, k, k, 2, D, PS)
        rt.gather_tokens_fp8([], pool, k, k, 2, D, PS)
    rt.page_copy_fp8([], pool, None, 2, D, 0, PS)
    rt.page_copy_fp8([(0, 0, 1, 0)], pool, None, 2, D, 0, PS)
    torch.cuda.synchronize()
    assert bool((pool == 77).all()) and bool((x == 1).all())


def test_every_code_reads_back_exactly():
    """All 256 codes with all exponent bytes that are written, in both K and V."""
    pool = torch.zeros(237, o.page_bytes(1), dtype=torch.uint8)
    pool[:, :4096] = torch.from_numpy(np.random.default_rng(1).permutation(np.tile(np.arange(256, dtype=np.uint8), 16)))
    pool[:, 4096:4128] = torch.arange(10, 247, dtype=torch.uint8)[:, None]
    bt = torch.arange(237, dtype=torch.int32).cuda()
    ko, vo = (torch.empty(237 * PS, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rt.gather_tokens_fp8([(bt, 0, 237 * PS, 0)], pool.cuda(), ko, vo, 1, D, PS)
    p = pool.numpy()
    want = [o.read(p, g, s, 1) for g in range(237) for s in range(PS)]
    _same(ko, np.stack([w[0] for w in want]))
    _same(vo, np.stack([w[1] for w in want]))


@pytest.mark.parametrize("hkv,r,hidden", [(8, 16, 1024), (2, 8, 2048), (1, 64, 1024), (3, 32, 1024), (8, 0, 0)])
def test_batch_with_rope_and_shrink(hkv, r, hidden):
    """Ragged sequences, one without adapter, one empty, far positions: K's rotation rounded once, C beside it."""
    rng = np.random.default_rng(hkv * 100 + r)
    spec = [(0, 1), (13, 40), (5, 0), (4091, 70), (100000, 3)]  # (pos0, n)
    rows = sum(n for _, n in spec)
    k, v = _rows(rng, rows, hkv, "plain"), _rows(rng, rows, hkv, "plain")
    k[::7] *= 100
    k[3, :, 9] = float("inf")
    x = torch.from_numpy(rng.standard_normal((rows, max(hidden, 1)))).to(torch.bfloat16)
    la = torch.from_numpy(rng.standard_normal((len(spec), 2, max(r, 1), max(hidden, 1))) / max(hidden, 1) ** 0.5).to(torch.bfloat16)
    cos, sin = rt.rope_tables(D, 100016, THETA, "cuda")
    width, used = 100016 // PS, 0
    tables, seqs, row0 = [], [], 0
    for i, (pos0, n) in enumerate(spec):
        bt = np.zeros(width, np.int32)
        first, last = pos0 // PS, (pos0 + n + PS - 1) // PS
        bt[first:last] = np.arange(used, used + last - first)
        used += last - first
        tables.append(torch.from_numpy(bt).cuda())
        seqs.append((tables[-1], tables[-1] if r else None, la[i].cuda() if r and i != 1 else None, pos0, n, row0))
        row0 += n
    pool = torch.zeros(used, o.page_bytes(hkv), dtype=torch.uint8, device="cuda")
    res = torch.zeros(used, max(1, rt.res_page_elems(PS, r)), dtype=torch.bfloat16, device="cuda")
    rt.produce_tokens_fp8(seqs, x.cuda() if r else None, k.cuda(), v.cuda(), (cos, sin), pool, res if r else None, hkv, D, r, PS)
    ko, vo = (torch.empty(rows, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rt.gather_tokens_fp8([(s[0], s[3], s[4], s[5]) for s in seqs], pool, ko, vo, hkv, D, PS)
    pos = np.concatenate([np.arange(p, p + n) for p, n in spec])
    co, si = _cos_sin(pos, cos, sin)
    kd = k.double().numpy()
    a, b = kd[..., :64], kd[..., 64:]
    with np.errstate(invalid="ignore"):
        turned = np.concatenate([a * co[:, None] - b * si[:, None], b * co[:, None] + a * si[:, None]], axis=-1)
    _same(ko, o.nearest(turned))
    _same(vo, o.nearest(v.double().numpy()))
    if r:
        # the residual pool is what the bf16 producer writes, bit for bit
        want = torch.zeros_like(res)
        base = torch.zeros(used, 2, hkv, PS * D, dtype=torch.bfloat16, device="cuda")
        rt.produce_tokens_batch(seqs, x.cuda(), k.cuda(), v.cuda(), (cos, sin), base, want, hkv, D, r, PS)
        assert torch.equal(res.view(torch.int16), want.view(torch.int16)) and res.any()


def test_cut_into_calls_writes_the_same():
    rng = np.random.default_rng(5)
    k, v = (_rows(rng, 61, 2, "plain").cuda() for _ in range(2))
    bt = torch.arange(5, dtype=torch.int32).cuda()
    rope = rt.rope_tables(D, 80, THETA, "cuda")
    pools = [torch.zeros(5, o.page_bytes(2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    rt.produce_tokens_fp8([(bt, None, None, 9, 61, 0)], None, k, v, rope, pools[0], None, 2, D, 0, PS)
    at = 0
    for n in (1, 2, 3, 5, 1, 17, 30, 2):
        rt.produce_tokens_fp8([(bt, None, None, 9 + at, n, at)], None, k, v, rope, pools[1], None, 2, D, 0, PS)
        at += n
    assert at == 61 and torch.equal(*pools)


def test_more_sequences_than_one_launch():
    rng = np.random.default_rng(6)
    n = [int(x) for x in rng.integers(0, 20, size=70)]
    row0 = np.concatenate([[0], np.cumsum(n)])
    k, v = (_rows(rng, int(row0[-1]), 2, "plain") for _ in range(2))
    bt = torch.arange(140, dtype=torch.int32).reshape(70, 2).cuda()
    pool = torch.zeros(140, o.page_bytes(2), dtype=torch.uint8, device="cuda")
    seqs = [(bt[i], None, None, i % 13, n[i], int(row0[i])) for i in range(70)]
    rt.produce_tokens_fp8(seqs, None, k.cuda(), v.cuda(), None, pool, None, 2, D, 0, PS)
    ko, vo = (torch.empty(k.shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rt.gather_tokens_fp8([(s[0], s[3], s[4], s[5]) for s in seqs], pool, ko, vo, 2, D, PS)
    _same(ko, o.nearest(k.double().numpy()))
    _same(vo, o.nearest(v.double().numpy()))


@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_page_copy(hkv):
    rng = np.random.default_rng(hkv)
    before = rng.integers(0, 256, size=(40, o.page_bytes(hkv)), dtype=np.uint8)
    pool = torch.from_numpy(before).cuda()
    res0 = torch.from_numpy(rng.standard_normal((40, 512))).to(torch.bfloat16).cuda()
    res = res0.clone()
    copies = [(0, s, 20 + s, s) for s in range(18)] + [(1, 1, 30, 5), (0, 3, 3, 16)]
    rt.page_copy_fp8(copies, pool, res, hkv, D, 16, PS)
    want = before.copy()
    i = np.arange(D)
    for _, s, d, nv in copies[:18]:
        for t in range(min(nv, PS)):
            for h in range(hkv):
                for j, where in enumerate((o.k_byte, o.v_byte)):
                    at = h * 4096 + j * 2048 + where(t, i)
                    want[d, at] = before[s, at]
                    e = hkv * 4096 + h * 32 + j * 16 + t
                    want[d, e] = before[s, e]
    assert np.array_equal(pool.cpu().numpy(), want)
    other = torch.cat([res0[:30], res0[31:]])
    assert torch.equal(torch.cat([res[:30], res[31:]]), other) and not torch.equal(res[30], res0[30])


def test_long_list_of_copies():
    pool = torch.from_numpy(np.random.default_rng(2).integers(0, 256, size=(600, o.page_bytes(1)), dtype=np.uint8)).cuda()
    want = pool.clone()
    want[300:, :4128] = pool[:300, :4128]
    rt.page_copy_fp8([(0, s, 300 + s, 16) for s in range(300)], pool, None, 1, D, 0, PS)
    assert torch.equal(pool[:, :4128], want[:, :4128])


def test_pool_above_four_gib():
    """Pages whose byte offsets pass 32 bits."""
    hkv = 8
    pages = (4 << 30) // o.page_bytes(hkv) + 40
    pool = torch.zeros(pages, o.page_bytes(hkv), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(8)
    k, v = (_rows(rng, 40, hkv, "plain") for _ in range(2))
    bt = torch.tensor([pages - 1, 3, pages - 7], dtype=torch.int32).cuda()
    rt.produce_tokens_fp8([(bt, None, None, 0, 40, 0)], None, k.cuda(), v.cuda(), None, pool, None, hkv, D, 0, PS)
    rt.page_copy_fp8([(0, pages - 1, pages - 2, 16), (0, 3, 4, 16)], pool, None, hkv, D, 0, PS)
    ko, vo = (torch.empty(40, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rt.gather_tokens_fp8([(torch.tensor([pages - 2, 4, pages - 7], dtype=torch.int32).cuda(), 0, 40, 0)], pool, ko, vo, hkv, D, PS)
    _same(ko, o.nearest(k.double().numpy()))
    _same(vo, o.nearest(v.double().numpy()))


def test_other_stream_and_graph():
    """The calls go to the stream they are given, and replay from a graph onto new rows."""
    rng = np.random.default_rng(9)
    k, v = (_rows(rng, 30, 2, "plain").cuda() for _ in range(2))
    bt = torch.arange(3, dtype=torch.int32).cuda()
    pool = torch.zeros(3, o.page_bytes(2), dtype=torch.uint8, device="cuda")
    ko, vo = (torch.zeros(30, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rope = rt.rope_tables(D, 48, THETA, "cuda")

    def both(stream=None):
        rt.produce_tokens_fp8([(bt, None, None, 5, 30, 0)], None, k, v, rope, pool, None, 2, D, 0, PS, stream)
        rt.gather_tokens_fp8([(bt, 5, 30, 0)], pool, ko, vo, 2, D, PS, stream)

    both()
    torch.cuda.synchronize()
    want = ko.clone(), vo.clone()
    side = torch.cuda.Stream()
    pool.zero_()
    ko.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert torch.equal(ko, want[0]) and torch.equal(vo, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(4):
        k.copy_(torch.randn_like(k))
        v.copy_(torch.randn_like(v))
        both()
        torch.cuda.synchronize()
        want = ko.clone(), vo.clone()
        pool.zero_()
        ko.zero_()
        vo.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ko, want[0]) and torch.equal(vo, want[1]), i


def test_refusals_on_the_gpu():
    pool = torch.zeros(2, o.page_bytes(2), dtype=torch.uint8, device="cuda")
    k = torch.zeros(40, 2, D, dtype=torch.bfloat16, device="cuda")
    bt = torch.zeros(2, dtype=torch.int32, device="cuda")
    good = dict(seqs=[(bt, None, None, 0, 4, 0)], x=None, k_raw=k, v=k, rope=None, base_fp8=pool, res_kv=None, hkv=2, d=D, r=0, page_size=PS)
    rt.produce_tokens_fp8(**good)
    la = torch.zeros(2, 16, 1024, dtype=torch.bfloat16, device="cuda")
    for bad in (dict(seqs=[(bt, None, None, 30, 4, 0)]), dict(seqs=[(bt, None, None, 0, 4, 37)]), dict(seqs=[(bt.long(), None, None, 0, 4, 0)]),
                dict(k_raw=k.float()), dict(v=k[:39]), dict(k_raw=k.transpose(0, 1)), dict(base_fp8=pool[:, :-128]), dict(hkv=1),
                dict(base_fp8=pool.view(torch.int8)), dict(rope=(k, k)), dict(seqs=[(bt, None, la, 0, 4, 0)], r=16),
                dict(seqs=[(bt, bt, la, 0, 4, 0)], r=16, x=k.reshape(40, 256)), dict(k_raw=k.cpu()), dict(seqs=[(None, None, None, 0, 4, 0)])):
        with pytest.raises(rt.FKVError):
            rt.produce_tokens_fp8(**{**good, **bad})
    ro = dict(seqs=[(bt, 0, 4, 0)], base_fp8=pool, k_out=k, v_out=k.clone(), hkv=2, d=D, page_size=PS)
    rt.gather_tokens_fp8(**ro)
    for bad in (dict(seqs=[(bt, 29, 4, 0)]), dict(seqs=[(bt, 0, 4, 38)]), dict(seqs=[(bt.cpu(), 0, 4, 0)]), dict(k_out=k.half()),
                dict(v_out=k[:, :1]), dict(base_fp8=pool.bfloat16())):
        with pytest.raises(rt.FKVError):
            rt.gather_tokens_fp8(**{**ro, **bad})
    for copies in ([(0, 0, 2, 4)], [(0, 2, 0, 4)], [(1, 0, 0, 4)], [(2, 0, 1, 4)], [(0, -1, 1, 4)]):
        with pytest.raises(rt.FKVError):
            rt.page_copy_fp8(copies, pool, None, 2, D, 0, PS)
    torch.cuda.synchronize()
