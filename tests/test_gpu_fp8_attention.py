"""ResidualAttention over an 8-bit base cache, against 64 bits and against the bf16 kernels on the same values.

Every cached value is exact in bf16, and the decode kernels scale their weights by powers of two only, so decode
over 8-bit pages has to give the bits that decode over bf16 pages with the same values gives.

Bound of an element's error against 64 bits, u = 2^-8 (half a bf16 step): u |O| for the output's rounding; 2 u A for the weights'
(numerator and, where the row sums take them rounded, denominator), A = sum p |v| / l with |v| = |V_base| + |C_V| |B_V|; and
2.1 D A for the scores', whose error is at most D = u scale max_key sum |q| |k| (sum over what is rounded before it enters a
product: K, or its low-rank part) -- a score error of D moves a weight by a factor of at most e^(2 D) after
normalisation.  fp32 sums add less than 1 % of that.  Beside it, since roundings are not all at their worst, the 2-norm of the
error is at most 1e-2 of the result's (the bar of the bf16 path's tests).  Unwritten slots hold NaN codes, exponent byte 255 and NaN rCache rows throughout.
"""
import ctypes

import numpy as np
import pytest
import torch

from oracle import fp8_cache as o
from paper_2604_06370_amd import _native as N
from paper_2604_06370_amd import runtime as rt
from paper_2604_06370_amd import workloads as W
from paper_2604_06370_amd.driver import LoadedWorkload

pytestmark = pytest.mark.gpu
PS, D, THETA = 16, 128, 500000.0
TOL_REL = 1e-2


class Problem:
    """Agents of `lens` tokens, the first `shared` of them common, rows[a] query rows each (decode: one)."""

    def __init__(self, seed, lens, shared, hq, hkv, r, rope, rows=None, bare=(), q_std=1.0, b_std=None, edit=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.lens, self.hq, self.hkv, self.r, self.rope, self.rows = list(lens), hq, hkv, r, rope and r > 0, rows
        n, width = len(lens), max(-(-x // PS) for x in lens) + 1
        common = shared // PS
        bt, nb = np.zeros((n, width), np.int32), common
        rbt, nr = np.zeros((n, width), np.int32), 0
        for a, x in enumerate(lens):
            pages = -(-x // PS)
            mine = min(common, pages)
            bt[a, :mine] = np.arange(mine)
            bt[a, mine:pages] = np.arange(nb, nb + pages - mine)
            nb += pages - mine
            rbt[a, :pages] = np.arange(nr, nr + pages)
            nr += pages
        rng = np.random.default_rng(seed)
        self.bt, self.rbt = rng.permutation(nb).astype(np.int32)[bt], rng.permutation(nr).astype(np.int32)[rbt]
        self.base = torch.from_numpy(self.bt).cuda()
        self.res_bt = torch.from_numpy(self.rbt).cuda()
        pool = torch.full((nb, o.page_bytes(hkv)), 255, dtype=torch.uint8, device="cuda")
        wide = torch.full((nb, 2, hkv, PS * D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.res_kv = torch.full((nr, max(1, rt.res_page_elems(PS, r))), float("nan"), dtype=torch.bfloat16, device="cuda") if r else None
        channel = torch.where(torch.rand(hkv, D, generator=g, device="cuda") < 0.03, 6.0, 1.0)
        sk, sv = normal(max(shared, 1), hkv, D) * channel, normal(max(shared, 1), hkv, D)
        self.k, self.v, self.ck, self.cv = [], [], [], []
        for a, x in enumerate(lens):
            k, v = normal(x, hkv, D) * channel, normal(x, hkv, D)
            m = min(common * PS, x)
            k[:m], v[:m] = sk[:m], sv[:m]
            if edit:
                edit(a, k, v)
            k, v = k.bfloat16(), v.bfloat16()
            rt.produce_tokens_fp8([(self.base[a], None, None, 0, x, 0)], None, k, v, None, pool, None, hkv, D, 0, PS)
            ko, vo = torch.empty_like(k), torch.empty_like(v)
            rt.gather_tokens_fp8([(self.base[a], 0, x, 0)], pool, ko, vo, hkv, D, PS)
            rt.scatter_tokens(self.base[a], None, 0, ko, vo, None, None, wide, self.res_kv, hkv, D, r, PS)
            self.k.append(ko)
            self.v.append(vo)
            if r:
                c = normal(2, x, r).bfloat16()
                rt.scatter_tokens(None, self.res_bt[a], 0, None, None, c[0].contiguous(), c[1].contiguous(), wide, self.res_kv, hkv, D, r, PS)
                self.ck.append(c[0])
                self.cv.append(c[1])
        self.pool, self.wide = pool, wide
        self.adapter = np.array([-1 if a in bare else a for a in range(n)], np.int32)
        self.b = (normal(n, 2, max(r, 1), hkv * D) * (b_std or (max(r, 1) ** -0.5))).bfloat16() if r else None
        self.q = (normal(sum(rows) if rows else n, hq, D) * q_std).bfloat16()
        self.cos_sin = rt.rope_tables(D, width * PS, THETA, "cuda") if self.rope else None
        self.dev_lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.dev_adapter = torch.from_numpy(self.adapter).cuda()
        self.indptr = torch.tensor(np.cumsum([0] + list(rows)).astype(np.int32), device="cuda") if rows else None

    def args(self, out, pool=None, **more):
        return rt.make_args(q=self.q, base_kv=self.pool if pool is None else pool, res_kv=self.res_kv, lora_b=self.b,
                            adapter_idx=self.dev_adapter if self.r else None, base_bt=self.base, res_bt=self.res_bt if self.r else None,
                            seq_lens=self.dev_lens, out=out, hq=self.hq, hkv=self.hkv, d=D, r=self.r, page_size=PS, rope=self.cos_sin, **more)

    def plan(self, **kw):
        return rt.DecodePlan(self.bt, np.array(self.lens, np.int32), self.hq, self.hkv, PS, r=self.r, rope=self.rope, **kw)

    def decode(self, wide=False, plan=None):
        plan = plan or self.plan()
        out = torch.full_like(self.q, 9.0)
        ws = torch.full((max(4, plan.info(D, self.r)["workspace_bytes"]) // 4,), float("nan"), dtype=torch.float32, device="cuda")
        call = rt.residual_attention_decode if wide else rt.residual_attention_decode_fp8
        call(self.args(out, pool=self.wide if wide else None, plan_dev=plan.device("cuda"), workspace=ws), plan)
        torch.cuda.synchronize()
        return out

    def prefill(self, wide=False, max_q=0):
        out = torch.full_like(self.q, 9.0)
        call = rt.residual_attention_prefill if wide else rt.residual_attention_prefill_fp8
        call(self.args(out, pool=self.wide if wide else None, q_indptr=self.indptr, n_q=sum(self.rows), max_q_per_agent=max_q or max(self.rows)))
        torch.cuda.synchronize()
        return out

    def reference(self):
        """Outputs in 64 bits, and the bound of each element's error."""
        u, g, scale = 2.0 ** -8, self.hq // self.hkv, D ** -0.5
        rows = self.rows or [1] * len(self.lens)
        outs, bounds, q0 = [], [], 0
        for a, x in enumerate(self.lens):
            m = rows[a]
            k, v = self.k[a].double(), self.v[a].double()
            va, low = v.abs(), torch.zeros_like(k)
            if self.r and self.adapter[a] >= 0:
                b = self.b[a].double().view(2, self.r, self.hkv, D)
                low = torch.einsum("tr,rhd->thd", self.ck[a].double(), b[0])
                if self.rope:
                    f = THETA ** (-torch.arange(64, device="cuda", dtype=torch.float64) * 2 / D)
                    ang = torch.arange(x, device="cuda", dtype=torch.float64)[:, None, None] * f
                    c, s, p, w = ang.cos(), ang.sin(), low[..., :64], low[..., 64:]
                    low = torch.cat([p * c - w * s, w * c + p * s], dim=-1)
                v = v + torch.einsum("tr,rhd->thd", self.cv[a].double(), b[1])
                va = va + torch.einsum("tr,rhd->thd", self.cv[a].double().abs(), b[1].abs())
            kk = k + low
            seen = torch.arange(x, device="cuda")[None] <= (x - m + torch.arange(m, device="cuda"))[:, None]
            q = self.q[q0:q0 + m].double().view(m, self.hkv, g, D)
            q0 += m
            z = torch.einsum("mhgd,thd->hgmt", q, kk) * scale
            p = torch.softmax(z.masked_fill(~seen, float("-inf")), dim=-1)
            out = torch.einsum("hgmt,thd->mhgd", p, v)
            big = torch.einsum("hgmt,thd->mhgd", p, va)
            # what is rounded before the score products: K whole (prefill) or its low-rank part, through W = B q without RoPE
            part = (kk.abs() + low.abs()) if self.rows else low.abs()
            if self.r and not self.rope and self.adapter[a] >= 0:
                wq = torch.einsum("mhgd,rhd->mhgr", q, b[0]).abs()
                extra = torch.einsum("mhgr,tr->hgmt", wq, self.ck[a].double().abs())
            else:
                extra = 0.0
            d = u * scale * (torch.einsum("mhgd,thd->hgmt", q.abs(), part) + extra)
            d = d.masked_fill(~seen, 0.0).amax(dim=-1).permute(2, 0, 1)[..., None]
            bounds.append((u * out.abs() + (2 * u + torch.expm1(2.1 * d)) * big).reshape(m, self.hq, D) * 1.01 + 1e-30)
            outs.append(out.reshape(m, self.hq, D))
        return torch.cat(outs), torch.cat(bounds)

    def check(self, out):
        ref, bound = self.reference()
        err = (out.double() - ref).abs()
        rel = float(err.norm() / ref.norm())
        print(f"rel {rel:.2e} worst share of the bound {float((err / bound).max()):.3f}", flush=True)
        assert torch.isfinite(out.float()).all() and (err <= bound).all() and rel <= TOL_REL


RANKS = [(0, False), (8, False), (8, True), (16, False), (16, True), (32, False), (32, True), (64, False), (64, True)]
SHORT = [1, 2, 15, 16, 17, 5, 31, 33]


@pytest.mark.parametrize("r,rope", RANKS)
@pytest.mark.parametrize("hq,hkv", [(8, 2), (64, 8), (4, 1), (12, 3)])
def test_decode_short_and_private(hq, hkv, r, rope):
    p = Problem(1, SHORT, 0, hq, hkv, r, rope, bare=(5,))
    out = p.decode()
    assert torch.equal(out, p.decode(wide=True))
    p.check(out)


@pytest.mark.parametrize("r,rope", RANKS)
@pytest.mark.parametrize("hq,hkv", [(32, 8), (16, 2)])
@pytest.mark.parametrize("n", [3, 7, 16, 33])
def test_decode_shared_prefix(hq, hkv, r, rope, n):
    """Items of one to four agent groups over a shared prefix, ragged suffixes, agents that end inside it."""
    lens = [700 + (37 * a) % 150 for a in range(n)]
    lens[n // 2] = 690
    p = Problem(2 + n, lens, 692, hq, hkv, r, rope, bare=(1,))
    out = p.decode()
    assert torch.equal(out, p.decode(wide=True))
    p.check(out)


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("pps,agents", [(1, 0), (4, 2), (64, 1), (7, 16)])
def test_decode_other_plans(rope, pps, agents):
    p = Problem(5, [900 + 5 * a for a in range(12)], 880, 32, 8, 16, rope)
    plan = p.plan(pages_per_split=pps, max_item_agents=agents)
    out = p.decode(plan=plan)
    assert torch.equal(out, p.decode(wide=True, plan=plan))
    p.check(out)


@pytest.mark.parametrize("rope", [False, True])
def test_decode_long_context_one_kv_head(rope):
    p = Problem(6, [40000, 39990, 40011, 1], 39985, 4, 1, 16, rope)
    out = p.decode()
    assert torch.equal(out, p.decode(wide=True))
    p.check(out)


@pytest.mark.parametrize("kind", ["sharp", "tiny", "huge", "zero", "scales", "nan"])
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("prefill", [False, True])
def test_values_at_the_edges(prefill, kind, rope):
    """Peaked rows, rows far below and above 1, zero rows, tokens of very different scales, a NaN in one agent's values."""
    def edit(a, k, v):
        if kind == "tiny":
            k *= 1e-30
            v *= 1e-30
        elif kind == "huge":
            v *= 1e30
        elif kind == "zero":
            k[::3], v[::2] = 0, 0
        elif kind == "scales":
            s = torch.exp2(torch.arange(v.shape[0], device="cuda") % 41 - 20.0)[:, None, None]
            v *= s
        elif kind == "nan" and a == 1:
            v[-1, 0, 3] = float("nan")

    lens = [130, 77, 300, 64]
    p = Problem(7, lens, 0, 32, 8, 16, rope, rows=[20, 1, 33, 64] if prefill else None, q_std=4.0 if kind == "sharp" else 1.0,
                b_std=1e-3 if kind in ("tiny", "huge", "nan") else None, edit=edit)
    run = p.prefill if prefill else p.decode
    out = run()
    if not prefill:
        both = torch.stack([out, run(wide=True)]).float()
        assert torch.equal(torch.isnan(both[0]), torch.isnan(both[1])) and torch.equal(both[0].nan_to_num(), both[1].nan_to_num())
    if kind == "nan":
        bad = torch.isnan(out.float())
        rows = slice(20, 21) if prefill else slice(1, 2)  # only agent 1's row, heads of KV head 0, dim 3
        assert bad[rows, :4, 3].all() and int(bad.sum()) == 4
        return
    ref, bound = p.reference()
    err = (out.double() - ref).abs()
    assert torch.isfinite(out.float()).all() and (err <= bound).all() and float(err.norm() / ref.norm()) <= TOL_REL


@pytest.mark.parametrize("r,rope", RANKS)
@pytest.mark.parametrize("hq,hkv", [(32, 8), (64, 8), (4, 1), (24, 3)])
def test_prefill_ragged_chunks(hq, hkv, r, rope):
    """Chunks of one token to several tiles, whole contexts, contexts that end inside a tile or page."""
    p = Problem(11, [1, 17, 200, 64, 333, 129], 0, hq, hkv, r, rope, rows=[1, 17, 5, 64, 130, 1], bare=(2,))
    p.check(p.prefill())


@pytest.mark.parametrize("r,rope", RANKS)
@pytest.mark.parametrize("lens,rows", [([2100], [2100]), ([5000, 4811], [70, 300]), ([65, 128, 192, 193], [64, 64, 1, 100])])
def test_prefill_tiles(r, rope, lens, rows):
    p = Problem(12, lens, 32, 32, 8, r, rope, rows=rows)
    p.check(p.prefill())


@pytest.mark.parametrize("r,rope", RANKS)
def test_prefill_middle_grids(r, rope):
    """Grids that fill the compute units with 128 rows per workgroup and not with 256: contexts of one tile to many, whole and partial."""
    p = Problem(14, [1000, 63, 250, 4130], 0, 32, 8, r, rope, rows=[250, 63, 250, 249], bare=(0,))
    p.check(p.prefill())


def _without_workspace(p, max_q=0):
    """The C call without scratch: one workgroup passes over all keys of a row."""
    out = torch.full_like(p.q, 9.0)
    args = p.args(out, q_indptr=p.indptr, n_q=sum(p.rows), max_q_per_agent=max_q or max(p.rows))
    N.check(N.fkv_residual_attention_prefill_fp8(ctypes.byref(args), torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("r,rope", RANKS)
@pytest.mark.parametrize("hq,hkv,lens,rows", [
    (64, 8, [9001], [1]),                        # one row per head over a long context, a workgroup per 256 keys
    (4, 1, [3000, 20, 1, 517], [4, 20, 1, 33]),  # contexts shorter than the splits: most of them are empty
    (32, 8, [4133, 2000], [64, 250]),            # 256 rows, a chunk that ends before the last block
])
def test_prefill_splits_long_contexts(hq, hkv, lens, rows, r, rope):
    p = Problem(15, lens, 0, hq, hkv, r, rope, rows=rows, bare=(0,) if len(lens) == 4 else ())
    width = p.base.shape[1]
    assert rt.prefill_fp8_workspace_bytes(hq, hkv, r, len(lens), max(rows), width) > 0
    p.check(p.prefill())
    p.check(_without_workspace(p))


def test_prefill_splits_with_the_callers_workspace():
    p = Problem(16, [5000, 700], 0, 32, 8, 16, True, rows=[3, 40])
    want, whole = p.prefill(), _without_workspace(p)
    need = rt.prefill_fp8_workspace_bytes(32, 8, 16, 2, 40, p.base.shape[1])
    kw = dict(q_indptr=p.indptr, n_q=43, max_q_per_agent=40)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")  # NaN, and a guard behind it
    out = torch.zeros_like(p.q)
    rt.residual_attention_prefill_fp8(p.args(out, workspace=ws[:need], **kw))
    torch.cuda.synchronize()
    assert torch.equal(out, want) and bool((ws[need:] == 255).all()) and not bool((ws[:need] == 255).all())
    args = p.args(out, workspace=ws[:need - 16], **kw)  # too small for the C call: no split
    N.check(N.fkv_residual_attention_prefill_fp8(ctypes.byref(args), torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert torch.equal(out, whole) and not torch.equal(out, want)


def test_prefill_splits_keep_unreached_rows_nan():
    p = Problem(17, [2000, 900], 0, 32, 8, 16, False, rows=[200, 20])
    out = p.prefill(max_q=64)
    ref, bound = p.reference()
    reached = torch.ones(220, dtype=torch.bool, device="cuda")
    reached[64:200] = False
    assert torch.isnan(out[~reached].float()).all()
    assert ((out.double() - ref).abs() <= bound)[reached].all()


def test_prefill_splits_in_a_graph_and_on_two_streams():
    ps = [Problem(18 + i, [6000, 333], 0, 32, 8, 16, i == 1, rows=[5, 60]) for i in range(2)]
    want = [p.prefill() for p in ps]
    outs = [torch.zeros_like(p.q) for p in ps]
    args = [p.args(out, q_indptr=p.indptr, n_q=65, max_q_per_agent=60) for p, out in zip(ps, outs)]
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(3):  # scratch of calls in flight at once is not shared
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for a, s in zip(args, streams):
            rt.residual_attention_prefill_fp8(a, s)
        torch.cuda.synchronize()
        assert all(torch.equal(out, w) for out, w in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for a in args:
            rt.residual_attention_prefill_fp8(a)
    for _ in range(4):
        for out in outs:
            out.zero_()
        graph.replay()
        eager = ps[0].prefill()
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0]) and all(torch.equal(out, w) for out, w in zip(outs, want))


def test_prefill_splits_on_a_forked_stream_of_a_graph():
    p = Problem(22, [6000, 70], 0, 32, 8, 16, True, rows=[5, 9])
    want, out = p.prefill(), torch.zeros_like(p.q)
    args = p.args(out, q_indptr=p.indptr, n_q=14, max_q_per_agent=9)
    assert rt.prefill_fp8_workspace_bytes(32, 8, 16, 2, 9, p.base.shape[1]) > 0
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        rt.residual_attention_prefill_fp8(args, side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        out.zero_()
        graph.replay()
        eager = p.prefill()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(eager, want)


@pytest.mark.parametrize("raw", [False, True])
def test_prefill_scratch_belongs_to_its_stream(raw):
    """Memory freed on the current stream with work pending there is not the scratch of a call on another stream."""
    p = Problem(21, [6000], 0, 32, 8, 16, False, rows=[5])
    want, out = p.prefill(), torch.zeros_like(p.q)
    args = p.args(out, q_indptr=p.indptr, n_q=5, max_q_per_agent=5)
    need = rt.prefill_fp8_workspace_bytes(32, 8, 16, 1, 5, p.base.shape[1])
    side, a = torch.cuda.Stream(), torch.full((4096, 4096), 1e-4, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for _ in range(3):
        held = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(4)]
        for _ in range(8):
            a = a @ a * 1e-3
        for x in held:
            x.fill_(255)
        del held, x
        rt.residual_attention_prefill_fp8(args, side.cuda_stream if raw else side)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        out.zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("r", [0, 16])
def test_prefill_understated_rows_are_nan(r):
    p = Problem(13, [400, 300], 0, 32, 8, r, False, rows=[200, 20])
    full = p.prefill()
    out = p.prefill(max_q=64)
    assert torch.isnan(out[64:200].float()).all()
    assert torch.equal(out[:64], full[:64]) and torch.equal(out[200:], full[200:])


def _held(wl):
    """The workload with the values that an 8-bit cache holds in place of its base rows."""
    for name in ("base_k", "base_v"):
        x = W.bf16_bits_to_f64(getattr(wl, name))
        setattr(wl, name, W.f32_to_bf16_bits(o.nearest(x).astype(np.float32)))
    return wl


@pytest.mark.parametrize("rope", [False, True])
def test_driver_serves_a_mixed_step(rope):
    """Forks, copy-on-write page copies, appended chunks, decode steps, the mixed step and its graph, all on 8-bit pages."""
    make = lambda: W.tree("fp8-mixed", 71, node_parent=[-1, 0], node_len=[203, 37], agent_node=[0, 1, 1, 0, 1, 0], suffix_lo=1,  # noqa: E731
                          suffix_hi=60, hq=32, hkv=8, r=16, b_std=0.25, chunk=[0, 40, 0, 0, 25, 0], zero_residual=[3])
    lw, lw16 = LoadedWorkload(make(), rope=rope, base_format="fp8"), LoadedWorkload(_held(make()), rope=rope)
    for a in range(6):
        n = int(lw.wl.seq_len[a])
        k, v = lw.read_base(a, 0, n)
        rows = lw16.wl.base_row[a][:n]
        for got, want in ((k, lw16.wl.base_k), (v, lw16.wl.base_v)):
            assert np.array_equal(got.view(torch.int16).cpu().numpy(), want[rows].view(np.int16))
    out, chunk = (x.clone() for x in lw.mixed())
    torch.cuda.synchronize()
    assert torch.equal(out, lw16.decode())
    diff = (chunk.double() - lw16.prefill().double())
    assert float(diff.norm() / chunk.double().norm()) <= TOL_REL
    graph = lw.capture_mixed_graph()
    for _ in range(4):
        lw._decode["out"].zero_()
        lw._prefill["out"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(lw._decode["out"], out) and torch.equal(lw._prefill["out"], chunk)
        lw.decode()
        torch.cuda.synchronize()
    rng, rng16 = np.random.default_rng(3), np.random.default_rng(3)
    for _ in range(20):
        for a in lw._decode["agents"]:
            lw.append_token(a, W.append_decode_token(lw.wl, a, rng))
            rows = W.append_decode_token(lw16.wl, a, rng16)
            for name in ("k", "v"):
                x = W.bf16_bits_to_f64(rows[name])
                rows[name] = W.f32_to_bf16_bits(o.nearest(x).astype(np.float32))
            lw16.append_token(a, rows)
        for w in (lw, lw16):
            sl = w.refresh_decode_tables()
            w._decode["plan"].covers(sl)
        assert torch.equal(lw.decode(), lw16.decode())
    lw.close()
    lw16.close()


def test_plan_serves_both_formats_on_two_streams():
    """Two 8-bit decodes at once on two streams with workspaces of their own, beside the bf16 one."""
    ps = [Problem(20 + i, [500 + 9 * a for a in range(9)], 480, 32, 8, 16, i == 1) for i in range(2)]
    want = [p.decode() for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    held = []
    for p, s in zip(ps, streams):
        plan, out = p.plan(), torch.zeros_like(p.q)
        ws = torch.empty(plan.info(D, 16)["workspace_bytes"] // 4, dtype=torch.float32, device="cuda")
        held.append((plan, out, ws, p.args(out, plan_dev=plan.device("cuda"), workspace=ws)))
    torch.cuda.synchronize()
    for _ in range(3):
        for (plan, _, _, args), s in zip(held, streams):
            rt.residual_attention_decode_fp8(args, plan, s)
    torch.cuda.synchronize()
    for (_, out, _, _), w in zip(held, want):
        assert torch.equal(out, w)


def test_attention_refusals():
    p = Problem(30, [40, 50], 0, 32, 8, 16, True, rows=[4, 5])
    out = torch.zeros_like(p.q)
    plan = p.plan()
    ws = torch.empty(plan.info(D, 16)["workspace_bytes"] // 4, dtype=torch.float32, device="cuda")
    kw = dict(plan_dev=plan.device("cuda"), workspace=ws)
    pf = dict(q_indptr=p.indptr, n_q=9, max_q_per_agent=5)
    bad_pool = p.pool[:, :-128].contiguous()
    for pool in (p.wide, bad_pool, p.pool.view(torch.int8), p.pool[:, ::2]):
        with pytest.raises(rt.FKVError):
            rt.residual_attention_decode_fp8(p.args(out, pool=pool, **kw), plan)
        with pytest.raises(rt.FKVError):
            rt.residual_attention_prefill_fp8(p.args(out, pool=pool, **pf))
    with pytest.raises(rt.FKVError):
        rt.residual_attention_decode(p.args(out, **kw), plan)
    with pytest.raises(rt.FKVError):
        rt.residual_attention_decode_noalloc(p.args(out, **kw), plan)
    with pytest.raises(rt.FKVError):
        rt.residual_attention_prefill(p.args(out, **pf))
    for field, value in (("d", 64), ("page_size", 32), ("r", 24), ("hq", 8), ("scale", float("nan")), ("max_pages", 1), ("base_kv", p.pool.data_ptr() + 8),
                         ("rope_max_pos", 16), ("workspace_bytes", 16), ("plan", None), ("n_agents", 3), ("seq_lens", None)):
        a = p.args(out, **kw)
        setattr(a, field, value)
        with pytest.raises(rt.FKVError, match="fkv_residual_attention_decode_fp8"):
            rt.residual_attention_decode_fp8(a, plan)
    for field, value in (("d", 64), ("r", 24), ("hq", 8), ("n_q", 0), ("q_indptr", None), ("rope_max_pos", 16), ("max_q_per_agent", 10),
                         ("base_kv", p.pool.data_ptr() + 8), ("scale", 0.0)):
        a = p.args(out, **pf)
        setattr(a, field, value)
        with pytest.raises(rt.FKVError, match="fkv_residual_attention_prefill_fp8"):
            rt.residual_attention_prefill_fp8(a)
    torch.cuda.synchronize()
