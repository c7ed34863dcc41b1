"""Pins of the 8-bit cache oracle, and refusals of the 8-bit entry points that need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import fp8_cache as o
from paper_2604_06370_amd import _native as N
from paper_2604_06370_amd import runtime as rt


def test_code_values_are_those_of_the_type():
    bits = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mine = o.values(np.arange(256, dtype=np.uint8).reshape(2, 128), np.zeros(2, np.int64)).reshape(-1)
    assert np.array_equal(np.isnan(bits), np.isnan(mine)) and np.array_equal(bits[~np.isnan(bits)], mine[~np.isnan(mine)])


def test_every_value_is_a_fixed_point():
    # largest magnitude 448 * 2^E in the row: every code keeps itself, zeros keep their sign bit
    for e in (-117, -3, 0, 119):
        row = np.concatenate([o.CODE_VALUES, [448.0]]) * 2.0 ** e
        for x in (row, -row):
            c, ee = o.codes(x[None])
            assert ee[0] == e and np.array_equal(o.values(c, ee)[0], x)


@pytest.mark.parametrize("x,want", [(1.0625, 1.0), (1.1875, 1.25), (-1.0625, -1.0), (17.0, 16.0), (19.0, 20.0), (2.0 ** -10, 0.0),
                                    (3 * 2.0 ** -10, 2.0 ** -8), (1.06250001, 1.125), (2.0 ** -10 * 1.0001, 2.0 ** -9)])
def test_rounding_is_to_nearest_even(x, want):
    row = np.zeros(128)
    row[0], row[1] = 300.0, x
    assert o.exponent(row) == 0 and o.nearest(row[None])[0, 1] == want


@pytest.mark.parametrize("amax,e", [(448.0, 0), (np.nextafter(448.0, 500), 1), (224.0, -1), (224.5, 0), (1.75 * 2.0 ** 127, 119), (3.38e38, 119),
                                    (0.0, -117), (1e-40, -117), (1.75 * 2.0 ** -110, -118 + 0)])
def test_exponent_borders(amax, e):
    row = np.zeros(128)
    row[7] = -amax
    assert o.exponent(row) == max(e, -117)


def test_values_that_are_not_finite_leave_the_others_alone():
    row = np.linspace(-1, 1, 128)
    want = o.nearest(row[None])[0]
    bad = row.copy()
    bad[3], bad[9] = np.inf, np.nan
    got = o.nearest(bad[None])[0]
    assert np.isnan(got[[3, 9]]).all()
    rest = np.setdiff1d(np.arange(128), [3, 9])
    assert np.array_equal(got[rest], want[rest])


def test_layout_is_a_bijection():
    t, i = np.meshgrid(np.arange(16), np.arange(128), indexing="ij")
    for where in (o.k_byte, o.v_byte):
        assert np.array_equal(np.sort(where(t, i).reshape(-1)), np.arange(2048))
    for hkv in (1, 2, 3, 8):
        assert rt.fp8_page_bytes(16, hkv, 128) == o.page_bytes(hkv)


def test_page_bytes_refuses_other_shapes():
    for ps, hkv, d in ((8, 8, 128), (16, 0, 128), (16, 8, 64)):
        assert N.fkv_fp8_page_bytes(ps, hkv, d) == 0
        with pytest.raises(rt.FKVError):
            rt.fp8_page_bytes(ps, hkv, d)


def _seq(pos0=0, n=1, row0=0, bt=16, res=16, a=16):
    return N.fkv_produce_seq(bt, res, a, pos0, n, row0)


# (pointers here are never followed: every call has to be refused before a launch)
@pytest.mark.parametrize("what,kw", [
    ("d", dict(d=64)), ("page size", dict(ps=32)), ("rank", dict(r=24)), ("heads", dict(hkv=0)), ("pool", dict(base=None)),
    ("k", dict(k=None)), ("rope pair", dict(sin=None)), ("rope length", dict(max_pos=0)), ("alignment", dict(k=24)),
    ("pool alignment", dict(base=8)), ("hidden", dict(hidden=1000)), ("no x", dict(x=None)), ("no res", dict(res=None)),
    ("position", dict(seq=_seq(pos0=-1))), ("count", dict(seq=_seq(n=-1))), ("row", dict(seq=_seq(row0=-1))),
    ("table", dict(seq=_seq(bt=None))), ("adapter alignment", dict(seq=_seq(a=24))), ("long", dict(seq=_seq(n=1 << 25), max_pos=1 << 30)),
    ("nseq", dict(nseq=-1)), ("seqs", dict(seq=None)),
])
def test_produce_refusals(what, kw):
    a = dict(seq=_seq(), nseq=1, x=16, hidden=1024, k=16, v=16, cos=16, sin=16, max_pos=64, base=16, res=16, hkv=2, d=128, r=16, ps=16)
    a.update(kw)
    seq = ctypes.byref(a["seq"]) if a["seq"] is not None else None
    st = N.fkv_produce_tokens_fp8(seq, a["nseq"], a["x"], a["hidden"], a["k"], a["v"], a["cos"], a["sin"], a["max_pos"], a["base"],
                                  a["res"], a["hkv"], a["d"], a["r"], a["ps"], None)
    assert st == N.FKV_ERR_INVALID and "fkv_produce_tokens_fp8" in N.fkv_last_error().decode()


@pytest.mark.parametrize("what,kw", [
    ("d", dict(d=64)), ("page size", dict(ps=32)), ("heads", dict(hkv=0)), ("pool", dict(base=None)), ("k", dict(k=None)),
    ("alignment", dict(v=24)), ("position", dict(seq=N.fkv_read_seq(16, -1, 1, 0))), ("count", dict(seq=N.fkv_read_seq(16, 0, -1, 0))),
    ("row", dict(seq=N.fkv_read_seq(16, 0, 1, -1))), ("table", dict(seq=N.fkv_read_seq(None, 0, 1, 0))),
    ("long", dict(seq=N.fkv_read_seq(16, 0, 1 << 25, 0))), ("nseq", dict(nseq=-1)), ("seqs", dict(seq=None)),
])
def test_gather_refusals(what, kw):
    a = dict(seq=N.fkv_read_seq(16, 0, 1, 0), nseq=1, base=16, k=16, v=16, hkv=2, d=128, ps=16)
    a.update(kw)
    seq = ctypes.byref(a["seq"]) if a["seq"] is not None else None
    st = N.fkv_gather_tokens_fp8(seq, a["nseq"], a["base"], a["k"], a["v"], a["hkv"], a["d"], a["ps"], None)
    assert st == N.FKV_ERR_INVALID and "fkv_gather_tokens_fp8" in N.fkv_last_error().decode()


@pytest.mark.parametrize("what,copies,kw", [
    ("d", [(0, 0, 1, 4)], dict(d=64)), ("page size", [(0, 0, 1, 4)], dict(ps=8)), ("pool", [(0, 0, 1, 4)], dict(base=None)),
    ("alignment", [(0, 0, 1, 4)], dict(base=24)), ("source", [(0, 0, 1, 4), (0, -1, 1, 4)], {}), ("which pool", [(2, 0, 1, 4)], {}),
    ("residual pool", [(1, 0, 1, 4)], dict(res=None)), ("n", [(0, 0, 1, 4)], dict(n=-1)),
])
def test_page_copy_refusals(what, copies, kw):
    a = dict(base=16, res=16, hkv=2, d=128, r=16, ps=16, n=len(copies))
    a.update(kw)
    arr = np.array(copies, dtype=np.int32)
    st = N.fkv_page_copy_list_fp8(arr.ctypes.data, a["n"], a["base"], a["res"], a["hkv"], a["d"], a["r"], a["ps"], None)
    assert st == N.FKV_ERR_INVALID and "fkv_page_copy_list_fp8" in N.fkv_last_error().decode()


def test_empty_calls_do_nothing():
    assert N.fkv_page_copy_list_fp8(None, 0, None, None, 2, 128, 16, 16, None) == N.FKV_OK
    assert N.fkv_produce_tokens_fp8(None, 0, None, 0, 16, 16, None, None, 0, 16, None, 2, 128, 0, 16, None) == N.FKV_OK
    seq = N.fkv_read_seq(None, 5, 0, 3)
    assert N.fkv_gather_tokens_fp8(ctypes.byref(seq), 1, 16, 16, 16, 2, 128, 16, None) == N.FKV_OK


def test_host_tensors_are_refused(monkeypatch):
    # the binding looks at every tensor before it takes an address: host memory never reaches a kernel
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    pool = torch.zeros(2, rt.fp8_page_bytes(16, 2, 128), dtype=torch.uint8)
    k = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    bt = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(rt.FKVError, match="current GPU"):
        rt.produce_tokens_fp8([(bt, None, None, 0, 4, 0)], None, k, k, None, pool, None, 2, 128, 0, 16)
    with pytest.raises(rt.FKVError, match="current GPU"):
        rt.gather_tokens_fp8([(bt, 0, 4, 0)], pool, k, k, 2, 128, 16)
    with pytest.raises(rt.FKVError, match="current GPU"):
        rt.page_copy_fp8([(0, 0, 1, 4)], pool, None, 2, 128, 0, 16)


def _attn(**kw):
    a = N.fkv_attn_args()
    for name in ("q", "base_kv", "res_kv", "lora_b", "adapter_idx", "base_bt", "res_bt", "seq_lens", "out", "q_indptr", "plan", "workspace"):
        setattr(a, name, 4096)
    a.n_agents, a.hq, a.hkv, a.d, a.r, a.page_size, a.max_pages, a.n_q, a.scale, a.workspace_bytes = 2, 8, 2, 128, 16, 16, 4, 5, 0.1, 1 << 20
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw", [dict(base_kv=4104), dict(base_kv=None), dict(d=64), dict(page_size=32), dict(r=24), dict(hq=6), dict(hq=2), dict(q=None),
                                dict(seq_lens=None), dict(scale=-1.0), dict(n_agents=0), dict(rope_cos=4096), dict(lora_b=None)])
def test_attention_refusals_without_a_gpu(kw):
    bt = np.zeros((2, 4), np.int32)
    plan = rt.DecodePlan(bt, np.array([20, 30], np.int32), 8, 2, 16, r=16)
    for name in ("prefill", "decode"):
        call = getattr(N, f"fkv_residual_attention_{name}_fp8")
        st = call(ctypes.byref(_attn(**kw)), *((plan.handle,) if name == "decode" else ()), None)
        assert st in (N.FKV_ERR_INVALID, N.FKV_ERR_UNSUPPORTED)
        assert f"fkv_residual_attention_{name}_fp8" in N.fkv_last_error().decode()


def test_prefill_workspace():
    # the smaller the grid the more workgroups share a row's keys; none where the grid fills the GPU or contexts are short
    need = lambda *a: rt.prefill_fp8_workspace_bytes(*a)  # noqa: E731
    assert need(32, 8, 16, 1, 1, 4096) == 32 * 16 * 32 * (128 + 4) * 4  # splits, tokens of a workgroup, heads, floats of a record
    assert need(32, 8, 16, 1, 1, 31) == 0 and need(32, 8, 16, 64, 4096, 4096) == 0
    assert need(32, 8, 16, 1, 1, 64) == need(32, 8, 16, 1, 1, 4096) * 4 // 32
    for bad in ((32, 8, 24, 1, 1, 64), (32, 5, 16, 1, 1, 64), (8, 8, 16, 1, 1, 64), (32, 8, 16, 0, 1, 64), (32, 8, 16, 1, 0, 64), (32, 8, 16, 1, 1, 0),
                (0, 0, 0, 0, 0, 0), (-32, -8, 16, 1, 1, 64), (32, 8, 16, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert need(*bad) == 0
    assert N.fkv_residual_attention_prefill_fp8(ctypes.byref(_attn(workspace=4104)), None) == N.FKV_ERR_INVALID
    assert "workspace" in N.fkv_last_error().decode()


def test_null_arguments_are_refused():
    assert N.fkv_residual_attention_prefill_fp8(None, None) == N.FKV_ERR_INVALID
    assert N.fkv_residual_attention_decode_fp8(None, None, None) == N.FKV_ERR_INVALID
    assert N.fkv_residual_attention_decode_fp8(ctypes.byref(_attn()), None, None) == N.FKV_ERR_INVALID


def test_pool_formats_are_kept_apart():
    # the binding refuses a pool of the other format before it calls the library
    args = _attn()
    args.base_pool = (torch.bfloat16, (4, 2, 2, 2048), True)
    for call in (rt.residual_attention_prefill_fp8, lambda a: rt.residual_attention_decode_fp8(a, None)):
        with pytest.raises(rt.FKVError, match="uint8"):
            call(args)
    args.base_pool = (torch.uint8, (4, rt.fp8_page_bytes(16, 2, 128)), True)
    for call in (rt.residual_attention_prefill, lambda a: rt.residual_attention_decode(a, None), lambda a: rt.residual_attention_decode_noalloc(a, None)):
        with pytest.raises(rt.FKVError, match="8-bit"):
            call(args)
    args.base_pool = (torch.uint8, (4, 128), True)
    with pytest.raises(rt.FKVError, match="fp8_page_bytes"):
        rt.residual_attention_prefill_fp8(args)
