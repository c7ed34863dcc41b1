"""Operators of the 8-bit base cache, as they are measured: the cache write that quantises, the read
back, and ResidualAttention (decode and chunked prefill) over the quantised pages.

A row of the cache is the 128 values of K or of V of one token and KV head.  It is held as 128 e4m3
codes and one exponent byte b, and stands for code * 2^(b - 127).  With amax the largest magnitude
among the row's finite values, E = b - 127 is the smallest integer in [-117, 119] with
amax <= 448 * 2^E; a code is x * 2^-E, clamped to +-448, rounded to nearest even; values that are not
finite become NaN.  A page of 16 tokens is [Hkv][2][2048] codes (K, then V), then [Hkv][2][16]
exponent bytes, then zeros up to a multiple of 128 bytes.

A case names an operation and the sizes of its inputs:

  op       write    every sequence's new tokens into the pages (K with RoPE, V, the LoRA shrink of
                    the hidden state), and those tokens read back
           read     ranges of cached tokens read back as bf16 rows
           decode   one query row per agent over its whole context
           prefill  every agent's chunk of new tokens attends causally to its context
  hq, hkv, r, rope          heads, LoRA rank, RoPE (write: of K; attention: of the rebuilt key)
  agents, trees, root       agents, dealt round-robin over trees whose tokens they share (root, 2 root, ...)
  suffix_lo, suffix_hi      private tokens of an agent before its chunk (read: tokens to read)
  chunk_lo, chunk_hi        new tokens of an agent (read: position of the first one)
  bare                      > 0: every bare-th agent has no adapter
  b_std, hidden             scale of the up-projections, width of the hidden state

Head dim 128 and pages of 16 tokens throughout.
"""
import math
import random

import numpy as np
import torch

own = False

D, PS, THETA = 128, 16, 500000.0
DEVICE = "cuda"
TINY, H8B, H70B, SHARE = (8, 2), (32, 8), (64, 8), (4, 1)


def _case(name, op, heads, r, rope, agents, **more):
    c = {"op": op, "hq": heads[0], "hkv": heads[1], "r": r, "rope": rope, "agents": agents, "trees": 1, "root": 0,
         "suffix_lo": 0, "suffix_hi": 0, "chunk_lo": 0, "chunk_hi": 0, "bare": 0, "b_std": 0.02, "hidden": 4096, **more}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the cache write of one decode step of 16 sequences: latency
        _case("write-8b-16x1", "write", H8B, 16, True, 16, suffix_lo=100, suffix_hi=4000, chunk_lo=1, chunk_hi=1),
        # full prompt chunks of 16 agents
        _case("write-8b-16x2048", "write", H8B, 16, True, 16, suffix_lo=1000, suffix_hi=1500, chunk_lo=2048, chunk_hi=2048),
        # K and V rows computed elsewhere, from odd positions, odd lengths, 70B heads
        _case("write-rows-8x700", "write", H70B, 0, False, 8, suffix_lo=1, suffix_hi=300, chunk_lo=301, chunk_hi=700),
        # a few tool results handed to another engine
        _case("read-tiny-3x77", "read", TINY, 0, False, 3, suffix_lo=5, suffix_hi=77, chunk_lo=1, chunk_hi=40),
        # long contexts handed on whole
        _case("read-8b-4x32k", "read", H8B, 0, False, 4, suffix_lo=32000, suffix_hi=32768, chunk_lo=0, chunk_hi=15),
        # a small model with a short system prompt: latency and launches
        _case("decode-tiny-rope", "decode", TINY, 8, True, 4, root=512, suffix_lo=64, suffix_hi=64),
        # 16 agents of one 8B-shaped model over a 32K document
        _case("decode-8b-16x32k", "decode", H8B, 16, False, 16, root=32768, suffix_lo=256, suffix_hi=4096),
        # the same with deferred RoPE
        _case("decode-8b-16x32k-rope", "decode", H8B, 16, True, 16, root=32768, suffix_lo=256, suffix_hi=4096),
        # 70B heads, rank 64, three documents, some agents on the base model
        _case("decode-70b-rope", "decode", H70B, 64, True, 12, trees=3, root=4096, suffix_lo=64, suffix_hi=4096, bare=5, b_std=0.05),
        # the prefill part of a decode-heavy step: few agents, short ragged chunks over a long context
        _case("prefill-8b-4x250", "prefill", H8B, 16, False, 4, root=32768, suffix_lo=256, suffix_hi=4096, chunk_lo=129, chunk_hi=250),
        # chunked prefill at larger chunks
        _case("prefill-8b-8x1024-rope", "prefill", H8B, 16, True, 8, root=8192, suffix_lo=100, suffix_hi=1000, chunk_lo=700, chunk_hi=1024),
        # 70B heads at rank 64, some agents on the base model
        _case("prefill-70b-6x500-rope", "prefill", H70B, 64, True, 6, trees=2, root=4000, suffix_lo=64, suffix_hi=1000, chunk_lo=200, chunk_hi=500, bare=4, b_std=0.05),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


# Caps of a drawn case, those of the largest listed ones: (agent, KV head, key) triples of decode,
# (query row, head, key) triples of prefill, bytes of hidden state and of K and V of write and read.
_DECODE_MOST, _PREFILL_MOST, _ROWS_MOST = 4_600_000, 2_400_000_000, 32768


def draw(rng):
    op = rng.choice(["write", "read", "decode", "decode", "decode", "prefill", "prefill"])
    heads, r, rope = rng.choice([H8B, H8B, H70B, TINY, SHARE]), rng.choice([0, 8, 16, 16, 32, 64]), rng.random() < 0.7
    hq, hkv = heads
    more = {"b_std": rng.choice([0.02, 0.05]), "bare": rng.choice([0, 0, 0, 2, 5])}
    if op == "write":
        agents, chunk = _log(rng, 1, 48), _log(rng, 1, 2048)
        agents = max(1, min(agents, _ROWS_MOST // chunk))
        lo = rng.randint(0, 40)
        return _case(None, op, heads, r, rope, agents, chunk_lo=max(1, chunk // rng.choice([1, 2, 4])), chunk_hi=chunk,
                     suffix_lo=lo, suffix_hi=lo + _log(rng, 1, 2000), hidden=rng.choice([1024, 4096, 8192 if agents * chunk <= 16384 else 4096]), **more)
    if op == "read":
        agents, n = _log(rng, 1, 40), _log(rng, 1, 32768)
        agents = max(1, min(agents, 4 * _ROWS_MOST // n))
        return _case(None, op, heads, 0, False, agents, suffix_lo=max(1, n // rng.choice([1, 2, 4])), suffix_hi=n, chunk_lo=0,
                     chunk_hi=rng.randint(0, 100))
    lo = _log(rng, 1, 1500)
    more.update(suffix_lo=lo, suffix_hi=_log(rng, lo, 4 * lo), trees=rng.choice([1, 1, 1, 2, 3]))
    most = lambda root: (root << (more["trees"] - 1)) + more["suffix_hi"]  # noqa: E731
    if op == "decode":
        agents, root = _log(rng, 1, 64), _log(rng, 16, 131072)
        while root > 16 and agents * hkv * most(root) > _DECODE_MOST:
            root = root * 2 // 3
        return _case(None, op, heads, r, rope, agents, root=root, **more)
    agents, chunk, root = _log(rng, 1, 16), _log(rng, 1, 2048), _log(rng, 16, 32768)
    while root > 16 and agents * hq * chunk * (most(root) + chunk) > _PREFILL_MOST:
        root = root * 2 // 3
    while agents > 1 and agents * hq * chunk * (most(root) + chunk) > _PREFILL_MOST:
        agents -= 1
    return _case(None, op, heads, r, rope, agents, root=root, chunk_lo=max(1, chunk // rng.choice([1, 2, 4])), chunk_hi=chunk, **more)


# ---- sizes that follow from a case alone ---------------------------------------------------------


def _sizes(c):
    rng, n = random.Random(29), c["agents"]
    suffix = [rng.randint(c["suffix_lo"], c["suffix_hi"]) for _ in range(n)]
    chunk = [rng.randint(c["chunk_lo"], c["chunk_hi"]) for _ in range(n)]
    adapter = [-1 if c["bare"] and a % c["bare"] == c["bare"] - 1 or not c["r"] else a for a in range(n)]
    if c["op"] in ("write", "read"):
        pos0, new = (suffix, chunk) if c["op"] == "write" else (chunk, suffix)
        return pos0, new, [p + m for p, m in zip(pos0, new)], adapter
    trees = [c["root"] << (a % c["trees"]) for a in range(n)]
    pos0 = [t + s for t, s in zip(trees, suffix)]
    new = chunk if c["op"] == "prefill" else [1] * n
    return pos0, new, [max(1, p + (m if c["op"] == "prefill" else 0)) for p, m in zip(pos0, new)], adapter


def _page_bytes(hkv):
    return hkv * 4096 + -(-hkv * 32 // 128) * 128


def _rank_tiles(r):
    return -(-r // 16)


# ---- the format, in elementary operations --------------------------------------------------------


def _power(e):
    """2^e in 64 bits, e an integer tensor."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x):
    """Rows [..., 128] in 64 bits: their codes (as e4m3 values) and exponents E."""
    fine = torch.isfinite(x)
    amax = torch.where(fine, x.abs(), 0.0).amax(dim=-1)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-117, 119)
    q = (x * _power(-e)[..., None]).clamp(-448.0, 448.0)
    step = _power((torch.frexp(q)[1] - 1).clamp(min=-6) - 3)
    q = torch.where(fine, torch.round(q / step) * step, math.nan)
    return q.float().to(torch.float8_e4m3fn), e


def _to_pages(k, v):
    """K and V of whole pages [pages][16][hkv][128] as the cache's bytes."""
    n, hkv = k.shape[0], k.shape[2]
    pool = torch.zeros(n, _page_bytes(hkv), dtype=torch.uint8, device=k.device)
    codes, exps = pool[:, : hkv * 4096].view(n, hkv, 2, 2048), pool[:, hkv * 4096: hkv * 4128].view(n, hkv, 2, 16)
    (qk, ek), (qv, ev) = _quantise(k.double()), _quantise(v.double())
    # K: dim 64 a + 32 b + 16 c + 4 g + e of token t at [a][g][t][b][c][e]; V: dim 64 a + 32 b + 16 c + i of token 4 u + e at [a][u][i][b][c][e]
    qk = qk.view(torch.uint8).view(n, 16, hkv, 2, 2, 2, 4, 4).permute(0, 2, 3, 6, 1, 4, 5, 7)
    qv = qv.view(torch.uint8).view(n, 4, 4, hkv, 2, 2, 2, 16).permute(0, 3, 4, 1, 7, 5, 6, 2)
    codes[:, :, 0], codes[:, :, 1] = qk.reshape(n, hkv, 2048), qv.reshape(n, hkv, 2048)
    exps[:, :, 0], exps[:, :, 1] = (ek + 127).to(torch.uint8).transpose(1, 2), (ev + 127).to(torch.uint8).transpose(1, 2)
    return pool


def _from_pages(pool, hkv):
    """K and V in 32 bits, [pages][16][hkv][128]."""
    n = pool.shape[0]
    codes = pool[:, : hkv * 4096].reshape(n, hkv, 2, 2048).view(torch.float8_e4m3fn).float()
    exps = (pool[:, hkv * 4096: hkv * 4128].reshape(n, hkv, 2, 16).int() << 23).view(torch.float32)
    k = codes[:, :, 0].reshape(n, hkv, 2, 4, 16, 2, 2, 4).permute(0, 4, 1, 2, 5, 6, 3, 7).reshape(n, 16, hkv, D)
    v = codes[:, :, 1].reshape(n, hkv, 2, 4, 16, 2, 2, 4).permute(0, 3, 7, 1, 2, 5, 6, 4).reshape(n, 16, hkv, D)
    return k * exps[:, :, 0].transpose(1, 2)[..., None], v * exps[:, :, 1].transpose(1, 2)[..., None]


def _rotate(x, cos, sin):
    a, b = x[..., : D // 2], x[..., D // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


# ---- what a program has in hand ------------------------------------------------------------------


def _rope_tables(positions):
    """cos and sin of position p and pair i at [p / 16][i / 16][p % 16 + 16 ((i % 16) / 4)][i % 4], as the library keeps them."""
    p = -(-positions // PS) * PS
    f = THETA ** (-torch.arange(D // 2, device=DEVICE, dtype=torch.float64) * 2 / D)
    ang = torch.arange(p, device=DEVICE, dtype=torch.float64)[:, None] * f
    lay = lambda t: t.float().view(p // PS, PS, 4, 4, 4).permute(0, 2, 3, 1, 4).reshape(p, D // 2).contiguous()  # noqa: E731
    return lay(ang.cos()), lay(ang.sin())


def _rope_rows(table):
    """A table in the order [position][pair]."""
    p = table.shape[0]
    return table.view(p // PS, 4, 4, PS, 4).permute(0, 3, 1, 2, 4).reshape(p, D // 2)


def _layout(c, g):
    """Block tables over randomly placed pages: base [agents][pages], residual likewise, pages of each pool."""
    pos0, new, total, _ = _sizes(c)
    n, width = c["agents"], -(-max(total) // PS) + 1
    base, res, nb, nr, first = np.zeros((n, width), np.int32), np.zeros((n, width), np.int32), 0, 0, {}
    for a, t in enumerate(total):
        p0, p1 = (pos0[a] // PS if c["op"] in ("write", "read") else 0), -(-t // PS)
        tree = a % c["trees"]
        shared = (c["root"] << tree) // PS if c["op"] in ("decode", "prefill") else 0
        if tree in first:
            base[a, :shared] = base[first[tree], :shared]
            p0 = max(p0, shared)
        else:
            first[tree] = a
        base[a, p0:p1] = np.arange(nb, nb + p1 - p0)
        nb += p1 - p0
        r0 = pos0[a] // PS if c["op"] == "write" else 0
        res[a, r0:p1] = np.arange(nr, nr + p1 - r0)
        nr += p1 - r0
    where = [torch.randperm(m, generator=g, device=DEVICE).int().cpu().numpy() for m in (nb, nr)]
    return where[0][base], where[1][res], nb, nr


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEVICE).manual_seed(seed)
    n, hq, hkv, r = c["agents"], c["hq"], c["hkv"], c["r"]
    pos0, new, total, adapter = _sizes(c)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.bfloat16).mul_(std)

    base, res, nb, nr = _layout(c, g)
    # keys have a few strong channels, the same for every token of a head
    channel = torch.where(torch.rand(hkv, D, generator=g, device=DEVICE) < 0.03, 6.0, 1.0).bfloat16()
    row0 = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    st = {"case": c, "base": torch.from_numpy(base).to(DEVICE), "row0": row0}
    if c["op"] == "write":
        rows = int(row0[-1])
        st.update(k=normal(rows, hkv, D) * channel, v=normal(rows, hkv, D), pool=torch.zeros(nb, _page_bytes(hkv), dtype=torch.uint8, device=DEVICE))
        if r:
            st.update(x=normal(rows, c["hidden"]), a=normal(n, 2, r, c["hidden"], std=c["hidden"] ** -0.5), res=torch.from_numpy(res).to(DEVICE),
                      res_kv=torch.zeros(nr, _rank_tiles(r) * 512, dtype=torch.bfloat16, device=DEVICE))
    else:
        st["pool"] = torch.cat([_to_pages(normal(m, PS, hkv, D) * channel, normal(m, PS, hkv, D)) for m in [min(2048, nb - i) for i in range(0, nb, 2048)]])
    if c["op"] in ("write", "read"):
        st["out"] = (torch.empty(int(row0[-1]), hkv, D, dtype=torch.bfloat16, device=DEVICE), torch.empty(int(row0[-1]), hkv, D, dtype=torch.bfloat16, device=DEVICE))
    st["rope"] = _rope_tables(base.shape[1] * PS) if c["rope"] else None
    if c["op"] in ("decode", "prefill"):
        st.update(q=normal(int(row0[-1]), hq, D), seq_lens=torch.tensor(total, dtype=torch.int32, device=DEVICE),
                  indptr=torch.from_numpy(row0).to(DEVICE), adapter=torch.tensor(adapter, dtype=torch.int32, device=DEVICE))
        if r:
            st.update(res=torch.from_numpy(res).to(DEVICE), res_kv=normal(nr, _rank_tiles(r) * 512), lora_b=normal(n, 2, r, hkv * D, std=c["b_std"]))
    if own and c["op"] in ("decode", "prefill"):  # the plan, workspace and argument block that a program keeps between steps
        from paper_2604_06370_amd import runtime as rt

        st["result"] = torch.empty_like(st["q"])
        common = dict(q=st["q"], base_kv=st["pool"], res_kv=st.get("res_kv"), lora_b=st.get("lora_b"), adapter_idx=st["adapter"] if r else None,
                      base_bt=st["base"], res_bt=st.get("res"), seq_lens=st["seq_lens"], out=st["result"], hq=hq, hkv=hkv, d=D, r=r, page_size=PS,
                      rope=st["rope"] if r else None)
        if c["op"] == "prefill":
            st["args"] = rt.make_args(**common, q_indptr=st["indptr"], n_q=int(row0[-1]), max_q_per_agent=max(new))
        else:
            st["plan"] = rt.DecodePlan(base, np.array(total, np.int32), hq, hkv, PS, r=r, rope=c["rope"] and r > 0)
            st["work"] = torch.empty(max(4, st["plan"].info(D, r)["workspace_bytes"]) // 4, dtype=torch.float32, device=DEVICE)
            st["args"] = rt.make_args(**common, plan_dev=st["plan"].device(DEVICE), workspace=st["work"])
    return st


# ---- one pass ------------------------------------------------------------------------------------


def run(state):
    c = state["case"]
    if own:
        return _run_own(state)
    return {"write": _plain_write, "read": _plain_read, "decode": _plain_attention, "prefill": _plain_attention}[c["op"]](state)


def _run_own(state):
    from paper_2604_06370_amd import runtime as rt

    c = state["case"]
    hkv, r, op = c["hkv"], c["r"], c["op"]
    if op == "decode":
        rt.residual_attention_decode_fp8(state["args"], state["plan"])
        return state["result"]
    if op == "prefill":
        rt.residual_attention_prefill_fp8(state["args"])
        return state["result"]
    pos0, new, _, adapter = _sizes(c)
    row0, base, (k, v) = state["row0"], state["base"], state["out"]
    if op == "write":
        seqs = [(base[a], state["res"][a] if r else None, state["a"][a] if adapter[a] >= 0 else None, pos0[a], new[a], int(row0[a])) for a in range(c["agents"])]
        rt.produce_tokens_fp8(seqs, state.get("x"), state["k"], state["v"], state["rope"], state["pool"], state.get("res_kv"), hkv, D, r, PS)
    rt.gather_tokens_fp8([(base[a], pos0[a], new[a], int(row0[a])) for a in range(c["agents"])], state["pool"], k, v, hkv, D, PS)
    return {"k": k, "v": v, "res": state["res_kv"]} if op == "write" and r else {"k": k, "v": v}


def _positions(c):
    """Agent and position of every new row."""
    pos0, new, _, _ = _sizes(c)
    agent = np.repeat(np.arange(c["agents"]), new)
    pos = np.arange(agent.size) - np.repeat(np.concatenate([[0], np.cumsum(new)[:-1]]), new) + np.repeat(pos0, new)
    return torch.from_numpy(agent).to(DEVICE), torch.from_numpy(pos).to(DEVICE)


def _plain_write(st):
    c, r = st["case"], st["case"]["r"]
    agent, pos = _positions(c)
    k, v = st["k"].double(), st["v"].double()  # a code next to a border needs the angles' products whole
    if c["rope"]:
        k = _rotate(k, _rope_rows(st["rope"][0])[pos].double()[:, None], _rope_rows(st["rope"][1])[pos].double()[:, None])
    (qk, ek), (qv, ev) = _quantise(k), _quantise(v)
    out = {"k": (qk.double() * _power(ek)[..., None]).bfloat16(), "v": (qv.double() * _power(ev)[..., None]).bfloat16()}
    if not r:
        return out
    # C = x A^T of each row's own adapter: rows of one sequence are padded to one length
    _, new, _, adapter = _sizes(c)
    n, m = c["agents"], max(new)
    x = torch.zeros(n, m, c["hidden"], device=DEVICE)
    at = torch.arange(agent.numel(), device=DEVICE) - torch.from_numpy(st["row0"]).to(DEVICE)[agent]
    x[agent, at] = st["x"].float()
    has = torch.tensor([a >= 0 for a in adapter], device=DEVICE)[agent]
    co = torch.matmul(x[:, None], st["a"].float().transpose(2, 3))[agent, :, at].bfloat16()  # [rows][2][r]
    res = torch.zeros_like(st["res_kv"])
    page, t, rho = st["res"][agent, pos // PS].long(), pos % PS, torch.arange(r, device=DEVICE)
    tile, i = (rho // 16 * 512)[None], rho % 16
    res[page[has, None], (tile + (16 * (i // 4) + t[:, None]) * 8 + i % 4)[has]] = co[has, 0]
    res[page[has, None], (tile + (16 * (t[:, None] // 4) + i) * 8 + 4 + t[:, None] % 4)[has]] = co[has, 1]
    return {**out, "res": res}


def _plain_read(st):
    agent, pos = _positions(st["case"])
    k, v = _from_pages(st["pool"], st["case"]["hkv"])
    page, t = st["base"][agent, pos // PS].long(), pos % PS
    return {"k": k[page, t].bfloat16(), "v": v[page, t].bfloat16()}


def _plain_attention(st):
    c = st["case"]
    n, hq, hkv, r, prefill = c["agents"], c["hq"], c["hkv"], c["r"], c["op"] == "prefill"
    _, new, total, _ = _sizes(c)
    pages, m, g = -(-max(total) // PS), max(new), hq // hkv
    keys = pages * PS
    k, v = (x[st["base"][:, :pages].long()].view(n, keys, hkv, D) for x in _from_pages(st["pool"], hkv))
    if r:
        tiles = st["res_kv"][st["res"][:, :pages].long()].view(n, pages, -1, 4, 16, 2, 4).float()  # [tile][lane group][lane][K|V][4]
        ck = tiles[..., 0, :].permute(0, 1, 4, 2, 3, 5).reshape(n, 1, keys, -1)[..., :r]
        cv = tiles[..., 1, :].permute(0, 1, 3, 5, 2, 4).reshape(n, 1, keys, -1)[..., :r]
        has = (st["adapter"] >= 0).float()[:, None, None, None]
        b = st["lora_b"].float().view(n, 2, r, hkv, D).transpose(2, 3) * has[..., None]
        past = (torch.arange(keys, device=DEVICE) < st["seq_lens"][:, None])[:, None, :, None]
        u = torch.matmul(torch.where(past, ck, 0.0), b[:, 0])
        if c["rope"]:
            u = _rotate(u, _rope_rows(st["rope"][0])[:keys], _rope_rows(st["rope"][1])[:keys])
        k = k.transpose(1, 2) + u
        v = v.transpose(1, 2) + torch.matmul(torch.where(past, cv, 0.0), b[:, 1])
    else:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    agent = torch.repeat_interleave(torch.arange(n, device=DEVICE), torch.tensor(new, device=DEVICE))
    at = torch.arange(agent.numel(), device=DEVICE) - st["indptr"].long()[agent]
    q = torch.zeros(n, m, hkv, g, D, device=DEVICE)
    q[agent, at] = st["q"].float().view(-1, hkv, g, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(n, hkv, m * g, D)
    s = torch.matmul(q, k.transpose(2, 3)).mul_(D ** -0.5).view(n, hkv, m, g, keys)
    lens, row = st["seq_lens"].long(), torch.arange(m, device=DEVICE)
    count = (st["indptr"][1:] - st["indptr"][:-1]).long()
    last = (lens - count)[:, None] + row if prefill else (lens - 1)[:, None]  # the last key that a row sees
    s.masked_fill_((torch.arange(keys, device=DEVICE) > last[..., None])[:, None, :, None], -math.inf)
    s = torch.exp(s.sub_(s.amax(dim=-1, keepdim=True)))
    o = torch.matmul(s.view(n, hkv, m * g, keys), v).view(n, hkv, m, g, D) / s.sum(dim=-1, keepdim=True)
    return o.permute(0, 2, 1, 3, 4)[agent, at].reshape(-1, hq, D).bfloat16()


# ---- the least a pass moves and computes ---------------------------------------------------------


def work(case):
    c = case
    n, hq, hkv, r = c["agents"], c["hq"], c["hkv"], c["r"]
    pos0, new, total, adapter = _sizes(c)
    rows, code, wide = sum(new), hkv * 258, hkv * D * 2 * 2  # a token's bytes in the cache and in bf16
    if c["op"] == "read":
        return {"bytes": rows * (code + wide), "flops": rows * hkv * D * 2}
    if c["op"] == "write":
        with_a = sum(m for m, a in zip(new, adapter) if a >= 0)
        tables = len({p for a in range(n) for p in range(pos0[a], total[a])}) * D * 4 if c["rope"] else 0
        return {"bytes": rows * (2 * wide + 2 * code) + with_a * (c["hidden"] * 2 + r * 4) + sum(a >= 0 for a in adapter) * 2 * r * c["hidden"] * 2 + tables,
                "flops": with_a * 4 * r * c["hidden"] + rows * hkv * D * 8}
    shared = sum(c["root"] << t for t in range(min(c["trees"], n)))
    own_tokens = sum(t - (c["root"] << (a % c["trees"])) for a, t in enumerate(total))
    res = [t if a >= 0 else 0 for t, a in zip(total, adapter)]
    nbytes = (shared + own_tokens) * code + sum(res) * r * 4 + sum(a >= 0 for a in adapter) * 2 * r * hkv * D * 2 + rows * hq * D * 4
    rope, flops = c["rope"] and r > 0, 0
    nbytes += max(total) * D * 4 if rope else 0
    for t, m, k in zip(total, new, res):
        seen = m * t - m * (m - 1) // 2
        flops += hq * seen * 4 * D
        if k:
            flops += hq * seen * 2 * r + m * hq * 2 * r * D
            flops += k * hkv * 2 * r * D if rope else hq * (seen * 2 * r + m * 2 * r * D)
    return {"bytes": nbytes, "flops": flops}


# ---- the same in 64 bits, from the definitions ---------------------------------------------------


def _e4m3_values():
    """The 127 values of codes 0 .. 126: 3 fraction bits, exponent bias 7, subnormals below 2^-6."""
    return torch.tensor([(c % 8) / 8 * 2.0 ** -6 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7) for c in range(127)], dtype=torch.float64, device=DEVICE)


def _nearest(x):
    """What the cache stands for after writing rows x [..., 128] (64 bits): a search among the values that a code can take."""
    scales = torch.tensor([2.0 ** e for e in range(-117, 120)], dtype=torch.float64, device=DEVICE)
    fine = torch.isfinite(x)
    scale = scales[torch.bucketize(torch.where(fine, x, 0.0).abs().amax(dim=-1, keepdim=True), 448.0 * scales[:-1])]
    val = _e4m3_values()
    mid = (val[1:] + val[:-1]) / 2
    z = x.abs() / scale
    code = torch.bucketize(z, mid)
    tie = z == mid[code.clamp(max=125)]
    code = torch.where(tie & (code % 2 == 1) & (code < 126), code + 1, code)
    return torch.where(fine, torch.copysign(val[code] * scale, x), math.nan)


def _cached(st, hkv, a, positions):
    """K and V [positions][hkv][128] of agent a in 64 bits, each value looked up by its byte's place."""
    page, t = st["base"][a, positions // PS].long()[:, None, None], (positions % PS)[:, None, None]
    h, i = torch.arange(hkv, device=DEVICE)[None, :, None], torch.arange(D, device=DEVICE)[None, None]
    key = (i // 64) * 1024 + (t + 16 * (i % 16 // 4)) * 16 + (i // 32 % 2) * 8 + 4 * (i % 32 // 16) + i % 4
    val = (i // 64) * 1024 + (i % 16 + 16 * (t // 4)) * 16 + (i // 32 % 2) * 8 + 4 * (i // 16 % 2) + t % 4
    half = torch.cat([_e4m3_values(), torch.full((1,), math.nan, dtype=torch.float64, device=DEVICE)])
    table = torch.cat([half, -half])
    scales = torch.tensor([2.0 ** (b - 127) for b in range(256)], dtype=torch.float64, device=DEVICE)
    found = []
    for j, where in enumerate((key, val)):
        scale = scales[st["pool"][page, hkv * 4096 + h * 32 + j * 16 + t].long()]
        found.append(table[st["pool"][page, h * 4096 + j * 2048 + where].long()] * scale)
    return found


def _turn(x, positions, table):
    """RoPE of rows [positions][..., 128] with a table of the library's order."""
    p, i = positions[:, None], torch.arange(D // 2, device=DEVICE)[None]
    at = (p // 16) * 1024 + (i // 16) * 256 + (p % 16 + 16 * (i % 16 // 4)) * 4 + i % 4
    co, si = (t.reshape(-1)[at].double() for t in table)
    co, si = (t.view(t.shape[0], *[1] * (x.dim() - 2), D // 2) for t in (co, si))
    return torch.cat([x[..., :64] * co - x[..., 64:] * si, x[..., 64:] * co + x[..., :64] * si], dim=-1)


def exact(case, seed):
    c = case
    st = prepare({k: v for k, v in c.items() if k != "name"}, seed)
    n, hq, hkv, r = c["agents"], c["hq"], c["hkv"], c["r"]
    g = hq // hkv
    pos0, new, total, adapter = _sizes(c)
    if c["op"] == "read":
        both = [_cached(st, hkv, a, torch.arange(pos0[a], total[a], device=DEVICE)) for a in range(n)]
        return {"k": torch.cat([x[0] for x in both]), "v": torch.cat([x[1] for x in both])}
    if c["op"] == "write":
        k, v, out = [], [], {}
        if r:
            out["res"] = torch.zeros(st["res_kv"].shape, dtype=torch.float64, device=DEVICE)
        for a in range(n):
            lo, hi = int(st["row0"][a]), int(st["row0"][a + 1])
            pos = torch.arange(pos0[a], total[a], device=DEVICE)
            key = st["k"][lo:hi].double()
            k.append(_nearest(_turn(key, pos, st["rope"]) if c["rope"] else key))
            v.append(_nearest(st["v"][lo:hi].double()))
            for j in range(2 if adapter[a] >= 0 else 0):
                co = st["x"][lo:hi].double() @ st["a"][a, j].double().t()
                for rho in range(r):
                    at = (16 * (rho % 16 // 4) + pos % PS) * 8 + rho % 4 if j == 0 else (16 * (pos % PS // 4) + rho % 16) * 8 + 4 + pos % 4
                    out["res"][st["res"][a, pos // PS].long(), rho // 16 * 512 + at] = co[:, rho]
        return {"k": torch.cat(k), "v": torch.cat(v), **out}
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEVICE)
    for a in range(n):
        t, m, row = total[a], new[a], int(st["row0"][a])
        pos = torch.arange(t, device=DEVICE)
        k, v = _cached(st, hkv, a, pos)
        if adapter[a] >= 0:
            page, s, rho = st["res"][a, pos // PS].long()[:, None], (pos % PS)[:, None], torch.arange(r, device=DEVICE)[None]
            ck = st["res_kv"][page, rho // 16 * 512 + (16 * (rho % 16 // 4) + s) * 8 + rho % 4].double()
            cv = st["res_kv"][page, rho // 16 * 512 + (16 * (s // 4) + rho % 16) * 8 + 4 + s % 4].double()
            u = (ck @ st["lora_b"][a, 0].double()).view(t, hkv, D)
            k = k + (_turn(u, pos, st["rope"]) if c["rope"] else u)
            v = v + (cv @ st["lora_b"][a, 1].double()).view(t, hkv, D)
        for h in range(hkv):
            for i in range(0, m, 512):
                j = min(i + 512, m)
                z = st["q"][row + i:row + j, h * g:(h + 1) * g].double().reshape(-1, D) @ k[:, h].t() / math.sqrt(D)
                if c["op"] == "prefill":
                    z.masked_fill_(pos > (t - m + torch.arange(i, j, device=DEVICE)).repeat_interleave(g)[:, None], -math.inf)
                p = torch.softmax(z, dim=1)
                out[row + i:row + j, h * g:(h + 1) * g] = (p @ v[:, h]).view(j - i, g, D)
    return out
