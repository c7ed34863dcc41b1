// ResidualAttention chunked prefill over 8-bit base pages, the kernel of all but small grids (Section 6 prefill kernel, Algorithm 1 with
// a block of query rows; fp8_cache.hpp has the page format, prefill_fp8.hip the scales of K and Q and that of small grids).
//
// One workgroup of eight waves = (agent a, KV head h, block of 256 query rows), one row group of 32 rows per wave and two waves per SIMD (within 256
// registers each): while one wave's products hold the matrix cores the other issues its vector work.  Four waves of 64 rows read
// half as much from LDS (every operand serves two products) and were slower, 895 against 920 TFLOP/s without adapters, 733 against 752
// at rank 16 with RoPE and 300 against 700 at rank 64, where their accumulators spilled: alone on its SIMD, a wave's vector instructions
// wait for its own products.
//
// Wave w stages half of page w % 4 of a tile (four pages): the quarters w / 4 and w / 4 + 2 of the head dim, rotate-half partners.
// Codes and rCache rows come to registers a tile ahead and leave as operands in LDS, K = K_base + RoPE_p(B_K^T C_K^T) in fp16 times
// 2^-e, V = code * 2^E in bf16, C_V.  The work goes in steps of 32 keys (half a tile); step i issues, product by product in a
// written order,
//   O^T += V^T P^T and acc_r^T += C_V^T P^T of step i - 1, beside the row maxima and weights of step i
//   S^T = K Q^T of step i + 1, beside half of the staging of the next tile
// so that every product has vector work next to it; one barrier per tile.  A change of the running maximum rescales the accumulators at the
// end of its step, when the products of the step before, which carry the old one, are in.
//
// Measured at 16 chunks of 1024 tokens over 9.5k tokens of context, 8B heads: 950 TFLOP/s without adapters (a large bf16 product of
// the library: 1140), 905 with rank 16 (prefill_fp8.hip's kernel at 256 rows: 823), 757 with RoPE (712), and 727 at rank 64 with RoPE
// over 70B heads (511).
//
// Where 256 rows leave compute units idle a workgroup has 128 rows in four row groups, and two key groups of four waves take one half
// of every tile each: one step per tile, beside all of its staging, with the values two tiles behind the scores; at the end the second
// group's rows are merged into the first's.  Four chunks of up to 250 tokens, 8B heads: rank 16 over 35k 939 us (prefill_fp8.hip's kernel
// at 128 rows: 1028), over 17k without adapters 415 (418), rank 32 with RoPE 592 (650), rank 64 with RoPE 869 (941) and without 625 (868).
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>
#include <utility>

#include "fp8_cache.hpp"
#include "lds_dma.hpp"
#include "mfma.hpp"
#include "prefill.hpp"

using namespace fkvk;

namespace fkvp {
namespace {

constexpr int D = 128, PS = 16, TILE_KEYS = 64, WAVES = 8;
constexpr float kNegInf = -INFINITY, kLazyRescale = 8.f;

template <int R, int KG>
struct Lay {
    static constexpr int ROWS = 32 * WAVES / KG, VT = KG == 1 ? 3 : 4;  // query rows; tiles of V and C_V kept
    static constexpr int RT = R == 0 ? 0 : (R + 15) / 16, NRB = (RT + 1) / 2;
    static constexpr bool LROW = RT == 1;  // rows 16..31 of the rank block are ones: the row sums come with acc_r
    // K [2 tiles][32-key block][step][lane] 16 B, V [VT tiles][page][32-dim block][lane] 16 B, C_V [VT tiles][page][32-rank block][lane] 16 B
    static constexpr int V_OFF = 2 * 16384, C_OFF = V_OFF + VT * 16384, C_TILE = 4 * NRB * 1024;
    static constexpr int B_OFF = C_OFF + VT * C_TILE, E_OFF = B_OFF + RT * 4096, MAIN = E_OFF + 64;
    static constexpr int EPI = R * D * 4 + ROWS * (R + 1) * 4;
    static constexpr int NF4 = 16 + 4 * (NRB > 0 ? NRB : 1) + 1;  // a wave's rows: oacc, racc, (m, l)
    static constexpr int BYTES = MAIN > EPI ? MAIN : EPI;
    static_assert(KG == 1 || WAVES / 2 * NF4 * 1024 <= BYTES, "merge area");
    static_assert(BYTES <= 160 * 1024, "LDS of one workgroup");
};

typedef __attribute__((address_space(3))) u32x4 *lds128;
typedef __attribute__((address_space(3))) u32x2 *lds64;
__device__ __forceinline__ void st128(uint32_t a, const u32x4 &v) { *reinterpret_cast<lds128>((uintptr_t)a) = v; }
__device__ __forceinline__ void st64(uint32_t a, const u32x2 &v) { *reinterpret_cast<lds64>((uintptr_t)a) = v; }
__device__ __forceinline__ u32x2 ld64(uint32_t a) { return *reinterpret_cast<const __attribute__((address_space(3))) u32x2 *>((uintptr_t)a); }

__device__ __forceinline__ f32x16 mfma32x32_f16(const u32x4 &a, const u32x4 &b, const f32x16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// f(integral_constant 0), f(1), ..., f(N - 1): steps whose index selects code, without leaving the unrolling to the optimiser's limits.
template <int... I, class F>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F &&f) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F &&f) {
    each(std::make_integer_sequence<int, N>{}, f);
}
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// A workgroup's place in the grid.
struct Place {
    int a, h, qb, split;
    __device__ __forceinline__ Place(const PrefillArgs &p, int block) {
        const int bpa = p.blocks_per_agent_head, local = block / kXcds;
        const int pair = local / (bpa * p.splits) * kXcds + block % kXcds;
        a = pair / p.hkv;
        h = pair % p.hkv;
        qb = local % bpa;
        split = local / bpa % p.splits;
    }
};

template <int R, int G, bool ROPE, int KG>
__device__ __forceinline__ void block(const PrefillArgs &p, unsigned char *lds, int a, int h, int tok_begin, int split) {
    using S = Lay<R, KG>;
    constexpr int RT = S::RT, RTX = RT > 0 ? RT : 1, NRB = S::NRB, NRBX = NRB > 0 ? NRB : 1, TPW = S::ROWS / G, VT = S::VT;
    constexpr bool LROW = S::LROW;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4, hh = lane >> 5, r32 = lane & 31;
    const int rg = wave % (WAVES / KG), kg = wave / (WAVES / KG);  // row group, key group
    const int hkv = p.hkv;
    const int64_t n = (int64_t)hkv * D;
    const int q0 = p.q_indptr[a], nq = p.q_indptr[a + 1] - q0;
    int L = p.seq_lens[a], P0 = L - nq;
    const int ad = R > 0 ? p.adapter_idx[a] : -1;
    const int tok_end = tok_begin + TPW < nq ? tok_begin + TPW : nq, last_pos = P0 + tok_end - 1;
    const int all_tiles = last_pos / TILE_KEYS + 1, per_split = (all_tiles + p.splits - 1) / p.splits, t0 = split * per_split;
    const int n_tiles = min(per_split, all_tiles - t0);  // of this split
    if (n_tiles <= 0) return empty_rows(p, split, a, h, G, tok_begin, tok_end);
    // from here on tiles, pages and positions are counted from the split's first
    const int page_t0 = t0 * (TILE_KEYS / PS);
    L -= t0 * TILE_KEYS;
    P0 -= t0 * TILE_KEYS;
    const int n_pages = (L + PS - 1) / PS;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)lds;
    const int32_t *btb = p.base_bt + (int64_t)a * p.max_pages + page_t0, *btr = R > 0 ? p.res_bt + (int64_t)a * p.max_pages + page_t0 : nullptr;
    const unsigned char *base = reinterpret_cast<const unsigned char *>(p.base_kv);
    int *page_exp = reinterpret_cast<int *>(lds + S::E_OFF);  // [2 tiles][page]

    // ---- staging: half `half` of page pw of a tile (pages past the sequence repeat its last one; their keys are masked): quarters
    // half and half + 2 of the head dim, whose dims are rotate-half partners ----
    const int pw = wave & 3, half = wave >> 2;
    u32x2 kw[2], vw[2];
    uint32_t ke, ve;
    u32x4 c[RTX];
    f32x4 cs[2], sn[2];
    auto page_of = [&](int tile) __attribute__((always_inline)) { return min(4 * tile + pw, n_pages - 1); };
    // (buffer loads: a scalar base and one lane offset; lane addresses of 64 bits would be kept in registers for the launch)
    const int off16 = lane * 16, off8 = lane * 16 + half * 8, off_ve = PS + 4 * grp, off_ke = col;
    // Page ids of this wave's pages of 64 tiles, one per lane, and of the 64 after them: an id read where it is used would hold up the wave.
    auto ids = [&](int chunk, int &b, int &r) __attribute__((always_inline)) {
        const int pg = min((64 * chunk + lane) * 4 + pw, n_pages - 1);
        b = btb[pg];
        r = R > 0 ? btr[pg] : 0;
    };
    int idb, idr, idb_next, idr_next;
    ids(0, idb, idr);
    ids(1, idb_next, idr_next);
    // What staging takes first (exponents, rCache, V) and last (K) is requested as soon as the tile before has used its registers.
    // Tiles in order, from 0.
    auto request = [&](int tile) __attribute__((always_inline)) {
        if (__builtin_expect(tile > 0 && (tile & 63) == 0, 0)) {
            idb = idb_next;
            idr = idr_next;
            ids((tile >> 6) + 1, idb_next, idr_next);
        }
        const uint64_t page = reinterpret_cast<uint64_t>(base) + (int64_t)__builtin_amdgcn_readlane(idb, tile & 63) * f8_page_bytes(hkv);
        const i32x4 blk = block_rsrc(page + (int64_t)h * kF8HeadBytes, kF8HeadBytes), ex = block_rsrc(page + f8_exp_off(hkv, h), 2 * PS);
        ke = buf_load_u8(ex, off_ke);
        ve = buf_load4(ex, off_ve);
        if constexpr (R > 0) {
            const i32x4 rb = block_rsrc(reinterpret_cast<uint64_t>(p.res_kv) + (int64_t)__builtin_amdgcn_readlane(idr, tile & 63) * (RT * 1024), RT * 1024);
#pragma unroll
            for (int t = 0; t < RT; ++t) c[t] = buf_load16_at(rb, off16, t * 1024);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) vw[j] = buf_load8_at(blk, off8, kF8Block + 1024 * j);
    };
    auto request_keys = [&](int tile) __attribute__((always_inline)) {  // (after request of the same tile)
        const uint64_t page = reinterpret_cast<uint64_t>(base) + (int64_t)__builtin_amdgcn_readlane(idb, tile & 63) * f8_page_bytes(hkv);
        const i32x4 blk = block_rsrc(page + (int64_t)h * kF8HeadBytes, kF8HeadBytes);
#pragma unroll
        for (int j = 0; j < 2; ++j) kw[j] = buf_load8_at(blk, off8, 1024 * j);
    };
    auto request_angles = [&](int tile, int w) __attribute__((always_inline)) {  // of frequency tile 2 half + w
        if constexpr (ROPE) {
            const int64_t at = (int64_t)(page_t0 + page_of(tile)) * (PS * D / 2 * 4);
            const i32x4 rc = block_rsrc(reinterpret_cast<uint64_t>(p.rope_cos) + at, PS * D / 2 * 4);
            const i32x4 rs = block_rsrc(reinterpret_cast<uint64_t>(p.rope_sin) + at, PS * D / 2 * 4);
            cs[w] = __builtin_bit_cast(f32x4, buf_load16_at(rc, off16, 2048 * half + 1024 * w));
            sn[w] = __builtin_bit_cast(f32x4, buf_load16_at(rs, off16, 2048 * half + 1024 * w));
        }
    };
    float b_sum = 0.f;
    // staging in parts, spread over the products of a tile's two steps
    struct Staging {
        uint32_t kd, vd, cd;
        float e, ks, inv;
        int ep;
        f32x4 vs;
        u32x2 ck[RTX];
        f32x4 x, y;
        u32x2 pk[2][2];  // [partner][tile of the quarter], packed
    };
    const uint32_t bkt = lds0 + S::B_OFF + half * 1024 + lane * 8;  // B_K^T fragments [rank tile][column tile][lane]
    constexpr int PARTS = 18;
    auto low_rank = [&](const Staging &g, int m, f32x4 u) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < RT; ++t) u = mfma16(ld64(bkt + (t * 8 + m) * 512), g.ck[t], u);
        return u;
    };
    auto base_key = [&](const Staging &g, int m) __attribute__((always_inline)) {
        const uint32_t w = kw[m / 4][m % 4];  // (tile m of the wave's: w or, its partner, 4 + w)
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, g.ks, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, g.ks, true);
        return f32x4{lo.x, lo.y, hi.x, hi.y};
    };
    auto stage_part = [&](Staging &g, int tile, auto part_tag) __attribute__((always_inline)) {
        constexpr int part = decltype(part_tag)::value;
        if constexpr (part == 2) request_angles(tile, 1);  // (tile 0: before the step)
        if constexpr (part == 0) {
            int lane = threadIdx.x & 63;
            asm("" : "+v"(lane));  // what follows from it is formed here, not kept for the launch
            const int col = lane & 15, grp = lane >> 4;
            const int vis = L - (4 * tile + pw) * PS;  // tokens of the page inside the sequence
            if (__builtin_expect(vis < PS, 0)) {  // unwritten values may be any bits, and meet zero weights
                const int left = max(0, min(4, vis - 4 * grp));
                const uint32_t m = left == 4 ? 0xffffffffu : (1u << (8 * left)) - 1u;
                ve &= m;
                ke = col < vis ? ke : 0u;
#pragma unroll
                for (int j = 0; j < 2; ++j) vw[j] = u32x2{vw[j].x & m, vw[j].y & m};
                if constexpr (R > 0) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const u32x2 v = mask4(u32x2{c[t].z, c[t].w}, vis, grp);
                        c[t] = col < vis ? u32x4{c[t].x, c[t].y, v.x, v.y} : u32x4{0, 0, v.x, v.y};
                    }
                }
            }
            // K: operand of step 2 kk + grp / 2, lane half grp % 2, row 16 (page % 2) + col; V, C_V: words of four tokens 4 grp .. + 3,
            // the lower or upper eight bytes of lane half grp % 2
            const uint32_t at = ((lane & 16) * 2 + (lane & 15)) * 16;  // of lane half grp % 2, row col
            g.kd = lds0 + (tile & 1) * 16384 + (pw >> 1) * 8192 + (pw & 1) * 256 + half * 2048 + (lane & 32) * 32 + at;
            g.vd = lds0 + S::V_OFF + (tile % VT) * 16384 + pw * 4096 + half * 1024 + (lane & 32) / 4 + at;
            g.cd = g.vd + (S::C_OFF - S::V_OFF) + (tile % VT) * (S::C_TILE - 16384) + pw * (NRB * 1024 - 4096) - half * 1024;
            g.e = (float)((int)ke - 127 + 9);
            if constexpr (R > 0) {
                typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
                u16x2 m = {0, 0};
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if constexpr (R == 8) c[t] = u32x4{grp < 2 ? c[t].x : 0u, grp < 2 ? c[t].y : 0u, col < 8 ? c[t].z : 0u, col < 8 ? c[t].w : 0u};
                    const u16x2 x = __builtin_bit_cast(u16x2, c[t].x & 0x7fff7fffu), y = __builtin_bit_cast(u16x2, c[t].y & 0x7fff7fffu);
                    m = __builtin_elementwise_max(__builtin_elementwise_max(x, y), m);
                }
                const uint32_t w = __builtin_bit_cast(uint32_t, m);
                const uint32_t bits = __float_as_uint(fmaxf(bf16_lo(w), bf16_hi(w)) * b_sum) >> 23;
                g.e = fmaxf(g.e, bits < 255u ? (float)((int)bits - 126) : -200.f);
            }
        } else if constexpr (part == 1) {
            g.ep = max(-100, min(126, (int)max_over_groups(max_over_row(g.e))));
        } else if constexpr (part == 2) {
            if (lane == 0) page_exp[(tile & 1) * 4 + pw] = g.ep;  // (both halves find the same)
            g.ks = __uint_as_float((uint32_t)max(0, min(254, (int)ke - g.ep)) << 23);
            g.inv = __uint_as_float((uint32_t)(127 - g.ep) << 23);
            g.vs = f32x4{f8_scale(ve & 255u), f8_scale((ve >> 8) & 255u), f8_scale((ve >> 16) & 255u), f8_scale(ve >> 24)};
        } else if constexpr (part < 7) {
            constexpr int i = part - 3;  // word i: dims 32 (half + 2 (i / 2)) + 16 (i % 2) + col
            const uint32_t w = vw[i / 2][i % 2];
            const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, true);
            st64(g.vd + (i / 2) * 2048 + (i % 2) * 256, u32x2{pack_bf16(lo.x * g.vs.x, lo.y * g.vs.y), pack_bf16(hi.x * g.vs.z, hi.y * g.vs.w)});
        } else if constexpr (part == 7) {
            if constexpr (R > 0) {
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    g.ck[t] = u32x2{pack_bf16(bf16_lo(c[t].x) * g.inv, bf16_hi(c[t].x) * g.inv), pack_bf16(bf16_lo(c[t].y) * g.inv, bf16_hi(c[t].y) * g.inv)};
                    if (half == 0) st64(g.cd + (t / 2) * 1024 + (t % 2) * 256, u32x2{c[t].z, c[t].w});
                }
            }
        } else if constexpr (part == 8) {
            request(tile + 1);
        } else if constexpr (part < 17) {
            constexpr int w = (part - 9) / 4, s = (part - 9) % 4;  // the wave's tiles w and 4 + w (rotate-half partners)
            if constexpr (s == 0) {
                if constexpr (R > 0) {
                    g.x = low_rank(g, w, ROPE ? f32x4{0, 0, 0, 0} : base_key(g, w));
                    g.y = low_rank(g, w + 4, ROPE ? f32x4{0, 0, 0, 0} : base_key(g, w + 4));
                } else {
                    g.x = base_key(g, w);
                    g.y = base_key(g, w + 4);
                }
            } else if constexpr (s == 1) {
                f32x4 x = g.x;
                if constexpr (ROPE) {
                    const f32x4 b = base_key(g, w);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(g.x[j], cs[w][j], __builtin_fmaf(-g.y[j], sn[w][j], b[j]));
                }
                g.pk[0][w] = u32x2{pack_f16(x.x, x.y), pack_f16(x.z, x.w)};
            } else if constexpr (s == 2) {
                f32x4 y = g.y;
                if constexpr (ROPE) {
                    const f32x4 b = base_key(g, w + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = __builtin_fmaf(g.y[j], cs[w][j], __builtin_fmaf(g.x[j], sn[w][j], b[j]));
                }
                g.pk[1][w] = u32x2{pack_f16(y.x, y.y), pack_f16(y.z, y.w)};
            } else if constexpr (w == 1) {
#pragma unroll
                for (int j = 0; j < 2; ++j) st128(g.kd + j * 4096, u32x4{g.pk[j][0].x, g.pk[j][0].y, g.pk[j][1].x, g.pk[j][1].y});
            }
        } else if constexpr (part == 17) {
            request_keys(tile + 1);
        }
    };

    // ---- queries (B operand: lane = row, dims 32 kk + 4 g + 0..3 and 16 further, g = 2 (st % 2) + hh), fp16 times 2^-eq ----
    int row_tok, eq;
    u32x4 qf[8];
    {
        const int rr = rg * 32 + r32, tk = tok_begin + rr / G;
        const bool ok = tk < nq;
        row_tok = ok ? tk : -1;
        const uint16_t *qr = p.q + ((int64_t)(q0 + (ok ? tk : 0)) * p.hq + h * G + rr % G) * D;
        float big = 0.f;
#pragma unroll
        for (int st = 0; st < 8; ++st) {
            const int dm = 32 * (st / 2) + 4 * (2 * (st % 2) + hh);
            u32x4 v = {0, 0, 0, 0};
            if (ok) {
                const u32x2 lo = ldg64(qr + dm), hi = ldg64(qr + dm + 16);
                v = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) big = fmaxf(big, fmaxf(fabsf(bf16_lo(v[i])), fabsf(bf16_hi(v[i]))));
            qf[st] = v;
        }
        eq = max(-100, min(126, (int)(__float_as_uint(max_over_halves(big)) >> 23) - 126));
        const float inv = __uint_as_float((uint32_t)(127 - eq) << 23);
#pragma unroll
        for (int st = 0; st < 8; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[st][i] = pack_f16(bf16_lo(qf[st][i]) * inv, bf16_hi(qf[st][i]) * inv);
    }
    request(0);
    request_keys(0);
    if constexpr (R > 0) {
        // B_K^T fragments: lane (c, g) of (tile t, column tile m) holds B_K[16t + 4g + 0..3][16m + c]; sums of the ranks' largest
        const uint16_t *bk = p.lora_b + (int64_t)ad * 2 * R * n + (int64_t)h * D;
        float mine = 0.f;
        for (int rho = wave; rho < R; rho += WAVES) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(bk + (int64_t)rho * n + 2 * lane);
            mine += max_over_groups(max_over_row(fmaxf(fabsf(bf16_lo(w)), fabsf(bf16_hi(w)))));
        }
        float *part = reinterpret_cast<float *>(lds + S::E_OFF);
        if (lane == 0) part[wave] = mine * 1.4143f;
        for (int idx = threadIdx.x; idx < RT * 512; idx += 64 * WAVES) {
            const int ln = idx & 63, m = (idx >> 6) & 7, t = idx >> 9;
            uint32_t w[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r0 = 16 * t + 4 * (ln >> 4) + 2 * j;
                const uint16_t lo = r0 < R ? bk[(int64_t)r0 * n + 16 * m + (ln & 15)] : (uint16_t)0;
                const uint16_t hi = r0 + 1 < R ? bk[(int64_t)(r0 + 1) * n + 16 * m + (ln & 15)] : (uint16_t)0;
                w[j] = (uint32_t)lo | ((uint32_t)hi << 16);
            }
            st64(lds0 + S::B_OFF + idx * 8, u32x2{w[0], w[1]});
        }
        if constexpr (LROW) {  // rows 16..31 of the rank block: ones, for the launch
            for (int idx = threadIdx.x; idx < VT * 4 * 64; idx += 64 * WAVES)
                if (idx & 16) st128(lds0 + S::C_OFF + idx * 16, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) b_sum += part[w];
        __syncthreads();
    }

    f32x16 oacc[4], racc[NRBX], s;  // s: scores of 32 keys
#pragma unroll
    for (int b = 0; b < 4; ++b) oacc[b] = f32x16{};
#pragma unroll
    for (int b = 0; b < NRBX; ++b) racc[b] = f32x16{};
    float m_run = kNegInf, lsum = 0.f;
    const float cl = p.scale_log2;

    // One step: PV: values of block pv_kb of tile pv_tile with the weights pf_in, beside (EXP) the weights of the scores s (32 keys from
    // key0; page exponents e0, e1) into pf_out; then QK: scores of block qk_kb of tile qk_tile into s, beside (STAGE) the first or second
    // half of the staging of tile st_tile.
    constexpr int NP = 8 + 2 * NRB, SLOTS = NP + 8, PRE = 2;  // products of the values, of a step; operands read ahead (four
    // spill at ranks over 16: 639 TFLOP/s at rank 64, not 700)
    u32x4 ahead[PRE];
    auto step = [&](auto exp_tag, auto qk_tag, auto pv_tag, auto stage_tag, u32x4 (&pf_in)[2], u32x4 (&pf_out)[2], int key0, int e0, int e1, int qk_tile,
                    int qk_kb, int pv_tile, int pv_kb, int next_tile, int next_kb, Staging &g, int st_tile) __attribute__((always_inline)) {
        constexpr bool EXP = decltype(exp_tag)::value, QK = decltype(qk_tag)::value, PV = decltype(pv_tag)::value;
        constexpr int STAGE = decltype(stage_tag)::value;  // 0: none, 1: first half of the parts, 2: second half, 3: all
        const uint32_t ka = lds0 + (qk_tile & 1) * 16384 + qk_kb * 8192 + lane * 16;
        const uint32_t va = lds0 + S::V_OFF + (pv_tile % VT) * 16384 + pv_kb * 8192 + lane * 16;
        const uint32_t ca = lds0 + S::C_OFF + (pv_tile % VT) * S::C_TILE + pv_kb * 2 * NRB * 1024 + lane * 16;
        const uint32_t vn = lds0 + S::V_OFF + (next_tile % VT) * 16384 + next_kb * 8192 + lane * 16;
        const uint32_t cn = lds0 + S::C_OFF + (next_tile % VT) * S::C_TILE + next_kb * 2 * NRB * 1024 + lane * 16;
        // operands in order: those of the values (page i / (4 + NRB), block i % (4 + NRB)), of the scores, then the next step's first
        auto frag = [&](auto slot_tag) __attribute__((always_inline)) -> u32x4 {
            constexpr int slot = decltype(slot_tag)::value;
            if constexpr (slot >= SLOTS) {
                constexpr int pg = (slot - SLOTS) / (4 + NRB), b = (slot - SLOTS) % (4 + NRB);
                return b < 4 ? lds_load(vn + pg * 4096 + b * 1024) : lds_load(cn + (pg * NRB + b - 4) * 1024);
            } else if constexpr (slot >= NP) {
                return QK ? lds_load(ka + (slot - NP) * 1024) : u32x4{};
            } else {
                constexpr int pg = slot / (4 + NRB), b = slot % (4 + NRB);
                if constexpr (!PV) return u32x4{};
                return b < 4 ? lds_load(va + pg * 4096 + b * 1024) : lds_load(ca + (pg * NRB + b - 4) * 1024);
            }
        };
        auto product = [&](auto slot_tag, const u32x4 &f) __attribute__((always_inline)) {
            constexpr int slot = decltype(slot_tag)::value;
            if constexpr (slot >= NP) {
                constexpr int i = slot - NP;
                if constexpr (QK) s = mfma32x32_f16(f, qf[i], i == 0 ? f32x16{} : s);
            } else if constexpr (PV) {
                constexpr int pg = slot / (4 + NRB), b = slot % (4 + NRB);
                if constexpr (b < 4) oacc[b] = mfma32x32(f, pf_in[pg], oacc[b]);
                else racc[b - 4] = mfma32x32(f, pf_in[pg], racc[b - 4]);
            }
        };
        float f[2], mx, alpha, tsum = 0.f;  // f [page]
        bool moved = false;
        if constexpr (EXP) {
            if (__builtin_expect(key0 + 31 > P0 + tok_begin, 0)) {  // causal mask
                const int lim = row_tok < 0 ? -1 : P0 + row_tok - key0 - 4 * hh;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 8 * (i / 4) + i % 4 <= lim ? s[i] : kNegInf;
            }
        }
        auto maxima = [&]() __attribute__((always_inline)) {
            f[0] = fminf(fmaxf(ldexpf(cl, e0 + eq), 1.2e-38f), 3e38f);  // neither 0 nor infinite: masked scores and zeros stay
            f[1] = fminf(fmaxf(ldexpf(cl, e1 + eq), 1.2e-38f), 3e38f);
            float x0 = fmaxf(s[0], s[1]), x1 = fmaxf(s[8], s[9]);
#pragma unroll
            for (int i = 2; i < 8; i += 2) {
                x0 = fmaxf(fmaxf(x0, s[i]), s[i + 1]);
                x1 = fmaxf(fmaxf(x1, s[8 + i]), s[9 + i]);
            }
            mx = fmaxf(x0 * f[0], x1 * f[1]);
        };
        auto weights = [&](auto pair_tag) __attribute__((always_inline)) {  // values 2 w, 2 w + 1 of the lane's 16
            constexpr int w = decltype(pair_tag)::value, i = 2 * w, pg = i / 8;
            const float m_use = m_run == kNegInf ? 0.f : m_run;
            const float w0 = fast_exp2(__builtin_fmaf(s[i], f[pg], -m_use)), w1 = fast_exp2(__builtin_fmaf(s[i + 1], f[pg], -m_use));
            uint32_t pk = pack_bf16(w0, w1);
            asm volatile("" : "+v"(pk));  // stays here: otherwise the compiler moves the weights past the branch below, behind the products
            pf_out[pg][(i % 8) / 2] = pk;
            if constexpr (!LROW) tsum = add_bf16_pair(pk, tsum);  // the weights as the products take them: their rounding cancels in O / l
        };
        auto beside = [&](auto slot_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(slot_tag)::value, FIRST = 2;
            if constexpr (EXP && i < NP) {
                if constexpr (i == 0) maxima();
                if constexpr (i == 1) {
                    mx = max_over_halves(mx);
                    moved = __builtin_amdgcn_ballot_w64(mx > m_run + kLazyRescale) != 0;
                    if (__builtin_expect(moved, 0)) {
                        const float m_new = fmaxf(m_run, mx);
                        alpha = fast_exp2(m_run - (m_new == kNegInf ? 0.f : m_new));
                        m_run = m_new;
                    }
                }
                if constexpr (i >= FIRST) {
                    constexpr int n = NP - FIRST, a0 = 8 * (i - FIRST) / n, a1 = 8 * (i + 1 - FIRST) / n;
                    each<a1 - a0>([&](auto q) __attribute__((always_inline)) { weights(std::integral_constant<int, a0 + q.value>{}); });
                }
                if constexpr (i == NP - 1) {
                    if (__builtin_expect(moved, 0)) {
#pragma unroll
                        for (int b = 0; b < 4; ++b) oacc[b] *= alpha;
#pragma unroll
                        for (int b = 0; b < NRB; ++b) racc[b] *= alpha;
                        lsum *= alpha;
                    }
                    if constexpr (!LROW) lsum += tsum;
                }
            }
            if constexpr (STAGE == 3) {
                constexpr int p0 = PARTS * i / SLOTS, p1 = PARTS * (i + 1) / SLOTS;
                each<p1 - p0>([&](auto k) __attribute__((always_inline)) { stage_part(g, st_tile, std::integral_constant<int, p0 + k.value>{}); });
            } else if constexpr (STAGE > 0 && i >= NP) {
                constexpr int HALF = PARTS / 2, q = i - NP, p0 = HALF * q / 8, p1 = HALF * (q + 1) / 8;
                each<p1 - p0>([&](auto k) __attribute__((always_inline)) {
                    stage_part(g, st_tile, std::integral_constant<int, (STAGE - 1) * HALF + p0 + k.value>{});
                });
            }
            fence();
        };
        u32x4 fr[SLOTS + PRE];
        each<PRE>([&](auto q) __attribute__((always_inline)) { fr[q.value] = ahead[q.value]; });
        fence();
        each<SLOTS>([&](auto slot_tag) __attribute__((always_inline)) {
            constexpr int slot = decltype(slot_tag)::value;
            product(slot_tag, fr[slot]);
            fr[slot + PRE] = frag(std::integral_constant<int, slot + PRE>{});
            beside(slot_tag);
        });
        each<PRE>([&](auto q) __attribute__((always_inline)) { ahead[q.value] = fr[SLOTS + q.value]; });
    };
    using T = std::true_type;
    using F = std::false_type;
    using N0 = std::integral_constant<int, 0>;
    using N1 = std::integral_constant<int, 1>;
    using N2 = std::integral_constant<int, 2>;
    using N3 = std::integral_constant<int, 3>;
    Staging g;
    u32x4 pa[2], pb[2];  // weights [page]: of a tile's second and first half; two key groups: of the tile before and of a tile

    request_angles(0, 0);
    each<PARTS>([&](auto i) __attribute__((always_inline)) { stage_part(g, 0, i); });  // (requests tile 1)
    __syncthreads();
    auto exps_of = [&](int tile) __attribute__((always_inline)) { return *reinterpret_cast<const i32x4 *>(page_exp + (tile & 1) * 4); };
    if constexpr (KG == 1) {
        // tile 0: no values yet
        i32x4 e = exps_of(0);
        request_angles(1, 0);
        step(F{}, T{}, F{}, N1{}, pa, pb, 0, 0, 0, 0, 0, 0, 0, 0, 0, g, 1);
        step(T{}, T{}, F{}, N2{}, pa, pb, 0, e.x, e.y, 0, 1, 0, 0, 0, 0, g, 1);
        for (int u = 1; u < n_tiles; ++u) {
            lds_fence_barrier();  // (not one that waits for the loads in flight) tile u is staged, tile u - 1's keys and tile u - 2's values are read
            const i32x4 en = exps_of(u);
            request_angles(u + 1, 0);
            step(T{}, T{}, T{}, N1{}, pb, pa, (u - 1) * TILE_KEYS + 32, e.z, e.w, u, 0, u - 1, 0, u - 1, 1, g, u + 1);
            step(T{}, T{}, T{}, N2{}, pa, pb, u * TILE_KEYS, en.x, en.y, u, 1, u - 1, 1, u, 0, g, u + 1);
            e = en;
        }
        // the last tile's second half, and its values
        step(T{}, F{}, T{}, N0{}, pb, pa, (n_tiles - 1) * TILE_KEYS + 32, e.z, e.w, 0, 0, n_tiles - 1, 0, n_tiles - 1, 1, g, 0);
        step(F{}, F{}, T{}, N0{}, pa, pb, 0, 0, 0, 0, 0, n_tiles - 1, 1, 0, 0, g, 0);
    } else {
        // Key group kg takes half kg of every tile, one step per tile: values of tile u - 2, weights of u - 1, scores of u.  (Before there
        // are weights, tile 0's values meet zeros.)
        auto pages_of = [&](int tile) __attribute__((always_inline)) { return *reinterpret_cast<const u32x2 *>(page_exp + (tile & 1) * 4 + 2 * kg); };
        u32x2 e = pages_of(0);
        pa[0] = pa[1] = u32x4{0, 0, 0, 0};
        request_angles(1, 0);
        step(F{}, T{}, F{}, N3{}, pa, pb, 0, 0, 0, 0, kg, 0, 0, 0, kg, g, 1);
        for (int u = 1; u < n_tiles; ++u) {
            lds_fence_barrier();  // tile u is staged, tile u - 1's keys and tile u - 3's values are read
            const u32x2 en = pages_of(u);
            request_angles(u + 1, 0);
            step(T{}, T{}, T{}, N3{}, pa, pb, (u - 1) * TILE_KEYS + 32 * kg, e.x, e.y, u, kg, max(u - 2, 0), kg, u - 1, kg, g, u + 1);
            pa[0] = pb[0];
            pa[1] = pb[1];
            e = en;
        }
        step(T{}, F{}, T{}, N0{}, pa, pb, (n_tiles - 1) * TILE_KEYS + 32 * kg, e.x, e.y, 0, 0, max(n_tiles - 2, 0), kg, n_tiles - 1, kg, g, 0);
        step(F{}, F{}, T{}, N0{}, pb, pa, 0, 0, 0, 0, 0, n_tiles - 1, kg, 0, 0, g, 0);
    }
    __syncthreads();
    if constexpr (KG == 2) {  // the second key group leaves its rows in LDS, the first merges them into its own
        constexpr int NF4 = S::NF4;
        f32x4 *buf = reinterpret_cast<f32x4 *>(lds) + rg * NF4 * 64 + lane;
        auto four = [](const f32x16 &x, int i) __attribute__((always_inline)) { return f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]}; };
        if (kg == 1) {
#pragma unroll
            for (int i = 0; i < 16; ++i) buf[i * 64] = four(oacc[i / 4], i % 4);
#pragma unroll
            for (int i = 0; i < 4 * NRB; ++i) buf[(16 + i) * 64] = four(racc[i / 4], i % 4);
            buf[(NF4 - 1) * 64] = f32x4{m_run, lsum, 0.f, 0.f};
        }
        __syncthreads();
        if (kg == 0) {
            const f32x4 ml = buf[(NF4 - 1) * 64];
            const float M = fmaxf(m_run, ml.x), Mu = M == kNegInf ? 0.f : M;
            const float w0 = fast_exp2(m_run - Mu), w1 = fast_exp2(ml.x - Mu);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const f32x4 x = buf[i * 64];
#pragma unroll
                for (int j = 0; j < 4; ++j) oacc[i / 4][4 * (i % 4) + j] = oacc[i / 4][4 * (i % 4) + j] * w0 + x[j] * w1;
            }
#pragma unroll
            for (int i = 0; i < 4 * NRB; ++i) {
                const f32x4 x = buf[(16 + i) * 64];
#pragma unroll
                for (int j = 0; j < 4; ++j) racc[i / 4][4 * (i % 4) + j] = racc[i / 4][4 * (i % 4) + j] * w0 + x[j] * w1;
            }
            lsum = lsum * w0 + ml.y * w1;
            m_run = M;
        }
        __syncthreads();
    }

    // ---- epilogue: O = (acc + acc_r . B_V[h]) / l; lane: row r32, dims 32 b + 8 (i / 4) + 4 hh + i % 4 ----
    const float l_run = LROW ? __shfl(racc[0][8], r32) : lsum + __shfl_xor(lsum, 32);
    // what the epilogue takes is derived again, from a copy that the compiler takes for another: kept over the loop it would be spilled
    int block_id = blockIdx.x;
    asm volatile("" : "+s"(block_id));
    const Place at(p, block_id);
    if constexpr (R > 0) {
        float *bv = reinterpret_cast<float *>(lds), *acc = bv + R * D;
        const int64_t n = (int64_t)p.hkv * D;
        const uint16_t *src = p.lora_b + ((int64_t)p.adapter_idx[at.a] * 2 + 1) * R * n + (int64_t)at.h * D;
        for (int e = threadIdx.x; e < R * D / 2; e += 64 * WAVES) {
            const uint32_t w = *reinterpret_cast<const uint32_t *>(src + (int64_t)(e / (D / 2)) * n + 2 * (e % (D / 2)));
            bv[2 * e] = bf16_lo(w);
            bv[2 * e + 1] = bf16_hi(w);
        }
#pragma unroll
        for (int b = 0; b < NRB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int rho = 32 * b + 8 * (i / 4) + 4 * hh + i % 4;
                if (rho < R && kg == 0) acc[(rg * 32 + r32) * (R + 1) + rho] = racc[b][i];
            }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll 2
        for (int rho = 0; rho < R; ++rho) {
            const float x = acc[(rg * 32 + r32) * (R + 1) + rho];
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(bv + rho * D + 32 * b + 8 * i + 4 * hh);
#pragma unroll
                    for (int j = 0; j < 4; ++j) oacc[b][4 * i + j] += x * v[j];
                }
        }
    }
    if (kg == 0 && row_tok >= 0 && p.splits > 1) {  // this split's partial rows
        float *rec = partial_row(p, at.split, at.a, row_tok, at.h * G + (rg * 32 + r32) % G);
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4 *>(rec + 32 * b + 8 * i + 4 * hh) =
                    f32x4{oacc[b][4 * i], oacc[b][4 * i + 1], oacc[b][4 * i + 2], oacc[b][4 * i + 3]};
        if (hh == 0) *reinterpret_cast<f32x4 *>(rec + D) = f32x4{m_run, l_run, 0.f, 0.f};
    } else if (kg == 0 && row_tok >= 0) {
        const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
        uint16_t *o = p.out + ((int64_t)(p.q_indptr[at.a] + row_tok) * p.hq + at.h * G + (rg * 32 + r32) % G) * D;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 v = {oacc[b][4 * i] * inv, oacc[b][4 * i + 1] * inv, oacc[b][4 * i + 2] * inv, oacc[b][4 * i + 3] * inv};
                *reinterpret_cast<u32x2 *>(o + 32 * b + 8 * i + 4 * hh) = pack4(v);
            }
    }
}

template <int R, int G, bool ROPE, int KG>
__global__ __launch_bounds__(64 * WAVES, 1) void prefill_fp8_stream_kernel(PrefillArgs p) {
    constexpr int TPW = Lay<R, KG>::ROWS / G;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[Lay<R, KG>::BYTES > Lay<0, KG>::BYTES ? Lay<R, KG>::BYTES : Lay<0, KG>::BYTES];
    const Place at(p, blockIdx.x);
    const int a = at.a, h = at.h, qb = at.qb, split = at.split;
    if (a >= p.n_agents) return;
    const int q0 = p.q_indptr[a], nq = p.q_indptr[a + 1] - q0;
    const int tok_begin = qb * TPW;
    const int bpa = p.blocks_per_agent_head;
    if (qb == bpa - 1 && split == 0 && nq > bpa * TPW) poison_unreached_rows(p, q0, nq, h, G, bpa * TPW);
    if (tok_begin >= nq) return;
    if (R > 0 && p.adapter_idx[a] >= 0) block<R, G, ROPE, KG>(p, lds, a, h, tok_begin, split);
    else block<0, G, false, KG>(p, lds, a, h, tok_begin, split);
}

template <int R, int G, bool ROPE, int KG>
hipError_t launch(const PrefillArgs &pa, hipStream_t st, void *const *ev) {
    const int pairs = (pa.n_agents * pa.hkv + kXcds - 1) / kXcds * kXcds;
    // timing events carry the kernel's own start and end timestamps (set by the launch)
    hipEvent_t e0 = ev ? static_cast<hipEvent_t>(ev[0]) : nullptr, e1 = ev ? static_cast<hipEvent_t>(ev[1]) : nullptr;
    hipExtLaunchKernelGGL((prefill_fp8_stream_kernel<R, G, ROPE, KG>), dim3(pairs * pa.blocks_per_agent_head * pa.splits), dim3(64 * WAVES), 0, st, e0, e1, 0, pa);
    return hipGetLastError();
}

template <int R, int G, int KG>
hipError_t launch(bool rope, const PrefillArgs &pa, hipStream_t st, void *const *ev) {
    return R > 0 && rope ? launch<R, G, (R > 0), KG>(pa, st, ev) : launch<R, G, false, KG>(pa, st, ev);
}

template <int G, int KG>
hipError_t dispatch(int r, bool rope, const PrefillArgs &pa, hipStream_t st, void *const *ev) {
    switch (r) {
    case 0: return launch<0, G, KG>(rope, pa, st, ev);
    case 8: return launch<8, G, KG>(rope, pa, st, ev);
    case 16: return launch<16, G, KG>(rope, pa, st, ev);
    case 32: return launch<32, G, KG>(rope, pa, st, ev);
    case 64: return launch<64, G, KG>(rope, pa, st, ev);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_fp8_stream(int r, int g, int rows, const PrefillArgs &pa, hipStream_t st, void *const *ev) {
    const bool rope = pa.rope_cos != nullptr;
    if (rows == 256) return g == 4 ? dispatch<4, 1>(r, rope, pa, st, ev) : dispatch<8, 1>(r, rope, pa, st, ev);
    return g == 4 ? dispatch<4, 2>(r, rope, pa, st, ev) : dispatch<8, 2>(r, rope, pa, st, ev);
}

}  // namespace fkvp
