// ResidualAttention chunked prefill over 8-bit base pages (Section 6 prefill kernel, Algorithm 1 with a block of
// query rows; fp8_cache.hpp has the page format).
//
// The kernel of small grids: one workgroup of eight waves = (agent a, KV head h, block of 64 query rows, split of the keys); its rows are
// (query token, query head of h), all of the same agent.  Wave w serves row group w % 2 (32 rows) as key group w / 2.  Per round of
// eight pages:
//   staging     wave w takes page w: its codes and rCache rows come to registers one round ahead, and leave as
//               matrix-core operands in LDS, where all waves read them: a value is converted once per workgroup.
//               K = K_base + RoPE_p(B_K^T C_K^T) (without tables no rotation), V = code * 2^E.
//   every wave  S^T = K Q^T, causal mask + online softmax, O^T += V^T P^T, acc_r^T += C_V^T P^T over the two pages of its key group
// and at the end the key groups' rows are merged and O = (O + acc_r . B_V[h]) / l (Eq. 4) is written in bf16, or, where the keys are
// split over workgroups, the partial rows for merge_splits_kernel.  prefill_fp8_stream.hip has the kernel of 256 and 128 rows.
//
// K and Q are fp16 here, 11 significant bits: the sum of a base key, exact in four bits, and its low-rank part would
// lose what bf16 keeps of it alone (error of the result 5.6e-3 with bf16 keys at 8B heads, rank 16, over 9000 tokens, 2-norm; 2.2e-3 in
// fp16).  For their range both are scaled by powers of two: Q by its row's largest magnitude, K by a bound of its page's,
// max(448 * 2^E over its tokens, the largest |C_K| * sum_rho sqrt(2) max_i |B_K[rho][i]|), so that it stays below 2; both
// exponents go into the softmax's factor of the page.  V stays bf16, in which it is exact.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "fp8_cache.hpp"
#include "lds_dma.hpp"
#include "mfma.hpp"
#include "prefill.hpp"

using namespace fkvk;

namespace fkvp {
namespace {

constexpr int D = 128, PS = 16;
constexpr int WAVES = 8, ROWS_PER_WAVE = 32, ROUND_PAGES = WAVES, ROUND_KEYS = ROUND_PAGES * PS;
constexpr int NRG = 2, KG = WAVES / NRG, ROWS = NRG * ROWS_PER_WAVE, GP = ROUND_PAGES / KG;  // row groups, key groups; pages of a key group per round
constexpr float kNegInf = -INFINITY, kLazyRescale = 8.f;

template <int R>
struct Shape {
    static constexpr int RT = R == 0 ? 0 : (R + 15) / 16, RTX = RT > 0 ? RT : 1;
    // LDS: K and V ([page][4 KB], fragment order), rCache pages [page][rank tile][1 KB], B_K^T fragments, page exponents
    static constexpr int V_OFF = ROUND_PAGES * 4096, C_OFF = 2 * V_OFF, B_OFF = C_OFF + RT * ROUND_PAGES * 1024;
    static constexpr int E_OFF = B_OFF + RT * 4096, MAIN = E_OFF + 64;
    static constexpr int EPI = R * D * 4 + ROWS * (R + 1) * 4;  // B_V and the rank accumulators of the epilogue
    static constexpr int NF4 = 2 * (8 + RT + 2);                // a wave's rows: oacc, racc, lacc, m
    static constexpr int MERGE = (KG / 2) * NRG * NF4 * 1024;
    static constexpr int B2 = MAIN > EPI ? MAIN : EPI;
    static constexpr int BYTES = B2 > MERGE ? B2 : MERGE;
    static_assert(BYTES <= 160 * 1024, "LDS of one workgroup");
};

// Four codes of V (four tokens of one dim) as bf16, each token with its own power of two.
__device__ __forceinline__ u32x2 value_word(uint32_t w, const f32x4 &scale) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, 1.f, true);
    return u32x2{pack_bf16(lo.x * scale.x, lo.y * scale.y), pack_bf16(hi.x * scale.z, hi.y * scale.w)};
}

template <int R, int G>
__global__ __launch_bounds__(64 * WAVES, 1) void prefill_fp8_kernel(PrefillArgs p) {
    using S = Shape<R>;
    constexpr int RT = S::RT, RTX = S::RTX, TPW = ROWS / G;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[S::BYTES];
    const int hkv = p.hkv, bpa = p.blocks_per_agent_head;
    const int xcd = blockIdx.x % kXcds, local = blockIdx.x / kXcds;
    const int pair = local / (bpa * p.splits) * kXcds + xcd, qb = local % bpa, split = local / bpa % p.splits;
    if (pair >= p.n_agents * hkv) return;
    const int a = pair / hkv, h = pair % hkv;
    const int q0 = p.q_indptr[a], nq = p.q_indptr[a + 1] - q0;
    const int tok_begin = qb * TPW;
    if (qb == bpa - 1 && split == 0 && nq > bpa * TPW) poison_unreached_rows(p, q0, nq, h, G, bpa * TPW);
    if (tok_begin >= nq) return;
    const int L = p.seq_lens[a], P0 = L - nq;
    const int ad = R > 0 ? p.adapter_idx[a] : -1;
    const bool use_res = ad >= 0, rope = use_res && p.rope_cos;

    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int rg = wave % NRG, kg = wave / NRG;
    const int64_t n = (int64_t)hkv * D;
    const int n_pages = (L + PS - 1) / PS;
    const int tok_end = tok_begin + TPW < nq ? tok_begin + TPW : nq, last_pos = P0 + tok_end - 1;
    // rounds of this split: n_rounds from r0 (rounds below are counted from r0)
    const int all_rounds = last_pos / ROUND_KEYS + 1, per_split = (all_rounds + p.splits - 1) / p.splits, r0 = split * per_split;
    const int n_rounds = min(per_split, all_rounds - r0);
    if (n_rounds <= 0) return empty_rows(p, split, a, h, G, tok_begin, tok_end);
    const int32_t *btb = p.base_bt + (int64_t)a * p.max_pages, *btr = R > 0 ? p.res_bt + (int64_t)a * p.max_pages : nullptr;
    const unsigned char *base = reinterpret_cast<const unsigned char *>(p.base_kv);

    // ---- staging: this wave's page of a round in registers ----
    u32x4 kw[2], vw[2];
    uint32_t ke, ve;
    u32x4 c[RTX];
    f32x4 cs[4], sn[4];
    // Page ids of this wave's pages of 64 rounds, one per lane, and of the 64 after them: an id read where it is used would hold up the wave.
    auto ids = [&](int chunk, int &b, int &r) __attribute__((always_inline)) {
        const int pg = min((r0 + 64 * chunk + lane) * ROUND_PAGES + wave, n_pages - 1);  // pages past the sequence repeat its last one; their keys are masked
        b = btb[pg];
        r = R > 0 ? btr[pg] : 0;
    };
    int idb, idr, idb_next, idr_next;
    ids(0, idb, idr);
    ids(1, idb_next, idr_next);
    auto request = [&](int round) __attribute__((always_inline)) {  // rounds in order, from 0
        if (__builtin_expect(round > 0 && (round & 63) == 0, 0)) {
            idb = idb_next;
            idr = idr_next;
            ids((round >> 6) + 1, idb_next, idr_next);
        }
        const int pg = min(ROUND_PAGES * (r0 + round) + wave, n_pages - 1);
        const unsigned char *page = base + (int64_t)__builtin_amdgcn_readlane(idb, round & 63) * f8_page_bytes(hkv);
        const unsigned char *blk = page + (int64_t)h * kF8HeadBytes + lane * 16;
        const unsigned char *ex = page + f8_exp_off(hkv, h);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            kw[j] = ldg128(blk + 1024 * j);
            vw[j] = ldg128(blk + kF8Block + 1024 * j);
        }
        ke = ex[col];
        ve = *reinterpret_cast<const uint32_t *>(ex + PS + 4 * grp);
        if constexpr (R > 0) {
            if (use_res) {
                const uint16_t *rb = p.res_kv + (int64_t)__builtin_amdgcn_readlane(idr, round & 63) * (RT * 512) + lane * 8;
#pragma unroll
                for (int t = 0; t < RT; ++t) c[t] = ldg128(rb + t * 512);
            }
            if (rope) {
                const int64_t at = (int64_t)pg * (PS * D / 2) + 4 * lane;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    cs[j] = *reinterpret_cast<const f32x4 *>(p.rope_cos + at + 256 * j);
                    sn[j] = *reinterpret_cast<const f32x4 *>(p.rope_sin + at + 256 * j);
                }
            }
        }
    };
    const u32x2 *bkt = reinterpret_cast<const u32x2 *>(lds + S::B_OFF);  // [rank tile][column tile][lane]
    int *page_exp = reinterpret_cast<int *>(lds + S::E_OFF);
    float b_sum = 0.f;  // sum over ranks of sqrt(2) max_i |B_K[rho][i]|
    auto stage = [&](int round) __attribute__((always_inline)) {
        const int vis = L - (ROUND_PAGES * (r0 + round) + wave) * PS;  // tokens of the page inside the sequence
        if (vis < PS) {  // unwritten values may be any bits, and meet zero weights
            const int left = max(0, min(4, vis - 4 * grp));
            const uint32_t m = left == 4 ? 0xffffffffu : (1u << (8 * left)) - 1u;
            ve &= m;
            ke = col < vis ? ke : 0u;
#pragma unroll
            for (int j = 0; j < 2; ++j) vw[j] = u32x4{vw[j].x & m, vw[j].y & m, vw[j].z & m, vw[j].w & m};
            if constexpr (R > 0) {
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const u32x2 v = mask4(u32x2{c[t].z, c[t].w}, vis, grp);
                    c[t] = col < vis ? u32x4{c[t].x, c[t].y, v.x, v.y} : u32x4{0, 0, v.x, v.y};
                }
            }
        }
        // the page's exponent: |K| < 2^e
        float e = (float)((int)ke - 127 + 9);
        if constexpr (R > 0) {
            if (use_res) {
                uint32_t m = 0;  // largest |C_K| of the lane, as two halves
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if constexpr (R == 8) c[t] = u32x4{grp < 2 ? c[t].x : 0u, grp < 2 ? c[t].y : 0u, c[t].z, c[t].w};  // rank padding
                    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
                    const u16x2 x = __builtin_bit_cast(u16x2, c[t].x & 0x7fff7fffu), y = __builtin_bit_cast(u16x2, c[t].y & 0x7fff7fffu);
                    m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_elementwise_max(x, y), __builtin_bit_cast(u16x2, m)));
                }
                const uint32_t bits = __float_as_uint(fmaxf(bf16_lo(m), bf16_hi(m)) * b_sum) >> 23;
                // (a token whose rCache row is not finite has no finite key whatever the exponent)
                e = fmaxf(e, bits < 255u ? (float)((int)bits - 126) : -200.f);
            }
        }
        const int ep = max(-100, min(126, (int)max_over_groups(max_over_row(e))));
        if (lane == 0) page_exp[wave] = ep;
        unsigned char *kd = lds + wave * 4096 + lane * 16;
        const float ks = __uint_as_float((uint32_t)max(0, min(254, (int)ke - ep)) << 23);
        const f32x4 vs = {f8_scale(ve & 255u), f8_scale((ve >> 8) & 255u), f8_scale((ve >> 16) & 255u), f8_scale(ve >> 24)};
#pragma unroll
        for (int q2 = 0; q2 < 4; ++q2) {
            const u32x2 v0 = value_word(vw[q2 / 2][2 * (q2 % 2)], vs), v1 = value_word(vw[q2 / 2][2 * (q2 % 2) + 1], vs);
            *reinterpret_cast<u32x4 *>(kd + S::V_OFF + 1024 * q2) = u32x4{v0.x, v0.y, v1.x, v1.y};
        }
        // K: word w of quarter kk is tile m = 2 kk + w, dims 16 m + 4 grp + 0..3 of token col
        auto base_key = [&](int m) __attribute__((always_inline)) {
            const uint32_t x = kw[m / 4][m % 4];
            const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x, ks, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x, ks, true);
            return f32x4{lo.x, lo.y, hi.x, hi.y};
        };
        auto store_keys = [&](int kk, const f32x4 &x, const f32x4 &y) __attribute__((always_inline)) {
            *reinterpret_cast<u32x4 *>(kd + 1024 * kk) =
                u32x4{pack_f16(x.x, x.y), pack_f16(x.z, x.w), pack_f16(y.x, y.y), pack_f16(y.z, y.w)};
        };
        if (!use_res) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) store_keys(kk, base_key(2 * kk), base_key(2 * kk + 1));
            return;
        }
        if constexpr (R > 0) {
            const float inv = __uint_as_float((uint32_t)(127 - ep) << 23);
            u32x2 ck[RT];  // C_K * 2^-e
#pragma unroll
            for (int t = 0; t < RT; ++t)
                ck[t] = u32x2{pack_bf16(bf16_lo(c[t].x) * inv, bf16_hi(c[t].x) * inv), pack_bf16(bf16_lo(c[t].y) * inv, bf16_hi(c[t].y) * inv)};
            auto low_rank = [&](int m, f32x4 u) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < RT; ++t) u = mfma16(bkt[(t * 8 + m) * 64 + lane], ck[t], u);
                return u;
            };
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {  // quarters kk and kk + 2: rotate-half partners
                f32x4 o[4];
                if (rope) {
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int m = 2 * kk + w;
                        const f32x4 x = low_rank(m, f32x4{0, 0, 0, 0}), y = low_rank(m + 4, f32x4{0, 0, 0, 0});
                        const f32x4 bx = base_key(m), by = base_key(m + 4);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            o[w][i] = __builtin_fmaf(x[i], cs[m][i], __builtin_fmaf(-y[i], sn[m][i], bx[i]));
                            o[w + 2][i] = __builtin_fmaf(y[i], cs[m][i], __builtin_fmaf(x[i], sn[m][i], by[i]));
                        }
                    }
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int m = 2 * kk + (w & 1) + 4 * (w >> 1);
                        o[w] = low_rank(m, base_key(m));
                    }
                }
                store_keys(kk, o[0], o[1]);
                store_keys(kk + 2, o[2], o[3]);
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if constexpr (R == 8) c[t] = u32x4{0, 0, col < 8 ? c[t].z : 0u, col < 8 ? c[t].w : 0u};
                *reinterpret_cast<u32x4 *>(lds + S::C_OFF + (wave * RT + t) * 1024 + lane * 16) = c[t];
            }
        }
    };

    // ---- queries: lane = row, in the contraction order of the stored K operands, as fp16 times 2^-eq ----
    int row_tok[2], eq[2];
    u32x4 qf[2][4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        const int rr = rg * ROWS_PER_WAVE + nt * 16 + col, tk = tok_begin + rr / G;
        const bool ok = tk < nq;
        row_tok[nt] = ok ? tk : -1;
        const uint16_t *qr = p.q + ((int64_t)(q0 + (ok ? tk : 0)) * p.hq + h * G + rr % G) * D;
        float big = 0.f;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            u32x4 v = {0, 0, 0, 0};
            if (ok) {
                const u32x2 lo = ldg64(qr + 32 * kk + 4 * grp), hi = ldg64(qr + 32 * kk + 16 + 4 * grp);
                v = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) big = fmaxf(big, fmaxf(fabsf(bf16_lo(v[i])), fabsf(bf16_hi(v[i]))));
            qf[nt][kk] = v;
        }
        eq[nt] = max(-100, min(126, (int)(__float_as_uint(max_over_groups(big)) >> 23) - 126));
        const float inv = __uint_as_float((uint32_t)(127 - eq[nt]) << 23);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i) qf[nt][kk][i] = pack_f16(bf16_lo(qf[nt][kk][i]) * inv, bf16_hi(qf[nt][kk][i]) * inv);
    }
    if constexpr (R > 0) {
        if (use_res) {  // lane (c, g) of fragment (tile t, column tile m): B_K[16t + 4g + 0..3][16m + c]
            u32x2 *dst = reinterpret_cast<u32x2 *>(lds + S::B_OFF);
            float *part = reinterpret_cast<float *>(lds);  // sums of the waves' ranks
            const uint16_t *bk = p.lora_b + (int64_t)ad * 2 * R * n + (int64_t)h * D;
            float mine = 0.f;
            for (int rho = wave; rho < R; rho += WAVES) {
                const uint32_t w = *reinterpret_cast<const uint32_t *>(bk + (int64_t)rho * n + 2 * lane);
                mine += max_over_groups(max_over_row(fmaxf(fabsf(bf16_lo(w)), fabsf(bf16_hi(w)))));
            }
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
                dst[idx] = u32x2{w[0], w[1]};
            }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) b_sum += part[w];
        }
    }

    f32x4 oacc[8][2], racc[RTX][2], lacc[2];
#pragma unroll
    for (int m = 0; m < 8; ++m) oacc[m][0] = oacc[m][1] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < RTX; ++t) racc[t][0] = racc[t][1] = f32x4{0, 0, 0, 0};
    lacc[0] = lacc[1] = f32x4{0, 0, 0, 0};
    float m_run[2] = {kNegInf, kNegInf};
    const float cl = p.scale_log2;
    const u32x4 kOnes = u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

    // Pages pg0 .. pg0 + GP - 1 of the round in LDS, keys from key0.
    auto step = [&](int pg0, int key0) __attribute__((always_inline)) {
        f32x4 sacc[GP][2];
        int ep[GP];
#pragma unroll
        for (int kt = 0; kt < GP; ++kt) {
            ep[kt] = page_exp[pg0 + kt];
            sacc[kt][0] = sacc[kt][1] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const u32x4 kf = *reinterpret_cast<const u32x4 *>(lds + (pg0 + kt) * 4096 + kk * 1024 + lane * 16);
                sacc[kt][0] = mfma32_f16(kf, qf[0][kk], sacc[kt][0]);
                sacc[kt][1] = mfma32_f16(kf, qf[1][kk], sacc[kt][1]);
            }
        }
        // causal mask and online softmax (rows in lanes): the maximum moves, and the accumulators are rescaled, only
        // where a row's scores exceed it by more than 2^kLazyRescale
        const bool full = key0 + GP * PS - 1 <= P0 + tok_begin;
        u32x2 pf[GP][2];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            if (!full) {
                const int lim = row_tok[nt] < 0 ? -1 : P0 + row_tok[nt] - key0 - 4 * grp;
#pragma unroll
                for (int kt = 0; kt < GP; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sacc[kt][nt][i] = kt * PS + i <= lim ? sacc[kt][nt][i] : kNegInf;
            }
            float mx = kNegInf, f[GP];
#pragma unroll
            for (int kt = 0; kt < GP; ++kt) {
                f[kt] = fminf(fmaxf(ldexpf(cl, ep[kt] + eq[nt]), 1.2e-38f), 3e38f);  // neither 0 nor infinite: masked scores and zeros stay
                float x = sacc[kt][nt][0];
#pragma unroll
                for (int i = 1; i < 4; ++i) x = fmaxf(x, sacc[kt][nt][i]);
                mx = fmaxf(mx, x * f[kt]);
            }
            mx = max_over_groups(mx);
            if (__builtin_amdgcn_ballot_w64(mx > m_run[nt] + kLazyRescale) != 0) {
                const float m_new = fmaxf(m_run[nt], mx);
                const float alpha = fast_exp2(m_run[nt] - (m_new == kNegInf ? 0.f : m_new));
#pragma unroll
                for (int m = 0; m < 8; ++m) oacc[m][nt] *= alpha;
#pragma unroll
                for (int t = 0; t < RT; ++t) racc[t][nt] *= alpha;
                lacc[nt] *= alpha;
                m_run[nt] = m_new;
            }
            const float m_use = m_run[nt] == kNegInf ? 0.f : m_run[nt];
#pragma unroll
            for (int kt = 0; kt < GP; ++kt) {
                f32x4 pv;
#pragma unroll
                for (int i = 0; i < 4; ++i) pv[i] = fast_exp2(__builtin_fmaf(sacc[kt][nt][i], f[kt], -m_use));
                pf[kt][nt] = pack4(pv);
            }
        }
        // values, two pages (32 keys) per product; row sums of the weights as the products take them
        u32x4 pb[2];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) pb[nt] = u32x4{pf[0][nt].x, pf[0][nt].y, pf[1][nt].x, pf[1][nt].y};
        const unsigned char *vb = lds + S::V_OFF + pg0 * 4096 + lane * 16;
#pragma unroll
        for (int q2 = 0; q2 < 4; ++q2) {
            const u32x4 v0 = *reinterpret_cast<const u32x4 *>(vb + q2 * 1024), v1 = *reinterpret_cast<const u32x4 *>(vb + 4096 + q2 * 1024);
            const u32x4 va = {v0.x, v0.y, v1.x, v1.y}, vc = {v0.z, v0.w, v1.z, v1.w};  // dims 32 q2 + col, 32 q2 + 16 + col
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                oacc[2 * q2][nt] = mfma32(va, pb[nt], oacc[2 * q2][nt]);
                oacc[2 * q2 + 1][nt] = mfma32(vc, pb[nt], oacc[2 * q2 + 1][nt]);
            }
        }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) lacc[nt] = mfma32(kOnes, pb[nt], lacc[nt]);
        if constexpr (R > 0) {
            if (use_res) {
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const unsigned char *cb = lds + S::C_OFF + (pg0 * RT + t) * 1024 + lane * 16 + 8;
                    const u32x2 c0 = *reinterpret_cast<const u32x2 *>(cb), c1 = *reinterpret_cast<const u32x2 *>(cb + RT * 1024);
                    const u32x4 ca = {c0.x, c0.y, c1.x, c1.y};
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) racc[t][nt] = mfma32(ca, pb[nt], racc[t][nt]);
                }
            }
        }
    };

    request(0);
    for (int round = 0; round < n_rounds; ++round) {
        lds_fence_barrier();  // the last round is read, the B_K^T fragments and rank sums are written (and read)
        stage(round);
        if (round + 1 < n_rounds) request(round + 1);
        lds_fence_barrier();  // (not one that waits for the loads in flight)
        const int key0 = (r0 + round) * ROUND_KEYS + kg * GP * PS;
        if (key0 <= last_pos) step(kg * GP, key0);
    }
    __syncthreads();

    // ---- key groups: the upper half leaves its rows in LDS, the lower half merges them into its own ----
#pragma unroll
    for (int half = KG / 2; half > 0; half /= 2) {
        f32x4 *buf = reinterpret_cast<f32x4 *>(lds) + lane;
        if (kg >= half && kg < 2 * half) {
            f32x4 *dst = buf + ((kg - half) * NRG + rg) * S::NF4 * 64;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
                for (int m = 0; m < 8; ++m) dst[(nt * (S::NF4 / 2) + m) * 64] = oacc[m][nt];
#pragma unroll
                for (int t = 0; t < RT; ++t) dst[(nt * (S::NF4 / 2) + 8 + t) * 64] = racc[t][nt];
                dst[(nt * (S::NF4 / 2) + 8 + RT) * 64] = f32x4{m_run[nt], lacc[nt][0], 0.f, 0.f};
            }
        }
        __syncthreads();
        if (kg < half) {
            const f32x4 *src = buf + (kg * NRG + rg) * S::NF4 * 64;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const f32x4 ml = src[(nt * (S::NF4 / 2) + 8 + RT) * 64];
                const float M = fmaxf(m_run[nt], ml.x), Mu = M == kNegInf ? 0.f : M;
                const float w0 = fast_exp2(m_run[nt] - Mu), w1 = fast_exp2(ml.x - Mu);
#pragma unroll
                for (int m = 0; m < 8; ++m) oacc[m][nt] = oacc[m][nt] * w0 + src[(nt * (S::NF4 / 2) + m) * 64] * w1;
#pragma unroll
                for (int t = 0; t < RT; ++t) racc[t][nt] = racc[t][nt] * w0 + src[(nt * (S::NF4 / 2) + 8 + t) * 64] * w1;
                lacc[nt][0] = lacc[nt][0] * w0 + ml.y * w1;
                m_run[nt] = M;
            }
        }
        __syncthreads();
    }

    // ---- epilogue: O = (acc + acc_r . B_V[h]) / l ----
    if constexpr (R > 0) {
        if (use_res) {
            float *bv = reinterpret_cast<float *>(lds), *acc = bv + R * D;
            const uint16_t *src = p.lora_b + ((int64_t)ad * 2 + 1) * R * n + (int64_t)h * D;
            for (int e = threadIdx.x; e < R * D; e += 64 * WAVES) bv[e] = bf16_to_f32(src[(int64_t)(e / D) * n + e % D]);
            if (kg == 0) {
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int t = 0; t < RT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * t + 4 * grp + i < R) acc[(rg * ROWS_PER_WAVE + nt * 16 + col) * (R + 1) + 16 * t + 4 * grp + i] = racc[t][nt][i];
            }
            __syncthreads();
            if (kg == 0) {
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll 2
                    for (int rho = 0; rho < R; ++rho) {
                        const float x = acc[(rg * ROWS_PER_WAVE + nt * 16 + col) * (R + 1) + rho];
#pragma unroll
                        for (int m = 0; m < 8; ++m) oacc[m][nt] += x * *reinterpret_cast<const f32x4 *>(bv + rho * D + 16 * m + 4 * grp);
                    }
            }
        }
    }
    if (kg > 0) return;
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        if (row_tok[nt] < 0) continue;
        if (p.splits > 1) {  // this split's partial rows
            float *rec = partial_row(p, split, a, row_tok[nt], h * G + (rg * ROWS_PER_WAVE + nt * 16 + col) % G);
#pragma unroll
            for (int m = 0; m < 8; ++m) *reinterpret_cast<f32x4 *>(rec + 16 * m + 4 * grp) = oacc[m][nt];
            if (grp == 0) *reinterpret_cast<f32x4 *>(rec + D) = f32x4{m_run[nt], lacc[nt][0], 0.f, 0.f};
            continue;
        }
        const float l = lacc[nt][0], inv = l > 0.f ? 1.f / l : 0.f;
        uint16_t *o = p.out + ((int64_t)(q0 + row_tok[nt]) * p.hq + h * G + (rg * ROWS_PER_WAVE + nt * 16 + col) % G) * D;
#pragma unroll
        for (int m = 0; m < 8; ++m) *reinterpret_cast<u32x2 *>(o + 16 * m + 4 * grp) = pack4(oacc[m][nt] * inv);
    }
}

// The splits' partial rows are merged: O = sum w acc / sum w l with w = 2^(m - max m).  Half a wave takes a query row: its lanes are the
// splits (32 at most), then four dims each.  A workgroup has eight query heads of one chunk token.  (acc_r . B_V[h] is in acc: done here
// it took 46 of 545 us at rank 64, as one wave per row 62, for four chunks of 250 in two splits.)
__global__ __launch_bounds__(256) void merge_splits_kernel(PrefillArgs p) {
    const int groups = (p.hq + 7) / 8, group = blockIdx.x % groups, at = blockIdx.x / groups;
    const int a = at / p.reach, tok = at % p.reach;
    const int q0 = p.q_indptr[a], nq = p.q_indptr[a + 1] - q0;
    if (tok >= nq) return;
    const int lane = threadIdx.x & 63, half = lane >> 5, c = lane & 31;
    const int row = 8 * group + 2 * uniform(threadIdx.x >> 6) + half, head = min(row, p.hq - 1);
    const int64_t step = (int64_t)p.n_agents * p.reach * p.hq * kPartFloats;
    const float *rec = partial_row(p, 0, a, tok, head);
    float m = kNegInf, l = 0.f;
    if (c < p.splits) {
        m = rec[c * step + D];
        l = rec[c * step + D + 1];
    }
    const uint64_t live = __builtin_amdgcn_ballot_w64(!(m == kNegInf && l == 0.f)) >> (32 * half);  // a split without keys has only m and l
    float M = m;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) M = fmaxf(M, __shfl_xor(M, x));
    const float w = fast_exp2(m - (M == kNegInf ? 0.f : M));
    float sum = w * l;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) sum += __shfl_xor(sum, x);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < p.splits; ++i) {
        const uint32_t u = __float_as_uint(w), lo = __builtin_amdgcn_readlane(u, i), hi = __builtin_amdgcn_readlane(u, 32 + i);
        const float wi = __uint_as_float(half ? hi : lo);
        const bool on = (live >> i) & 1;
        const f32x4 x = *reinterpret_cast<const f32x4 *>(rec + i * step + 4 * c);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += on ? wi * x[j] : 0.f;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    if (row < p.hq) *reinterpret_cast<u32x2 *>(p.out + ((int64_t)(q0 + tok) * p.hq + head) * D + 4 * c) = pack4(o * inv);
}

// Rows of a workgroup, and workgroups that share its keys.  An (agent, KV head) pair keeps to one XCD, so a grid takes as many passes
// as the fullest XCD's workgroups over its compute units, and a grid that leaves half of them or more idle splits the keys over
// them; its cost is the passes, times that of a key at so many rows, over the splits.  Fewer rows have to be 5 % better.
// Time per key, grids of one pass (us per 1024 keys at 256 / 128 / 64 rows): rank 0 29.8 / 20.4 / 15.2, 16 36.4 / 25.7 /
// 22.0, with RoPE 39.4 / 29.0 / 26.8, 64 with RoPE 67.4 / 47.7 / 67.0: rank 64 takes 128 rows at least.  (32 rows took as long as 64.)
// Measured as the rule chooses (rows x splits) and beside it, us: four chunks of up to 250 over 35k, rank 16, 256 x 2 698, 128 x 1 877,
// 256 x 3 856; one of 100 over 9k, rank 16, RoPE, 256 x 16 57, 64 x 1 237, 128 x 8 63, 64 x 8 89; one token of two agents over 60k,
// 64 x 16 133, 64 x 1 1480, 64 x 32 128; eight of up to 1024 over 9k, 256 x 1 1577, 128 x 1 1861, 256 x 2 1722; two of 300 over 500 tokens,
// rank 32, RoPE, 256 x 3 63, 128 x 1 59, 64 x 1 87.
struct Grid {
    int rows, splits;
};
Grid grid_of(int64_t pairs, int64_t max_q, int g, int r, int max_pages, bool split) {
    constexpr int kXcdCus = kCus / kXcds, kSplitPages = 16;  // a split has 256 keys or more
    constexpr struct {
        int rows;
        float cost;
    } kForms[3] = {{256, 1.f}, {128, 0.72f}, {64, 0.6f}};
    const int64_t per_xcd = (pairs + kXcds - 1) / kXcds;
    const int most = split ? std::min(kXcdCus, std::max(1, max_pages / kSplitPages)) : 1;
    Grid best = {256, 1};
    float least = INFINITY;
    for (const auto &f : kForms) {
        if (f.rows < 128 && r > 32) continue;
        const int64_t wgs = per_xcd * ((max_q * g + f.rows - 1) / f.rows);
        const int splits = (int)std::max<int64_t>(1, std::min<int64_t>(most, kXcdCus / wgs));
        const float c = f.cost * (float)((wgs * splits + kXcdCus - 1) / kXcdCus) / splits;
        if (c < least * 0.95f) least = c, best = {f.rows, splits};
    }
    return best;
}
int64_t parts_bytes(const Grid &gr, int n_agents, int64_t max_q, int hq, int g) {
    const int64_t reach = (max_q * g + gr.rows - 1) / gr.rows * (gr.rows / g);
    return (int64_t)gr.splits * n_agents * reach * hq * kPartFloats * 4;
}

template <int R, int G>
hipError_t launch(const PrefillArgs &pa, hipStream_t st, void *const *ev) {
    const int pairs = (pa.n_agents * pa.hkv + kXcds - 1) / kXcds * kXcds;
    // timing events carry the kernel's own start and end timestamps (set by the launch)
    hipEvent_t e0 = ev ? static_cast<hipEvent_t>(ev[0]) : nullptr, e1 = ev ? static_cast<hipEvent_t>(ev[1]) : nullptr;
    hipExtLaunchKernelGGL((prefill_fp8_kernel<R, G>), dim3(pairs * pa.blocks_per_agent_head * pa.splits), dim3(64 * WAVES), 0, st, e0, e1, 0, pa);
    return hipGetLastError();
}

template <int G>
hipError_t dispatch(int r, const PrefillArgs &pa, hipStream_t st, void *const *ev) {
    switch (r) {
    case 0: return launch<0, G>(pa, st, ev);
    case 8: return launch<8, G>(pa, st, ev);
    case 16: return launch<16, G>(pa, st, ev);
    case 32: return launch<32, G>(pa, st, ev);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_fp8(int r, int g, int64_t max_q, PrefillArgs pa, void *workspace, size_t workspace_bytes, hipStream_t st, void *const *ev) {
    const int64_t pairs = (int64_t)pa.n_agents * pa.hkv;
    Grid gr = grid_of(pairs, max_q, g, r, pa.max_pages, true);
    if (gr.splits > 1 && (!workspace || (int64_t)workspace_bytes < parts_bytes(gr, pa.n_agents, max_q, pa.hq, g)))
        gr = grid_of(pairs, max_q, g, r, pa.max_pages, false);
    pa.blocks_per_agent_head = (int)((max_q * g + gr.rows - 1) / gr.rows);
    pa.splits = gr.splits;
    pa.reach = pa.blocks_per_agent_head * (gr.rows / g);
    pa.parts = static_cast<float *>(workspace);
    void *first[2] = {ev ? ev[0] : nullptr, nullptr};
    void *const *ev1 = gr.splits > 1 ? (ev ? first : nullptr) : ev;
    hipError_t e = gr.rows >= 128 ? launch_fp8_stream(r, g, gr.rows, pa, st, ev1)
                   : g == 4       ? dispatch<4>(r, pa, st, ev1)
                                  : dispatch<8>(r, pa, st, ev1);
    if (e != hipSuccess || gr.splits == 1) return e;
    hipExtLaunchKernelGGL(merge_splits_kernel, dim3(pa.n_agents * pa.reach * ((pa.hq + 7) / 8)), dim3(256), 0, st, nullptr, ev ? static_cast<hipEvent_t>(ev[1]) : nullptr, 0,
                          pa);
    return hipGetLastError();
}

}  // namespace fkvp

extern "C" int64_t fkv_prefill_fp8_workspace_bytes(int32_t hq, int32_t hkv, int32_t r, int32_t n_agents, int32_t max_q, int32_t max_pages) {
    const int g = hkv > 0 && hq > 0 && hq % hkv == 0 ? hq / hkv : 0;
    if ((g != 4 && g != 8) || (r != 0 && r != 8 && r != 16 && r != 32 && r != 64) || n_agents < 1 || max_q < 1 || max_pages < 1) return 0;
    if ((int64_t)n_agents * hkv >= 1 << 24 || max_q >= 1 << 28) return 0;  // (no split there, and their products stay in 64 bits)
    const fkvp::Grid gr = fkvp::grid_of((int64_t)n_agents * hkv, max_q, g, r, max_pages, true);
    return gr.splits > 1 ? fkvp::parts_bytes(gr, n_agents, max_q, hq, g) : 0;
}
