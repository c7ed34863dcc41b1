// ResidualAttention decode for gfx950 (Section 5.3, Algorithm 1): the merge of the partial rows, and
// the entry points.  The kernels over the pages are in decode_kernels.hpp, their 8-bit instances are
// built by decode_fp8.hip.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <mutex>
#include <string>

#include "decode_kernels.hpp"
#include "internal.hpp"

using namespace fkvk;
using namespace fkvd;

namespace {

// Log-sum-exp merge of one agent's partials and Stage 3 of Algorithm 1 for one query
// row (agent a, query head j of KV head h = j / G), by one workgroup of CW waves:
//   O = (sum_k w_k acc_k + (sum_k w_k acc_r,k) . B_V[h]) / L,
//   w_k = 2^(m_k - M), M = max_k m_k, L = sum_k w_k l_k.
// An agent's partials are contiguous; wave w merges partials w, w + CW, ... (all of its
// share in flight at once): lane i < NV reads float4 i of every record (acc, then acc_r)
// and lane NV its (m, l); lanes past NV read float4 0 and drop it.  The waves' results
// meet in LDS and wave 0 merges them and applies Stage 3.  B_V is read at the start, as
// it does not depend on the partials.
// Waves per row: four, or sixteen when the rows are fewer than half the compute units and each
// has many partials (one KV head per GPU: a row's partials are then all the parallelism there
// is; measured on 16 agents x 4 query heads with 278 partials per row, 12.3 -> 8.8 us).
constexpr int kCombineWaves = 4, kCombineWavesFewRows = 16;
constexpr int kCus = 256;  // compute units of the GPU
constexpr int combine_batch(int cw) { return cw == kCombineWaves ? 12 : 8; }  // partials in flight per wave

__device__ __forceinline__ void lse_merge(float &M, float &L, f32x4 &acc, float mk, float lk, const f32x4 &v) {
    const float Mn = fmaxf(M, mk);
    const float Mu = Mn == kNegInf ? 0.f : Mn;
    const float e0 = fast_exp2(M - Mu), e1 = fast_exp2(mk - Mu);
    L = L * e0 + lk * e1;
    acc = acc * e0 + v * e1;
    M = Mn;
}

template <int R, int G, int CW>
__global__ __launch_bounds__(64 * CW) void decode_combine_kernel(DecodeArgs p) {
    constexpr int NV = (D + R) / 4;  // float4s of acc and acc_r; (m, l) follow
    constexpr int RB = R > 0 ? R : 1;
    constexpr int BATCH = combine_batch(CW);
    __shared__ f32x4 s_acc[CW > 1 ? CW - 1 : 1][NV + 1];
    const int row = blockIdx.x;
    const int wave = uniform(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int hq = p.hq;
    const int a = row / hq, j = row - a * hq;
    const int h = j / G, jj = j - h * G;
    const int32_t *ptr = p.plan + p.off_ptr;
    const int k0 = ptr[a], K = ptr[a + 1] - k0;
    const int ad = R > 0 ? p.adapter_idx[a] : -1;
    const int stride = p.ws_stride;
    const i32x4 rs = workspace_rsrc(p.ws, p.ws_bytes);
    // byte offsets: record of partial k0 for this row, lane's float4 (lanes past NV: float4 0)
    const int rec0 = (int)(((int64_t)k0 * G * p.hkv + jj * p.hkv + h) * stride * 4) + (lane <= NV ? 16 * lane : 0);
    const int kstride = G * p.hkv * stride * 4;

    // B_V[rho][h*D + 4 lane .. +3] for the output dims of lanes 0..31 of wave 0, requested at
    // the start: in registers of wave 0 for the four-wave merge; for the sixteen-wave one (at
    // most 128 registers per lane) in LDS, each wave copying a share of it.
    constexpr bool kBvRegs = CW == kCombineWaves;
    __shared__ u32x2 s_bv[(R > 0 && !kBvRegs) ? R * (D / 4) : 1];
    const uint16_t *bv_row = p.lora_b + ((int64_t)(ad >= 0 ? ad : 0) * 2 + 1) * R * p.hkv * D + (int64_t)h * D;
    u32x2 bv[kBvRegs ? RB : 1];
    if constexpr (R > 0 && kBvRegs) {
        if (wave == 0) {
#pragma unroll
            for (int rho = 0; rho < R; ++rho)
                bv[rho] = ad >= 0 ? ldg64(bv_row + (int64_t)rho * p.hkv * D + 4 * (lane & 31)) : u32x2{0, 0};
        }
    } else if constexpr (R > 0) {
        for (int i = threadIdx.x; i < R * (D / 4); i += 64 * CW)
            s_bv[i] = ad >= 0 ? ldg64(bv_row + (int64_t)(i / (D / 4)) * p.hkv * D + 4 * (i % (D / 4))) : u32x2{0, 0};
    }

    f32x4 acc = {0, 0, 0, 0};
    float M = kNegInf, L = 0.f;
    for (int kb = wave; kb < K; kb += BATCH * CW) {
        f32x4 v[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u)
            v[u] = kb + u * CW < K ? raw_buffer_load_v4f32(rs, rec0 + (kb + u * CW) * kstride, 0, kDeviceCoherent)
                                   : f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            // past the last partial: weight zero (m = -inf in lane NV, zeros elsewhere)
            if (!(kb + u * CW < K && lane <= NV)) v[u] = f32x4{lane == NV ? kNegInf : 0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) lse_merge(M, L, acc, __shfl(v[u].x, NV), __shfl(v[u].y, NV), v[u]);
    }
    if constexpr (CW > 1) {
        // lane NV's acc holds (L, 0, 0, 0) scaled alongside; carry (M, L) there instead
        if (wave > 0 && lane <= NV) s_acc[wave - 1][lane] = lane == NV ? f32x4{M, L, 0.f, 0.f} : acc;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll 3
        for (int w = 0; w < CW - 1; ++w) {
            const f32x4 v = lane <= NV ? s_acc[w][lane] : f32x4{0, 0, 0, 0};
            lse_merge(M, L, acc, __shfl(v.x, NV), __shfl(v.y, NV), lane < NV ? v : f32x4{0, 0, 0, 0});
        }
    }
    // Stage 3 (Eq. 4): lanes 0..31 own output dims 4 lane .. +3; acc_r sits in lanes 32..
    f32x4 o = acc;
    auto apply_bv = [&](int rho, u32x2 b) __attribute__((always_inline)) {
        const float ar = __shfl(acc[rho % 4], D / 4 + rho / 4);
        o[0] += ar * bf16_lo(b.x);
        o[1] += ar * bf16_hi(b.x);
        o[2] += ar * bf16_lo(b.y);
        o[3] += ar * bf16_hi(b.y);
    };
    if constexpr (R > 0 && kBvRegs) {
#pragma unroll
        for (int rho = 0; rho < R; ++rho) apply_bv(rho, bv[rho]);
    } else if constexpr (R > 0) {
        // eight ranks per LDS wait keeps the sixteen-wave merge within its registers
        for (int r0 = 0; r0 < R; r0 += 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) apply_bv(r0 + i, s_bv[(r0 + i) * (D / 4) + (lane & 31)]);
        }
    }
    const float inv = L > 0.f ? 1.f / L : 0.f;
    if (lane < D / 4) {
        uint16_t *dst = p.out + ((int64_t)a * hq + j) * D + 4 * lane;
        *reinterpret_cast<u32x2 *>(dst) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
    }
}

template <int R, int G>
hipError_t launch_merge(const DecodeArgs &da, bool wide_merge, hipStream_t st, hipEvent_t e2) {
    if (!wide_merge)
        hipExtLaunchKernelGGL((decode_combine_kernel<R, G, kCombineWaves>), dim3(da.n_rows), dim3(64 * kCombineWaves), 0, st,
                              nullptr, e2, 0, da);
    else
        hipExtLaunchKernelGGL((decode_combine_kernel<R, G, kCombineWavesFewRows>), dim3(da.n_rows),
                              dim3(64 * kCombineWavesFewRows), 0, st, nullptr, e2, 0, da);
    return hipGetLastError();
}

template <int G>
hipError_t dispatch_merge(int r, const DecodeArgs &da, bool wide, hipStream_t st, hipEvent_t e2) {
    switch (r) {
    case 0: return launch_merge<0, G>(da, wide, st, e2);
    case 8: return launch_merge<8, G>(da, wide, st, e2);
    case 16: return launch_merge<16, G>(da, wide, st, e2);
    case 32: return launch_merge<32, G>(da, wide, st, e2);
    case 64: return launch_merge<64, G>(da, wide, st, e2);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace

namespace fkv {
fkv_status validate_attn_common(const fkv_attn_args *a, const char *who);
int64_t plan_max_pages(const fkv_plan *plan);
}  // namespace fkv

namespace {

// The decode entry points: checks, then the split and merge launches with the partial rows
// in `workspace` (`workspace_bytes` long).  fp8: args' base pool holds 8-bit pages.
fkv_status decode_impl(const fkv_attn_args *a, const fkv_plan *plan, void *stream, void *workspace,
                       size_t workspace_bytes, bool fp8 = false) {
    const std::string who = fp8 ? "fkv_residual_attention_decode_fp8" : "fkv_residual_attention_decode";
    fkv_status st = fkv::validate_attn_common(a, who.c_str());
    if (st != FKV_OK) return st;
    if (!plan || !a->plan || !workspace)
        return fkv::fail(FKV_ERR_INVALID, who + ": plan (host and device copy) and workspace are required");
    const auto &w = plan->words;
    const int g = a->hq / a->hkv;
    if (plan->n_agents != a->n_agents || plan->hkv != a->hkv || plan->g != g)
        return fkv::fail(FKV_ERR_INVALID, who + ": plan was built for other n_agents / heads");
    fkv_plan_info info;
    fkv_decode_plan_info(plan, a->d, a->r, &info);
    if ((int64_t)workspace_bytes < info.workspace_bytes)
        return fkv::fail(FKV_ERR_INVALID, who + ": workspace too small");
    if (a->max_pages < fkv::plan_max_pages(plan))
        return fkv::fail(FKV_ERR_INVALID, who + ": block-table rows shorter than the plan's "
                                          "page capacity");
    if (a->rope_cos && (int64_t)a->rope_max_pos < fkv::plan_max_pages(plan) * a->page_size)
        return fkv::fail(FKV_ERR_INVALID, who + ": RoPE table shorter than the longest sequence");
    if (g != 4 && g != 8)
        return fkv::fail(FKV_ERR_UNSUPPORTED, who + ": query heads per KV head must be 4 or 8");
    const bool rope_on = a->rope_cos != nullptr && a->r > 0;
    if (w[fkv::H_RANK] != a->r || w[fkv::H_ROPE] != (rope_on ? 1 : 0))
        return fkv::fail(FKV_ERR_INVALID, who + ": the plan was built for another rank or "
                                          "RoPE setting");
    const int hpb = w[fkv::H_HEADS_PER_BLOCK];
    if (hpb != fkv::decode_heads_per_block(a->hkv, rope_on))
        return fkv::fail(FKV_ERR_INVALID, who + ": plan built for another head blocking");
    if (w[fkv::H_MAX_ITEM_AGENTS] > fkv::decode_item_agent_cap(g, a->hkv, a->r, rope_on))
        return fkv::fail(FKV_ERR_INVALID, who + ": the plan puts more agents in a work item "
                                          "than this kernel takes");
    if (w[fkv::H_PAGES_PER_SPLIT] > fkv::kMaxPagesSingle)
        return fkv::fail(FKV_ERR_INVALID, who + ": plan items longer than the kernel takes");
    if (w[fkv::H_OFF_DESC] < 0)
        return fkv::fail(FKV_ERR_INVALID, who + ": plan has no block descriptors");
    DecodeArgs da;
    da.q = static_cast<const uint16_t *>(a->q);
    da.base_kv = static_cast<const uint16_t *>(a->base_kv);
    da.res_kv = static_cast<const uint16_t *>(a->res_kv);
    da.lora_b = static_cast<const uint16_t *>(a->lora_b);
    da.adapter_idx = a->adapter_idx;
    da.base_bt = a->base_bt;
    da.res_bt = a->res_bt;
    da.seq_lens = a->seq_lens;
    da.rope_cos = a->rope_cos;
    da.rope_sin = a->rope_sin;
    da.plan = a->plan;
    da.ws = static_cast<float *>(workspace);
    da.out = static_cast<uint16_t *>(a->out);
    da.hq = a->hq;
    da.hkv = a->hkv;
    da.max_pages = a->max_pages;
    da.ws_stride = ws_stride_of(a->r);
    da.off_items = w[fkv::H_OFF_ITEMS];
    da.off_blocks = w[fkv::H_OFF_BLOCKS];
    da.off_ptr = w[fkv::H_OFF_AGENT_PTR];
    da.off_zero = w[fkv::H_OFF_ZERO];
    da.off_desc = w[fkv::H_OFF_DESC];
    da.scale_log2 = a->scale * 1.4426950408889634f;
    da.rope_max_pos = a->rope_cos ? a->rope_max_pos : 0;
    da.ws_bytes = fkv::decode_partials_bytes(plan, a->d, a->r);
    if (da.ws_bytes >= 0x7fffffff)
        return fkv::fail(FKV_ERR_UNSUPPORTED, who + ": partial rows above 2 GiB");
    da.n_rows = a->n_agents * a->hq;
    const int nb = w[fkv::H_N_BLOCKS];
    hipStream_t hs = static_cast<hipStream_t>(stream);
    // Merge with sixteen waves per row when there are fewer rows than half the compute units
    // and each row has many partials (at least 128 on average); four otherwise.
    const int64_t total_partials = w[w[fkv::H_OFF_AGENT_PTR] + a->n_agents];
    const bool wide = (int64_t)a->n_agents * a->hq < kCus / 2 && total_partials >= 128LL * a->n_agents;
    const int wa = w[fkv::H_AGENTS_PER_ITEM];  // agents per wave that the plan was laid out for
    // timing events carry the kernels' own start and end timestamps (set by the launch)
    void *const *ev = a->timing_events;
    hipEvent_t e0 = ev ? static_cast<hipEvent_t>(ev[0]) : nullptr, e1 = ev ? static_cast<hipEvent_t>(ev[1]) : nullptr,
               e2 = ev ? static_cast<hipEvent_t>(ev[2]) : nullptr;
    hipError_t e = fp8 ? launch_pages_fp8(a->r, g, rope_on, da, nb, wa, hs, e0, e1) : dispatch_pages<false>(a->r, g, rope_on, da, nb, wa, hs, e0, e1);
    if (e == hipSuccess) e = g == 4 ? dispatch_merge<4>(a->r, da, wide, hs, e2) : dispatch_merge<8>(a->r, da, wide, hs, e2);
    if (e != hipSuccess) return fkv::fail(FKV_ERR_HIP, who + ": launch failed: " + hipGetErrorString(e));
    return FKV_OK;
}

// Partial rows of fkv_residual_attention_decode_noalloc: one array per GPU, held from the
// library's first use on that GPU until the process ends.  Host code never passes the
// array's name to a kernel (on the host it names a stand-in, not device memory): each
// device's address comes from hipGetSymbolAddress with that device current.
constexpr size_t kNoAllocBytes = FKV_NOALLOC_WORKSPACE_BYTES;
__device__ __attribute__((aligned(256))) unsigned char scratch[kNoAllocBytes];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void *g_scratch_addr[kMaxDevices] = {};

fkv_status scratch_address(void **out) {
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess)
        return fkv::fail(FKV_ERR_HIP, std::string("fkv_residual_attention_decode_noalloc: hipGetDevice: ") + hipGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices)
        return fkv::fail(FKV_ERR_UNSUPPORTED, "fkv_residual_attention_decode_noalloc: device index above 63");
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_addr[dev]) {
        void *p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !p)
            return fkv::fail(FKV_ERR_HIP, std::string("fkv_residual_attention_decode_noalloc: hipGetSymbolAddress: ") +
                                              hipGetErrorString(e));
        g_scratch_addr[dev] = p;
    }
    *out = g_scratch_addr[dev];
    return FKV_OK;
}

}  // namespace

extern "C" fkv_status fkv_residual_attention_decode(const fkv_attn_args *a, const fkv_plan *plan, void *stream) {
    fkv::clear_error();
    if (!a) return fkv::fail(FKV_ERR_INVALID, "fkv_residual_attention_decode: null args");
    return decode_impl(a, plan, stream, a->workspace, a->workspace_bytes);
}

extern "C" fkv_status fkv_residual_attention_decode_fp8(const fkv_attn_args *a, const fkv_plan *plan, void *stream) {
    fkv::clear_error();
    if (!a) return fkv::fail(FKV_ERR_INVALID, "fkv_residual_attention_decode_fp8: null args");
    if ((uintptr_t)a->base_kv & 15)
        return fkv::fail(FKV_ERR_INVALID, "fkv_residual_attention_decode_fp8: the base pool must be aligned to 16 bytes");
    return decode_impl(a, plan, stream, a->workspace, a->workspace_bytes, true);
}

extern "C" fkv_status fkv_residual_attention_decode_noalloc(const fkv_attn_args *a, const fkv_plan *plan, void *stream) {
    fkv::clear_error();
    if (!a || !plan) return fkv::fail(FKV_ERR_INVALID, "fkv_residual_attention_decode_noalloc: null argument");
    fkv_plan_info info;
    fkv_status st = fkv_decode_plan_info(plan, a->d, a->r, &info);
    if (st != FKV_OK) return st;
    if (info.workspace_bytes > (int64_t)kNoAllocBytes)
        return fkv::fail(FKV_ERR_INVALID, "fkv_residual_attention_decode_noalloc: the plan's partial rows (" +
                                              std::to_string(info.workspace_bytes) + " bytes) exceed the " +
                                              std::to_string(kNoAllocBytes) + "-byte static workspace");
    void *ws = nullptr;
    st = scratch_address(&ws);
    if (st != FKV_OK) return st;
    return decode_impl(a, plan, stream, ws, kNoAllocBytes);
}
