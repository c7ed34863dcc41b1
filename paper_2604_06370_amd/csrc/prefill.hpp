// What the two prefill kernels and their entry point share.
#pragma once

#include <hip/hip_runtime.h>

#include "mfma.hpp"

namespace fkvp {

struct PrefillArgs {
    const uint16_t *q, *base_kv, *res_kv, *lora_b;
    const int32_t *adapter_idx, *base_bt, *res_bt, *seq_lens, *q_indptr;
    const float *rope_cos, *rope_sin;
    uint16_t *out;
    int32_t n_agents, hq, hkv, max_pages, blocks_per_agent_head;
    float scale_log2;
    int32_t rope_rows;  // positions the RoPE tables hold
    // 8-bit pages: each agent's keys are split over `splits` workgroups, which leave partial rows in `parts`, records of kPartFloats
    // floats [split][agent][token of the chunk, of `reach`][query head]: acc[128] (with acc_r . B_V[h]), m, l, and two to align
    float *parts;
    int32_t splits, reach;
};

constexpr int kPartFloats = 128 + 4;
constexpr int kXcds = 8;
constexpr int kCus = 256;  // compute units of the GPU

// Rows of an agent's chunk that its query blocks do not reach (a max_q_per_agent below the
// agent's row count) are written as NaN by the agent's last block, so the shortfall shows in
// the output instead of leaving stale memory there.
__device__ __forceinline__ void poison_unreached_rows(const PrefillArgs &p, int q0, int nq, int h, int g, int reach) {
    using namespace fkvk;
    const uint32_t nan2 = 0x7fc07fc0u;  // two bf16 quiet NaNs
    for (int64_t i = threadIdx.x; i < (int64_t)(nq - reach) * g * 32; i += blockDim.x) {
        const int64_t row = i / 32, c = i % 32;
        const int tok = reach + (int)(row / g), j = (int)(row % g);
        uint16_t *orow = p.out + ((int64_t)(q0 + tok) * p.hq + h * g + j) * 128;
        *reinterpret_cast<u32x2 *>(orow + 4 * c) = u32x2{nan2, nan2};
    }
}

// Launch of the pipelined kernel (prefill_stream.hip) with 128 or 256 query rows per workgroup.
hipError_t launch_stream(int r, int g, bool rope, bool rows128, const PrefillArgs &pa, hipStream_t st, void *const *ev);

__device__ __forceinline__ float *partial_row(const PrefillArgs &p, int split, int a, int tok, int head) {
    return p.parts + ((((int64_t)split * p.n_agents + a) * p.reach + tok) * p.hq + head) * kPartFloats;
}
// A workgroup without keys in its split leaves rows of no weight.
__device__ __forceinline__ void empty_rows(const PrefillArgs &p, int split, int a, int h, int g, int tok_begin, int tok_end) {
    for (int i = threadIdx.x; i < (tok_end - tok_begin) * g; i += blockDim.x)
        *reinterpret_cast<fkvk::f32x4 *>(partial_row(p, split, a, tok_begin + i / g, h * g + i % g) + 128) =
            fkvk::f32x4{-INFINITY, 0.f, 0.f, 0.f};
}

// Launch of the kernels over 8-bit base pages (prefill_fp8.hip) for chunks of up to max_q tokens, which sets the fields of the grid. Keys are
// split only where `workspace` has the bytes for it.
hipError_t launch_fp8(int r, int g, int64_t max_q, PrefillArgs pa, void *workspace, size_t workspace_bytes, hipStream_t st, void *const *ev);

// The one of all but small grids (prefill_fp8_stream.hip): 256 or 128 query rows per workgroup.
hipError_t launch_fp8_stream(int r, int g, int rows, const PrefillArgs &pa, hipStream_t st, void *const *ev);

}  // namespace fkvp
