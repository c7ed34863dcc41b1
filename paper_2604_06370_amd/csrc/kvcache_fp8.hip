// The 8-bit base cache beside the attention: reading rows back, and copy-on-write page copies (Section 5.2).
// What writes it is the producer (kvcache.hip); the page layout stands in fp8_cache.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "fp8_cache.hpp"
#include "internal.hpp"
#include "mfma.hpp"

using namespace fkvk;

namespace {

constexpr int PS = 16, D = 128;

// ---------------------------------------------------------------------------
// Read back: K and V of positions pos0 .. pos0 + n - 1 of up to 32 sequences as bf16 rows, exactly the values
// that the cache stands for.  The inverse of the cache write: a wave takes four slots of a page and one head; a lane reads two
// words of K (dims 4c .. + 3 and 64 further of its token) and two of V (one dim of four tokens, transposed over
// the lanes), and stores 8 bytes of each half of its token's rows, 128 contiguous bytes per token.
constexpr int kReadMaxSeqs = 32, kReadHeads = 2;
struct ReadSeq {
    const int32_t *bt;
    int64_t pos0, row0;
    int32_t n, first;  // rows; its first workgroup
};
struct ReadArgs {
    ReadSeq seq[kReadMaxSeqs];
    int32_t nseq, hkv;
    const unsigned char *base;
    uint16_t *k, *v;
};

__global__ __launch_bounds__(256) void gather_fp8_kernel(ReadArgs a) {
    const int bid = blockIdx.x;
    int s = 0;
    for (int j = 1; j < a.nseq; ++j)
        if (a.seq[j].first <= bid) s = j;
    const ReadSeq &q = a.seq[s];
    const int n_hg = (a.hkv + kReadHeads - 1) / kReadHeads;
    const int lb = bid - q.first, h0 = (lb % n_hg) * kReadHeads, nh = min(kReadHeads, a.hkv - h0);
    const int64_t pp = q.pos0 / PS + lb / n_hg;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int k = lane >> 4, c = lane & 15, t = 4 * wave + k;
    const int64_t tf = pp * PS - q.pos0 + 4 * wave, tj = tf + k;  // rows of the wave's first token and of the lane's
    if (tf + 3 < 0 || tf >= q.n) return;
    const unsigned char *pg = a.base + (int64_t)q.bt[pp] * f8_page_bytes(a.hkv);
    uint32_t w[kReadHeads][4];
    uint32_t ek[kReadHeads], ev[kReadHeads];
#pragma unroll
    for (int i = 0; i < kReadHeads; ++i) {
        if (i >= nh) break;
        const unsigned char *blk = pg + (int64_t)(h0 + i) * kF8HeadBytes;
        const unsigned char *kb = blk + f8_k_word(t, c), *vb = blk + kF8Block + f8_v_word(wave, k, c);
        w[i][0] = *reinterpret_cast<const uint32_t *>(kb);
        w[i][1] = *reinterpret_cast<const uint32_t *>(kb + 1024);
        w[i][2] = *reinterpret_cast<const uint32_t *>(vb);
        w[i][3] = *reinterpret_cast<const uint32_t *>(vb + 1024);
        const unsigned char *ex = pg + f8_exp_off(a.hkv, h0 + i) + t;
        ek[i] = ex[0];
        ev[i] = ex[16];
    }
    const bool ok = tj >= 0 && tj < q.n;
#pragma unroll
    for (int i = 0; i < kReadHeads; ++i) {
        if (i >= nh) break;
        const uint32_t v0 = f8_transpose(w[i][2], k), v1 = f8_transpose(w[i][3], k);
        if (!ok) continue;
        const int64_t dst = ((q.row0 + tj) * a.hkv + h0 + i) * D + 4 * c;
        *reinterpret_cast<u32x2 *>(a.k + dst) = f8_to_bf16(w[i][0], f8_scale(ek[i]));
        *reinterpret_cast<u32x2 *>(a.k + dst + 64) = f8_to_bf16(w[i][1], f8_scale(ek[i]));
        *reinterpret_cast<u32x2 *>(a.v + dst) = f8_to_bf16(v0, f8_scale(ev[i]));
        *reinterpret_cast<u32x2 *>(a.v + dst + 64) = f8_to_bf16(v1, f8_scale(ev[i]));
    }
}

// ---------------------------------------------------------------------------
// Page copies: the first n_valid slots of page src into page dst, 16 bytes per thread and step.  A K chunk
// belongs to one slot, a V chunk to four (its words are [tokens 4g .. 4g + 3] of four dims), the exponent bytes
// of a head's K (V) are one chunk.  Residual pages go through fkv_page_copy_list as they are.
constexpr int kCopyMax = 128;  // copies per launch (2 KB of kernel arguments)
struct CopyList {
    fkv_page_copy c[kCopyMax];
};

__device__ __forceinline__ u32x4 merge_bytes(const u32x4 &from, const u32x4 &to, uint32_t mask) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (from[i] & mask) | (to[i] & ~mask);
    return r;
}

__global__ __launch_bounds__(256) void page_copy_fp8_kernel(unsigned char *base, int hkv, CopyList l) {
    const fkv_page_copy c = l.c[blockIdx.x];
    const int nv = min(c.n_valid, PS);
    if (nv <= 0 || c.src == c.dst) return;
    const int64_t page = f8_page_bytes(hkv);
    const u32x4 *src = reinterpret_cast<const u32x4 *>(base + (int64_t)c.src * page);
    u32x4 *dst = reinterpret_cast<u32x4 *>(base + (int64_t)c.dst * page);
    const int codes = hkv * (kF8HeadBytes / 16), all = codes + hkv * 2;
    for (int i = (int)(blockIdx.y * blockDim.x + threadIdx.x); i < all; i += (int)(gridDim.y * blockDim.x)) {
        if (i >= codes) {
            u32x4 m;  // bytes below n_valid
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = max(0, min(4, nv - 4 * j));
                m[j] = b == 4 ? 0xffffffffu : (1u << (8 * b)) - 1u;
            }
            const u32x4 from = src[i], to = dst[i];
            u32x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = (from[j] & m[j]) | (to[j] & ~m[j]);
            dst[i] = o;
            continue;
        }
        const bool value = (i >> 7) & 1;  // 128 chunks per block: K, then V of a head
        const int lane = i & 63;
        if (!value) {
            if ((lane & 15) < nv) dst[i] = src[i];
        } else {
            const int n = nv - 4 * (lane >> 4);
            if (n >= 4) dst[i] = src[i];
            else if (n > 0) dst[i] = merge_bytes(src[i], dst[i], (1u << (8 * n)) - 1u);
        }
    }
}

fkv_status launched(const char *fn) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? FKV_OK : fkv::fail(FKV_ERR_HIP, std::string(fn) + ": " + hipGetErrorString(e));
}

}  // namespace

extern "C" {

int64_t fkv_fp8_page_bytes(int32_t page_size, int32_t hkv, int32_t d) {
    return page_size == PS && d == D && hkv >= 1 ? f8_page_bytes(hkv) : 0;
}

fkv_status fkv_gather_tokens_fp8(const fkv_read_seq *seqs, int32_t nseq, const void *base_fp8, void *k_out, void *v_out, int32_t hkv,
                                 int32_t d, int32_t page_size, void *stream) {
    fkv::clear_error();
    const std::string fn = "fkv_gather_tokens_fp8";
    if (nseq < 0 || (nseq > 0 && !seqs) || hkv < 1 || d != D || page_size != PS)
        return fkv::fail(FKV_ERR_INVALID, fn + ": needs d = 128, page_size = 16");
    if (!base_fp8 || !k_out || !v_out) return fkv::fail(FKV_ERR_INVALID, fn + ": pool, K or V missing");
    if (((uintptr_t)base_fp8 | (uintptr_t)k_out | (uintptr_t)v_out) & 15)
        return fkv::fail(FKV_ERR_INVALID, fn + ": device pointers must be aligned to 16 bytes");
    const int64_t n_hg = (hkv + kReadHeads - 1) / kReadHeads;
    auto groups = [&](const fkv_read_seq &q) {
        return q.n == 0 ? (int64_t)0 : ((q.pos0 + q.n - 1) / PS - q.pos0 / PS + 1) * n_hg;
    };
    for (int32_t i = 0; i < nseq; ++i) {
        const fkv_read_seq &q = seqs[i];
        const std::string who = fn + ": sequence " + std::to_string(i) + ": ";
        if (q.pos0 < 0 || q.n < 0 || q.row0 < 0) return fkv::fail(FKV_ERR_INVALID, who + "negative position, count or row");
        if (q.n > (int64_t)1 << 24 || groups(q) > INT32_MAX / kReadMaxSeqs)
            return fkv::fail(FKV_ERR_INVALID, who + "too many tokens in one call");
        if (q.n > 0 && !q.bt_base) return fkv::fail(FKV_ERR_INVALID, who + "base table missing");
    }
    for (int32_t c0 = 0; c0 < nseq; c0 += kReadMaxSeqs) {
        ReadArgs a{};
        a.hkv = hkv;
        a.base = static_cast<const unsigned char *>(base_fp8);
        a.k = static_cast<uint16_t *>(k_out);
        a.v = static_cast<uint16_t *>(v_out);
        int64_t blocks = 0;
        for (int32_t i = c0; i < std::min(nseq, c0 + kReadMaxSeqs); ++i) {
            if (seqs[i].n == 0) continue;
            a.seq[a.nseq++] = ReadSeq{seqs[i].bt_base, seqs[i].pos0, seqs[i].row0, (int32_t)seqs[i].n, (int32_t)blocks};
            blocks += groups(seqs[i]);
        }
        if (a.nseq == 0) continue;
        hipLaunchKernelGGL(gather_fp8_kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), a);
        const fkv_status st = launched("fkv_gather_tokens_fp8");
        if (st != FKV_OK) return st;
    }
    return FKV_OK;
}

fkv_status fkv_page_copy_list_fp8(const fkv_page_copy *copies, int32_t n, void *base_fp8, void *res_kv, int32_t hkv, int32_t d,
                                  int32_t r, int32_t page_size, void *stream) {
    fkv::clear_error();
    const std::string fn = "fkv_page_copy_list_fp8";
    if (n < 0 || (n > 0 && !copies) || hkv < 1 || r < 0 || d != D || page_size != PS)
        return fkv::fail(FKV_ERR_INVALID, fn + ": needs d = 128, page_size = 16");
    if (n == 0) return FKV_OK;
    if (!base_fp8 || (r > 0 && !res_kv)) return fkv::fail(FKV_ERR_INVALID, fn + ": pool pointer missing");
    if ((uintptr_t)base_fp8 & 15) return fkv::fail(FKV_ERR_INVALID, fn + ": the pool must be aligned to 16 bytes");
    for (int32_t i = 0; i < n; ++i)
        if (copies[i].src < 0 || copies[i].dst < 0 || (copies[i].pool != FKV_POOL_BASE && copies[i].pool != FKV_POOL_RES))
            return fkv::fail(FKV_ERR_INVALID, fn + ": copy " + std::to_string(i) + " names no page");
    const unsigned parts = (unsigned)std::min<int64_t>(16, ((int64_t)hkv * (kF8HeadBytes / 16 + 2) + 255) / 256);
    // base copies 128 per launch; residual ones likewise, on their own kernel
    CopyList l{};
    fkv_page_copy res[kCopyMax];
    int32_t nl = 0, nres = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (copies[i].pool == FKV_POOL_BASE) l.c[nl++] = copies[i];
        else res[nres++] = copies[i];
        if (nl == kCopyMax || (i == n - 1 && nl > 0)) {
            hipLaunchKernelGGL(page_copy_fp8_kernel, dim3((unsigned)nl, parts), dim3(256), 0, static_cast<hipStream_t>(stream),
                               static_cast<unsigned char *>(base_fp8), hkv, l);
            const fkv_status st = launched("fkv_page_copy_list_fp8");
            if (st != FKV_OK) return st;
            nl = 0;
        }
        if (nres == kCopyMax || (i == n - 1 && nres > 0)) {
            const fkv_status st = fkv_page_copy_list(res, nres, base_fp8, res_kv, hkv, d, r, page_size, stream);
            if (st != FKV_OK) return st;
            nres = 0;
        }
    }
    return FKV_OK;
}

}  // extern "C"
