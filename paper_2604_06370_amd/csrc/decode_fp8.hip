// The decode kernels over 8-bit base pages (decode_kernels.hpp with F8; fp8_cache.hpp has the format).
#include "decode_kernels.hpp"

namespace fkvd {

hipError_t launch_pages_fp8(int r, int g, bool rope, const DecodeArgs &da, int n_blocks, int wave_agents, hipStream_t st,
                            hipEvent_t e0, hipEvent_t e1) {
    return dispatch_pages<true>(r, g, rope, da, n_blocks, wave_agents, st, e0, e1);
}

}  // namespace fkvd
