// The batch calls over a cache of 8-bit codes.
#include "quant_cache.hpp"

namespace cake {

hipError_t launch_append_q8(int dtype, const float* qkv, void* q, void* values, const Q8View& v, const cake_rope& rope, int n_q, int max_rows, hipStream_t st) {
    return launch_append<8>(dtype, qkv, q, values, v, rope, n_q, max_rows, st);
}

hipError_t launch_attention_q8(int dtype, const void* q, void* out, const Q8View& v, int n_q, int max_rows, int max_len, int window, int sinks,
                               const AttnWs& ws, hipStream_t st) {
    return launch_attention<8>(dtype, q, out, v, n_q, max_rows, max_len, window, sinks, ws, st);
}

}  // namespace cake
