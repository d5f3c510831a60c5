// Attention over pages of fp16 and fp32 rows; 8-bit ones in attention_paged8.hip.
#include "attention_paged.h"

namespace d3 {

int launch_attention_paged(const PagedAttnArgs& a, int hd, int kv_dtype, int n_cu, hipStream_t s) {
    if (kv_dtype == D3_F32) return hd == 64 ? launch<float, 64>(a, n_cu, s) : launch<float, 128>(a, n_cu, s);
    if (kv_dtype == D3_F16) return hd == 64 ? launch<f16_t, 64>(a, n_cu, s) : launch<f16_t, 128>(a, n_cu, s);
    return launch_attention_paged8(a, hd, kv_dtype, n_cu, s);
}

}  // namespace d3
