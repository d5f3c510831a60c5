// Attention over pages of 8-bit rows with a scale for each row and head.
#include "attention_paged.h"

namespace d3 {

int launch_attention_paged8(const PagedAttnArgs& a, int hd, int kv_dtype, int n_cu, hipStream_t s) {
    if (kv_dtype == D3_I8) return hd == 64 ? launch<i8_t, 64>(a, n_cu, s) : launch<i8_t, 128>(a, n_cu, s);
    if (kv_dtype == D3_E4M3) return hd == 64 ? launch<e4m3_t, 64>(a, n_cu, s) : launch<e4m3_t, 128>(a, n_cu, s);
    return (int)hipErrorInvalidValue;
}

}  // namespace d3
