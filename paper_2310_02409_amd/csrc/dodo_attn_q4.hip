// dodo_nugget_attention_q4: nugget attention (Eq. 13 / Eq. 9 of the Dodo paper) over a nugget cache held in 4 bits.
// The cache is unpacked into the workspace and attended over from there.
#include "dodo_common.h"

namespace dodo {
namespace {

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace
}  // namespace dodo

extern "C" size_t dodo_nugget_attention_q4_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t d_h, int32_t max_q,
                                                           int32_t max_k, int32_t max_local, int64_t Kt, int dtype) {
  using namespace dodo;
  if (B <= 0 || H <= 0 || H_kv <= 0 || d_h <= 0 || max_q <= 0 || max_k < 0 || max_local < 0 || Kt < 0 || !dtype_ok(dtype)) return 0;
  const size_t attention = dodo_nugget_attention_workspace_bytes_grouped(B, H, H_kv, d_h, max_q, max_k, max_local, dtype);
  return round256(attention) + 2 * round256(static_cast<size_t>(Kt) * H_kv * d_h * elem_bytes(dtype));
}

extern "C" int dodo_nugget_attention_q4(const void* Q, const uint8_t* Kc, const uint8_t* Ks, const uint8_t* Vc, const uint8_t* Vs,
                                        const void* Kl, const void* Vl, const int32_t* cu_q, const int32_t* cu_nuggets,
                                        const int32_t* cu_local, int32_t B, int32_t H, int32_t H_kv, int32_t d_h, int32_t max_q,
                                        int32_t max_k, int32_t max_local, int64_t Kt, float softmax_scale, int dtype, int layout,
                                        void* O, float* lse, void* ws, size_t ws_bytes, void* stream) {
  using namespace dodo;
  if (B < 0 || H <= 0 || H_kv <= 0 || d_h <= 0 || max_q < 0 || max_k < 0 || max_local < 0 || Kt < 0) return DODO_ERR_INVALID_ARG;
  if (H % H_kv != 0) return DODO_ERR_INVALID_ARG;
  if (layout != DODO_LAYOUT_TOKEN_MAJOR && layout != DODO_LAYOUT_HEAD_MAJOR) return DODO_ERR_INVALID_ARG;
  if (!(softmax_scale == softmax_scale)) return DODO_ERR_INVALID_ARG;
  if (B == 0 || max_q == 0) return DODO_OK;
  if (!Q || !O || !cu_q || !cu_nuggets || !cu_local) return DODO_ERR_INVALID_ARG;
  if (Kt == 0) max_k = 0;
  if (max_k > 0 && (!Kc || !Ks || !Vc || !Vs)) return DODO_ERR_INVALID_ARG;
  if (max_local > 0 && (!Kl || !Vl)) return DODO_ERR_INVALID_ARG;
  if (!dtype_ok(dtype)) return DODO_ERR_UNSUPPORTED;
  if (d_h != 64 && d_h != 128) return DODO_ERR_UNSUPPORTED;
  if (!aligned16(Q) || !aligned16(O) || !aligned16(Kc) || !aligned16(Vc) || !aligned16(Kl) || !aligned16(Vl) || !aligned16(ws) ||
      ((reinterpret_cast<uintptr_t>(Ks) | reinterpret_cast<uintptr_t>(Vs)) & 3u) != 0)
    return DODO_ERR_UNSUPPORTED;
  if (ws_bytes < dodo_nugget_attention_q4_workspace_bytes(B, H, H_kv, d_h, max_q, max_k, max_local, Kt, dtype) || (ws_bytes > 0 && !ws))
    return DODO_ERR_WORKSPACE_TOO_SMALL;
  const size_t attention = dodo_nugget_attention_workspace_bytes_grouped(B, H, H_kv, d_h, max_q, max_k, max_local, dtype);
  const size_t cache = round256(static_cast<size_t>(Kt) * H_kv * d_h * elem_bytes(dtype));
  char* Kn = static_cast<char*>(ws) + round256(attention);
  char* Vn = Kn + cache;
  if (max_k > 0) {
    const int rc = dodo_unpack_nuggets_q4(Kc, Ks, Vc, Vs, Kt * H_kv, d_h, dtype, Kn, Vn, stream);
    if (rc != DODO_OK) return rc;
  }
  return dodo_nugget_attention(Q, Kn, Vn, Kl, Vl, cu_q, cu_nuggets, cu_local, B, H, H_kv, d_h, max_q, max_k, max_local, Kt,
                               softmax_scale, dtype, layout, O, lse, attention ? ws : nullptr, attention, stream);
}
