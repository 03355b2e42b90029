// Attention of rows that share the beginnings of their sequences (dck_paged_shared_attention,
// dck_quant_shared_attention).
#include "paged.cuh"

namespace dck {

size_t paged_shared_workspace(const PagedView& v, DecodeKind kind, int B, int max_len, int max_own, int sms) {
  return paged_decode_workspace(v, kind, B, max_len, sms);
}

// Every row by itself.
cudaError_t launch_paged_shared(const PagedDecodeArgs& a, DecodeKind kind, int sms, cudaStream_t s) {
  return launch_paged_decode(a, kind, sms, s);
}

}  // namespace dck
