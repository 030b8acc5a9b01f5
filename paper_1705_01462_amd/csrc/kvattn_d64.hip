// kvattn_d64.hip -- attention over the quantized cache (kvattn_kernel.h), heads of 64 channels.
#include "kvattn_kernel.h"

namespace fgq {

fgq_status launch_kv_attn_d64(const KvAttnArgs& a, int nt, bool share, hipStream_t st) {
  if (a.G == 32) return launch_bits<64, 32>(a, nt, share, st);
  return launch_bits<64, 64>(a, nt, share, st);
}

}  // namespace fgq
