// kvattn_d256.hip -- attention over the quantized cache (kvattn_kernel.h), heads of 256 channels.
#include "kvattn_kernel.h"

namespace fgq {

fgq_status launch_kv_attn_d256(const KvAttnArgs& a, int nt, bool share, hipStream_t st) {
  if (a.G == 32) return launch_bits<256, 32>(a, nt, share, st);
  if (a.G == 64) return launch_bits<256, 64>(a, nt, share, st);
  return launch_bits<256, 128>(a, nt, share, st);
}

}  // namespace fgq
