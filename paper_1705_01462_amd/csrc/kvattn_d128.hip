// kvattn_d128.hip -- attention over the quantized cache (kvattn_kernel.h), heads of 128 channels.
#include "kvattn_kernel.h"

namespace fgq {

fgq_status launch_kv_attn_d128(const KvAttnArgs& a, int nt, bool share, hipStream_t st) {
  if (a.G == 32) return launch_bits<128, 32>(a, nt, share, st);
  if (a.G == 64) return launch_bits<128, 64>(a, nt, share, st);
  return launch_bits<128, 128>(a, nt, share, st);
}

}  // namespace fgq
