// kvcache.h -- the layout of a quantized, paged key/value cache, shared by the
// kernels that write, read back and attend over it.
//
// A page holds P tokens of every key head; for one head its bytes are
//   codes of the P keys    [P][D * bits / 8]   (4 bits: even channel in the low nibble)
//   codes of the P values  [P][D * bits / 8]
//   parameters of the keys   uint32 [D / G][P]   (low half: bf16 lo, high half: bf16 step)
//   parameters of the values uint32 [D / G][P]
// so that a run of tokens is one run of bytes in each part, the parameters of
// four consecutive tokens are one 16-byte load, and a token is written without
// touching bytes of another.  With P a multiple of 16 every part starts at a
// multiple of 16 bytes.
#pragma once

#include "fgq_internal.h"

namespace fgq {

__host__ __device__ inline int64_t kv_row_bytes(int32_t D, int32_t bits) { return static_cast<int64_t>(D) * bits / 8; }
__host__ __device__ inline int64_t kv_head_bytes(int32_t P, int32_t D, int32_t bits, int32_t G) {
  return 2 * P * (kv_row_bytes(D, bits) + 4 * (D / G));
}

struct KvGeom {
  int64_t num_pages;
  int32_t Hkv, D, P, bits, G;
};

// Launchers; arguments already validated.
fgq_status launch_kv_write(const void* k, const void* v, int32_t type, int64_t T, const int64_t (&stride)[4],
                           const int64_t* slots, const KvGeom& c, uint8_t* cache, hipStream_t st);
fgq_status launch_kv_read(const int64_t* slots, int64_t T, const KvGeom& c, const uint8_t* cache, int32_t type,
                          void* k, void* v, hipStream_t st);

}  // namespace fgq
