// kvcache.hip -- fgq_kv_write and fgq_kv_read: tokens quantized as they are
// written into the cache (kvcache.h), and read back as values.
//
// A lane holds eight consecutive channels, so a group of G channels is G / 8
// neighbouring lanes that agree on its minimum and maximum by exchanges within
// the wave; one pass over the data, bound by its bytes.
//
// lo is the minimum rounded down to bf16 and step the range over the number of
// steps rounded up to bf16 (to bf16 because the exponent range of every input
// type has to fit): every value then lies within [lo, lo + L * step], so it is
// at most half a step from the value its code stands for.
#include "elem.h"
#include "kvcache.h"
#include "rowquant.h"

namespace fgq {
namespace {

constexpr int kThreads = 256;

struct KvArgs {
  const void* src[2];
  void* dst[2];
  int64_t st[2], sh[2];  // strides of src in elements: token, head
  const int64_t* slots;
  uint8_t* cache;
  int64_t T, num_slots, items;
  int32_t Hkv, D, P, G, row, ng;
  int64_t head_bytes;
};

// Which eight channels this thread has: token, head, eighth of the head.
struct Item {
  int64_t t;
  int h, d8;
};
__device__ inline Item item_of(const KvArgs& a, int64_t i) {
  const int n8 = a.D / 8;
  const int64_t th = i / n8;
  return Item{th / a.Hkv, static_cast<int>(th % a.Hkv), static_cast<int>(i % n8)};
}

template <int kType, int kBits>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvArgs a) {
#pragma clang fp contract(off)
  constexpr float L = kBits == 4 ? 15.0f : 255.0f;
  const int z = blockIdx.y;  // 0: keys, 1: values
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const bool have = i < a.items;
  const Item it = item_of(a, have ? i : 0);
  const int64_t slot = have ? a.slots[it.t] : -1;
  float v[8];
  values8<kType>(load8<kType>(a.src[z], it.t * a.st[z] + it.h * a.sh[z] + 8 * it.d8), v);
  float lo = v[0], hi = v[0];
  uint32_t big = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo = fminf(lo, v[j]);
    hi = fmaxf(hi, v[j]);
    big = max(big, abs_bits(v[j]));
  }
  const int lanes = a.G / 8;  // 4, 8 or 16: whole groups in every wave
  for (int off = 1; off < lanes; off *= 2) {
    lo = fminf(lo, __shfl_xor(lo, off));
    hi = fmaxf(hi, __shfl_xor(hi, off));
    big = max(big, static_cast<uint32_t>(__shfl_xor(static_cast<int>(big), off)));
  }
  uint32_t u = __float_as_uint(lo);
  u = (static_cast<int32_t>(u) < 0 ? u + 0xFFFFu : u) & 0xFFFF0000u;
  lo = __uint_as_float(u);
  const float s = (hi * 0.5f - lo * 0.5f) * (2.0f / L);
  uint32_t t = (__float_as_uint(s) + 0xFFFFu) & 0xFFFF0000u;
  if (__uint_as_float(t) < 0x1p-120f) t = 0;
  float inv = t ? 1.0f / __uint_as_float(t) : 0.0f;
  if (big >= 0x7F800000u || u == 0xFF800000u) {  // not finite (or lo is not, in bf16): the group reads back NaN
    u = t = 0x7FC00000u;
    inv = 0.0f;
  }
  uint32_t c[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) c[j] = static_cast<uint32_t>(fminf(fmaxf(rintf((v[j] - lo) * inv), 0.0f), L));
  if (slot < 0 || slot >= a.num_slots) return;
  const int64_t page = slot / a.P;
  const int at = static_cast<int>(slot % a.P);
  const int64_t base = (page * a.Hkv + it.h) * a.head_bytes;
  const int64_t limit = a.num_slots / a.P * a.Hkv * a.head_bytes;
  const int64_t cd = base + static_cast<int64_t>(z * a.P + at) * a.row + it.d8 * kBits;
  if (check_store(kSiteStoreCache, cd, kBits, limit)) {
    if constexpr (kBits == 4) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) w |= c[j] << (4 * j);
      *reinterpret_cast<uint32_t*>(a.cache + cd) = w;
    } else {
      uint64_t w = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) w |= static_cast<uint64_t>(c[j]) << (8 * j);
      *reinterpret_cast<uint64_t*>(a.cache + cd) = w;
    }
  }
  if (it.d8 % lanes == 0) {
    const int64_t pp = base + 2LL * a.P * a.row + 4LL * ((z * a.ng + it.d8 / lanes) * a.P + at);
    if (check_store(kSiteStoreCache, pp, 4, limit)) *reinterpret_cast<uint32_t*>(a.cache + pp) = u >> 16 | t;
  }
}

template <int kType, int kBits>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvArgs a) {
  const int z = blockIdx.y;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= a.items) return;
  const Item it = item_of(a, i);
  const int64_t slot = a.slots[it.t];
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (slot >= 0 && slot < a.num_slots) {
    const int64_t page = slot / a.P;
    const int at = static_cast<int>(slot % a.P);
    const uint8_t* base = a.cache + (page * a.Hkv + it.h) * a.head_bytes;
    const uint8_t* cd = base + static_cast<int64_t>(z * a.P + at) * a.row + it.d8 * kBits;
    const uint32_t par = *reinterpret_cast<const uint32_t*>(
        base + 2LL * a.P * a.row + 4LL * ((z * a.ng + 8 * it.d8 / a.G) * a.P + at));
    const float lo = bf16_f32(par & 0xFFFFu), step = __uint_as_float(par & 0xFFFF0000u);
    uint64_t w;
    if constexpr (kBits == 4)
      w = *reinterpret_cast<const uint32_t*>(cd);
    else
      w = *reinterpret_cast<const uint64_t*>(cd);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = fmaf(step, static_cast<float>(w >> (kBits * j) & ((1 << kBits) - 1)), lo);
  }
  if (check_store(kSiteStoreY, 8 * i, 8, 8 * a.items)) store8<kType>(a.dst[z], 8 * i, v);
}

KvArgs kv_args(const KvGeom& c, int64_t T, const int64_t* slots) {
  KvArgs a{};
  a.slots = slots;
  a.T = T;
  a.num_slots = c.num_pages * c.P;
  a.items = T * c.Hkv * (c.D / 8);
  a.Hkv = c.Hkv;
  a.D = c.D;
  a.P = c.P;
  a.G = c.G;
  a.row = static_cast<int32_t>(kv_row_bytes(c.D, c.bits));
  a.ng = c.D / c.G;
  a.head_bytes = kv_head_bytes(c.P, c.D, c.bits, c.G);
  return a;
}

}  // namespace

fgq_status launch_kv_write(const void* k, const void* v, int32_t type, int64_t T, const int64_t (&stride)[4],
                           const int64_t* slots, const KvGeom& c, uint8_t* cache, hipStream_t st) {
  KvArgs a = kv_args(c, T, slots);
  a.src[0] = k;
  a.src[1] = v;
  a.st[0] = stride[0];
  a.sh[0] = stride[1];
  a.st[1] = stride[2];
  a.sh[1] = stride[3];
  a.cache = cache;
  const dim3 grid(static_cast<uint32_t>(ceil_div(a.items, kThreads)), 2);
  return with_type(type, [&](auto t) {
    if (c.bits == 4)
      hipLaunchKernelGGL((kv_write_kernel<decltype(t)::value, 4>), grid, dim3(kThreads), 0, st, a);
    else
      hipLaunchKernelGGL((kv_write_kernel<decltype(t)::value, 8>), grid, dim3(kThreads), 0, st, a);
    return last_launch();
  });
}

fgq_status launch_kv_read(const int64_t* slots, int64_t T, const KvGeom& c, const uint8_t* cache, int32_t type,
                          void* k, void* v, hipStream_t st) {
  KvArgs a = kv_args(c, T, slots);
  a.dst[0] = k;
  a.dst[1] = v;
  a.cache = const_cast<uint8_t*>(cache);
  const dim3 grid(static_cast<uint32_t>(ceil_div(a.items, kThreads)), 2);
  return with_type(type, [&](auto t) {
    if (c.bits == 4)
      hipLaunchKernelGGL((kv_read_kernel<decltype(t)::value, 4>), grid, dim3(kThreads), 0, st, a);
    else
      hipLaunchKernelGGL((kv_read_kernel<decltype(t)::value, 8>), grid, dim3(kThreads), 0, st, a);
    return last_launch();
  });
}

}  // namespace fgq
