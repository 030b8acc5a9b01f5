// kvattn.hip -- attention over the quantized cache: how a call is divided
// (rows, workgroups, splits of the keys), and the join of split keys.
#include "kvattn.h"

#include <algorithm>

#include "igemm.h"

namespace fgq {
namespace {

constexpr int kJoinThreads = 256;

// A workgroup a row: the splits' outputs weighted by 2^(their maximum - the
// largest), over the sum of the weighted sums.  Each wave takes every fourth
// split, several in flight; the order of the additions is fixed.
template <int kType, int kD>
__global__ __launch_bounds__(kJoinThreads) void kv_attn_join_kernel(KvAttnArgs a) {
  constexpr int kWaves = kJoinThreads / 64, kC = kD / 64, kAhead = 4;
  typedef float vec __attribute__((ext_vector_type(kC), aligned(4)));
  __shared__ float smax[kWaves], ssum[kWaves], so[kWaves][kD];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t item = blockIdx.x;
  const int head = static_cast<int>(item % a.Hq);
  const int i = static_cast<int>(item / a.Hq % a.max_q), b = static_cast<int>(item / a.Hq / a.max_q);
  const int64_t q0 = max(0, min(a.cu_q[b], static_cast<int>(a.T)));
  const int64_t q1 = max(q0, min(static_cast<int64_t>(a.cu_q[b + 1]), a.T));
  if (i >= q1 - q0) return;
  const int64_t row = (q0 + i) * a.Hq + head;
  const float* p = a.part + row * a.splits * (kD + 2);
  // this lane's split of each 64: maxima and sums
  float mx = -INFINITY;
  for (int s = threadIdx.x; s < a.splits; s += kJoinThreads) mx = fmaxf(mx, p[s * (kD + 2) + kD]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
  if (lane == 0) smax[wave] = mx;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, smax[w]);
  const float base = mx == -INFINITY ? 0.0f : mx;
  float sum = 0.0f;
  vec v = {};
  for (int s0 = wave; s0 < a.splits; s0 += kWaves * kAhead) {
    vec o[kAhead];
    float m[kAhead], l[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int s = min(s0 + kWaves * u, a.splits - 1);
      const float* ps = p + static_cast<int64_t>(s) * (kD + 2);
      o[u] = *reinterpret_cast<const vec*>(ps + kC * lane);
      m[u] = ps[kD];
      l[u] = ps[kD + 1];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (s0 + kWaves * u < a.splits) {
        const float w = exp2f(m[u] - base);
        sum += w * l[u];
        v += w * o[u];
      }
  }
  if (lane == 0) ssum[wave] = sum;
#pragma unroll
  for (int c = 0; c < kC; ++c) so[wave][kC * lane + c] = reinterpret_cast<const float*>(&v)[c];
  __syncthreads();
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += ssum[w];
  if (threadIdx.x < kD) {
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) x += so[w][threadIdx.x];
    const int64_t at = row * kD + threadIdx.x;
    if (check_store(kSiteStoreY, at, 1, a.T * a.Hq * kD)) Elem<kType>::put(a.o, at, sum == 0.0f ? 0.0f : x / sum);
  }
  if (threadIdx.x == 0 && a.lse && check_store(kSiteStoreY, row, 1, a.T * a.Hq))
    a.lse[row] = sum > 0.0f ? (mx + log2f(sum)) * 0.6931471805599453f : (sum == 0.0f ? -INFINITY : sum);
}

template <int kType>
void launch_join(const KvAttnArgs& a, int64_t items, hipStream_t st) {
  const dim3 grid(static_cast<uint32_t>(items)), wg(kJoinThreads);
  if (a.D == 64)
    hipLaunchKernelGGL((kv_attn_join_kernel<kType, 64>), grid, wg, 0, st, a);
  else if (a.D == 128)
    hipLaunchKernelGGL((kv_attn_join_kernel<kType, 128>), grid, wg, 0, st, a);
  else
    hipLaunchKernelGGL((kv_attn_join_kernel<kType, 256>), grid, wg, 0, st, a);
}

struct Plan {
  int nt, tiles, splits, split_keys;
  int max_splits;  // no less than splits, and no less for more keys
  bool share, wide;
};

// How a call is divided; wide: the form with eight waves exists.  max_keys: the
// most keys of a sequence, as far as the host knows.
//
// Few rows, or too few workgroups for a unit each: the waves share rows and
// divide the keys, else they have rows of their own, four times as many a
// workgroup, and one expansion of the codes.  us, rows of their own and shared,
// 32 heads on 8, 4 bits, one sequence: 128 queries on 4096 keys (32 workgroups
// of 128 rows) 176, 50; 512 on 32768 (128) 1336, 562; 1024 on 16384 (256) 678,
// 553; 2048 on 8192 (512) 426, 511.  Heads of 256, on 8192: 512 queries 882, 585;
// 768 882, 858; 1024 on 16384 1753, 2211.
//
// Keys are split until there are three workgroups a unit (us, two sequences of
// 131072 keys and 16 (sequence, key head) pairs: 1.5 a unit 88, 3 70, 6 80, 12
// 88; 48 sequences of up to 8191: 85, 80, 82, 84), but not below 256 keys, two
// steps of each of four waves.
Plan plan(int32_t D, int blocks, bool wide, int32_t Hq, int32_t Hkv, int64_t B, int64_t max_q, int64_t max_keys, int64_t window) {
  Plan p{};
  const int64_t rows = max_q * (Hq / Hkv), cus = ig::device_cus();
  p.share = rows <= 64 || B * Hkv * ceil_div(rows, 128) <= (D == 256 ? cus / 2 : cus);
  p.nt = rows <= 16 ? 1 : blocks;
  p.tiles = static_cast<int>(ceil_div(rows, 16 * p.nt * (p.share ? 1 : 4)));
  // keys that a tile's rows can see, and its first step's alignment
  const int64_t keys = (window ? std::min(max_keys, window + max_q) : max_keys) + kKvAttnAlign;
  p.splits = 1;
  if (p.share) {
    const int64_t wgs = B * Hkv * p.tiles;
    p.splits = static_cast<int>(std::max<int64_t>(1, std::min({keys / kKvAttnSplit, 3 * cus / wgs, int64_t{1024}})));
    // Some hundred keys and few workgroups: eight waves take them without a join
    // (us: 8 pairs of 777 keys 11.7 instead of 13.7, 192 pairs of a window of 512
    // 11.5 instead of 15.9; 64 pairs of 4096 keys 34 instead of 19.4).
    if (wide && wgs <= cus && keys > 256 && keys <= 1024) {
      p.wide = true;
      p.splits = 1;
    }
  }
  p.max_splits = p.splits;
  p.split_keys = static_cast<int>(round_up(ceil_div(keys, p.splits), kKvAttnSplit));
  p.splits = static_cast<int>(ceil_div(keys, p.split_keys));
  return p;
}

}  // namespace

size_t kv_attn_ws_bytes(int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int64_t B, int64_t max_q, int64_t max_keys) {
  // of any group size and window
  const Plan p = plan(D, 2, false, Hq, Hkv, B, max_q, max_keys, 0);
  return p.max_splits == 1 ? 0 : static_cast<size_t>(T) * Hq * p.max_splits * (D + 2) * sizeof(float);
}

fgq_status launch_kv_attn(KvAttnArgs a, void* ws, hipStream_t st) {
  const Plan p = plan(a.D, kv_attn_blocks(a.D, a.G), kv_attn_has_wide(a.D, a.G), a.Hq, a.Hkv, a.B, a.max_q,
                      a.max_pages * a.P, a.window);
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.wide = p.wide ? 1 : 0;
  a.split_keys = p.split_keys;
  a.part = static_cast<float*>(ws);
  const fgq_status rc = a.D == 64    ? launch_kv_attn_d64(a, p.nt, p.share, st)
                        : a.D == 128 ? launch_kv_attn_d128(a, p.nt, p.share, st)
                                     : launch_kv_attn_d256(a, p.nt, p.share, st);
  if (rc != FGQ_OK || p.splits == 1) return rc;
  const int64_t items = static_cast<int64_t>(a.B) * a.max_q * a.Hq;
  if (a.type == FGQ_F16)
    launch_join<FGQ_F16>(a, items, st);
  else
    launch_join<FGQ_BF16>(a, items, st);
  return last_launch();
}

}  // namespace fgq
