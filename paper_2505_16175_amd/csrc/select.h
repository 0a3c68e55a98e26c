// The k-th largest of a list of 32-bit keys, found by one workgroup of 1024 threads: the threshold of a TopK.
//   * A round spreads the current key range [lo, lo + span] over up to 2048 buckets of equal power-of-two width (bucket =
//     (key - lo) >> sh), counts keys per bucket with LDS atomics, turns the counts into suffix sums (two buckets per thread,
//     shuffles inside a wavefront, 16 wavefront totals through LDS) and picks the bucket in which the k-th largest key falls;
//     the range shrinks to that bucket. Because the buckets follow the data's own range, real scores (which share sign and
//     exponent) spread over them and the atomics rarely collide; one ballot per batch folds a digit shared by many lanes into
//     a single atomic, so that a constant score vector does not serialise either.
//   * As soon as the bucket holds at most 256 keys they are copied to a list and ranked directly (every candidate counts the
//     candidates above and equal to it). Otherwise another round runs on the bucket; a bucket of width one is exact. The width
//     shrinks by 2^11 per round: at most 3 rounds.
#pragma once
#include "qp_internal.h"

namespace qp {

constexpr int SEL_THREADS = 1024;
constexpr int SEL_WAVES = SEL_THREADS / 64;
constexpr int SEL_BITS = 11;
constexpr int SEL_NB = 1 << SEL_BITS;  // buckets per round, two per thread
constexpr int SEL_LIST = 256;          // a bucket of at most this many keys is ranked directly
constexpr int SEL_UNROLL = 2;          // independent reads of keys in LDS per thread and loop trip
constexpr int SEL_MAX_ROUNDS = 4;      // 3 suffice for 32-bit keys; the bound makes termination explicit
static_assert(SEL_NB == 2 * SEL_THREADS, "two buckets per thread");

__device__ __forceinline__ uint32_t order_key(float s) {
  s += 0.f;  // -0.0 -> +0.0 so that the two zeros tie
  const uint32_t u = __float_as_uint(s);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);  // ascending in s
}

struct SelectLds {
  __attribute__((aligned(16))) uint32_t hist[SEL_NB];  // 16: wave_a then is too, which is read by fours. Zero at entry, and again when the search returns
  uint32_t list[SEL_LIST];
  uint32_t wave_a[SEL_WAVES];
  uint32_t sel_bucket, sel_need, sel_count, sel_key, list_n;  // list_n: zero at entry
};

// Every key of key_at(0) .. key_at(n - 1) once, by whole wavefronts: f(key, whether there is one).
template <int UNROLL, class KeyAt>
struct EachKey {
  KeyAt key_at;
  int n;
  template <class F>
  __device__ __forceinline__ void operator()(F f) const {
    const int n_round = (n + SEL_THREADS - 1) / SEL_THREADS * SEL_THREADS;  // whole wavefronts take part
    for (int j0 = threadIdx.x; j0 < n_round; j0 += UNROLL * SEL_THREADS) {
      uint32_t kk[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) kk[u] = j0 + u * SEL_THREADS < n ? key_at(j0 + u * SEL_THREADS) : 0u;
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) f(kk[u], j0 + u * SEL_THREADS < n);  // beyond n_round no lane has one
    }
  }
};
template <int UNROLL = SEL_UNROLL, class KeyAt>
__device__ __forceinline__ EachKey<UNROLL, KeyAt> each_key(KeyAt key_at, int n) {
  return EachKey<UNROLL, KeyAt>{key_at, n};
}

// thr: the rank-th largest of the keys that `each` hands to the workgroup's threads, as far as they are inside [lo, hi]
// (1 <= rank <= their number); need: how many keys equal to it are among the first `rank` (>= 1). `each` brings whole wavefronts;
// `scan` hands out the same keys and need not (the list's pass has no ballot: n rounded up to the wavefronts costs a short TopK
// 0.7 us of 12). The workgroup has met at a barrier behind what it wrote to `lds` and to the keys. FOLD: keys that share a bucket
// are counted together first (above). Without it that is done for the smallest keys alone, by wavefronts that have many of them
// (`many_low`, the same in all lanes): entries that nothing looked at weigh 0.
template <bool FOLD = true, class Each, class Scan>
__device__ __forceinline__ void select_threshold(Each each, Scan scan, uint32_t lo, uint32_t hi, uint32_t rank, SelectLds& lds,
                                                 uint32_t& thr, uint32_t& need, bool many_low = false) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t span = hi - lo;          // keys still in play: lo <= key <= lo + span
  need = rank;                      // of T among them, counted from the largest
  thr = lo;
  for (int round = 0; round < SEL_MAX_ROUNDS; ++round) {
    const int bits = span ? 32 - __builtin_clz(span) : 0;
    const int sh = bits > SEL_BITS ? bits - SEL_BITS : 0;
    auto count_key = [&](uint32_t key, bool in) {
      const uint32_t off = key - lo;
      bool act = in && off <= span;  // a key below lo wraps to a large offset
      const uint32_t bin = off >> sh;
      const unsigned long long am = __ballot(act);
      if (FOLD && am != 0) {  // fold the first active lane's bucket when many lanes share it
        const int leader = __ffsll((long long)am) - 1;
        const uint32_t b0 = (uint32_t)__builtin_amdgcn_readlane((int)bin, leader);
        const bool mine = act && bin == b0;
        const unsigned long long same = __ballot(mine);
        if (__popcll(same) >= 8) {
          if (lane == leader) atomicAdd(&lds.hist[b0], (uint32_t)__popcll(same));
          if (mine) act = false;
        }
      }
      if (act) atomicAdd(&lds.hist[bin], 1u);
    };
    if (!FOLD && many_low) {
      uint32_t low = 0;  // of this wavefront's keys in the first bucket
      each([&](uint32_t key, bool in) {
        const bool first = in && (key - lo) >> sh == 0;
        low += (uint32_t)__popcll(__ballot(first));
        count_key(key, in && !first);
      });
      if (lane == 0) atomicAdd(&lds.hist[0], low);
    } else {
      each(count_key);
    }
    __syncthreads();
    // suffix sums over the buckets: this thread owns buckets 2 tid and 2 tid + 1 (and clears them for a next round)
    const uint2 hb = *(const uint2*)&lds.hist[2 * tid];
    *(uint2*)&lds.hist[2 * tid] = make_uint2(0u, 0u);
    const uint32_t own = hb.x + hb.y;
    uint32_t suf = own;  // inclusive suffix over the wavefront's lanes
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t t = __shfl_down(suf, o, 64);
      if (lane + o < 64) suf += t;
    }
    if (lane == 0) lds.wave_a[wave] = suf;
    __syncthreads();
    uint32_t above = suf - own;  // keys in buckets above 2 tid + 1
#pragma unroll
    for (int w = 1; w < SEL_WAVES; ++w) above += w > wave ? lds.wave_a[w] : 0u;
    const uint32_t suf1 = above + hb.y, suf0 = suf1 + hb.x;
    if (suf1 >= need && above < need) {  // exactly one (thread, bucket) holds the crossing
      lds.sel_bucket = 2 * tid + 1;
      lds.sel_need = need - above;
      lds.sel_count = hb.y;
    } else if (suf0 >= need && suf1 < need) {
      lds.sel_bucket = 2 * tid;
      lds.sel_need = need - suf1;
      lds.sel_count = hb.x;
    }
    __syncthreads();
    const uint32_t first = lds.sel_bucket << sh;  // offset of the chosen bucket's first key
    need = lds.sel_need;
    const uint32_t count = lds.sel_count;
    lo += first;
    span = min(span - first, (sh ? (1u << sh) : 1u) - 1u);
    thr = lo;
    if (sh == 0) break;  // buckets were single keys: T = lo, `need` of its copies survive
    if (count <= SEL_LIST) {
      // rank the bucket's keys directly
      scan([&](uint32_t key, bool in) {
        if (in && key - lo <= span) {
          const uint32_t p = atomicAdd(&lds.list_n, 1u);
          if (p < (uint32_t)SEL_LIST) lds.list[p] = key;  // always true: the bucket holds `count` keys
        }
      });
      __syncthreads();
      if (tid < (int)count) {
        const uint32_t x = lds.list[tid];
        uint32_t g = 0, e = 0;
        for (uint32_t m = 0; m < count; ++m) {
          const uint32_t y = lds.list[m];
          g += y > x;
          e += y == x;
        }
        if (g < need && need <= g + e) {  // equal candidates write the same values
          lds.sel_key = x;
          lds.sel_need = need - g;
        }
      }
      __syncthreads();
      thr = lds.sel_key;
      need = lds.sel_need;
      break;
    }
  }
}

}  // namespace qp
