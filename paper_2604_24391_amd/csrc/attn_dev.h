// Device code that the attention kernels over token caches share (qattn.hip, pattn.hip): the deal of
// key blocks over workgroups, what a row sees of a block, loads.
#pragma once

#include <hip/hip_runtime.h>

#include "fc_internal.h"
#include "gemm_dev.h"
#include "qcache.h"

namespace fc {
namespace {

constexpr int kKeyBlock = 64;                // keys that a wave takes at a time
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNegInf = -__builtin_inff();

// LDS words that lanes of one wave write in parts and read whole, and the order between the two.
typedef uint16_t __attribute__((may_alias)) part16;
typedef uint32_t __attribute__((may_alias)) part32;
typedef uint8_t __attribute__((may_alias)) part8;
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// The bits of a block's 64 keys below `seen` (relative to the block's first).
__device__ __forceinline__ uint64_t seen_bits(int seen) {
  return seen >= 64 ? ~0ull : (seen <= 0 ? 0ull : (1ull << seen) - 1ull);
}
// Eight query elements, their signs turned where the scale is negative.
__device__ __forceinline__ bf16x8 load_q(const uint16_t *src, uint32_t flip) {
  u32x4 w = *reinterpret_cast<const u32x4 *>(src);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] ^= flip;
  return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Splits that the key blocks of one tile of rows are dealt over (kernels of many rows): lengths are known on
// the device only, so the grid has room for `splits`, and a short item uses no more than leaves
// each of them `least` blocks.
template <class A>
__device__ __forceinline__ int splits_used(int kmax, const A &a) {
  return max(1, min(a.splits, (kmax + a.least * kKeyBlock - 1) / (a.least * kKeyBlock)));
}
// Kernels of few rows deal a.slots workgroups of each key-value head over the items by their lengths, `per`
// blocks to each: with the same number for every item, the longest one of a ragged batch would
// keep few CUs busy to the end.  Items take ceil(blocks / per) slots in order; per is the smallest
// number with which they suffice, but at least four blocks (one per wave).
struct Share {
  int item, start, used, per;       // the item, its first slot, its slots, blocks of each
  int held, m;                      // its rows held and new
};
// Sums over a wave's lanes up to each one, by moves within the vector unit: rows of 16 lanes first, then a
// row's sum to the next one, then the first half's to the second.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row_bcast:15 to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // row_bcast:31 to rows 2 and 3
  return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }
// The share of the item that slot `slot` falls to (item -1: none).
template <class A>
__device__ __forceinline__ Share share_of(const A &a, int slot) {
  const int lane = threadIdx.x & 63;
  int held = 0, m = 0;                // of item i + lane
  auto blocks = [&](int i) {
    const int j = min(i + lane, a.B - 1);
    held = min(max(a.len[j], 0), a.cap);
    m = min(a.n_new ? min(max(a.n_new[j], 0), a.n) : a.n, a.cap - held);
    return i + lane < a.B && m > 0 ? (held + m + kKeyBlock - 1) / kKeyBlock : 0;
  };
  if (a.slots == a.B) {               // one workgroup for each item
    held = q_held(a.len, slot, a.cap), m = q_new(a.n_new, slot, a.n, held, a.cap);
    return Share{m > 0 ? slot : -1, slot, 1, (a.cap + kKeyBlock - 1) / kKeyBlock, held, m};
  }
  int x = blocks(0);
  if (a.B == 1) {
    const int n = __builtin_amdgcn_readfirstlane(x), per = max(4, (n + a.slots - 1) / a.slots), used = (n + per - 1) / per;
    return Share{slot < used ? 0 : -1, 0, used, per, __builtin_amdgcn_readfirstlane(held), __builtin_amdgcn_readfirstlane(m)};
  }
  // The calls' checks hold an 8-bit cache of heads of 64 dims and more to 2^42 bytes and a paged cache's table
  // to 2^36 rows, whatever its pool, so all items hold up to 2^36 rows: 2^30 blocks, and one more for
  // each of up to 65535 items (a paged capacity is a multiple of 16).  With at least three slots for two
  // items, all + slots and lo + hi stay below 2^31.
  auto slots_of = [&](int per) {      // per 0: the blocks themselves
    int all = 0;
    for (int i = 0; i < a.B; i += 64) {
      if (a.B > 64) x = blocks(i);
      all += wave_sum(per ? (int)((unsigned)(x + per - 1) / (unsigned)per) : x);
    }
    return all;
  };
  const int all = slots_of(0);
  int lo = max(4, (all + a.slots - 1) / a.slots), hi = max(lo, (all + a.slots - a.B - 1) / (a.slots - a.B));
  while (lo < hi) {                   // hi suffices: the quotients round up by less than one each
    const int mid = (lo + hi) / 2;
    if (slots_of(mid) <= a.slots) hi = mid;
    else lo = mid + 1;
  }
  const int per = lo;
  if (a.B > 64) x = blocks(0);
  int run = 0;
  for (int i = 0;;) {
    const int u = (int)((unsigned)(x + per - 1) / (unsigned)per);
    const int inc = wave_scan(u);
    const int at = run + inc - u;
    const unsigned long long hit = __ballot(slot >= at && slot < at + u);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      return Share{i + l, __builtin_amdgcn_readlane(at, l), __builtin_amdgcn_readlane(u, l), per,
                   __builtin_amdgcn_readlane(held, l), __builtin_amdgcn_readlane(m, l)};
    }
    run += __builtin_amdgcn_readlane(inc, 63);
    i += 64;
    if (i >= a.B) return Share{-1, 0, 0, per, 0, 0};
    x = blocks(i);
  }
}
// LDS DMA of 4 B per lane to lds + 4 * lane (lds must be wave-uniform), as dma16.
__device__ __forceinline__ void dma4(const void *gp, uint32_t lds) {
  const uint32_t l = __builtin_amdgcn_readfirstlane(lds);
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\t"
      "global_load_lds_dword %1, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(gp), "s"(l)
      : "memory");
}

// N KB as dma16, the i-th from base + off[i] + 1024 i (base wave-uniform, off in bytes) to lds + 1024 i: an
// instruction's offset counts on both sides.  One M0 serves them.
template <int N>
__device__ __forceinline__ void dma16_run(uint64_t base, const int (&off)[N], uint32_t lds) {
  static_assert(N == 2 || N == 4);
  uint32_t saved;
  if constexpr (N == 2)
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %4\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %3\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:%c5\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(off[0]), "v"(off[1]), "s"(base), "s"(lds), "i"(1024)
        : "memory");
  else
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %6\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %5\n\t"
        "global_load_lds_dwordx4 %2, %5 offset:%c7\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:2 * %c7\n\t"
        "global_load_lds_dwordx4 %4, %5 offset:3 * %c7\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "s"(lds), "i"(1024)
        : "memory");
}
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// The kernel's arguments read anew, which keeps no register between two reads.
template <class A>
__device__ __forceinline__ A args_again() {
  typedef const __attribute__((address_space(4))) uint32_t *Words;
  Words p = (Words)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  struct { uint32_t w[sizeof(A) / 4]; } x;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(A) / 4); ++i) x.w[i] = p[i];
  return __builtin_bit_cast(A, x);
}

// Counts lie 256 bytes apart: side by side their atomics wait for one another (1 token of 256 in 64
// items 114 us instead of 60, 40 items of 300 over 500 keys 174 instead of 148).
constexpr int kQueueStep = 64;

}  // namespace
}  // namespace fc
