// The 8-bit token cache: rows appended (rotary positions on up to three axes, keys and
// values quantised by block) and rows evicted by the attention weight they have received.
//
//   append: K rows (a, b) -> (a cos t - b sin t, b cos t + a sin t) for the pairs
//           (i, i + hd / 2), t = pos[axis(i)] theta^(-2 i / hd); codes e4m3(x / s) with s the
//           block's scale.  It moves bytes: every q, k and v element is read and written once.
//   evict:  the kept rows' indexes by a radix select over the weights' bits, then each block
//           of kept rows gathered, scaled anew and written.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "fc_internal.h"
#include "qcache.h"

namespace fc {
namespace {

constexpr int kQThreads = 256;

struct AppendArgs {
  const uint16_t *q, *k, *v;                  // q may be null (no queries)
  long q_row, k_row, v_row;                   // elements from one token to the next
  long q_item, k_item, v_item;                // and from one item to the next
  const int32_t *pos, *len, *n_new;
  long pos_axis;                              // elements from one axis to the next
  uint16_t *q_out;
  uint8_t *kc, *vc;
  float *ks, *vs, *weight;
  int n, H, KV, cap, sec0, sec1;              // pairs below sec0 take axis 0, below sec1 axis 1
  Quot by_g;                                  // division by H / KV
  double lo[8], hi[8];                        // lo[i % 8] hi[i / 8] = theta^(-2 i / hd) / (2 pi) turns
};

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ void unpack8(uint4 u, float *x) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// Rounded to nearest even; a NaN stays one.
__device__ __forceinline__ uint4 pack8(const float *x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
    w[i] = __builtin_bit_cast(uint32_t, p);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A projection's row, read once: no place in the memory-side cache, which the writes need (a prompt
// of 8192 rows 41.6 -> 35.6 us).
__device__ __forceinline__ uint4 load_row16(const uint16_t *p) {
  const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// One block of 64 rows of one key-value head of one item: the new rows in it, the queries of
// its group at those tokens, and, where the scale grows, the rows held in it before.  A workgroup
// owns the block, so that its largest number is known before the first code is written.  Memory
// bounds it: 8192 rows of 28 + 4 + 4 heads (143 MB) 35.4 us, 4.0 TB/s, against 4.85 of a plain copy;
// a token's row 5.5 us, one latency after the other (lengths, positions, rows).
template <int HD>
__global__ __launch_bounds__(kQThreads) void k_qappend(AppendArgs a) {
  constexpr int HALF = HD / 2, TPR = HD / 16;       // threads of one row of pairs, 8 pairs each
  constexpr int RPP = kQThreads / TPR;              // rows of one pass
  constexpr int KP = kQBlock / RPP;                 // passes over a block's rows
  constexpr int VT = HD / 8, VP = kQBlock / (kQThreads / VT);
  constexpr int VSTR = kQBlock + 4;                 // value columns in LDS, off the bank period
  __shared__ float2 cs[kQBlock][HALF];
  __shared__ __align__(16) uint8_t vt[HD * VSTR];
  __shared__ float red[2][kQThreads / 64];
  const int b = blockIdx.y / a.KV, kv = blockIdx.y % a.KV, tid = threadIdx.x;
  const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
  const int blk = held / kQBlock + blockIdx.x, j0 = blk * kQBlock;
  const int lo = max(held, j0), cnt = min(held + m, j0 + kQBlock) - lo;
  if (cnt <= 0) return;
  const int i0 = lo - held, at = lo - j0;            // first new row's token, its place in the block
  const long hb = (long)b * a.KV + kv, nblk = a.cap / kQBlock;
  const float ks_old = at ? a.ks[hb * nblk + blk] : 0.f, vs_old = at ? a.vs[hb * nblk + blk] : 0.f;

  // the keys' and values' loads first; the angles are computed while they fly
  const int sub = tid % TPR, row = tid / TPR, p0 = sub * 8, vsub = tid % VT, vrow = tid / VT;
  uint4 klo[KP], khi[KP], vr[VP];
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    const int t = min(p * RPP + row, cnt - 1);
    const uint16_t *src = a.k + (long)b * a.k_item + (long)(i0 + t) * a.k_row + kv * HD + p0;
    klo[p] = *reinterpret_cast<const uint4 *>(src);
    khi[p] = *reinterpret_cast<const uint4 *>(src + HALF);
  }
#pragma unroll
  for (int p = 0; p < VP; ++p) {
    const int t = min(p * (kQThreads / VT) + vrow, cnt - 1);
    vr[p] = *reinterpret_cast<const uint4 *>(a.v + (long)b * a.v_item + (long)(i0 + t) * a.v_row + kv * HD + vsub * 8);
  }
  // angles in turns, reduced in 64 bits: float32 would lose those of far positions
  for (int x = tid; x < cnt * HALF; x += kQThreads) {
    const int t = x / HALF, p = x % HALF;
    const long ax = p < a.sec0 ? 0 : (p < a.sec1 ? 1 : 2);
    const double turn = (double)a.pos[ax * a.pos_axis + (long)b * a.n + i0 + t] * (a.lo[p & 7] * a.hi[p >> 3]);
    float s, c;
    sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
    cs[t][p] = make_float2(c, s);
  }
  __syncthreads();

  // keys: rotated in float32, held in registers until the block's scale is known (rows repeated
  // behind the last one set no other scale)
  float kr[KP][16], kmax = 0.f, vmax = 0.f;
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    const int t = min(p * RPP + row, cnt - 1);
    float x[8], y[8];
    unpack8(klo[p], x);
    unpack8(khi[p], y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 r = cs[t][p0 + e];
      kr[p][e] = x[e] * r.x - y[e] * r.y;
      kr[p][8 + e] = y[e] * r.x + x[e] * r.y;
      kmax = fmaxf(kmax, fmaxf(finite_abs(kr[p][e]), finite_abs(kr[p][8 + e])));
    }
  }
#pragma unroll
  for (int p = 0; p < VP; ++p) {
    float x[8];
    unpack8(vr[p], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) vmax = fmaxf(vmax, finite_abs(x[e]));
  }
  kmax = wave_max(kmax);
  vmax = wave_max(vmax);
  if (tid % 64 == 0) red[0][tid / 64] = kmax, red[1][tid / 64] = vmax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQThreads / 64; ++w) kmax = fmaxf(kmax, red[0][w]), vmax = fmaxf(vmax, red[1][w]);
  const float ks = fmaxf(scale_of(kmax), ks_old), vs = fmaxf(scale_of(vmax), vs_old);
  const float ki = 1.f / ks, vi = 1.f / vs;          // exact: powers of two
  if (tid == 0) a.ks[hb * nblk + blk] = ks, a.vs[hb * nblk + blk] = vs;

  uint8_t *kb = a.kc + (hb * a.cap + j0) * HD, *vb = a.vc + (hb * nblk + blk) * (long)(HD * kQBlock);
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    const int t = p * RPP + row;
    if (t < cnt) {
      float *x = kr[p];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] *= ki;
      uint8_t *dst = kb + (at + t) * HD + p0;
      *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_e4m3(x[0], x[1], x[2], x[3]), pack_e4m3(x[4], x[5], x[6], x[7]));
      *reinterpret_cast<uint2 *>(dst + HALF) = make_uint2(pack_e4m3(x[8], x[9], x[10], x[11]), pack_e4m3(x[12], x[13], x[14], x[15]));
    }
  }
  // held rows under the larger scale
  if (at && ks > ks_old) {
    const float ratio = ks_old * ki;
    for (int x = tid; x < at * HD / 4; x += kQThreads) {
      uint32_t *w = reinterpret_cast<uint32_t *>(kb) + x;
      *w = rescale_e4m3(*w, ratio);
    }
  }
  // values by columns: through LDS, then the bytes of the rows concerned and no others
#pragma unroll
  for (int p = 0; p < VP; ++p) {
    const int t = p * (kQThreads / VT) + vrow;
    if (t < cnt) {
      float x[8];
      unpack8(vr[p], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= vi;
      const uint32_t c0 = pack_e4m3(x[0], x[1], x[2], x[3]), c1 = pack_e4m3(x[4], x[5], x[6], x[7]);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        vt[(vsub * 8 + e) * VSTR + at + t] = (uint8_t)((e < 4 ? c0 : c1) >> (8 * (e & 3)));
    }
  }
  const bool again = at && vs > vs_old;
  if (again) {
    const float ratio = vs_old * vi;
    for (int x = tid; x < HD * at; x += kQThreads) {
      const int d = x / at, j = x % at;
      vt[d * VSTR + j] = (uint8_t)rescale_e4m3(vb[d * kQBlock + j], ratio);
    }
  }
  __syncthreads();
  const int from = again ? 0 : at, to = at + cnt;
  if (from == 0 && to == kQBlock) {
    for (int x = tid; x < HD * kQBlock / 16; x += kQThreads) {
      const uint32_t *w = reinterpret_cast<const uint32_t *>(vt + x / 4 * VSTR + x % 4 * 16);
      reinterpret_cast<uint4 *>(vb)[x] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
    for (int x = tid; x < HD * (to - from); x += kQThreads) {
      const int d = x / (to - from), j = from + x % (to - from);
      vb[d * kQBlock + j] = vt[d * VSTR + j];
    }
  }
  // a new row has received no weight yet
  if (a.weight && tid < cnt) a.weight[hb * a.cap + lo + tid] = 0.f;

  if (!a.q) return;
  // queries: four rows' loads at a time
  const int G = a.H / a.KV, rows = cnt * G;
  const uint16_t *qs = a.q + (long)b * a.q_item + (long)i0 * a.q_row + kv * G * HD + p0;
  uint16_t *qd = a.q_out + ((long)b * a.n + i0) * a.H * HD + kv * G * HD + p0;
  for (int x0 = row; x0 < rows; x0 += 4 * RPP) {
    uint4 lo4[4], hi4[4];
    int t[4], g[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int x = min(x0 + u * RPP, rows - 1);
      t[u] = a.by_g(x), g[u] = x - t[u] * G;
      const uint16_t *src = qs + (long)t[u] * a.q_row + g[u] * HD;
      lo4[u] = load_row16(src);
      hi4[u] = load_row16(src + HALF);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (x0 + u * RPP >= rows) break;
      float v[8], w[8], y[16];
      unpack8(lo4[u], v);
      unpack8(hi4[u], w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 r = cs[t[u]][p0 + e];
        y[e] = v[e] * r.x - w[e] * r.y;
        y[8 + e] = w[e] * r.x + v[e] * r.y;
      }
      uint16_t *dst = qd + ((long)t[u] * a.H + g[u]) * HD;
      *reinterpret_cast<uint4 *>(dst) = pack8(y);
      *reinterpret_cast<uint4 *>(dst + HALF) = pack8(y + 8);
    }
  }
}

// ------------------------------------------------------------------------------- evict
struct EvictArgs {
  const uint8_t *k, *v;
  const float *ks, *vs, *weight;
  uint8_t *k2, *v2;
  float *ks2, *vs2, *weight2;      // weight2 may be null
  const int32_t *len;
  int32_t *kept, *left;            // left may be null
  int KV, cap, cap2, keep, sink, recent;
};

constexpr int kPickThreads = 1024;

// Weights in an order of unsigned integers; a NaN and what lies below the finite numbers
// count as the lowest finite one, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(fmaxf(w, -3.402823466e38f) + 0.f);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

constexpr int kPickWaves = kPickThreads / 64;

// Sum of a number over the threads before this one (waves in order, lanes in order); total: over all.
__device__ __forceinline__ int pick_scan(int x, int *wsum, int &total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 63) wsum[w] = inc;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < kPickWaves; ++i) {
    if (i < w) base += wsum[i];
    total += wsum[i];
  }
  return base + inc - x;
}

constexpr int kPickBins = 2048;
// The digits of a key: bits 31-21, 20-10, 9-0.
template <int STEP>
struct Digit {
  static constexpr int shift = STEP == 0 ? 21 : (STEP == 1 ? 10 : 0), bits = STEP == 2 ? 10 : 11;
  __device__ static bool counts(uint32_t u, uint32_t prefix) {
    if constexpr (STEP == 0) return u != 0u;
    else return u >> (shift + bits) == prefix;
  }
  __device__ static int of(uint32_t u) { return u >> shift & ((1 << bits) - 1); }
};
// Places left in the selection: the digits of the smallest kept key found so far, and how many rows
// of that prefix stay.
struct Places {
  uint32_t prefix;
  int need;
};
// A digit more, from its counts: thread t holds those of bins 2047 - 2 t and 2046 - 2 t, so that a scan
// runs from the largest key down.
template <int STEP>
__device__ __forceinline__ Places next_digit(Places p, int c0, int c1, int *wsum, int *found) {
  int total;
  const int bin = kPickBins - 1 - 2 * (int)threadIdx.x, before = pick_scan(c0 + c1, wsum, total);
  if (before < p.need && before + c0 >= p.need) found[0] = bin, found[1] = p.need - before;
  else if (before + c0 < p.need && before + c0 + c1 >= p.need) found[0] = bin - 1, found[1] = p.need - before - c0;
  __syncthreads();
  return Places{STEP == 0 ? (uint32_t)found[0] : p.prefix << Digit<STEP>::bits | (uint32_t)found[0], found[1]};
}
// f(row, its key) for the rows row0 + lane + 64 i, i < runs, of a wave.  Keys of rows that compete, [lo,
// hi), are at least 0x00800000 (the lowest finite number's); the others, which stay whatever their
// weight or lie behind the last row, get 0.  N loads at a time, the last ones repeated where the
// run ends.
template <int N, class F>
__device__ __forceinline__ void each_key(const float *w, int row0, int runs, int lo, int hi, int cap, F f) {
  const int lane = threadIdx.x & 63;
  for (int i = 0; i < runs; i += N) {
    const int j0 = row0 + 64 * i, j1 = row0 + 64 * runs;
    float x[N];
    if (j0 + 64 * N <= j1 && j0 >= lo && j0 + 64 * N <= hi) {      // all of them compete
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = w[j0 + lane + 64 * e];
#pragma unroll
      for (int e = 0; e < N; ++e) f(j0 + lane + 64 * e, weight_key(x[e]));
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = w[min(j0 + lane + 64 * e, cap - 1)];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int j = j0 + lane + 64 * e;
        if (j0 + 64 * e < j1) f(j, j >= lo && j < hi ? weight_key(x[e]) : 0u);
      }
    }
  }
}
// The kept ones of a workgroup's rows written down in order: those above the smallest kept key, those
// that stay whatever their weight (key 0, below n), and of those that equal it what `need` leaves after
// the `tie` before; `out` rows are kept before.  each(f) as each_key, a wave's rows behind those of the
// waves before it.
template <class Each>
__device__ __forceinline__ void write_kept(Each each, Places p, int n, int keep, int out, int tie, int *wabove, int *wties,
                                           int32_t *kept) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto stays = [&](int r, uint32_t u) { return u > p.prefix || (u == 0u && r < n); };
  int above = 0, ties = 0;
  each([&](int r, uint32_t u) {
    above += __popcll(__ballot(stays(r, u)));
    ties += __popcll(__ballot(u == p.prefix));
  });
  if (lane == 0) wabove[wave] = above, wties[wave] = ties;
  __syncthreads();
  for (int i = 0; i < wave; ++i) {
    out += wabove[i] + min(max(p.need - tie, 0), wties[i]);
    tie += wties[i];
  }
  const unsigned long long below = (1ull << lane) - 1ull;
  each([&](int r, uint32_t u) {
    const unsigned long long t = __ballot(u == p.prefix);
    const bool stay = stays(r, u) || (u == p.prefix && tie + __popcll(t & below) < p.need);
    tie += __popcll(t);
    const unsigned long long k = __ballot(stay);
    const int to = out + __popcll(k & below);
    out += __popcll(k);
    if (stay && to < keep) kept[to] = r;
  });
}

// The kept rows of one head in ascending order, by one workgroup.  A radix select over 11, 11 and 10
// bits of the weights' keys finds the smallest kept key and how many rows of that key stay (the lowest
// ones); then every wave counts, and writes down, what stays of its own run of rows.
// Weights share few exponents, so the first digit's counts stand in 4 copies, one for every fourth
// lane (16 where there are more rows to count): with one the lanes of a wave wait for each other.  IT > 0: a lane holds IT keys in
// registers (up to 1024 IT rows; 64 of them spill: 90 us for 65536 rows against 57); IT = 0 reads
// the weights anew in each pass, where the workspace has no room for the counts of several
// workgroups.  Latency bounds it, a chain of passes and barriers: 7.5 us for 2176 rows.
template <int IT>
__global__ __launch_bounds__(kPickThreads) void k_qevict_pick(EvictArgs a) {
  constexpr int COPIES = IT ? 4 : 16;                 // fewer to clear and to add up for few rows
  __shared__ __align__(16) int hist[kPickBins * COPIES];  // 128 KB of 16 copies: one workgroup on a CU
  __shared__ int wsum[kPickWaves], wabove[kPickWaves], wties[kPickWaves], found[2];
  const int b = blockIdx.x / a.KV, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = q_held(a.len, b, a.cap);
  const float *w = a.weight + (long)blockIdx.x * a.cap;
  int32_t *kept = a.kept + (long)blockIdx.x * a.keep;
  if (a.left && tid == 0 && blockIdx.x % a.KV == 0) a.left[b] = min(n, a.keep);
  if (n <= a.keep) {
    for (int j = tid; j < a.keep; j += kPickThreads) kept[j] = j < n ? j : -1;
    return;
  }
  const int lo = a.sink, hi = n - a.recent;              // rows that compete: [lo, hi)
  const int take = a.keep - a.sink - a.recent;           // < hi - lo
  const int runs = IT ? IT : (n + kPickThreads - 1) / kPickThreads, row0 = wave * runs * 64;
  uint32_t key[IT ? IT : 1];
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int j = row0 + lane + 64 * i;
    const uint32_t u = weight_key(w[min(j, a.cap - 1)]);   // no branch: the loads overlap
    key[i] = j >= lo && j < hi ? u : 0u;
  }
  auto each = [&](auto f) {
    if constexpr (IT > 0) {
#pragma unroll
      for (int i = 0; i < IT; ++i) f(row0 + lane + 64 * i, key[i]);
    } else {
      each_key<16>(w, row0, runs, lo, hi, a.cap, f);
    }
  };
  Places p{~0u, take};                 // take 0: no row is above or ties
  if (take > 0) {
    auto digit = [&](auto tag) {
      constexpr int step = decltype(tag)::value, copies = step == 0 ? COPIES : 1;
      for (int x = tid; x < kPickBins * copies / 4; x += kPickThreads) reinterpret_cast<int4 *>(hist)[x] = make_int4(0, 0, 0, 0);
      __syncthreads();
      each([&](int, uint32_t u) {
        if (Digit<step>::counts(u, p.prefix)) atomicAdd(&hist[Digit<step>::of(u) * copies + (step == 0 ? lane & (COPIES - 1) : 0)], 1);
      });
      __syncthreads();
      int c[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int bin = kPickBins - 1 - 2 * tid - e;
        c[e] = 0;
        if constexpr (step == 0) {
#pragma unroll
          for (int x = 0; x < COPIES / 4; ++x) {
            const int4 y = reinterpret_cast<const int4 *>(hist)[bin * (COPIES / 4) + x];
            c[e] += y.x + y.y + y.z + y.w;
          }
        } else {
          c[e] = hist[bin];
        }
      }
      p = next_digit<step>(p, c[0], c[1], wsum, found);
    };
    digit(std::integral_constant<int, 0>{});
    digit(std::integral_constant<int, 1>{});
    digit(std::integral_constant<int, 2>{});
  }
  write_kept(each, p, n, a.keep, 0, 0, wabove, wties, kept);
}

// The same by `parts` workgroups of each head, a kernel to a digit: each counts its own rows, the next
// one adds the parts' counts up and finds the digit; the last one also finds from them how many rows
// stay before its own.  The counts of a head are read by as many workgroups as it has, which share an
// XCD's L2 where the heads are a multiple of 8 (heads fastest: workgroups go round the 8 in turn).
// For caches of more than 16384 rows: 32 heads of 65536 take 30 us against 57 by one workgroup each,
// 4 of 262144 with their move 100 against 214, but 4 of 16384 35 against 28 (launches).
constexpr int kMaxParts = 8;
struct PickArgs {
  EvictArgs e;
  int *count;                          // [head][3 digits][part][kPickBins]
  Places *places;                      // [head][2]: after the first and the second digit
  int *above;                          // [head][part] rows above the prefix of the first two digits
  int parts;
};
// Counts of a digit's bins 2046 - 2 t (x) and 2047 - 2 t (y) in every part.
struct PartCounts {
  int2 c[kMaxParts];
  int c0 = 0, c1 = 0;                  // y and x summed
};
__device__ __forceinline__ int *part_bins(const PickArgs &a, int step, int part) {
  return a.count + (((long)blockIdx.x * 3 + step) * a.parts + part) * kPickBins + kPickBins - 2 - 2 * (int)threadIdx.x;
}
__device__ __forceinline__ PartCounts all_parts(const PickArgs &a, int step) {
  PartCounts p;
#pragma unroll
  for (int i = 0; i < kMaxParts; ++i) p.c[i] = *reinterpret_cast<const int2 *>(part_bins(a, step, min(i, a.parts - 1)));
#pragma unroll
  for (int i = 0; i < kMaxParts; ++i)
    if (i < a.parts) p.c0 += p.c[i].y, p.c1 += p.c[i].x;
  return p;
}
// A wave's rows: from row0 on, `runs` times 64; its workgroup's start at `start`.
struct PartRows {
  int start, row0, runs;
};
__device__ __forceinline__ PartRows part_rows(const PickArgs &a, int n) {
  const int runs = (n + kPickThreads * a.parts - 1) / (kPickThreads * a.parts), start = blockIdx.y * runs * kPickThreads;
  return PartRows{start, start + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * runs * 64, runs};
}

template <int STEP>
__global__ __launch_bounds__(kPickThreads) void k_qevict_count(PickArgs a) {
  constexpr int COPIES = STEP == 0 ? 4 : 1;
  __shared__ __align__(16) int hist[kPickBins * COPIES];
  __shared__ int wsum[kPickWaves], found[2];
  const EvictArgs &e = a.e;
  const int head = blockIdx.x, tid = threadIdx.x, n = q_held(e.len, head / e.KV, e.cap);
  const int take = e.keep - e.sink - e.recent;
  if (n <= e.keep || take == 0) return;
  for (int x = tid; x < kPickBins * COPIES / 4; x += kPickThreads) reinterpret_cast<int4 *>(hist)[x] = make_int4(0, 0, 0, 0);
  Places p{~0u, take};
  if constexpr (STEP > 0) {
    if (STEP == 2) p = a.places[head * 2];
    const PartCounts c = all_parts(a, STEP - 1);
    p = next_digit<STEP - 1>(p, c.c0, c.c1, wsum, found);
    if (blockIdx.y == 0 && tid == 0) a.places[head * 2 + STEP - 1] = p;
  }
  __syncthreads();
  const PartRows rows = part_rows(a, n);
  int above = 0;
  each_key<8>(e.weight + (long)head * e.cap, rows.row0, rows.runs, e.sink, n - e.recent, e.cap, [&](int, uint32_t u) {
    if (Digit<STEP>::counts(u, p.prefix)) atomicAdd(&hist[Digit<STEP>::of(u) * COPIES + (tid & (COPIES - 1))], 1);
    if constexpr (STEP == 2) above += u >> Digit<2>::bits > p.prefix;
  });
  __syncthreads();
  int c[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int bin = kPickBins - 2 - 2 * tid + i;
    if constexpr (COPIES == 4) {
      const int4 y = reinterpret_cast<const int4 *>(hist)[bin];
      c[i] = y.x + y.y + y.z + y.w;
    } else {
      c[i] = hist[bin];
    }
  }
  *reinterpret_cast<int2 *>(part_bins(a, STEP, blockIdx.y)) = make_int2(c[0], c[1]);
  if constexpr (STEP == 2) {
    int total;
    pick_scan(above, wsum, total);
    if (tid == 0) a.above[head * a.parts + blockIdx.y] = total;
  }
}

__global__ __launch_bounds__(kPickThreads) void k_qevict_write(PickArgs a) {
  __shared__ int wsum[kPickWaves], wabove[kPickWaves], wties[kPickWaves], found[2];
  const EvictArgs &e = a.e;
  const int head = blockIdx.x, part = blockIdx.y, b = head / e.KV, tid = threadIdx.x, n = q_held(e.len, b, e.cap);
  int32_t *kept = e.kept + (long)head * e.keep;
  if (e.left && tid == 0 && head % e.KV == 0 && part == 0) e.left[b] = min(n, e.keep);
  if (n <= e.keep) {
    for (int j = part * kPickThreads + tid; j < e.keep; j += a.parts * kPickThreads) kept[j] = j < n ? j : -1;
    return;
  }
  const int lo = e.sink, hi = n - e.recent, take = e.keep - e.sink - e.recent;
  const PartRows rows = part_rows(a, n);
  // rows kept before this part's: those whatever their weight, those above the smallest kept key, ties
  int out = min(rows.start, lo) + max(min(rows.start, n) - hi, 0), tie = 0;
  Places p{~0u, 0};
  if (take > 0) {
    const PartCounts c = all_parts(a, 2);
    p = next_digit<2>(a.places[head * 2 + 1], c.c0, c.c1, wsum, found);
    const int digit = p.prefix & 1023u, top = kPickBins - 1 - 2 * tid;
    int above = 0, ties = 0;
#pragma unroll
    for (int i = 0; i < kMaxParts; ++i)
      if (i < part) {
        above += (top > digit ? c.c[i].y : 0) + (top - 1 > digit ? c.c[i].x : 0);
        ties += (top == digit ? c.c[i].y : 0) + (top - 1 == digit ? c.c[i].x : 0);
      }
    if (tid < part) above += a.above[head * a.parts + tid];
    int total;
    pick_scan(above, wsum, total);
    out += total;
    __syncthreads();
    pick_scan(ties, wsum, tie);
    out += min(p.need, tie);
  }
  const float *w = e.weight + (long)head * e.cap;
  write_kept([&](auto f) { each_key<8>(w, rows.row0, rows.runs, lo, hi, e.cap, f); }, p, n, e.keep, out, tie, wabove, wties, kept);
}

// One block of 64 kept rows of one head: gathered, scaled anew, written.  Key rows are read alone;
// values lie by columns, so each source block with a kept row in it is read whole (8 KB at hd
// 128), four at a time through LDS, where single bytes cost nothing.  Memory bounds it: 32 heads,
// 16384 of 62000 rows each (400 MB read, by the counters, and 137 written) 123 us, 4.4 TB/s.  Two
// blocks at a time 142, eight 156 (LDS leaves fewer workgroups); neighbours on one XCD, or loads past
// the memory-side cache: no gain.
template <int HD>
__global__ __launch_bounds__(kQThreads) void k_qevict_move(EvictArgs a) {
  constexpr int TPR = HD / 16, RPP = kQThreads / TPR, KP = kQBlock / RPP;
  constexpr int TPD = kQThreads / HD, KPT = kQBlock / TPD;   // threads of a value column, keys of each
  constexpr int GROUP = 4, VSTR = kQBlock + 4;               // source blocks at a time; off the bank period
  constexpr int CPT = HD * kQBlock / 16 / kQThreads;         // 16-byte pieces of a block for each thread
  __shared__ int src[kQBlock];
  __shared__ float scale[2][kQBlock];                        // of each row's keys and values
  __shared__ float red[2][kQThreads / 64];
  __shared__ __align__(16) uint8_t vt[GROUP][HD * VSTR];
  const int hb = blockIdx.y, b = hb / a.KV, blk = blockIdx.x, j0 = blk * kQBlock, tid = threadIdx.x;
  const int n = q_held(a.len, b, a.cap), left = min(n, a.keep), cnt = min(left - j0, kQBlock);
  if (cnt <= 0) return;
  // (the last row again behind the end, so that src stays ascending)
  if (tid < kQBlock) src[tid] = min(max(a.kept[(long)hb * a.keep + j0 + min(tid, cnt - 1)], 0), a.cap - 1);
  __syncthreads();
  const long nblk = a.cap / kQBlock, nblk2 = a.cap2 / kQBlock;
  const float *ks = a.ks + hb * nblk, *vs = a.vs + hb * nblk;
  const int sub = tid % TPR, row = tid / TPR;
  uint4 kr[KP];
  float kmul[KP], kmax = 0.f;
  float mul = 0.f;
  if (tid < 2 * kQBlock) mul = (tid < kQBlock ? ks : vs)[src[tid % kQBlock] / kQBlock];
#pragma unroll
  for (int p = 0; p < KP; ++p)
    kr[p] = *reinterpret_cast<const uint4 *>(a.k + ((long)hb * a.cap + src[p * RPP + row]) * HD + sub * 16);
  const int d = tid / TPD, v0 = tid % TPD * KPT;
  const uint8_t *vb = a.v + (long)hb * a.cap * HD;
  uint32_t vc[KPT / 4];                 // codes of the thread's keys of its column
  float vmul[KPT], vmax = 0.f;
#pragma unroll
  for (int i = 0; i < KPT / 4; ++i) vc[i] = 0;
  const int b0 = src[0] / kQBlock, b1 = src[cnt - 1] / kQBlock;
  for (int g = b0; g <= b1; g += GROUP) {
    uint4 x[GROUP][CPT];
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
#pragma unroll
      for (int c = 0; c < CPT; ++c)
        x[i][c] = *reinterpret_cast<const uint4 *>(vb + (long)min(g + i, b1) * (HD * kQBlock) + (c * kQThreads + tid) * 16);
    if (g > b0) __syncthreads();        // the group before has been read
    else if (tid < 2 * kQBlock) scale[tid / kQBlock][tid % kQBlock] = mul;
#pragma unroll
    for (int i = 0; i < GROUP; ++i)
#pragma unroll
      for (int c = 0; c < CPT; ++c) {
        const int p = c * kQThreads + tid;
        uint32_t *to = reinterpret_cast<uint32_t *>(&vt[i][p / 4 * VSTR + p % 4 * 16]);
        to[0] = x[i][c].x, to[1] = x[i][c].y, to[2] = x[i][c].z, to[3] = x[i][c].w;
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int s = src[v0 + i], at = s / kQBlock - g;
      if (at >= 0 && at < GROUP) vc[i / 4] |= (uint32_t)vt[at][d * VSTR + s % kQBlock] << (8 * (i % 4));
    }
  }
#pragma unroll
  for (int i = 0; i < KPT; ++i) vmul[i] = scale[1][v0 + i];
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    kmul[p] = scale[0][p * RPP + row];
    const uint32_t w[4] = {kr[p].x, kr[p].y, kr[p].z, kr[p].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = unpack_e4m3(w[i]);
      kmax = fmaxf(kmax, kmul[p] * fmaxf(fmaxf(finite_abs(x.x), finite_abs(x.y)), fmaxf(finite_abs(x.z), finite_abs(x.w))));
    }
  }
#pragma unroll
  for (int i = 0; i < KPT / 4; ++i) {
    const float4 x = unpack_e4m3(vc[i]);
    vmax = fmaxf(vmax, fmaxf(fmaxf(finite_abs(x.x) * vmul[4 * i], finite_abs(x.y) * vmul[4 * i + 1]),
                             fmaxf(finite_abs(x.z) * vmul[4 * i + 2], finite_abs(x.w) * vmul[4 * i + 3])));
  }
  kmax = wave_max(kmax);
  vmax = wave_max(vmax);
  if (tid % 64 == 0) red[0][tid / 64] = kmax, red[1][tid / 64] = vmax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQThreads / 64; ++w) kmax = fmaxf(kmax, red[0][w]), vmax = fmaxf(vmax, red[1][w]);
  const float ksn = scale_of(kmax), vsn = scale_of(vmax), ki = 1.f / ksn, vi = 1.f / vsn;
  if (tid == 0) a.ks2[hb * nblk2 + blk] = ksn, a.vs2[hb * nblk2 + blk] = vsn;
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    const int t = p * RPP + row;
    if (t < cnt) {
      const float r = kmul[p] * ki;
      *reinterpret_cast<uint4 *>(a.k2 + ((long)hb * a.cap2 + j0 + t) * HD + sub * 16) =
          make_uint4(rescale_e4m3(kr[p].x, r), rescale_e4m3(kr[p].y, r), rescale_e4m3(kr[p].z, r), rescale_e4m3(kr[p].w, r));
    }
  }
  uint8_t *vd = a.v2 + ((long)hb * nblk2 + blk) * (HD * kQBlock) + d * kQBlock + v0;
#pragma unroll
  for (int i = 0; i < KPT / 4; ++i) {
    const float4 x = unpack_e4m3(vc[i]);
    vc[i] = pack_e4m3(x.x * (vmul[4 * i] * vi), x.y * (vmul[4 * i + 1] * vi), x.z * (vmul[4 * i + 2] * vi), x.w * (vmul[4 * i + 3] * vi));
  }
  if (cnt == kQBlock) {
#pragma unroll
    for (int i = 0; i < KPT / 16; ++i)
      reinterpret_cast<uint4 *>(vd)[i] = make_uint4(vc[4 * i], vc[4 * i + 1], vc[4 * i + 2], vc[4 * i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < KPT; ++i)
      if (v0 + i < cnt) vd[i] = (uint8_t)(vc[i / 4] >> (8 * (i % 4)));
  }
  if (a.weight2 && tid < cnt) a.weight2[(long)hb * a.cap2 + j0 + tid] = a.weight[(long)hb * a.cap + src[tid]];
}

}  // namespace

fc_status launch_qcache_append(fc_ctx *ctx, const fc_qcache &c, const fc_rope_axes &rope,
                               const fc_qkv_rows &x, const int32_t *pos, const int32_t *len,
                               const int32_t *n_new, uint16_t *q_out, int B, int n, hipStream_t st) {
  AppendArgs a{};
  a.q = x.q, a.k = x.k, a.v = x.v;
  a.q_row = x.q_row, a.k_row = x.k_row, a.v_row = x.v_row;
  a.q_item = x.q_item, a.k_item = x.k_item, a.v_item = x.v_item;
  a.pos = pos, a.len = len, a.n_new = n_new, a.pos_axis = (long)B * n;
  a.q_out = q_out;
  a.kc = c.k, a.vc = c.v, a.ks = c.k_scale, a.vs = c.v_scale, a.weight = c.weight;
  a.n = n, a.H = x.n_heads, a.KV = c.n_kv_heads, a.cap = c.capacity;
  a.by_g = quot_by(a.H / a.KV);
  const int half = c.head_dim / 2;
  const bool one = !(rope.section[0] || rope.section[1] || rope.section[2]);
  a.sec0 = one ? half : rope.section[0];
  a.sec1 = one ? half : rope.section[0] + rope.section[1];
  // two powers and products of them (sixteen calls of pow take as long as a small launch): with pow
  // within one unit in the last place, 2 2^-53, a factor is within 23 2^-53 and their product within 44
  const double r = std::pow(rope.theta, -2.0 / c.head_dim), r8 = std::pow(rope.theta, -16.0 / c.head_dim);
  a.lo[0] = 1.0 / (2.0 * M_PI), a.hi[0] = 1.0;
  for (int i = 1; i < 8; ++i) a.lo[i] = a.lo[i - 1] * r, a.hi[i] = a.hi[i - 1] * r8;
  // the new rows start inside a block, so one more may be touched than they fill
  const dim3 grid((unsigned)((n + 2 * kQBlock - 2) / kQBlock), (unsigned)(B * c.n_kv_heads));
  ProfScope ps(ctx, st, "fc_qappend");
  if (c.head_dim == 128)
    hipLaunchKernelGGL(k_qappend<128>, grid, dim3(kQThreads), 0, st, a);
  else
    hipLaunchKernelGGL(k_qappend<64>, grid, dim3(kQThreads), 0, st, a);
  FC_LAUNCH_OK(st, "k_qappend");
  return FC_OK;
}

fc_status launch_qcache_evict(fc_ctx *ctx, const fc_qcache &s, const fc_qcache &d, const int32_t *len,
                              int keep, int sink, int recent, int32_t *kept, int32_t *len_out, int B,
                              hipStream_t st) {
  EvictArgs a{};
  a.k = s.k, a.v = s.v, a.ks = s.k_scale, a.vs = s.v_scale, a.weight = s.weight;
  a.k2 = d.k, a.v2 = d.v, a.ks2 = d.k_scale, a.vs2 = d.v_scale, a.weight2 = d.weight;
  a.len = len, a.kept = kept, a.left = len_out;
  a.KV = s.n_kv_heads, a.cap = s.capacity, a.cap2 = d.capacity;
  a.keep = keep, a.sink = sink, a.recent = recent;
  // the workgroups of a head: as many as run at once, each with 4096 rows at least, where their counts fit
  const long heads = (long)B * a.KV;
  long parts = std::min<long>(std::min<long>(kMaxParts, a.cap / 4096), std::max<long>(1, 2L * ctx->num_cus / heads));
  parts = std::min<long>(parts, ((long)ctx->part_elems - (4 + kMaxParts) * heads) / (heads * 3 * kPickBins));
  if (a.cap > 16 * kPickThreads && parts > 1) {
    PickArgs p{a, reinterpret_cast<int *>(ctx->part), nullptr, nullptr, (int)parts};
    p.places = reinterpret_cast<Places *>(p.count + heads * 3 * parts * kPickBins);
    p.above = reinterpret_cast<int *>(p.places + 2 * heads);
    const dim3 grid((unsigned)heads, (unsigned)parts), block(kPickThreads);
    ProfScope ps(ctx, st, "fc_qevict_pick");
    hipLaunchKernelGGL(k_qevict_count<0>, grid, block, 0, st, p);
    FC_LAUNCH_OK(st, "k_qevict_count");
    hipLaunchKernelGGL(k_qevict_count<1>, grid, block, 0, st, p);
    FC_LAUNCH_OK(st, "k_qevict_count");
    hipLaunchKernelGGL(k_qevict_count<2>, grid, block, 0, st, p);
    FC_LAUNCH_OK(st, "k_qevict_count");
    hipLaunchKernelGGL(k_qevict_write, grid, block, 0, st, p);
    FC_LAUNCH_OK(st, "k_qevict_write");
  } else {
    ProfScope ps(ctx, st, "fc_qevict_pick");
    const dim3 grid((unsigned)heads), block(kPickThreads);
    if (a.cap <= 4 * kPickThreads) hipLaunchKernelGGL(k_qevict_pick<4>, grid, block, 0, st, a);
    else if (a.cap <= 8 * kPickThreads) hipLaunchKernelGGL(k_qevict_pick<8>, grid, block, 0, st, a);
    else if (a.cap <= 16 * kPickThreads) hipLaunchKernelGGL(k_qevict_pick<16>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(k_qevict_pick<0>, grid, block, 0, st, a);
    FC_LAUNCH_OK(st, "k_qevict_pick");
  }
  const dim3 grid((unsigned)((keep + kQBlock - 1) / kQBlock), (unsigned)(B * a.KV));
  ProfScope ps(ctx, st, "fc_qevict_move");
  if (s.head_dim == 128)
    hipLaunchKernelGGL(k_qevict_move<128>, grid, dim3(kQThreads), 0, st, a);
  else
    hipLaunchKernelGGL(k_qevict_move<64>, grid, dim3(kQThreads), 0, st, a);
  FC_LAUNCH_OK(st, "k_qevict_move");
  return FC_OK;
}

}  // namespace fc
