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

// One block of 64 rows of one key-value head of one item: the new rows in it, the queries of
// its group at those tokens, and, where the scale grows, the rows held in it before.
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

  // keys: rotated in float32, held in registers until the block's scale is known
  const int sub = tid % TPR, row = tid / TPR, p0 = sub * 8;
  float kr[KP][16], kmax = 0.f;
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    const int t = p * RPP + row;
    if (t < cnt) {
      const uint16_t *src = a.k + (long)b * a.k_item + (long)(i0 + t) * a.k_row + kv * HD + p0;
      float x[8], y[8];
      unpack8(*reinterpret_cast<const uint4 *>(src), x);
      unpack8(*reinterpret_cast<const uint4 *>(src + HALF), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 r = cs[t][p0 + e];
        kr[p][e] = x[e] * r.x - y[e] * r.y;
        kr[p][8 + e] = y[e] * r.x + x[e] * r.y;
        kmax = fmaxf(kmax, fmaxf(finite_abs(kr[p][e]), finite_abs(kr[p][8 + e])));
      }
    }
  }
  const int vsub = tid % VT, vrow = tid / VT;
  uint4 vr[VP];
  float vmax = 0.f;
#pragma unroll
  for (int p = 0; p < VP; ++p) {
    const int t = p * (kQThreads / VT) + vrow;
    if (t < cnt) {
      vr[p] = *reinterpret_cast<const uint4 *>(a.v + (long)b * a.v_item + (long)(i0 + t) * a.v_row +
                                               kv * HD + vsub * 8);
      float x[8];
      unpack8(vr[p], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) vmax = fmaxf(vmax, finite_abs(x[e]));
    }
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
  const int G = a.H / a.KV;
  for (int x = row; x < cnt * G; x += RPP) {
    const int t = x / G, h = kv * G + x % G;
    const uint16_t *src = a.q + (long)b * a.q_item + (long)(i0 + t) * a.q_row + (long)h * HD + p0;
    float u[8], w[8], y[16];
    unpack8(*reinterpret_cast<const uint4 *>(src), u);
    unpack8(*reinterpret_cast<const uint4 *>(src + HALF), w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 r = cs[t][p0 + e];
      y[e] = u[e] * r.x - w[e] * r.y;
      y[8 + e] = w[e] * r.x + u[e] * r.y;
    }
    uint16_t *dst = a.q_out + (((long)b * a.n + i0 + t) * a.H + h) * HD + p0;
    *reinterpret_cast<uint4 *>(dst) = pack8(y);
    *reinterpret_cast<uint4 *>(dst + HALF) = pack8(y + 8);
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
  const float low = -3.402823466e38f;
  w = (w >= low ? w : low) + 0.f;
  const uint32_t u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int pick_scan(int f, int *wsum, int *tot) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const unsigned long long bits = __ballot(f);
  const int pre = __popcll(bits & ((1ull << lane) - 1ull));
  __syncthreads();
  if (lane == 0) wsum[w] = __popcll(bits);
  __syncthreads();
  int base = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kPickThreads / 64; ++i) {
    if (i < w) base += wsum[i];
    all += wsum[i];
  }
  *tot = all;
  return base + pre;
}

// The kept rows of one head in ascending order: a radix select over 8 bits of the keys at a
// time finds the smallest kept key and how many rows of that key stay (the lowest ones).
__global__ __launch_bounds__(kPickThreads) void k_qevict_pick(EvictArgs a) {
  __shared__ int hist[256];
  __shared__ int wsum[kPickThreads / 64];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  const int b = blockIdx.x / a.KV, tid = threadIdx.x;
  const int n = q_held(a.len, b, a.cap);
  const float *w = a.weight + (long)blockIdx.x * a.cap;
  int32_t *kept = a.kept + (long)blockIdx.x * a.keep;
  const int left = min(n, a.keep);
  if (a.left && tid == 0 && blockIdx.x % a.KV == 0) a.left[b] = left;
  if (n <= a.keep) {
    for (int j = tid; j < a.keep; j += kPickThreads) kept[j] = j < n ? j : -1;
    return;
  }
  const int lo = a.sink, hi = n - a.recent;              // rows that compete: [lo, hi)
  const int take = a.keep - a.sink - a.recent;           // < hi - lo
  uint32_t prefix = 0;
  int need = take;
  if (take > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int x = tid; x < 256; x += kPickThreads) hist[x] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kPickThreads) {
        const uint32_t u = weight_key(w[j]);
        if (shift == 24 || (u >> (shift + 8)) == prefix) atomicAdd(&hist[(u >> shift) & 255u], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int d = 255, above = 0;
        while (d > 0 && above + hist[d] < need) above += hist[d--];
        s_prefix = prefix << 8 | (uint32_t)d;
        s_need = need - above;
      }
      __syncthreads();
      prefix = s_prefix;
      need = s_need;
    }
  }
  // rows above the smallest kept key and the first `need` rows equal to it
  int out = 0, ties = 0;
  for (int j = 0; j < n; j += kPickThreads) {
    const int r = j + tid;
    const bool end = r < n && (r < lo || r >= hi);
    const uint32_t u = r < n ? weight_key(w[r]) : 0u;
    const bool mid = r < n && !end && take > 0;
    int all;
    const bool tie = mid && u == prefix;
    const int at = ties + pick_scan(tie, wsum, &all);
    ties += all;
    const bool stay = end || (mid && u > prefix) || (tie && at < need);
    const int p = out + pick_scan(stay, wsum, &all);
    out += all;
    if (stay && p < a.keep) kept[p] = r;
  }
}

// One block of 64 kept rows of one head: gathered, scaled anew, written.
template <int HD>
__global__ __launch_bounds__(kQThreads) void k_qevict_move(EvictArgs a) {
  constexpr int TPR = HD / 16, RPP = kQThreads / TPR, KP = kQBlock / RPP;
  constexpr int TPD = kQThreads / HD, KPT = kQBlock / TPD;   // threads of a value column, keys of each
  __shared__ int src[kQBlock];
  __shared__ float red[2][kQThreads / 64];
  const int hb = blockIdx.y, b = hb / a.KV, blk = blockIdx.x, j0 = blk * kQBlock, tid = threadIdx.x;
  const int n = q_held(a.len, b, a.cap), left = min(n, a.keep), cnt = min(left - j0, kQBlock);
  if (cnt <= 0) return;
  if (tid < kQBlock)
    src[tid] = tid < cnt ? min(max(a.kept[(long)hb * a.keep + j0 + tid], 0), a.cap - 1) : 0;
  __syncthreads();
  const long nblk = a.cap / kQBlock, nblk2 = a.cap2 / kQBlock;
  const float *ks = a.ks + hb * nblk, *vs = a.vs + hb * nblk;
  const int sub = tid % TPR, row = tid / TPR;
  uint4 kr[KP];
  float kmul[KP], kmax = 0.f;
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    const int t = p * RPP + row;
    if (t < cnt) {
      const int s = src[t];
      kr[p] = *reinterpret_cast<const uint4 *>(a.k + ((long)hb * a.cap + s) * HD + sub * 16);
      kmul[p] = ks[s / kQBlock];
      const uint32_t w[4] = {kr[p].x, kr[p].y, kr[p].z, kr[p].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x = unpack_e4m3(w[i]);
        kmax = fmaxf(kmax, kmul[p] * fmaxf(fmaxf(finite_abs(x.x), finite_abs(x.y)), fmaxf(finite_abs(x.z), finite_abs(x.w))));
      }
    }
  }
  const int d = tid / TPD, v0 = tid % TPD * KPT;
  const uint8_t *vb = a.v + (long)hb * a.cap * HD + d * kQBlock;
  float vr[KPT], vmax = 0.f;
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    vr[i] = 0.f;
    if (v0 + i < cnt) {
      const int s = src[v0 + i];
      vr[i] = unpack_e4m3(vb[(long)(s / kQBlock) * (HD * kQBlock) + s % kQBlock]).x * vs[s / kQBlock];
      vmax = fmaxf(vmax, finite_abs(vr[i]));
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    kmax = fmaxf(kmax, __shfl_xor(kmax, o));
    vmax = fmaxf(vmax, __shfl_xor(vmax, o));
  }
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
  uint32_t w[KPT / 4];
#pragma unroll
  for (int i = 0; i < KPT / 4; ++i)
    w[i] = pack_e4m3(vr[4 * i] * vi, vr[4 * i + 1] * vi, vr[4 * i + 2] * vi, vr[4 * i + 3] * vi);
  if (cnt == kQBlock) {
#pragma unroll
    for (int i = 0; i < KPT / 16; ++i)
      reinterpret_cast<uint4 *>(vd)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < KPT; ++i)
      if (v0 + i < cnt) vd[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
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
  const int half = c.head_dim / 2;
  const bool one = !(rope.section[0] || rope.section[1] || rope.section[2]);
  a.sec0 = one ? half : rope.section[0];
  a.sec1 = one ? half : rope.section[0] + rope.section[1];
  for (int i = 0; i < 8; ++i) {
    a.lo[i] = std::pow(rope.theta, -2.0 * i / c.head_dim) / (2.0 * M_PI);
    a.hi[i] = std::pow(rope.theta, -16.0 * i / c.head_dim);
  }
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
  {
    ProfScope ps(ctx, st, "fc_qevict_pick");
    hipLaunchKernelGGL(k_qevict_pick, dim3((unsigned)(B * a.KV)), dim3(kPickThreads), 0, st, a);
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
