// Attention of new rows over the 8-bit token cache.
//
//   S_ij = c q_i . k_j over the rows j <= held + i that the key mask shows,
//   P = softmax_j(S), out_i = sum_j P_ij v_j (a row that sees no key: 0),
//   weight_j += sum over the rows i and the query heads of j's group of P_ij (on request).
//
// The G query heads of a group share their keys, so the n tokens of an item make R = n G rows
// of a matrix product per key-value head: row r is head r % G of the group at token r / G.
// S^T = K Q^T and O^T = V^T P^T: a lane then holds one query row, so the softmax's running
// maximum and sum, and the rescaling of O, are per-lane scalars.  Both A operands are read as
// the cache stores them (K by rows, V by columns of a block), each with 16-byte loads that
// cover whole 64-byte pieces, and P is already in the layout of the second product's B operand:
// the rows of an S^T tile are permuted so that a lane's 16 probabilities of a block belong to
// 16 neighbouring keys.  e4m3 numbers are dequantised to bfloat16, which is exact, and the
// products run on the bfloat16 matrix instructions: those of 8 bits align the products to the
// largest before they add them (7e-6 of sum |q k| at worst on normal data; bfloat16 2e-8), which
// the added-up weights, float32 numbers, would show.  P is rounded to bfloat16 for the second
// product (half a step, 2^-8 of each term of a float32 sum whose terms err apart).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attn_dev.h"
#include "fc_internal.h"
#include "qcache.h"

namespace fc {
namespace {

struct QAttnArgs {
  const uint8_t *k, *v;
  const float *ks, *vs;
  float *weight;
  const uint16_t *q;
  uint16_t *out;
  const int32_t *len, *n_new;
  const uint8_t *mask;               // [B][cap], or null
  float2 *ml;                        // running maximum (log2) and sum of each split's rows,
  float *part;                       // unnormalised outputs: k_qattn [KV][slots][R][hd], k_qattn_rows as
                                     // k_qattn_join_rows has it
  int2 *plan;                        // [B] k_qattn: an item's first slot and its slots
  float *lse;                        // [B KV][R] log2 of each row's sum, or null
  float *logit;                      // [B KV][R][cap] scores (log2), or null
  float c;                           // scale log2(e)
  int B, n, H, KV, G, cap, splits, least, tile_rows, slots;
  int *queue, pieces;                // k_qattn_rows: 8 counts of pieces taken behind the first ones, or null
  Quot by_g;                         // division by G
  uint32_t flip;                     // sign bits of a query pair to turn
};

// Eight e4m3 codes (two words) times a power of two, as bfloat16 (exact).
__device__ __forceinline__ bf16x8 dequant8(uint32_t w0, uint32_t w1, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Values enter the products 2^-17 smaller than they are, and an output's last factor makes up for
// it.  Scales reach 2^120, where codes of 256 and more stand for numbers beyond bfloat16 and 0 times
// one (a hidden row's) would be NaN, and outputs are sums of up to 2^8 |v| a row before their division.
// 17 is as far as the least number, 2^-109, stays a normal bfloat16; powers of two round nothing.
// Blocks that nobody sees may hold any scale: what comes out is finite.
constexpr uint32_t kValueDown = 17;
constexpr float kValueUp = 131072.f;
__device__ __forceinline__ float value_scale(float s) {
  return __uint_as_float((max(__float_as_uint(s) & 0x7FFFFFFFu, (127u + kQLowExp) << 23)) - (kValueDown << 23));
}
// What an unnormalised output is multiplied with, from its row's sum (a row that sees no key: 0).
__device__ __forceinline__ float output_factor(float l) { return l == 0.f ? 0.f : kValueUp / l; }
// Bytes of w that hold a NaN (0x7f or 0xff): their top bits, and as 0x01 each.
__device__ __forceinline__ uint32_t nan_tops(uint32_t w) { return (w & 0x7F7F7F7Fu) + 0x01010101u; }
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return nan_tops(w) >> 7 & 0x01010101u; }
// The four low bits of such bytes, side by side.
__device__ __forceinline__ uint32_t byte_bits(uint32_t n) { return (n * 0x01020408u) >> 24 & 15u; }
// The four low bits of b as bytes of 0xff.
__device__ __forceinline__ uint32_t bit_bytes(uint32_t b) { return ((b & 15u) * 0x00204081u & 0x01010101u) * 255u; }
// Bytes of w that are not zero, as 0xff each.
__device__ __forceinline__ uint32_t set_bytes(uint32_t w) {
  return ((((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w) >> 7 & 0x01010101u) * 255u;
}
// log2 of the sum of 2^S of a row from its maximum and sum: the probability of key j is 2^(S_j - L).
// A row that sees no key gets +inf (every weight 0).
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.f ? __builtin_inff() : (m == kNegInf ? 0.f : m) + __log2f(l);
}
__device__ __forceinline__ float prob(float y, float L) { return y == kNegInf ? 0.f : exp2_fast(y - L); }

// All rows of an item (MT tiles of 16: up to 32) against a run of its key blocks, which go round the 4
// waves; these are joined in LDS.  An item's only slot writes the outputs, several their parts.
// HBM bounds it over long caches (MT = 1: about 1000 vector cycles for a block's 16 KB, at 8 waves on
// a CU several times what HBM delivers), so loads run ahead: each next block's keys are read when the
// scores have used theirs, its values after the outputs.  Eight items of 40000 to 65535 rows (433 MB)
// take 70 us, 6.1 TB/s.  Short shares are bound by latency: sixteen items of 2200 to 4200 rows (54 MB, in
// the memory-side cache) 15 us, 3.6 TB/s, where a wave has three or four blocks and reads one more that
// it does not use; one of 2176 6.5 us, most of it the launch and one pass.  Two tiles (17 to 32 rows)
// take 366 registers at hd 128, one wave on a SIMD: 4 tokens of those sixteen items 30 us with the join.
//
// NT: loads without a place in the memory-side cache, for caches well beyond its 256 MB: 433 MB take
// 75.6 us so and 83.6 otherwise, 337 MB 67.2 and 61.5, 54 MB 25.2 and 20.8 (part of what fits is
// still there from the step before).
template <bool NT>
__device__ __forceinline__ u32x4 load16(const uint8_t *p) {
  const u32x4 *q = reinterpret_cast<const u32x4 *>(p);
  return NT ? __builtin_nontemporal_load(q) : *q;
}

template <int HD, int MT, bool NT>
__global__ __launch_bounds__(256) void k_qattn(QAttnArgs a) {
  constexpr int KC = HD / 64;                   // 16-byte pieces of a key row that a lane holds
  constexpr int DT = HD / 16;                   // output tiles of 16 dims
  constexpr int OS = HD + 4;
  __shared__ float sm_o[4][16][OS];
  __shared__ float2 sm_ml[4][16 * MT];
  __shared__ float sm_l[16], sm_lse[16 * MT];
  __shared__ uint64_t sm_nan[4][HD];
  const Share sh = share_of(a, blockIdx.x);
  if (sh.item < 0) return;
  const int b = sh.item, kv = blockIdx.y, hb = b * a.KV + kv, R = a.n * a.G;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, l16 = lane & 15;
  const int held = sh.held, m = sh.m, rows = m * a.G;   // m > 0
  const int kmax = held + m;                    // keys that any row sees
  const int kall = held + 1;                    // keys that every row sees, but for the mask
  const int blocks = (kmax + kQBlock - 1) / kQBlock, blo = (blockIdx.x - sh.start) * sh.per;
  const int bhi = min(blocks - blo, sh.per) + blo;
  const long slot = (long)kv * a.slots + blockIdx.x;
  if (a.plan && kv == 0 && blo == 0 && tid == 0) a.plan[b] = make_int2(sh.start, sh.used);
  const int nblk = a.cap / kQBlock;
  // S^T row m of tile t is key (m / 4) 16 + 4 t + m % 4
  const uint8_t *kbase = a.k + (long)hb * a.cap * HD + ((l16 >> 2) * 16 + (l16 & 3)) * HD + g * 16;
  const uint8_t *vbase = a.v + (long)hb * a.cap * HD + l16 * kQBlock + g * 16;
  const uniform_floats ksb = as_uniform(a.ks + (long)hb * nblk), vsb = as_uniform(a.vs + (long)hb * nblk);
  u32x4 kw[4][KC], vw[DT];
  auto load_k = [&](int blk) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < KC; ++i)
        kw[t][i] = load16<NT>(kbase + (long)blk * (HD * kQBlock) + 4 * t * HD + 64 * i);
  };
  auto load_v = [&](int blk) {
#pragma unroll
    for (int d = 0; d < DT; ++d) vw[d] = load16<NT>(vbase + (long)blk * (HD * kQBlock) + 16 * d * kQBlock);
  };
  // mask bytes of the lane's 16 keys, a block ahead as well
  const uint8_t *mbase = a.mask ? a.mask + (long)b * a.cap + g * 16 : nullptr;
  u32x4 mw = {~0u, ~0u, ~0u, ~0u};
  const int at0 = min(blo + wave, nblk - 1);
  if (mbase) mw = *reinterpret_cast<const u32x4 *>(mbase + at0 * kQBlock);
  load_k(at0);
  load_v(at0);
  float ks = ksb[at0], vs = value_scale(vsb[at0]);
  bf16x8 q[MT][2 * KC];
  int seen[MT];                                 // keys that the lane's row sees
  f32x4 o[MT][DT];
  float mx[MT], sum[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = 16 * t + l16, tok = a.by_g(min(r, rows - 1));
    seen[t] = r < rows ? held + tok + 1 : 0;
    const uint16_t *src = a.q + (((long)b * a.n + tok) * a.H + kv * a.G + min(r, rows - 1) - tok * a.G) * HD;
#pragma unroll
    for (int i = 0; i < KC; ++i) {
      q[t][2 * i] = load_q(src + 64 * i + g * 16, a.flip);
      q[t][2 * i + 1] = load_q(src + 64 * i + g * 16 + 8, a.flip);
    }
    mx[t] = kNegInf, sum[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0, 0, 0, 0};
  }

  for (int blk = blo + wave; blk < bhi; blk += 4) {
    const int j0 = blk * kQBlock, next = min(blk + 4, nblk - 1);
    const float ks_next = ksb[next], vs_next = value_scale(vsb[next]);
    const bool full = !a.mask && j0 + kQBlock <= kall;
    uint32_t vis[4] = {~0u, ~0u, ~0u, ~0u};      // the lane's 16 keys that some row may see, by bytes
    if (!full) {
      if (mbase) {
#pragma unroll
        for (int i = 0; i < 4; ++i) vis[i] = set_bytes(mw[i]);
        mw = *reinterpret_cast<const u32x4 *>(mbase + next * kQBlock);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int left = kmax - (j0 + g * 16 + 4 * i);   // keys from this word on
        vis[i] &= left >= 4 ? ~0u : (left <= 0 ? 0u : (1u << (8 * left)) - 1u);
      }
    }
    // 0 x NaN is NaN, so where some row may not see the block whole (what none sees may hold anything)
    // a NaN becomes 0, and NaN is what the rows that see it get for it afterwards.
    bool odd = false;
    if (!full) {
      uint32_t any = 0;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) any |= nan_tops(vw[d][i]);
      odd = __any((any & 0x80808080u) != 0);
      if (odd) {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          uint32_t bits = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t n = nan_bytes(vw[d][i]);
            vw[d][i] &= ~(n * 255u);
            bits |= byte_bits(n) << (4 * i);
          }
          reinterpret_cast<part16 *>(&sm_nan[wave][16 * d + l16])[g] = (uint16_t)bits;
        }
        wave_lds_order();
      }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      f32x4 s[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[x] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KC; ++i) {
          s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequant8(kw[x][i][0], kw[x][i][1], ks), q[t][2 * i], s[x], 0, 0, 0);
          s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequant8(kw[x][i][2], kw[x][i][3], ks), q[t][2 * i + 1], s[x], 0, 0, 0);
        }
      }
      if (t == MT - 1) load_k(next);
      float top = kNegInf;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y = s[x][e] * a.c;
          if (!full) {
            const int j = j0 + g * 16 + 4 * x + e;
            y = (j < seen[t] && (vis[x] >> (8 * e) & 1u)) ? y : kNegInf;
          }
          s[x][e] = y;
          top = fmaxf(top, y);
        }
      if (a.logit && seen[t]) {
        float *to = a.logit + ((long)hb * R + 16 * t + l16) * a.cap + j0 + g * 16;
#pragma unroll
        for (int x = 0; x < 4; ++x) *reinterpret_cast<f32x4 *>(to + 4 * x) = s[x];
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float mn = fmaxf(mx[t], top);
      const float ref = mn == kNegInf ? 0.f : mn;
      const float corr = exp2_fast(mx[t] - ref);
      mx[t] = mn;
      float add = 0.f;
      bf16x8 p[2];
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = exp2_fast(s[x][e] - ref);
          add += y;
          p[x >> 1][(x & 1) * 4 + e] = (__bf16)y;
        }
      sum[t] = sum[t] * corr + add;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        o[t][d] *= corr;
        o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequant8(vw[d][0], vw[d][1], vs), p[0], o[t][d], 0, 0, 0);
        o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequant8(vw[d][2], vw[d][3], vs), p[1], o[t][d], 0, 0, 0);
      }
      if (odd) {
        uint64_t keys = 0;               // that the lane's row sees
#pragma unroll
        for (int i = 0; i < 4; ++i) keys |= (uint64_t)byte_bits(vis[i] & 0x01010101u) << (16 * g + 4 * i);
        keys |= __shfl_xor(keys, 16);
        keys |= __shfl_xor(keys, 32);
        keys &= seen_bits(seen[t] - j0);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (sm_nan[wave][16 * d + 4 * g + e] & keys) o[t][d][e] = __builtin_nanf("");
      }
    }
    load_v(next);
    ks = ks_next, vs = vs_next;
  }

  // the four waves' parts of each row, joined; a lane's group g holds the sum over its own keys
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    float s = sum[t];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (g == 0) sm_ml[wave][16 * t + l16] = make_float2(mx[t], s);
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    __syncthreads();
    const float2 w0 = sm_ml[0][16 * t + l16], w1 = sm_ml[1][16 * t + l16], w2 = sm_ml[2][16 * t + l16],
                 w3 = sm_ml[3][16 * t + l16];
    const float mt = fmaxf(fmaxf(w0.x, w1.x), fmaxf(w2.x, w3.x)), ref = mt == kNegInf ? 0.f : mt;
    const float f = exp2_fast(mx[t] - ref);
    const float l = w0.y * exp2_fast(w0.x - ref) + w1.y * exp2_fast(w1.x - ref) +
                    w2.y * exp2_fast(w2.x - ref) + w3.y * exp2_fast(w3.x - ref);
    // O^T: lane (g, l16) holds dims 16 d + 4 g + e of row l16
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) sm_o[wave][l16][16 * d + 4 * g + e] = o[t][d][e] * f;
    const int rt = 16 * t;
    if (wave == 0 && g == 0) {
      if (a.ml && rt + l16 < rows) a.ml[slot * R + rt + l16] = make_float2(mt, l);
      if (a.lse && rt + l16 < rows) a.lse[(long)hb * R + rt + l16] = log_sum(mt, l);
      sm_l[l16] = l;
      sm_lse[rt + l16] = log_sum(mt, l);
    }
    __syncthreads();
    for (int x = tid; x < 16 * HD / 4; x += 256) {
      const int row = x / (HD / 4), d = x % (HD / 4) * 4, r = rt + row;
      if (r >= rows) continue;
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[e] = sm_o[0][row][d + e] + sm_o[1][row][d + e] + sm_o[2][row][d + e] + sm_o[3][row][d + e];
      if (a.part) {
        *reinterpret_cast<float4 *>(a.part + (slot * R + r) * HD + d) =
            make_float4(y[0], y[1], y[2], y[3]);
      } else {
        const float inv = output_factor(sm_l[row]);
        const bf16x4 w = {(__bf16)(y[0] * inv), (__bf16)(y[1] * inv), (__bf16)(y[2] * inv), (__bf16)(y[3] * inv)};
        *reinterpret_cast<bf16x4 *>(a.out + (((long)b * a.n + a.by_g(r)) * a.H + kv * a.G + r - a.by_g(r) * a.G) * HD + d) = w;
      }
    }
  }
  // one workgroup saw every key of these rows: their weights too (the scores it wrote above)
  if (a.logit && !a.part) {
    __syncthreads();
    for (int j = tid; j < kmax; j += 256) {
      float w = 0.f;
      for (int r = 0; r < rows; ++r) w += prob(a.logit[((long)hb * R + r) * a.cap + j], sm_lse[r]);
      a.weight[(long)hb * a.cap + j] += w;
    }
  }
}

// More than 32 rows: 4 waves of 32 each (2 up to 64 rows, where the others would hold places and idle:
// 46 us against 32 for sixteen items of 52 rows of 8 heads over 5000 keys) share the key blocks,
// which the DMA brings into LDS a block ahead (16 KB each at hd 128), in e4m3: half of the bytes that
// bfloat16 tiles would be read back as, at the price that every wave converts them for itself.  32 x
// 32 matrix instructions; a lane holds one row and, of a block's keys, the 32 of its half wave.
// Sixteen frames of up to 1024 tokens, 28 heads, over 2200 to 4200 rows (0.51 TFLOP) take 542 us, 0.95
// PFLOP/s (564 on another box), a prompt of 8192 (0.48 TFLOP) 472.  Matrix instructions take 41 and 45 %
// of a SIMD's cycles and vector ones (softmax, conversions) 60 and 64: together the whole, so at two waves
// on a SIMD little of the one runs under the other.  The clock is 2.2 GHz of 2.4, in the first launches
// after a pause 2.0 (595 us).  Scores a block ahead of the softmax (two ways), three waves on a SIMD or
// prefetched operands come out the same; 64 rows in a wave, or blocks converted once per workgroup, slower
// (by half, by a tenth); without the exponentials it is 8 % faster, without the keys' conversion 5.  256
// tokens over 2176 rows: 22 us, eight or nine blocks one after the other on 224 workgroups, and their
// start and end.
//
// LDS rows are 16-byte pieces, stored at piece ^ f(row) so that the 16 lanes that a read serves
// together (0-3, 12-15, 20-23, 24-27 and the other 16 of each half) fall on different banks.
template <int HD>
__device__ __forceinline__ int key_swz(int row) {
  return HD == 128 ? ((row >> 1) & 3) | ((row >> 5) << 2) : (row >> 2) & 3;
}
__device__ __forceinline__ int val_swz(int dim) { return (dim >> 2) & 3; }

// Pieces of work are numbered by pairs (item and key-value head), then splits, then tiles of rows, the
// last rows, which see most keys, first.  Workgroups go round the 8 XCDs in turn and start in order:
// an XCD that kept to its pairs, as P is often a multiple of 8, would make the others wait whenever its
// items are the longer ones, so the pairs move on by one with each round of them (8 items of 10 to
// 4000 rows: 244 to 135 us; all of one length: up to 1 % slower).
// QUEUE: as many workgroups as run at once, each going on with the next piece of its XCD's pairs, whose
// keys are in its L2, then with the others' (queue: pieces taken of each).  Batches whose items bring
// different numbers of tokens (n_new is given; what it holds the host does not know) go this way from
// four rounds of workgroups on, counted as if every token were there; in fewer a last round that is not
// full falls to few CUs (3.5 rounds of equal items: 392 us so, 357 without).  With the queue and without:
// sixteen frames of 704 to 1024 tokens, seven rounds, 522 and 541 us, with a key mask 608 and 665; of
// 1024 each 624 and 660; 48 items of 171 to 256 tokens 345 and 348; 300 of 64 over 1000 keys 406 and 403;
// where most tokens are missing the pieces without rows cost more so: 200 of 1024 tokens 127 and 129, 60
// of them 89 and 55.
template <int HD, int NW, bool QUEUE>
__global__ __launch_bounds__(64 * NW, 2) void k_qattn_rows(QAttnArgs args) {
  constexpr int PC = HD / 16;                   // 16-byte pieces of a key row
  constexpr int DT = HD / 32;                   // output tiles of 32 dims
  constexpr int TILE = kQBlock * HD;            // bytes of a block's keys, and of its values
  constexpr int DMAS = TILE / 1024 / NW;        // DMA instructions of a wave for either
  constexpr int ROWS = 32 * NW;
  constexpr int STAGES = 2;
  __shared__ __align__(1024) uint8_t sm[STAGES][2][TILE];
  __shared__ uint64_t sm_nan[NW][HD];
  __shared__ __align__(16) uint8_t sm_mask[STAGES][NW][256];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  auto work = [&](const QAttnArgs &a, int id) {
    const int P = a.B * a.KV, R = a.n * a.G;
    const int rest = id / P, hb = QUEUE ? id % P : (id % P + rest) % P, split = rest % a.splits;
    const int r0 = ((R + ROWS - 1) / ROWS - 1 - rest / a.splits) * ROWS;
    const int b = hb / a.KV, kv = hb % a.KV;
    const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
    const int rows = m * a.G;
    if (r0 >= rows) return;
    const int kmax = held + a.by_g(min(r0 + ROWS, rows) - 1) + 1;
    const int blocks = (kmax + kQBlock - 1) / kQBlock, used = splits_used(kmax, a);
    if (split >= used) return;
    const int blo = (int)((long)blocks * split / used), bhi = (int)((long)blocks * (split + 1) / used);

    const long nblk = a.cap / kQBlock;
    const uint8_t *kbase = a.k + (long)hb * a.cap * HD, *vbase = a.v + (long)hb * a.cap * HD;
    const uniform_floats ksb = as_uniform(a.ks + hb * nblk), vsb = as_uniform(a.vs + hb * nblk);
    int ksrc[DMAS], vsrc[DMAS];
#pragma unroll
    for (int i = 0; i < DMAS; ++i) {
      const int p = (wave * DMAS + i) * 64 + lane, kr = p / PC, vr = p / 4;
      ksrc[i] = kr * HD + ((p % PC) ^ key_swz<HD>(kr)) * 16;
      vsrc[i] = vr * kQBlock + ((p & 3) ^ val_swz(vr)) * 16;
    }
    auto fetch = [&](int blk, int stage) {
      const long at = (long)blk * TILE;
#pragma unroll
      for (int i = 0; i < DMAS; ++i) dma16(kbase + at + ksrc[i], lds_addr(&sm[stage][0][(wave * DMAS + i) * 1024]));
#pragma unroll
      for (int i = 0; i < DMAS; ++i) dma16(vbase + at + vsrc[i], lds_addr(&sm[stage][1][(wave * DMAS + i) * 1024]));
      // a block's 64 mask bytes for each wave (four times over: a DMA writes 4 bytes for every lane)
      if (a.mask) dma4(a.mask + (long)b * a.cap + blk * kQBlock + (lane & 15) * 4, lds_addr(&sm_mask[stage][wave][0]));
    };

    const int w0 = r0 + 32 * wave, r = w0 + l32, tok = a.by_g(min(r, rows - 1)), head = kv * a.G + min(r, rows - 1) - tok * a.G;
    const int seen = r < rows ? held + tok + 1 : 0;                              // keys that the lane's row sees
    const int wmax = w0 < rows ? held + a.by_g(min(w0 + 32, rows) - 1) + 1 : 0;  // that any row of the wave sees
    const int wall = held + a.by_g(w0) + 1;                                      // that every one does
    const long at_q = (((long)b * a.n + tok) * a.H + head) * HD;
    bf16x8 q[HD / 16];
    {
      const uint16_t *src = a.q + at_q;
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        q[2 * i] = load_q(src + (2 * i + h) * 16, a.flip);
        q[2 * i + 1] = load_q(src + (2 * i + h) * 16 + 8, a.flip);
      }
    }
    loads_done();
    fetch(blo, 0);

    // S^T row x of tile t is key ((x / 4) % 2) 32 + 16 t + x / 8 4 + x % 4
    const int kr = ((l32 >> 2) & 1) * 32 + (l32 >> 3) * 4 + (l32 & 3);
    const int koff = kr * HD, kx = key_swz<HD>(kr), voff = l32 * kQBlock, vx = val_swz(l32);
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float ref = kNegInf, sum = 0.f;   // exponents are taken relative to ref

    int stage = 0;
    float ks = ksb[blo], vs = value_scale(vsb[blo]);
    for (int blk = blo; blk < bhi; ++blk, stage ^= 1) {
      wait_vm<0>();                    // this wave's part of the block; the barrier adds the others', and
      lds_barrier();                   // every wave has left the other stage
      if (blk + 1 < bhi) fetch(blk + 1, stage ^ 1);
      if (w0 >= rows) continue;        // it only brings its part of the blocks
      const int j0 = blk * kQBlock, ahead = min(blk + 1, bhi - 1);
      const float ks_next = ksb[ahead], vs_next = value_scale(vsb[ahead]);
      f32x16 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
      for (int i = 0; i < HD / 32; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x4 w = *reinterpret_cast<const u32x4 *>(&sm[stage][0][koff + t * 16 * HD + (((2 * i + h) ^ kx) * 16)]);
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dequant8(w[0], w[1], ks), q[2 * i], s[t], 0, 0, 0);
          s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dequant8(w[2], w[3], ks), q[2 * i + 1], s[t], 0, 0, 0);
        }
      // the keys that the mask shows, and whether some row of the wave may not see the block whole
      uint64_t shown = ~0ull;
      if (a.mask) shown = __ballot(sm_mask[stage][wave][lane] != 0);
      const bool later = j0 + kQBlock > wall, part = later || shown != ~0ull;
      uint32_t mine = ~0u;             // the lane's 32 keys that some row may see
      uint32_t odd = 0;                // those of its halves where some value is NaN
      if (part) {
        const uint64_t some = shown & seen_bits(wmax - j0);
        mine = (uint32_t)(some >> (32 * h));
        if (later) {
          const uint32_t sees = mine & (uint32_t)(seen_bits(seen - j0) >> (32 * h));
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (!(sees >> (16 * t + e) & 1u)) s[t][e] = kNegInf;
        } else {                       // the same keys for every row: the scalar unit spreads them over the halves
          const uint32_t lo = (uint32_t)some, hi = (uint32_t)(some >> 32);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint64_t lanes = (uint64_t)(uint32_t)((int)(hi << (31 - 16 * t - e)) >> 31) << 32 |
                                     (uint32_t)((int)(lo << (31 - 16 * t - e)) >> 31);
              s[t][e] = __builtin_amdgcn_inverse_ballot_w64(lanes) ? s[t][e] : kNegInf;
            }
        }
      }
      float top = kNegInf;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; e += 2) top = fmaxf(fmaxf(top, s[t][e]), s[t][e + 1]);
      top = fmaxf(top, __shfl_xor(top, 32)) * a.c;
      // the reference follows the maximum only where it is 2^8 behind: most blocks need not touch O,
      // and its sums stay within float32 while rows times their largest value are below 2^137
      // (each row's by its own scores alone: another row's may come from keys that are hidden from it)
      if (__any(top > ref + 8.f)) {
        const bool up = top > ref + 8.f;
        const float corr = up ? exp2_fast(ref - top) : 1.f;
        ref = up ? top : ref;
        sum *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= corr;
      }
      const float sub = ref == kNegInf ? 0.f : ref;
      // 16 keys of the lane at a time: their values, their exponentials, their products
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 vw[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d)
          vw[d] = *reinterpret_cast<const u32x4 *>(&sm[stage][1][voff + d * 32 * kQBlock + (((2 * h + t) ^ vx) * 16)]);
        if (part) {                    // as in k_qattn
          uint32_t any = 0;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int x = 0; x < 4; ++x) any |= nan_tops(vw[d][x]);
          if (__any((any & 0x80808080u) != 0)) {
            odd |= 0xFFFFu << (16 * t);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
              uint32_t bits = 0;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const uint32_t n = nan_bytes(vw[d][x]);
                vw[d][x] &= ~(n * 255u);
                bits |= byte_bits(n) << (4 * x);
              }
              reinterpret_cast<part16 *>(&sm_nan[wave][32 * d + l32])[2 * h + t] = (uint16_t)bits;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          bf16x8 p;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float y = exp2_fast(fmaf(s[t][8 * i + e], a.c, -sub));
            sum += y;
            p[e] = (__bf16)y;
          }
#pragma unroll
          for (int d = 0; d < DT; ++d)
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(dequant8(vw[d][2 * i], vw[d][2 * i + 1], vs), p, o[d], 0, 0, 0);
        }
      }
      if (odd) {
        const uint32_t keep = mine & odd, other = __shfl_xor(keep, 32);
        const uint64_t keys = ((uint64_t)(h ? keep : other) << 32 | (h ? other : keep)) & seen_bits(seen - j0);
        wave_lds_order();
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (sm_nan[wave][32 * d + 8 * (e / 4) + 4 * h + e % 4] & keys) o[d][e] = __builtin_nanf("");
      }
      ks = ks_next, vs = vs_next;
    }

    sum += __shfl_xor(sum, 32);
    if (r >= rows) return;
    const long at = (long)hb * R + r;
    if (a.splits > 1) {
      const long to = (long)split * P * R + at;
      if (h == 0) a.ml[to] = make_float2(ref, sum);
      f32x4 *dst = reinterpret_cast<f32x4 *>(a.part) + (((long)split * P + hb) * ((R + 31) / 32) + w0 / 32) * (HD / 8) * 64 + lane;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) dst[(4 * d + j) * 64] = f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
    } else {
      if (a.lse && h == 0) a.lse[at] = log_sum(ref, sum);
      const float inv = output_factor(sum);
      uint16_t *dst = a.out + at_q;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x4 w = {(__bf16)(o[d][4 * j] * inv), (__bf16)(o[d][4 * j + 1] * inv), (__bf16)(o[d][4 * j + 2] * inv), (__bf16)(o[d][4 * j + 3] * inv)};
          *reinterpret_cast<bf16x4 *>(dst + 32 * d + 8 * j + 4 * h) = w;
        }
    }
  };
  if constexpr (!QUEUE) {
    work(args, blockIdx.x);
  } else {
    __shared__ int sm_next;
    int id = blockIdx.x, from = blockIdx.x % 8;
    for (int done = 0;;) {             // queues found empty
      const QAttnArgs a = args_again<QAttnArgs>();
      work(a, id);
      for (;;) {
        __syncthreads();
        if (tid == 0) sm_next = (int)gridDim.x + 8 * atomicAdd(&a.queue[kQueueStep * from], 1) + from;
        __syncthreads();
        id = __builtin_amdgcn_readfirstlane(sm_next);
        if (id < a.pieces) break;
        if (++done == 8) return;
        from = (from + 1) % 8;
      }
    }
  }
}

__global__ void k_qattn_queue(int *queue) { queue[kQueueStep * threadIdx.x] = 0; }

// The parts of one row joined by one workgroup: their outputs weighted by 2^(m_s - m) and divided
// by the sum; 4 to 5 us beside a launch's 3.6.  With scores written down (R <= 32 rows), further workgroups turn them into the
// weight that each key receives: 4 R bytes a key written and read, against the 2 R hd multiplications
// and the hd bytes of the keys that computing them again costs.
constexpr int kWeightKeys = 256;

template <int HD>
__global__ __launch_bounds__(256) void k_qattn_join(QAttnArgs a, int join_rows) {
  constexpr int TPR = HD / 4, SG = 256 / TPR;
  __shared__ float sm_y[SG][HD];
  __shared__ float2 sm_ml[SG];
  __shared__ float sm_lse[32];
  __shared__ f32x4 sm_w[4][kWeightKeys / 4];
  const int hb = blockIdx.y, b = hb / a.KV, kv = hb % a.KV, tid = threadIdx.x;
  const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
  const int R = a.n * a.G, rows = m * a.G, r = blockIdx.x;
  // part s of row r: at + s step
  const int2 sh = a.plan[b];          // not written for an item without rows, which returns below
  const long step = R, at0 = ((long)kv * a.slots + sh.x) * R;
  const int used = sh.y;
  if (r < join_rows) {
    if (r >= rows) return;
    const int sg = tid / TPR, d = tid % TPR * 4;
    const long at = at0 + r;
    float mt = kNegInf, l = 0.f;
    f32x4 y = {0, 0, 0, 0};
    for (int s = sg; s < used; s += SG) {
      const float2 z = a.ml[s * step + at];
      const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part + (s * step + at) * HD + d);
      const float mn = fmaxf(mt, z.x), ref = mn == kNegInf ? 0.f : mn;
      const float f = exp2_fast(mt - ref), h = exp2_fast(z.x - ref);
      mt = mn;
      l = l * f + z.y * h;
      y = y * f + x * h;
    }
    if (tid % TPR == 0) sm_ml[sg] = make_float2(mt, l);
    __syncthreads();
    float top = kNegInf;
#pragma unroll
    for (int i = 0; i < SG; ++i) top = fmaxf(top, sm_ml[i].x);
    const float ref = top == kNegInf ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < SG; ++i) sum += sm_ml[i].y * exp2_fast(sm_ml[i].x - ref);
    *reinterpret_cast<f32x4 *>(&sm_y[sg][d]) = y * exp2_fast(mt - ref);
    __syncthreads();
    if (tid < TPR) {
      f32x4 t = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < SG; ++i) t += *reinterpret_cast<const f32x4 *>(&sm_y[i][d]);
      t *= output_factor(sum);
      const bf16x4 w = {(__bf16)t[0], (__bf16)t[1], (__bf16)t[2], (__bf16)t[3]};
      *reinterpret_cast<bf16x4 *>(a.out + (((long)b * a.n + a.by_g(r)) * a.H + kv * a.G + r - a.by_g(r) * a.G) * HD + d) = w;
      if (a.lse && tid == 0) a.lse[(long)hb * R + r] = log_sum(top, sum);
    }
    return;
  }
  const int j0 = (r - join_rows) * kWeightKeys, seen = held + m;
  if (m == 0 || j0 >= seen) return;
  {
    // 8 threads to a row
    const int row = tid / 8;
    float mt = kNegInf, l = 0.f;
    if (row < rows)
      for (int s = tid % 8; s < used; s += 8) {
        const float2 z = a.ml[s * step + at0 + row];
        const float mn = fmaxf(mt, z.x), ref = mn == kNegInf ? 0.f : mn;
        l = l * exp2_fast(mt - ref) + z.y * exp2_fast(z.x - ref);
        mt = mn;
      }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      const float m2 = __shfl_xor(mt, o), l2 = __shfl_xor(l, o);
      const float mn = fmaxf(mt, m2), ref = mn == kNegInf ? 0.f : mn;
      l = l * exp2_fast(mt - ref) + l2 * exp2_fast(m2 - ref);
      mt = mn;
    }
    if (tid % 8 == 0) sm_lse[row] = log_sum(mt, l);
  }
  __syncthreads();
  // 64 threads of four keys each for every fourth row
  const int lane = tid & 63, part = tid >> 6, j = j0 + 4 * lane;
  f32x4 w = {0, 0, 0, 0};
  if (j < seen)
    for (int i = part; i < rows; i += 4) {
      const f32x4 y = *reinterpret_cast<const f32x4 *>(a.logit + ((long)hb * R + i) * a.cap + j);
      const float L = sm_lse[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] += prob(y[e], L);
    }
  sm_w[part][lane] = w;
  __syncthreads();
  if (part || j >= seen) return;
  w = (w + sm_w[1][lane]) + (sm_w[2][lane] + sm_w[3][lane]);
  float *to = a.weight + (long)hb * a.cap + j;
  if (j + 4 <= seen) {
    *reinterpret_cast<f32x4 *>(to) += w;
  } else {
    for (int e = 0; e < seen - j; ++e) to[e] += w[e];
  }
}

// The same for k_qattn_rows, whose rows are many and splits few: a workgroup joins 32 dims of 32 rows,
// eight splits' parts in flight at a time.  Parts lie as that kernel's lanes hold them, [split][pair]
// [32 rows][HD / 8][half wave][row] by four dims, so that both kernels move runs of 1 KB (7168 rows of
// four parts, 15 MB: 5.8 us; that kernel writes rows of 512 bytes 3 us slower).
template <int HD>
__global__ __launch_bounds__(256) void k_qattn_join_rows(QAttnArgs a) {
  constexpr int DT = HD / 32;
  const int hb = blockIdx.y, b = hb / a.KV, kv = hb % a.KV, tile = blockIdx.x / DT, dt = blockIdx.x % DT;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = 32 * dt + 8 * wave + lane / 32 * 4;
  const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
  const int R = a.n * a.G, rows = m * a.G, r = tile * 32 + lane % 32;
  if (r >= rows) return;
  const int last = min(r / a.tile_rows * a.tile_rows + a.tile_rows, rows) - 1;
  const int used = splits_used(held + a.by_g(last) + 1, a);
  const long step = (long)a.B * a.KV * R, at = (long)hb * R + r, R32 = (R + 31) / 32;
  const long pstep = (long)a.B * a.KV * R32 * (HD / 8) * 64;
  const f32x4 *part = reinterpret_cast<const f32x4 *>(a.part) + ((hb * R32 + tile) * (HD / 8) + 4 * dt + wave) * 64 + lane;
  float mt = kNegInf, l = 0.f;
  f32x4 y = {0, 0, 0, 0};
  for (int s0 = 0; s0 < used; s0 += 8) {
    float2 z[8];
    f32x4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = min(s0 + i, used - 1);
      z[i] = a.ml[p * step + at];
      x[i] = part[p * pstep];
    }
    float mn = mt;
#pragma unroll
    for (int i = 0; i < 8; ++i) mn = fmaxf(mn, z[i].x);
    const float ref = mn == kNegInf ? 0.f : mn, f = exp2_fast(mt - ref);
    mt = mn;
    l *= f;
    y *= f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float h = exp2_fast(z[i].x - ref);
      if (s0 + i >= used) break;
      l += z[i].y * h;
      y += x[i] * h;
    }
  }
  y *= output_factor(l);
  const int tok = a.by_g(r);
  const bf16x4 w = {(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
  *reinterpret_cast<bf16x4 *>(a.out + (((long)b * a.n + tok) * a.H + kv * a.G + r - tok * a.G) * HD + d) = w;
  if (a.lse && d == 0) a.lse[at] = log_sum(mt, l);
}

// The weight that each key receives, from scores computed again: 4 waves hold 64 keys each in
// registers, as bfloat16, and the rows' queries pass by through LDS, 64 between barriers (32: 10 %
// slower).  S^T puts the keys in a lane's registers, so its sums over rows stay there until the end.
// Row ranges are dealt over `row_splits` workgroups, whose sums the next kernel adds up in order.
// A prompt of 8192 rows (0.24 TFLOP) takes 278 us (306 in the first launches after a pause), 38 % of the
// matrix unit's cycles: the other terms, an exponential and two more vector instructions for 32 matrix
// cycles, and one barrier for 64 rows, add to the products (53 % of cycles) rather than hide behind them
// at two waves on a SIMD (252 registers: the keys are 64, scores and sums 64); without the exponentials
// it is a tenth faster.
constexpr int kWaveKeys = 64, kGroupKeys = 4 * kWaveKeys;

template <int HD>
__global__ __launch_bounds__(256, 2) void k_qattn_weight(QAttnArgs a, float *wpart, int row_splits) {
  constexpr int PC = HD / 8;                    // 16-byte pieces of a query row
  constexpr int ROWS = 64;                      // of a stage: two products' worth between barriers
  constexpr int TILE = ROWS * HD * 2, DMAS = TILE / 16 / 256;
  __shared__ __align__(1024) uint8_t sm[3][TILE];
  __shared__ float sm_l[3][4][ROWS];            // a wave's copy of the stage's row sums
  const int P = a.B * a.KV, R = a.n * a.G;
  const int rest = blockIdx.x / P, hb = (blockIdx.x % P + rest) % P, rs = rest % row_splits, j0 = rest / row_splits * kGroupKeys;
  const int b = hb / a.KV, kv = hb % a.KV;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
  const int rows = m * a.G, seen = held + m;
  if (m == 0 || j0 >= seen) return;
  // stages of rows that see a key of the group, and this workgroup's part of them
  const int t0 = (int)((long)max(0, j0 - held) * a.G / ROWS), t1 = (rows + ROWS - 1) / ROWS;
  const int lo = t0 + (int)((long)(t1 - t0) * rs / row_splits), hi = t0 + (int)((long)(t1 - t0) * (rs + 1) / row_splits);

  const int w0 = j0 + kWaveKeys * wave, blk = min(w0, a.cap - kQBlock) / kQBlock;
  const float ks = a.ks[hb * (long)(a.cap / kQBlock) + blk];
  bf16x8 k[2][HD / 16];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) {
      // S^T row x of tile t is key 32 t + x
      const u32x4 w = *reinterpret_cast<const u32x4 *>(
          a.k + ((long)hb * a.cap + (long)blk * kQBlock + 32 * t + l32) * HD + (2 * i + h) * 16);
      k[t][2 * i] = dequant8(w[0], w[1], ks);
      k[t][2 * i + 1] = dequant8(w[2], w[3], ks);
    }
  // a stage's rows lie over the tokens from that of its first row on; rows behind the last one are
  // read as the last one
  const float *lse = a.lse + (long)hb * R;
  const int skip = (a.H - a.G) * HD;  // from a token's last head of the group to the next one's first
  auto fetch = [&](int tile, int stage) {
    const int t = __builtin_amdgcn_readfirstlane(a.by_g(tile * ROWS)), g = tile * ROWS - t * a.G, last = rows - 1 - tile * ROWS;
    const uint16_t *qb = a.q + (((long)b * a.n + t) * a.H + kv * a.G) * HD;
#pragma unroll
    for (int i = 0; i < DMAS; ++i) {
      const int p = (wave * DMAS + i) * 64 + lane, row = p / PC, r = min(row, last) + g;
      const int piece = (p % PC) ^ (HD == 128 ? row & 15 : (row >> 1) & 7);
      dma16(qb + (unsigned)(a.by_g(r) * skip + r * HD + piece * 8), lds_addr(&sm[stage][(wave * DMAS + i) * 1024]));
    }
    dma4(lse + min(tile * ROWS + lane, rows - 1), lds_addr(&sm_l[stage][wave][0]));
  };
  f32x16 acc[2];
  const float c = a.flip ? -a.c : a.c;   // the queries' signs are as they came
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  loads_done();
  if (lo < hi) fetch(lo, 0);
  if (lo + 1 < hi) fetch(lo + 1, 1);
  const int qx = HD == 128 ? l32 & 15 : (l32 >> 1) & 7;
  bf16x8 q[HD / 16];                  // the coming 32 rows, and their sums
  float L = 0.f;
  auto queries = [&](int st, int half) {
    const uint8_t *qt = sm[st] + (32 * half + l32) * HD * 2;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x)     // piece of 8 elements: dims (2 i + h) 16 + 8 x
        q[2 * i + x] = *reinterpret_cast<const bf16x8 *>(qt + ((2 * (2 * i + h) + x) ^ qx) * 16);
    L = sm_l[st][wave][32 * half + l32];
  };
  auto arrived = [&](bool ahead) {
    if (ahead) wait_vm<DMAS + 1>();
    else wait_vm<0>();
    lds_barrier();
  };
  if (lo < hi) {
    arrived(lo + 1 < hi);
    queries(0, 0);
  }
  int stage = 0;
  for (int tile = lo; tile < hi; ++tile) {
    const int next = stage == 2 ? 0 : stage + 1;
    if (tile + 2 < hi) fetch(tile + 2, next == 2 ? 0 : next + 1);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int r0 = tile * ROWS + 32 * half;
      f32x16 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[0][i], q[i], s[0], 0, 0, 0);
        s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[1][i], q[i], s[1], 0, 0, 0);
      }
      const float sub = L;
      if (half == 0) {
        queries(stage, 1);
      } else if (tile + 1 < hi) {
        arrived(tile + 2 < hi);
        queries(next, 0);
      }
      const int r = r0 + l32;
      if (r0 + 32 <= rows && w0 + kWaveKeys <= held + a.by_g(r0) + 1) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[t][e] += exp2_fast(fmaf(s[t][e], c, -sub));
      } else {
        const int see = r < rows ? held + a.by_g(r) + 1 : 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p = exp2_fast(fmaf(s[t][e], c, -sub));
            acc[t][e] += w0 + 32 * t + 8 * (e / 4) + 4 * h + e % 4 < see ? p : 0.f;
          }
      }
    }
    stage = next;
  }
  // Summed over the 32 rows of a half wave: at each step a lane hands half of its keys' sums to the
  // lane across and adds that one's other half, until it holds one key's.
  float w[32];
#pragma unroll
  for (int e = 0; e < 32; ++e) w[e] = acc[e / 16][e % 16];
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int e = 0; e < o; ++e) {
      const bool up = l32 & o;
      w[e] = (up ? w[e + o] : w[e]) + __shfl_xor(up ? w[e] : w[e + o], o);
    }
  const int j = w0 + 32 * (l32 / 16) + 8 * (l32 % 16 / 4) + 4 * h + l32 % 4;
  if (j >= seen) return;
  const float x = a.mask && !a.mask[(long)b * a.cap + j] ? 0.f : w[0];
  const long out = (long)hb * a.cap + j;
  if (wpart) wpart[(long)rs * P * a.cap + out] = x;
  else a.weight[out] += x;
}

__global__ __launch_bounds__(256) void k_qattn_weight_add(QAttnArgs a, const float *wpart, int row_splits) {
  const int hb = blockIdx.y, b = hb / a.KV, j = blockIdx.x * 256 + threadIdx.x;
  const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
  if (m == 0 || j >= held + m) return;
  const long P = (long)a.B * a.KV;
  float w = 0.f;
  for (int i = 0; i < row_splits; ++i) w += wpart[(i * P + hb) * a.cap + j];
  a.weight[(long)hb * a.cap + j] += w;
}

template <int HD>
fc_status run_qattn(fc_ctx *ctx, QAttnArgs &a, bool weigh, hipStream_t st) {
  const long R = (long)a.n * a.G, pairs = (long)a.B * a.KV;
  const bool many = R > 32;
  const int MT = R <= 16 ? 1 : 2, NW = R <= 64 ? 2 : 4, tile = many ? 32 * NW : 16 * MT;
  const long tiles = (R + tile - 1) / tile;
  const long per = pairs * R, padded = many ? pairs * ((R + 31) / 32 * 32) : per, ws = (long)ctx->part_elems;
  auto up4 = [](long x) { return (x + 3) / 4 * 4; };
  // scores of 32 rows or fewer are written down for the weights, where they fit beside the parts
  // of two slots an item; else the weights compute them again from each row's sum
  const bool logit = weigh && !many && per * a.cap + 2 * up4(2 * per) + 2 * per * HD + up4(2L * a.B) <= ws;
  const long side = !weigh ? 0 : logit ? per * a.cap : up4(per), plan = up4(2L * a.B);
  if (side > ws)
    return fail(FC_ERR_CAPACITY, "fc_qcache_attention: the sums of %ld rows exceed the context's workspace", per);
  if (weigh && !logit && (a.cap + kGroupKeys - 1L) / kGroupKeys * pairs > (1L << 24) - 1)
    return fail(FC_ERR_UNSUPPORTED, "fc_qcache_attention: weights of %ld heads of %d rows in one call", pairs, a.cap);
  long splits = 1, slots = a.B;
  if (many) {
    // Workgroups for every CU, as long as each has four blocks; as many as run at once (eight waves on a
    // CU), as long as each has eight, for what its part of the outputs costs (63 rows of 4 heads over
    // 4000 keys 15.0 us so, with two 16.5, with eight 17.8; 1792 rows over 2176 42.5, with four to fill
    // all places 44.3, with twelve 47.9).
    const long units = pairs * tiles, blocks = a.cap / kQBlock, spread = std::min<long>(ctx->num_cus / units, blocks / 4);
    const long places = 8L / NW * ctx->num_cus;
    splits = std::min<long>(places / units, blocks / 8);
    a.least = spread >= splits ? 4 : 8;
    splits = std::max<long>(1, std::max(spread, splits));
    // Where they do not fill the places once, more, of 16 blocks at least, if these fill their last round
    // better by a tenth (360 tiles over 4600 keys in four splits 122 us, 142 in one; 200 over 7400 in
    // five 116, in two 124; 336 over 3200 in three 105, 103 in one).
    auto filled = [&](long s) { return (double)(units * s) / ((units * s + places - 1) / places * places); };
    if (units < places)
      for (long s = splits + 1; s <= 8 && blocks / s >= 16; ++s)
        if (filled(s) > filled(splits) + 0.1) splits = s;
    splits = std::max<long>(1, std::min<long>(splits, (ws - side - plan) / (up4(2 * per) + padded * HD)));
  } else {
    // One workgroup's loads keep a CU's path to memory busy; two, where a mask adds vector work to
    // each block, where head_dim 64 halves the loads in flight, or where an item would have fewer
    // than four slots and their lengths come out uneven (long caches: 8 items of 4 heads 72.7 us
    // with one, 75.6 with two; 19 of 8 heads 51.0 and 46.1, masked 69 and 50; 37 of 4 heads of 64
    // dims 39.7 and 36.9).  Four blocks at least to a slot, one per wave.
    slots = ctx->num_cus / a.KV;
    if (a.mask || HD == 64 || slots < 4L * a.B) slots = 2L * ctx->num_cus / a.KV;
    slots = std::min<long>(slots, a.cap / kQBlock / 4 * a.B);
    slots = std::max<long>(a.B, std::min<long>(slots, (ws - side - plan - 4) / (a.KV * R * (HD + 2))));
  }
  const bool parts = many ? splits > 1 : slots > a.B;
  a.splits = (int)splits;
  a.tile_rows = tile;
  a.slots = many ? 0 : (int)slots;
  float *at = ctx->part;
  if (logit) a.logit = at;
  else if (weigh) a.lse = at;
  at += side;
  if (parts) {
    a.plan = reinterpret_cast<int2 *>(at);
    at += plan;
    a.part = at;
    a.ml = reinterpret_cast<float2 *>(at + (many ? splits * padded : slots * a.KV * R) * HD);
  }
  if (many) {
    if (pairs * tiles * splits > (1L << 24) - 1)   // nothing has been launched yet
      return fail(FC_ERR_UNSUPPORTED, "fc_qcache_attention: %ld row tiles of %ld heads in one call", tiles, pairs);
    a.pieces = (int)(pairs * tiles * splits);
    const int once = (HD == 64 ? 3 : 2) * ctx->num_cus / 8 * 8;   // workgroups that run at once
    if (NW == 4 && !parts && a.B > 1 && a.n_new && a.pieces >= 4 * once && at - ctx->part + 8 * kQueueStep <= ws) {
      a.queue = reinterpret_cast<int *>(at);
      hipLaunchKernelGGL(k_qattn_queue, dim3(1), dim3(8), 0, st, a.queue);
      FC_LAUNCH_OK(st, "k_qattn_queue");
    }
    ProfScope ps(ctx, st, "fc_qattn_rows");
    if (a.queue) hipLaunchKernelGGL((k_qattn_rows<HD, 4, true>), dim3((unsigned)once), dim3(256), 0, st, a);
    else if (NW == 4) hipLaunchKernelGGL((k_qattn_rows<HD, 4, false>), dim3((unsigned)a.pieces), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_qattn_rows<HD, 2, false>), dim3((unsigned)a.pieces), dim3(128), 0, st, a);
    FC_LAUNCH_OK(st, "k_qattn_rows");
  } else {
    const dim3 grid((unsigned)a.slots, (unsigned)a.KV);
    ProfScope ps(ctx, st, "fc_qattn");
    const bool big = pairs * a.cap * HD * 2 > (384L << 20);
    if (MT == 1 && big) hipLaunchKernelGGL((k_qattn<HD, 1, true>), grid, dim3(256), 0, st, a);
    else if (MT == 1) hipLaunchKernelGGL((k_qattn<HD, 1, false>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_qattn<HD, 2, false>), grid, dim3(256), 0, st, a);
    FC_LAUNCH_OK(st, "k_qattn");
  }
  if (parts) {
    ProfScope ps(ctx, st, "fc_qattn_join");
    if (many) {
      hipLaunchKernelGGL(k_qattn_join_rows<HD>, dim3((unsigned)((R + 31) / 32 * (HD / 32)), (unsigned)pairs), dim3(256), 0, st, a);
      FC_LAUNCH_OK(st, "k_qattn_join_rows");
    } else {
      const long more = logit ? (a.cap + kWeightKeys - 1) / kWeightKeys : 0;
      hipLaunchKernelGGL(k_qattn_join<HD>, dim3((unsigned)(R + more), (unsigned)pairs), dim3(256), 0, st, a, (int)R);
      FC_LAUNCH_OK(st, "k_qattn_join");
    }
  }
  if (weigh && !logit) {
    const long groups = (a.cap + kGroupKeys - 1) / kGroupKeys, all = pairs * groups;
    // workgroups for four on every CU, each with 256 rows at least, where their sums fit
    long rs = std::max<long>(1, std::min(4L * ctx->num_cus / all, (R + 255) / 256));
    rs = std::max<long>(1, std::min<long>(rs, (ws - up4(per)) / (pairs * a.cap)));
    float *wpart = rs > 1 ? ctx->part + up4(per) : nullptr;   // the splits' parts are joined by now
    {
      ProfScope ps(ctx, st, "fc_qattn_weight");
      hipLaunchKernelGGL(k_qattn_weight<HD>, dim3((unsigned)(all * rs)), dim3(256), 0, st, a, wpart, (int)rs);
      FC_LAUNCH_OK(st, "k_qattn_weight");
    }
    if (rs > 1) {
      ProfScope ps(ctx, st, "fc_qattn_weight_add");
      hipLaunchKernelGGL(k_qattn_weight_add, dim3((unsigned)((a.cap + 255) / 256), (unsigned)pairs), dim3(256), 0, st, a, wpart, (int)rs);
      FC_LAUNCH_OK(st, "k_qattn_weight_add");
    }
  }
  return FC_OK;
}

}  // namespace

fc_status launch_qcache_attention(fc_ctx *ctx, const fc_qcache &c, const uint16_t *q,
                                  const int32_t *len, const int32_t *n_new,
                                  const uint8_t *key_mask, uint16_t *out, int n_heads, float scale,
                                  bool accumulate, int B, int n, hipStream_t st) {
  QAttnArgs a{};
  a.k = c.k, a.v = c.v, a.ks = c.k_scale, a.vs = c.v_scale, a.weight = c.weight;
  a.q = q, a.out = out, a.len = len, a.n_new = n_new, a.mask = key_mask;
  // a negative scale turns the queries' signs instead; scale 0: a number that leaves scores of any
  // ordinary size at 0 and hidden ones at -inf
  a.c = std::min(std::max(std::fabs(scale) * kLog2e, 1.2e-38f), 3.4e38f);
  a.flip = scale < 0.f ? 0x80008000u : 0u;
  a.B = B, a.n = n, a.H = n_heads, a.KV = c.n_kv_heads, a.G = n_heads / c.n_kv_heads, a.cap = c.capacity;
  a.by_g = quot_by(a.G);
  return c.head_dim == 128 ? run_qattn<128>(ctx, a, accumulate, st) : run_qattn<64>(ctx, a, accumulate, st);
}

}  // namespace fc
