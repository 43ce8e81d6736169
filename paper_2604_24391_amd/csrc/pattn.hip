// Attention of new rows over the paged token cache.
//
//   S_ij = c q_i . k_j over the rows j <= held + i that have a page and that the key mask shows,
//   P = softmax_j(S), out_i = sum_j P_ij v_j (a row that sees no key: 0).
//
// Laid out as the attention over the 8-bit cache (qattn.hip): the n tokens of an item make R = n G rows
// of a matrix product per key-value head, S^T = K Q^T and O^T = V^T P^T, so that a lane holds one
// query row and its softmax is per-lane scalars; the rows of an S^T tile are permuted so that a
// lane's probabilities are those of neighbouring keys, the B operand of the second product as it
// stands.  Operands are bfloat16 as the cache stores them.  P is rounded to bfloat16 for the second
// product (half a step, 2^-8 of each term of a float32 sum whose terms err apart).  k_pattn divides by the
// sum of unrounded ones, k_pattn_rows by that of rounded ones, which it adds up in pairs.
//
// Probabilities and their sums are held 2^-25 smaller than they are, which their quotient does not
// show: there is room for a running reference 2^16 behind a row's largest probability, and sums of
// outputs before the division still stay within float32 for 2^9 rows of bfloat16's largest numbers.
// At the other end a product or a sum below 2^-126 may be lost: for each key seen up to 2^-125 of a sum that is
// divided by 2^-25 or more, 2^-100 of an output.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_dev.h"
#include "fc_internal.h"
#include "pcache.h"

namespace fc {
namespace {

struct PAttnArgs {
  const uint16_t *k, *v;
  PageTable t;
  const uint16_t *q;
  uint16_t *out;
  const int32_t *len, *n_new;
  const uint8_t *mask;               // [B][cap], or null
  float2 *ml;                        // reference (log2) and sum of each split's rows
  float *part;                       // unnormalised outputs: k_pattn [KV][slots][R][hd], k_pattn_rows as
                                     // k_pattn_join_rows has it
  int2 *plan;                        // [B] k_pattn: an item's first slot and its slots
  float c;                           // scale log2(e)
  int B, n, H, KV, G, cap, splits, least, tile_rows, slots;
  int head_xcds;                     // k_pattn: XCDs of a head, or 0: heads along the grid's other axis
  int row_tiles, stride;             // k_pattn_rows: of a pair; pairs whose pieces take turns
  int *queue, pieces;                // k_pattn_rows: 8 counts of pieces taken behind the first ones, or null
  int back;                          // and from which one on an XCD takes its pieces from the last one back, or 0
  Quot by_g;                         // division by G
  uint32_t flip;                     // sign bits of a query pair to turn
};

constexpr float kProbDown = 25.f;    // log2
constexpr float kProbMost = 0x1p-9f; // as they are held: 2^16

__device__ __forceinline__ float output_factor(float l) { return l == 0.f ? 0.f : 1.f / l; }

// Values that are not finite.  0 times one is NaN, so where some row may not see a block whole they become
// 0 before the product, and what the rows that see them get for them is added afterwards.
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
// Their kinds, for one column of 64 keys: NaN, +inf, -inf.
struct OddKeys {
  uint64_t kind[3];
};
// Eight values of a column: those that are not finite become 0; their bits by kind.
__device__ __forceinline__ void take_odd(u32x4 &w, uint32_t *bits) {
  bits[0] = bits[1] = bits[2] = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint32_t x = w[i] >> (16 * s) & 0xFFFFu;
      if ((x & 0x7F80u) != 0x7F80u) continue;
      bits[(x & 0x7Fu) ? 0 : (x >> 15) + 1] |= 1u << (2 * i + s);
      w[i] &= s ? 0x0000FFFFu : 0xFFFF0000u;
    }
}
// What a row that sees `keys` of the column gets for them.
__device__ __forceinline__ float odd_sum(const OddKeys &o, uint64_t keys) {
  const bool up = o.kind[1] & keys, down = o.kind[2] & keys;
  const float inf = __builtin_inff();
  return (o.kind[0] & keys) || (up && down) ? __builtin_nanf("") : up ? inf : down ? -inf : 0.f;
}

template <bool NT>
__device__ __forceinline__ u32x4 load16(const uint16_t *p) {
  const u32x4 *q = reinterpret_cast<const u32x4 *>(p);
  return NT ? __builtin_nontemporal_load(q) : *q;
}

// All rows of an item (MT tiles of 16: up to 32) against a run of its key blocks, which go round the 4
// waves; these are joined in LDS.  An item's only slot writes the outputs, several their parts.
// Loads run ahead: each next block's keys are read when the scores have used theirs, its values after
// the outputs, its page numbers a block before both.
template <int HD, int MT, bool NT>
__global__ __launch_bounds__(256, HD == 128 && MT == 2 ? 1 : 2) void k_pattn(PAttnArgs a) {
  constexpr int KC = HD / 32;                   // 16-byte pieces of a key row that a lane holds
  constexpr int DT = HD / 16;                   // output tiles of 16 dims
  constexpr int OS = HD + 4;
  // Whether a wave's last look ahead is made too: short shares are better off without (sixteen items of 2200
  // rows 20.0 and 16.9 us, of up to 4200 25.2 and 23.6; one of 2176 10.9 and 9.8), but the branch costs
  // where loads are what bounds it (eight long ones 149.6 and 152.6) and with two row tiles (27.0 and 27.8).
  constexpr bool ALWAYS = NT || MT == 2;
  __shared__ float sm_o[4][16][OS];
  __shared__ float2 sm_ml[4][16 * MT];
  __shared__ float sm_l[16];
  __shared__ OddKeys sm_odd[4][HD];
  // Workgroups go round the 8 XCDs; each of these keeps to one head (several share it where there are fewer),
  // so that pages that several items hold come out of its L2 (sixteen answers on one history 17.1 to 16.5 us,
  // 64 items of their own 67.9 to 68.8).
  const int xcd = blockIdx.x % 8, turn = blockIdx.x / 8;
  const int kv = a.head_xcds ? xcd / a.head_xcds : blockIdx.y;
  const int my_slot = a.head_xcds ? turn * a.head_xcds + xcd % a.head_xcds : blockIdx.x;
  if (my_slot >= a.slots) return;
  const Share sh = share_of(a, my_slot);
  if (sh.item < 0) return;
  const int b = sh.item, R = a.n * a.G;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, l16 = lane & 15;
  const int held = sh.held, m = sh.m, rows = m * a.G;   // m > 0
  const int kmax = held + m;                    // keys that any row sees
  const int kall = held + 1;                    // keys that every row sees, but for the mask
  const int blocks = (kmax + kKeyBlock - 1) / kKeyBlock, blo = (my_slot - sh.start) * sh.per;
  const int bhi = min(blocks - blo, sh.per) + blo;
  const long slot = (long)kv * a.slots + my_slot;
  if (a.plan && kv == 0 && blo == 0 && tid == 0) a.plan[b] = make_int2(sh.start, sh.used);
  // S^T row m of tile t is key (m / 4) 16 + 4 t + m % 4
  const int in_page = (1 << a.t.shift) - 1;
  const uint16_t *kbase = a.k + (l16 & 3) * HD + g * 8, *vbase = a.v + l16 * kPTile;
  auto rows_of = [&](int page, int j) { return ((((long)page * a.KV + kv) << a.t.shift) + (j & in_page)) * HD; };
  // page of the 16 keys that lane group x holds in block blk (blocks behind the last one are read as it)
  auto page_of = [&](int blk, int x) { return a.t.entry(b, min((blk * kKeyBlock + 16 * x) >> a.t.shift, a.t.width - 1)); };
  u32x4 kw[4][KC], vw[2][DT];
  auto load_k = [&](int blk, int page) {
    const uint16_t *p = kbase + rows_of(a.t.safe(page), blk * kKeyBlock + (l16 >> 2) * 16);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < KC; ++i) kw[t][i] = load16<NT>(p + 4 * t * HD + 32 * i);
  };
  auto load_v = [&](int blk, int page) {
    const uint16_t *p = vbase + rows_of(a.t.safe(page), blk * kKeyBlock + g * 16);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int d = 0; d < DT; ++d) vw[s][d] = load16<NT>(p + s * (HD * kPTile) + 16 * d * kPTile);
  };
  // the block that a wave goes on with; its last one again, which the L2 holds, where it has no other
  auto behind = [&](int blk) { return blk + 4 < bhi ? blk + 4 : blk; };
  int at = min(blo + wave, bhi - 1), next = behind(at);
  int kp = page_of(at, l16 >> 2), vp = page_of(at, g);
  int kp_next = page_of(next, l16 >> 2), vp_next = page_of(next, g);
  // mask bytes of the lane's 16 keys, a block ahead as well
  const uint8_t *mbase = a.mask ? a.mask + (long)b * a.cap : nullptr;
  u32x4 mw = {~0u, ~0u, ~0u, ~0u};
  auto load_mask = [&](int blk) {
    mw = *reinterpret_cast<const u32x4 *>(mbase + min(blk * kKeyBlock + 16 * g, a.cap - 16));
  };
  if (mbase) load_mask(at);
  load_k(at, kp);
  load_v(at, vp);
  bf16x8 q[MT][KC];
  int seen[MT];                                 // keys that the lane's row sees
  f32x4 o[MT][DT];
  float mx[MT], sum[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int r = 16 * t + l16, tok = a.by_g(min(r, rows - 1));
    seen[t] = r < rows ? held + tok + 1 : 0;
    const uint16_t *src = a.q + (((long)b * a.n + tok) * a.H + kv * a.G + min(r, rows - 1) - tok * a.G) * HD;
#pragma unroll
    for (int i = 0; i < KC; ++i) q[t][i] = load_q(src + 32 * i + g * 8, a.flip);
    mx[t] = kNegInf, sum[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0, 0, 0, 0};
  }

  for (int blk = blo + wave; blk < bhi; blk += 4) {
    const int j0 = blk * kKeyBlock, jg = j0 + 16 * g;
    next = behind(blk);
    const int after = behind(next);
    const bool whole = __all(a.t.there(vp));
    const bool full = !a.mask && j0 + kKeyBlock <= kall && whole;
    uint32_t vis = 0xFFFFu;                       // the lane's 16 keys that some row may see
    if (!full) {
      if (mbase) {
        vis = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) vis |= (mw[i] >> (8 * e) & 0xFFu ? 1u : 0u) << (4 * i + e);
        load_mask(next);
      }
      const int left = kmax - jg;
      vis &= left >= 16 ? 0xFFFFu : (left <= 0 ? 0u : (1u << left) - 1u);
      if (!a.t.there(vp)) vis = 0;
    }
    bool odd = false;
    if (!full) {
      uint32_t any = 0;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) any |= odd_halves(vw[s][d][i]);
      odd = __any(any != 0);
      if (odd) {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          uint32_t lo[3], hi[3];
          take_odd(vw[0][d], lo);
          take_odd(vw[1][d], hi);
#pragma unroll
          for (int x = 0; x < 3; ++x)
            reinterpret_cast<part16 *>(&sm_odd[wave][16 * d + l16].kind[x])[g] = (uint16_t)(lo[x] | hi[x] << 8);
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
        for (int i = 0; i < KC; ++i)
          s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kw[x][i]), q[t][i], s[x], 0, 0, 0);
      }
      if (t == MT - 1 && (ALWAYS || blk + 4 < bhi)) load_k(next, kp_next);
      const uint32_t sees = full ? 0xFFFFu : vis & (uint32_t)seen_bits(seen[t] - jg);
      float top = kNegInf;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y = s[x][e] * a.c;
          if (!full) y = sees >> (4 * x + e) & 1u ? y : kNegInf;
          s[x][e] = y;
          top = fmaxf(top, y);
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
          const float y = exp2_fast(s[x][e] - (ref + kProbDown));
          add += y;
          p[x >> 1][(x & 1) * 4 + e] = (__bf16)y;
        }
      sum[t] = sum[t] * corr + add;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        o[t][d] *= corr;
        o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw[0][d]), p[0], o[t][d], 0, 0, 0);
        o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw[1][d]), p[1], o[t][d], 0, 0, 0);
      }
      if (odd) {
        uint64_t keys = (uint64_t)sees << (16 * g);   // that the lane's row sees
        keys |= __shfl_xor(keys, 16);
        keys |= __shfl_xor(keys, 32);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][d][e] += odd_sum(sm_odd[wave][16 * d + 4 * g + e], keys);
      }
    }
    if (ALWAYS || blk + 4 < bhi) load_v(next, vp_next);
    kp = kp_next, vp = vp_next;
    kp_next = page_of(after, l16 >> 2), vp_next = page_of(after, g);
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
      sm_l[l16] = l;
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
        *reinterpret_cast<float4 *>(a.part + (slot * R + r) * HD + d) = make_float4(y[0], y[1], y[2], y[3]);
      } else {
        const float inv = output_factor(sm_l[row]);
        const bf16x4 w = {(__bf16)(y[0] * inv), (__bf16)(y[1] * inv), (__bf16)(y[2] * inv), (__bf16)(y[3] * inv)};
        *reinterpret_cast<bf16x4 *>(a.out + (((long)b * a.n + a.by_g(r)) * a.H + kv * a.G + r - a.by_g(r) * a.G) * HD + d) = w;
      }
    }
  }
}

// The parts of one row joined by one workgroup: their outputs weighted by 2^(m_s - m) and divided by the
// sum.
template <int HD>
__global__ __launch_bounds__(256) void k_pattn_join(PAttnArgs a) {
  constexpr int TPR = HD / 4, SG = 256 / TPR;
  __shared__ float sm_y[SG][HD];
  __shared__ float2 sm_ml[SG];
  const int hb = blockIdx.y, b = hb / a.KV, kv = hb % a.KV, tid = threadIdx.x;
  const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
  const int R = a.n * a.G, rows = m * a.G, r = blockIdx.x;
  if (r >= rows) return;
  // part s of row r: at + s R
  const int2 sh = a.plan[b];          // (written, as the item has rows)
  const long at = ((long)kv * a.slots + sh.x) * R + r;
  const int used = sh.y, sg = tid / TPR, d = tid % TPR * 4;
  float mt = kNegInf, l = 0.f;
  f32x4 y = {0, 0, 0, 0};
  for (int s = sg; s < used; s += SG) {
    const float2 z = a.ml[(long)s * R + at];
    const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part + ((long)s * R + at) * HD + d);
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
  }
}

// More than 32 rows: 4 waves of 32 each (2 up to 64 rows) share the key blocks, which the DMA brings into
// LDS a block ahead (32 KB at hd 128).  32 x 32 matrix instructions; a lane holds one row and, of half a
// block's keys, the 16 of its half wave.
//
// Pieces of work are numbered pair by pair (item and key-value head), eight pairs taking turns as
// workgroups go round the 8 XCDs (fewer where their number is no multiple of eight), the last rows, which
// see most keys, first: an XCD works on one or two pairs at a time, whose keys its L2 holds (sixteen frames
// 634 us with all pairs at once, 597 so).  Items of one batch differ in length, so from two rounds of
// workgroups on pieces come from queues: as many workgroups as run at once, each going on with the next
// piece of its XCD's pairs, then with the others' (eight items of 10 to 4000 rows and 300 new ones
// 165 us before and 114 now, of 1024 397 and 323, ragged 310 and 254; of equal length 312 without queues
// and 319 with).
//
// A wave goes half a block (32 keys) at a time: beside the exponentials of its scores run the products
// of the next half's scores and of the last half's values, one exponential to a product, so that matrix
// and vector unit work at the same time (with each kind in a run of its own two waves on a SIMD took
// the sum of both: 544 us for a prompt of 8192 rows of 28 heads; with the values' products alone in a
// run 499; 457 now).  Keys are therefore brought a block ahead of values, and operands are read from
// LDS four products before their use (eight: the same).  No maximum is looked for (see `step`): a third
// fewer vector instructions.  Page numbers come by vector loads a block ahead, as a scalar load would
// have every wait for LDS wait for it.
//
// That prompt (0.48 TFLOP) takes 435 to 457 us back to back, 1.05 to 1.1 PFLOP/s.  Counted, at 470 us a
// launch, it has 812 thousand cycles, a clock of 1.73 GHz of 2.4, and the matrix unit busy for 57 % of
// them: power holds the clock there, and cycles saved come back in part as a lower one (from 893
// thousand at 1.82 GHz).  A run's loads share one asm block and its
// address serves keys and values: 457 to 443 us on one card, as scalar instructions take turns with the
// others.  Two row tiles in a wave would halve what LDS delivers for each product, but the compiler
// keeps no 128 output registers out of the vector unit's way there (650 us). 256 tokens over 2176 rows:
// 21 us, eight or nine blocks one after the other on 224 workgroups, and their start and end.
//
// A row of keys is 16-byte pieces, stored at piece ^ f(row) so that the 16 lanes that a read serves
// together (0-3, 12-15, 20-23, 24-27 and the other 16 of each half) fall on different banks; columns of
// values lie side by side as they are.
template <int HD>
__device__ __forceinline__ int pkey_swz(int row) {
  return HD == 128 ? row & 15 : (row >> 1) & 7;
}

// Both numbers of a pair of bfloat16 and c added up.
__device__ __forceinline__ float pair_sum(uint32_t pair, float c) {
  const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), one, c, false);
}

template <int HD, int NW, bool QUEUE>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void k_pattn_rows(PAttnArgs args) {
  constexpr int PC = HD / 8;                    // 16-byte pieces of a key row
  constexpr int DT = HD / 32;                   // output tiles of 32 dims
  constexpr int KS = HD / 16;                   // products of a tile of scores
  constexpr int TILE = kKeyBlock * HD * 2;      // bytes of a block's keys, and of its values
  constexpr int DMAS = TILE / 1024 / NW;        // DMA instructions of a wave for either
  constexpr int SUBS = 4 / NW;                  // runs of 16 rows that a wave brings, DMAS / SUBS instructions each
  constexpr int ROWS = 32 * NW;
  __shared__ __align__(1024) uint8_t sm_k[2][TILE], sm_v[2][TILE];
  __shared__ OddKeys sm_odd[2][HD];
  __shared__ int sm_flag[2][NW];
  __shared__ __align__(16) uint8_t sm_mask[2][NW][256];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  auto work = [&](const PAttnArgs &a, int id) {
    const int P = a.B * a.KV, R = a.n * a.G;   // pairs of item and key-value head, rows of each
    const int seq = id / a.stride, per = a.row_tiles * a.splits, rest = seq % per;
    const int hb = id % a.stride + a.stride * (seq / per), split = rest % a.splits;
    const int r0 = (a.row_tiles - 1 - rest / a.splits) * ROWS;
    const int b = hb / a.KV, kv = hb % a.KV;
    const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
    const int rows = m * a.G;
    if (r0 >= rows) return;
    const int kmax = held + a.by_g(min(r0 + ROWS, rows) - 1) + 1;
    const int blocks = (kmax + kKeyBlock - 1) / kKeyBlock, used = splits_used(kmax, a);
    if (split >= used) return;
    const int blo = (int)((long)blocks * split / used), bhi = (int)((long)blocks * (split + 1) / used);

    // Pages of a block's four runs of 16 rows (blocks behind the last one are read as it).  They are loaded
    // by lanes (0 to 3: a run each) a block before they are looked at: scalar loads would have every
    // wait for LDS wait for them too.
    struct Pages {
      int run[SUBS];                   // those of the runs that this wave brings
      uint32_t there;                  // the runs that have one
    };
    auto entries_of = [&](int blk) {
      return a.t.entry(b, min((4 * min(blk, bhi - 1) + (lane & 3)) >> (a.t.shift - 4), a.t.width - 1));
    };
    auto unpack = [&](int e) {
      Pages p;
#pragma unroll
      for (int u = 0; u < SUBS; ++u) p.run[u] = __builtin_amdgcn_readlane(e, wave * SUBS + u);
      p.there = (uint32_t)__ballot(a.t.there(e)) & 15;
      return p;
    };
    auto there = [&](const Pages &p) -> uint64_t {   // keys that have one
      if (p.there == 15) return ~0ull;
      uint64_t m = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (p.there >> x & 1) m |= 0xFFFFull << (16 * x);
      return m;
    };
    const int in_page = (1 << a.t.shift) - 1;
    // bytes from a pool's start to where run u of this wave's of block blk begins
    auto run_at = [&](int blk, const Pages &p, int u) {
      const int j = min(blk, bhi - 1) * kKeyBlock + 16 * (wave * SUBS + u);
      return uniform(((((long)a.t.safe(p.run[u]) * a.KV + kv) << a.t.shift) + (j & in_page)) * (2 * HD));
    };
    constexpr int PER = DMAS / SUBS;
    // a lane's bytes of a run's first KB of keys (piece ^ f(row)): those of the i-th KB are 64 i away in an exclusive or
    const int ksrc = lane / PC * (HD * 2) + ((lane % PC) ^ pkey_swz<HD>(lane / PC)) * 16;
    // Where in the pools a wave's runs of a block lie.
    struct Source {
      uint64_t at[SUBS];
    };
    auto source = [&](int blk, const Pages &p) {
      Source s;
#pragma unroll
      for (int u = 0; u < SUBS; ++u) s.at[u] = run_at(blk, p, u);
      return s;
    };
    const uint64_t k_pool = (uint64_t)(uintptr_t)a.k, v_pool = (uint64_t)(uintptr_t)a.v;
    // the u-th run of either
    auto fetch_k = [&](const Source &src, int stage, int u) {
      int off[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) off[i] = ksrc ^ (64 * i);
      dma16_run<PER>(k_pool + src.at[u], off, lds_addr(&sm_k[stage][(wave * DMAS + u * PER) * 1024]));
    };
    auto fetch_v = [&](const Source &src, int stage, int u) {
      int off[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) off[i] = lane * 16;
      dma16_run<PER>(v_pool + src.at[u], off, lds_addr(&sm_v[stage][(wave * DMAS + u * PER) * 1024]));
    };
    auto each_run = [&](auto f) {
#pragma unroll
      for (int u = 0; u < SUBS; ++u) f(u);
    };
    // a block's 64 mask bytes for each wave (four times over: a DMA writes 4 bytes for every lane)
    auto fetch_mask = [&](int blk, int stage) {
      dma4(a.mask + (long)b * a.cap + min(min(blk, bhi - 1) * kKeyBlock + (lane & 15) * 4, a.cap - 4), lds_addr(&sm_mask[stage][wave][0]));
    };

    const int w0 = r0 + 32 * wave, r = w0 + l32, tok = a.by_g(min(r, rows - 1)), head = kv * a.G + min(r, rows - 1) - tok * a.G;
    const int seen = r < rows ? held + tok + 1 : 0;                              // keys that the lane's row sees
    const int wall = held + a.by_g(w0) + 1;                                      // that every row of the wave sees
    const int gall = held + a.by_g(r0) + 1;                                      // that every row of the workgroup does
    const long at_q = (((long)b * a.n + tok) * a.H + head) * HD;
    bf16x8 q[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) q[i] = load_q(a.q + at_q + 16 * i + 8 * h, a.flip);
    const int e0 = entries_of(blo), e1 = entries_of(blo + 1);
    int e2 = entries_of(blo + 2);
    Pages pg = unpack(e0), pg1 = unpack(e1), pg2;   // of the blocks blk, blk + 1, blk + 2
    loads_done();
    Source src = source(blo, pg), src1 = source(blo + 1, pg1);   // of the blocks whose values and whose keys come next
    each_run([&](int u) { fetch_k(src, 0, u); });
    if (a.mask) fetch_mask(blo, 0);
    each_run([&](int u) { fetch_v(src, 0, u); });

    // S^T row x of a half block is key x with bits 2 and 3 of x exchanged
    const int kr = (l32 & 19) | ((l32 >> 2) & 1) << 3 | ((l32 >> 3) & 1) << 2;
    const int koff = kr * HD * 2 + (h ^ pkey_swz<HD>(kr)) * 16;   // piece h; piece 2 i + h is 32 i away in an exclusive or
    const int voff = (h * HD + l32) * 16;
    auto key_frag = [&](int stage, int half, int at, int i) {
      return *reinterpret_cast<const bf16x8 *>(&sm_k[stage][(at ^ (32 * i)) + half * 64 * HD]);
    };
    auto value_frag = [&](int stage, int half, int t, int d) {
      return *reinterpret_cast<const bf16x8 *>(&sm_v[stage][voff + ((4 * half + 2 * t) * HD + 32 * d) * 16]);
    };
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    float ref = kNegInf, sum = 0.f, sub = kProbDown;   // exponents are taken relative to ref, ref + kProbDown
    // a lane's sum of probabilities of 16 keys beyond which ref is looked at (any, as long as its row has seen no key)
    float limit = r < rows ? -1.f : __builtin_inff();
    f32x16 sa, sb;                    // scores of a block's halves

    // What a row does not see of a half block, given its scores and the keys shown.
    auto hide = [&](f32x16 &s, int j0, uint32_t shown) {
      if (j0 + 32 <= wall && shown == ~0u) return;
      // the lane's 16 keys: 16 i + 8 h + e
      const uint32_t sees = (shown & (uint32_t)seen_bits(seen - j0)) >> (8 * h);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!(sees >> (16 * (e / 8) + e % 8) & 1u)) s[e] = kNegInf;
    };
    // Values that are not finite, of the runs that this wave has brought, where not every row may see them:
    // they become 0, and their places are listed.
    auto clean = [&](int stage) {
      uint32_t any = 0;
      u32x4 *at = reinterpret_cast<u32x4 *>(&sm_v[stage][wave * DMAS * 1024]) + lane;
#pragma unroll
      for (int i = 0; i < DMAS; ++i) {
        const u32x4 w = at[64 * i];
#pragma unroll
        for (int x = 0; x < 4; ++x) any |= odd_halves(w[x]);
      }
      const bool odd = __any(any != 0);
      if (odd)
#pragma unroll 1
        for (int i = 0; i < DMAS; ++i) {
          u32x4 w = at[64 * i];
          uint32_t bits[3];
          take_odd(w, bits);
          at[64 * i] = w;
          const int p = (wave * DMAS + i) * 64 + lane;
#pragma unroll
          for (int x = 0; x < 3; ++x) reinterpret_cast<part8 *>(&sm_odd[stage][p % HD].kind[x])[p / HD] = (uint8_t)bits[x];
        }
      if (lane == 0) sm_flag[stage][wave] = odd;
    };
    // and what the rows that see them get for them
    auto add_odd = [&](int blk, int stage, uint64_t shown) {
      uint64_t listed = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w)
        if (sm_flag[stage][w]) listed |= (NW == 4 ? 0xFFFFull : 0xFFFFFFFFull) << (64 / NW * w);
      if (__builtin_amdgcn_readfirstlane((int)(listed != 0)) == 0) return;
      const uint64_t keys = listed & shown & seen_bits(seen - blk * kKeyBlock);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] += odd_sum(sm_odd[stage][32 * d + 8 * (e / 4) + 4 * h + e % 4], keys);
    };
    auto both_halves = [&](float x) {
      const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
    };

    // A step of 32 keys, whose scores are in s: their exponentials beside the products of the next step's scores
    // and of the values of the step before, one to each (two at hd 64), so that neither unit waits for the
    // other.  Operands are read from LDS AHEAD products before their use.
    //
    // Exponents are taken relative to ref, which follows a row's largest score only where the sum of a lane's
    // probabilities shows that it has been left 2^16 behind (or where the row has seen no key yet): most
    // steps need not look for their maximum, nor touch O (2^9: 495 us for the prompt above, 471 so).
    // Each row's ref follows its own scores alone: another row's may come from keys that are hidden from
    // it, and would show in how this one's are rounded.
    constexpr int SLOTS = KS + 2 * DT, PM = 16 / SLOTS, AHEAD = 4;
    bf16x8 frag[AHEAD];
    u32x4 p[2][2];                    // probabilities of the last two steps
    // the operand of product i: keys of the next step's half (next_half of the block at key stage ks), then values
    // of the step before (the other half of the block at stage vs)
    auto operand = [&](int ks, int vs, int half, int i) {
      return i < KS ? key_frag(ks, half, koff, i) : value_frag(vs, half, (i - KS) / DT, (i - KS) % DT);
    };
    auto read_ahead = [&](int ks, int vs, int half) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) frag[i] = operand(ks, vs, half, i);
    };
    // half: of the block that the next scores and the last values are of; first: the one behind the barrier, which
    // loads go with; last: no scores are left; start: no values yet
    enum { kFirst = 1, kLast = 2, kStart = 4 };
    auto step = [&](auto key_stage, auto value_stage, auto which, auto kind, f32x16 &s, f32x16 &next, int j_next, uint32_t show_next) {
      constexpr int ks = decltype(key_stage)::value, vs = decltype(value_stage)::value, half = decltype(which)::value;
      constexpr int what = decltype(kind)::value;
      constexpr int parity = half ^ 1;          // of the step itself: the second half's scores follow the first's
      float add = 0.f;
      float y[16];
      auto exps = [&](int from, int to) {
#pragma unroll
        for (int e = from; e < to; ++e) y[e] = exp2_fast(fmaf(s[e], a.c, -sub));
      };
      auto pack = [&](int from, int to) {
#pragma unroll
        for (int e = from; e < to; e += 2) {
          const bf16x2 w = {(__bf16)y[e], (__bf16)y[e + 1]};
          uint32_t u = __builtin_bit_cast(uint32_t, w);
          asm volatile("" : "+v"(u));   // rounded here: the pairs' registers are needed
          p[parity][e / 8][e % 8 / 2] = u;
          add = pair_sum(u, add);
        }
      };
#pragma unroll
      for (int e = 0; e < 16; ++e) next[e] = 0.f;
      auto slot = [&](auto at) {
        constexpr int i = decltype(at)::value;
        if constexpr (i < KS) {
          if constexpr (!(what & kLast)) next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % AHEAD], q[i], next, 0, 0, 0);
        } else if constexpr (!(what & kStart)) {
          constexpr int x = i - KS;
          o[x % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % AHEAD], __builtin_bit_cast(bf16x8, p[parity ^ 1][x / DT]), o[x % DT], 0, 0, 0);
        }
        auto read = [&](auto product) {
          constexpr int f = decltype(product)::value;
          if constexpr (f < SLOTS && !(f < KS ? what & kLast : what & kStart)) frag[f % AHEAD] = operand(ks, vs, half, f);
          if constexpr (f >= SLOTS && (what & kFirst) && !(what & kLast)) frag[f % AHEAD] = operand(ks, vs, half ^ 1, f - SLOTS);
        };
        // two at a time take half the waits (the prompt above 444 us and 435), but not beside the queue's registers
        // (16 items of 1024 rows over 3000: 769 and 777)
        if constexpr (QUEUE) read(std::integral_constant<int, i + AHEAD>());
        else if constexpr (i % 2) read(std::integral_constant<int, i + AHEAD - 1>()), read(std::integral_constant<int, i + AHEAD>());
        if constexpr ((what & kFirst) && !(what & kLast)) {   // the loads of the blocks to come
          constexpr int apart = SLOTS / (2 * SUBS), x = i / apart;
          if constexpr (i % apart == 0 && x < SUBS) fetch_k(src1, vs, x);
          else if constexpr (i % apart == 0 && x < 2 * SUBS) fetch_v(src, ks, x - SUBS);
        }
        exps(PM * i, PM * (i + 1));
        if constexpr (PM == 2) {
          if constexpr (i > 0) pack(2 * i - 2, 2 * i);
        } else {
          if constexpr (i > 0 && i % 2 == 0) pack(i - 2, i);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      slot(std::integral_constant<int, 0>()), slot(std::integral_constant<int, 1>()), slot(std::integral_constant<int, 2>()), slot(std::integral_constant<int, 3>());
      slot(std::integral_constant<int, 4>()), slot(std::integral_constant<int, 5>()), slot(std::integral_constant<int, 6>()), slot(std::integral_constant<int, 7>());
      if constexpr (SLOTS == 16) {
        slot(std::integral_constant<int, 8>()), slot(std::integral_constant<int, 9>()), slot(std::integral_constant<int, 10>()), slot(std::integral_constant<int, 11>());
        slot(std::integral_constant<int, 12>()), slot(std::integral_constant<int, 13>()), slot(std::integral_constant<int, 14>()), slot(std::integral_constant<int, 15>());
      }
      pack(14, 16);
      if (const uint64_t over = __ballot(add > limit)) {
        const uint64_t rows_over = over | over << 32 | over >> 32;   // of either half wave
        float top = kNegInf;
#pragma unroll
        for (int e = 0; e < 16; e += 2) top = fmaxf(fmaxf(top, s[e]), s[e + 1]);
        top = both_halves(top) * a.c;
        const bool up = __builtin_amdgcn_inverse_ballot_w64(rows_over) && top > ref;
        const float corr = up ? exp2_fast(ref - top) : 1.f;
        ref = up ? top : ref;
        sub = (ref == kNegInf ? 0.f : ref) + kProbDown;
        limit = ref == kNegInf ? limit : kProbMost;
        sum *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= corr;
        add = 0.f;
        exps(0, 16);
        pack(0, 16);
      }
      sum += add;
      if constexpr (!(what & kLast)) hide(next, j_next, show_next);
    };
    // a block's keys that have a page and that the mask shows
    auto shown_of = [&](int stage, const Pages &pages) {
      uint64_t m = there(pages);
      if (a.mask) m &= __ballot(sm_mask[stage][wave][lane] != 0);
      return m;
    };
    std::integral_constant<int, 0> zero;
    std::integral_constant<int, 1> one;

    // The first block's scores, and its first step, which has no values to multiply.
    wait_vm<0>();
    lds_barrier();
    uint64_t show = shown_of(0, pg);
    if (w0 < rows) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sa[e] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i) sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_frag(0, 0, koff, i), q[i], sa, 0, 0, 0);
      hide(sa, blo * kKeyBlock, (uint32_t)show);
      read_ahead(0, 0, 1);
      step(zero, zero, one, std::integral_constant<int, kStart>(), sa, sb, blo * kKeyBlock + 32, (uint32_t)(show >> 32));
    }
    src = src1;
    each_run([&](int u) { fetch_k(src, 1, u); });
    if (a.mask) fetch_mask(blo + 1, 1);
    // When block blk begins, its values and the keys of the next one have come: the second step of its scores, with
    // the values of its first half, and the first step of the next block's, with those of its second.
    auto block = [&](auto st, auto other, auto goes_on, int blk) {
      constexpr int stage = decltype(st)::value;   // of its values, and of the keys of the block after the next
      constexpr bool more = decltype(goes_on)::value;
      const bool partly = a.mask || blk * kKeyBlock + kKeyBlock > gall || there(pg) != ~0ull;
      wait_vm<0>();                    // this wave's parts of the blocks; the barrier adds the others', and
      if (partly) clean(stage);
      lds_barrier();                   // every wave has left what the loads below write over
      pg2 = unpack(e2);                // (come with the loads waited for above)
      uint64_t ahead = 0;
      if (more) {
        src = src1;
        src1 = source(blk + 2, pg2);
        e2 = entries_of(blk + 3);
        ahead = shown_of(stage ^ 1, pg1);
        if (a.mask) fetch_mask(blk + 2, stage);
      }
      if (w0 < rows) {
        const int j1 = blk * kKeyBlock + kKeyBlock;
        if constexpr (more) {
          read_ahead(stage ^ 1, stage, 0);
          step(other, st, zero, std::integral_constant<int, kFirst>(), sb, sa, j1, (uint32_t)ahead);
          step(other, st, one, zero, sa, sb, j1 + 32, (uint32_t)(ahead >> 32));
        } else {
#pragma unroll
          for (int i = KS; i < KS + AHEAD; ++i) frag[i % AHEAD] = operand(stage ^ 1, stage, 0, i);
          step(other, st, zero, std::integral_constant<int, kLast>(), sb, sa, j1, 0u);
#pragma unroll
          for (int x = 0; x < 2 * DT; ++x)
            o[x % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_frag(stage, 1, x / DT, x % DT), __builtin_bit_cast(bf16x8, p[1][x / DT]), o[x % DT], 0, 0, 0);
        }
        if (partly) add_odd(blk, stage, show);
      } else if (more) {               // it only brings its part of the blocks
        each_run([&](int u) { fetch_k(src1, stage, u); });
        each_run([&](int u) { fetch_v(src, stage ^ 1, u); });
      }
      show = ahead;
      pg = pg1, pg1 = pg2;
    };
    int blk = blo;
    for (; blk + 2 < bhi; blk += 2) {
      block(zero, one, std::true_type(), blk);
      block(one, zero, std::true_type(), blk + 1);
    }
    if (blk + 1 < bhi) {
      block(zero, one, std::true_type(), blk);
      block(one, zero, std::false_type(), blk + 1);
    } else {
      block(zero, one, std::false_type(), blk);
    }

    sum += __shfl_xor(sum, 32);
    if (r >= rows) return;
    if (a.splits > 1) {
      const long to = (long)split * P * R + (long)hb * R + r;
      if (h == 0) a.ml[to] = make_float2(ref, sum);
      f32x4 *dst = reinterpret_cast<f32x4 *>(a.part) + (((long)split * P + hb) * ((R + 31) / 32) + w0 / 32) * (HD / 8) * 64 + lane;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) dst[(4 * d + j) * 64] = f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
    } else {
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
    const int turn = blockIdx.x / 8, last = gridDim.x / 8 - 1;
    work(args, args.back && turn >= args.back ? 8 * (last - (turn - args.back)) + blockIdx.x % 8 : blockIdx.x);
  } else {
    __shared__ int sm_next;
    int id = blockIdx.x, from = blockIdx.x % 8;
    for (int done = 0;;) {             // queues found empty
      const PAttnArgs a = args_again<PAttnArgs>();
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

__global__ void k_pattn_queue(int *queue) { queue[kQueueStep * threadIdx.x] = 0; }

// The same for k_pattn_rows, whose rows are many and splits few: a workgroup joins 32 dims of 32 rows,
// eight splits' parts in flight at a time.  Parts lie as that kernel's lanes hold them, [split][pair]
// [32 rows][HD / 8][half wave][row] by four dims, so that both kernels move runs of 1 KB.
template <int HD>
__global__ __launch_bounds__(256) void k_pattn_join_rows(PAttnArgs a) {
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
}

template <int HD>
fc_status run_pattn(fc_ctx *ctx, PAttnArgs &a, hipStream_t st) {
  const long R = (long)a.n * a.G, pairs = (long)a.B * a.KV;
  const bool many = R > 32;
  const int MT = R <= 16 ? 1 : 2, NW = R <= 64 ? 2 : 4, tile = many ? 32 * NW : 16 * MT;
  const long tiles = (R + tile - 1) / tile;
  const long per = pairs * R, padded = many ? pairs * ((R + 31) / 32 * 32) : per, ws = (long)ctx->part_elems;
  auto up4 = [](long x) { return (x + 3) / 4 * 4; };
  const long plan = up4(2L * a.B), all_blocks = (a.cap + kKeyBlock - 1) / kKeyBlock;
  long splits = 1, slots = a.B;
  if (many) {
    // What a number of splits costs in microseconds, from the capacity, as lengths are on the device: blocks one
    // after the other, for one wave on a SIMD or two that share it, and the parts, written and read, with
    // the join's launch.  (A frame of 256 rows over 2176: 43, 31, 27, 30 us with 1, 2, 4, 8 splits, over
    // 8320: 144, 81, 51, 46; a prompt of 1000: 26 and 35 with 1 and 2.)
    const long units = pairs * tiles;
    const double blocks = all_blocks * (HD == 128 ? 1.05 : 0.65), part = padded * HD * 8 / 4.5e6;
    auto cost = [&](long s) {
      const double waves = (double)units * s * NW / (4. * ctx->num_cus);
      return blocks / s * (waves <= 1 ? 1 : 1.25 * std::ceil(waves / 2)) + (s > 1 ? 4 + s * part : 0.);
    };
    a.least = 4;
    for (long places : {4L, 8L}) {       // up to a wave on each SIMD, up to two
      const long most = std::min<long>(places * ctx->num_cus / NW / units, all_blocks / 4);
      const long s = std::min<long>(most, std::lround(std::sqrt(blocks * (places == 4 ? 1 : 1.25) / part)));
      if (s > 1 && cost(s) < cost(splits)) splits = s;
    }
    splits = std::max<long>(1, std::min<long>(splits, (ws - plan) / (up4(2 * per) + padded * HD)));
  } else {
    slots = ctx->num_cus / a.KV;
    if (a.mask || HD == 64 || slots < 4L * a.B) slots = 2L * ctx->num_cus / a.KV;
    slots = std::min<long>(slots, all_blocks / 4 * a.B);
    slots = std::max<long>(a.B, std::min<long>(slots, (ws - plan - 4) / (a.KV * R * (HD + 2))));
  }
  const bool parts = many ? splits > 1 : slots > a.B;
  a.splits = (int)splits;
  a.tile_rows = tile;
  a.slots = many ? 0 : (int)slots;
  float *at = ctx->part;
  if (parts) {
    a.plan = reinterpret_cast<int2 *>(at);
    at += plan;
    a.part = at;
    a.ml = reinterpret_cast<float2 *>(at + (many ? splits * padded : slots * a.KV * R) * HD);
  }
  if (many) {
    if (pairs * tiles * splits > (1L << 24) - 1)   // nothing has been launched yet
      return fail(FC_ERR_UNSUPPORTED, "fc_pcache_attention: %ld row tiles of %ld heads in one call", tiles, pairs);
    a.pieces = (int)(pairs * tiles * splits);
    a.row_tiles = (int)tiles;
    a.stride = pairs % 8 == 0 ? 8 : pairs % 4 == 0 ? 4 : pairs % 2 == 0 ? 2 : 1;
    // A CU gets a second workgroup when each has one: the shortest go to the CUs of the longest (a prompt of
    // 2048: 50 to 47 us; four of 4096 in 4 heads of 64, whose pairs also begin at once: 79 to 64).
    const int round = 4 / NW * (ctx->num_cus / 8 * 8);
    if (splits == 1 && a.pieces % 8 == 0 && a.pieces > round && a.pieces <= 2 * round) {
      if (pairs % 8 == 0) a.stride = (int)pairs;
      if (a.stride == pairs) a.back = round / 8;
    }
    // workgroups that run at once (without a queue a CU has three at hd 64: 1024 pieces 96 us with and 84, 2048
    // 152 and 175)
    const int once = 2 * ctx->num_cus / 8 * 8;
    if (NW == 4 && !parts && a.B > 1 && a.pieces >= (HD == 64 ? 3 : 2) * once && 8 * kQueueStep <= ws) {
      a.queue = reinterpret_cast<int *>(at);
      hipLaunchKernelGGL(k_pattn_queue, dim3(1), dim3(8), 0, st, a.queue);
      FC_LAUNCH_OK(st, "k_pattn_queue");
    }
    ProfScope ps(ctx, st, "fc_pattn_rows");
    if (a.queue) hipLaunchKernelGGL((k_pattn_rows<HD, 4, true>), dim3((unsigned)once), dim3(256), 0, st, a);
    else if (NW == 4) hipLaunchKernelGGL((k_pattn_rows<HD, 4, false>), dim3((unsigned)a.pieces), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_pattn_rows<HD, 2, false>), dim3((unsigned)a.pieces), dim3(128), 0, st, a);
    FC_LAUNCH_OK(st, "k_pattn_rows");
  } else {
    a.head_xcds = 8 % a.KV == 0 ? 8 / a.KV : 0;
    const dim3 grid = a.head_xcds ? dim3((unsigned)((a.slots + a.head_xcds - 1) / a.head_xcds * 8)) : dim3((unsigned)a.slots, (unsigned)a.KV);
    ProfScope ps(ctx, st, "fc_pattn");
    const bool big = std::min(pairs * a.cap, ((long)a.t.pages * a.KV) << a.t.shift) * HD * 4 > (384L << 20);
    if (MT == 1 && big) hipLaunchKernelGGL((k_pattn<HD, 1, true>), grid, dim3(256), 0, st, a);
    else if (MT == 1) hipLaunchKernelGGL((k_pattn<HD, 1, false>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_pattn<HD, 2, false>), grid, dim3(256), 0, st, a);
    FC_LAUNCH_OK(st, "k_pattn");
  }
  if (parts) {
    ProfScope ps(ctx, st, "fc_pattn_join");
    if (many)
      hipLaunchKernelGGL(k_pattn_join_rows<HD>, dim3((unsigned)((R + 31) / 32 * (HD / 32)), (unsigned)pairs), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(k_pattn_join<HD>, dim3((unsigned)R, (unsigned)pairs), dim3(256), 0, st, a);
    FC_LAUNCH_OK(st, "k_pattn_join");
  }
  return FC_OK;
}

}  // namespace

fc_status launch_pcache_attention(fc_ctx *ctx, const fc_pcache &c, const uint16_t *q, const int32_t *len,
                                  const int32_t *n_new, const uint8_t *key_mask, uint16_t *out, int n_heads,
                                  float scale, int B, int n, hipStream_t st) {
  PAttnArgs a{};
  a.k = c.k, a.v = c.v, a.t = page_table(c);
  a.q = q, a.out = out, a.len = len, a.n_new = n_new, a.mask = key_mask;
  // as in launch_qcache_attention
  a.c = std::min(std::max(std::fabs(scale) * kLog2e, 1.2e-38f), 3.4e38f);
  a.flip = scale < 0.f ? 0x80008000u : 0u;
  a.B = B, a.n = n, a.H = n_heads, a.KV = c.n_kv_heads, a.G = n_heads / c.n_kv_heads, a.cap = c.max_pages * c.page_rows;
  a.by_g = quot_by(a.G);
  return c.head_dim == 128 ? run_pattn<128>(ctx, a, st) : run_pattn<64>(ctx, a, st);
}

}  // namespace fc
