// The paged token cache: rows appended to their pages, and the pages themselves: items that go on from
// others' rows, grow and end, pages copied where several would write them, live pages moved together.
//
//   append: K rows (a, b) -> (a cos t - b sin t, b cos t + a sin t) for the pairs (i, i + hd / 2),
//           t = pos[axis(i)] theta^(-2 i / hd).  It moves bytes: every q, k and v element is read and
//           written once.
//   step:   table'[b] = the first ceil(len / R) entries of table[src b]; holders counted anew; the
//           k-th page needed (items in order, a copy's before those behind the kept rows) is the k-th
//           page without holders.
//   compact: the k-th live page from number L on to the k-th free page below it, L the live pages.
// The state is small (a few thousand numbers) and its parts depend on each other, so one workgroup
// makes the plan of a step, and a second launch moves the rows of all layers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "fc_internal.h"
#include "pcache.h"

namespace fc {
namespace {

// ------------------------------------------------------------------------------- append
constexpr int kPThreads = 256;

struct PAppendArgs {
  const uint16_t *q, *k, *v;                  // q may be null (no queries)
  long q_row, k_row, v_row;                   // elements from one token to the next
  long q_item, k_item, v_item;                // and from one item to the next
  const int32_t *pos, *len, *n_new;
  long pos_axis;                              // elements from one axis to the next
  uint16_t *q_out, *kc, *vc;
  PageTable t;
  int n, H, KV, cap, sec0, sec1;              // pairs below sec0 take axis 0, below sec1 axis 1
  double lo[8], hi[8];                        // lo[i % 8] hi[i / 8] = theta^(-2 i / hd) / (2 pi) turns
};

__device__ __forceinline__ void unpack8(u32x4 w, float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// Rounded to nearest even; a NaN stays one.
__device__ __forceinline__ u32x4 pack8(const float *x) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
    w[i] = __builtin_bit_cast(uint32_t, p);
  }
  return w;
}

// Eight rows of an item's cache, those that one group of value columns holds: all heads of the new
// tokens among them, so that a workgroup computes its angles once and writes whole 16-byte columns.
// A prompt of 8192 tokens of 36 heads of 128 (151 MB): 24 to 25 us, 6 TB/s, bound by HBM and the
// memory-side cache.  One token of 64 items: 4.4 us, one chain of length, position, angle and row
// (angles and rows of values asked for at once).
template <int HD>
__global__ __launch_bounds__(kPThreads) void k_pappend(PAppendArgs a) {
  constexpr int HALF = HD / 2, TPR = HD / 16;       // threads of one row of pairs, 8 pairs each
  __shared__ float2 cs[kPTile][HALF];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int held = q_held(a.len, b, a.cap), m = q_new(a.n_new, b, a.n, held, a.cap);
  const int group = held / kPTile + (int)blockIdx.x, j0 = group * kPTile;
  if (group >= a.cap / kPTile) return;
  const int lo = max(held, j0), cnt = min(held + m, j0 + kPTile) - lo;
  if (cnt <= 0) return;
  const int i0 = lo - held, at = lo - j0;            // first new row's token, its place in the group
  const int page = a.t.entry(b, j0 >> a.t.shift);
  const bool there = a.t.there(page);
  // angles in turns, reduced in 64 bits: float32 would lose those of far positions
  for (int x = tid; x < cnt * HALF; x += kPThreads) {
    const int t = x / HALF, p = x % HALF;
    const long ax = p < a.sec0 ? 0 : (p < a.sec1 ? 1 : 2);
    const double turn = (double)a.pos[ax * a.pos_axis + (long)b * a.n + i0 + t] * (a.lo[p & 7] * a.hi[p >> 3]);
    float s, c;
    sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
    cs[t][p] = make_float2(c, s);
  }
  __syncthreads();

  const int R = 1 << a.t.shift;
  const long in_page = (long)(j0 & (R - 1)) * HD;
  // rows of keys and queries, head by head; TPR threads to a row
  const int sub = tid % TPR, p0 = sub * 8, heads = a.KV + (a.q ? a.H : 0);
  for (int x = tid / TPR; x < cnt * heads; x += kPThreads / TPR) {
    const int t = x / heads, h = x % heads;
    const bool key = h < a.KV;
    if (key && !there) continue;
    const uint16_t *src = key ? a.k + (long)b * a.k_item + (long)(i0 + t) * a.k_row + h * HD
                              : a.q + (long)b * a.q_item + (long)(i0 + t) * a.q_row + (long)(h - a.KV) * HD;
    float u[8], w[8], y[16];
    unpack8(*reinterpret_cast<const u32x4 *>(src + p0), u);
    unpack8(*reinterpret_cast<const u32x4 *>(src + p0 + HALF), w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 r = cs[t][p0 + e];
      y[e] = u[e] * r.x - w[e] * r.y;
      y[8 + e] = w[e] * r.x + u[e] * r.y;
    }
    uint16_t *dst = key ? a.kc + (((long)page * a.KV + h) << a.t.shift) * HD + in_page + (at + t) * HD
                        : a.q_out + (((long)b * a.n + i0 + t) * a.H + h - a.KV) * HD;
    *reinterpret_cast<u32x4 *>(dst + p0) = pack8(y);
    *reinterpret_cast<u32x4 *>(dst + p0 + HALF) = pack8(y + 8);
  }
  if (!there) return;
  // values: eight columns of the group's rows to a thread
  for (int x = tid; x < a.KV * (HD / 8); x += kPThreads) {
    const int h = x / (HD / 8), d = x % (HD / 8) * 8;
    const uint16_t *src = a.v + (long)b * a.v_item + (long)i0 * a.v_row + h * HD + d;
    uint16_t *dst = a.vc + (((long)page * a.KV + h) << a.t.shift) * HD + in_page + d * kPTile;
    u32x4 r[kPTile];
#pragma unroll
    for (int t = 0; t < kPTile; ++t) r[t] = *reinterpret_cast<const u32x4 *>(src + (long)min(t, cnt - 1) * a.v_row);
    if (cnt == kPTile) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t u = r[2 * i][e / 2], v = r[2 * i + 1][e / 2];
          w[i] = e % 2 ? u >> 16 | (v & 0xFFFF0000u) : (u & 0xFFFFu) | v << 16;
        }
        *reinterpret_cast<u32x4 *>(dst + e * kPTile) = w;
      }
    } else {
#pragma unroll
      for (int t = 0; t < kPTile; ++t)
        if (t < cnt)
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[e * kPTile + at + t] = (uint16_t)(r[t][e / 2] >> (e % 2 * 16));
    }
  }
}

// ------------------------------------------------------------------------------- pages
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
constexpr int kPlanPages = 7168;              // pages whose counts a plan holds in LDS: up to 8 bytes each, 56 KB

// Rows that a plan has copied or moved: a tile is eight rows of one head.
struct PageMove {
  int from, to, tiles;
};

// The numbers of a plan in the context's workspace, of `step_numbers` (or `compact_numbers`) floats.
struct PlanWs {
  int *count;                                 // moves
  PageMove *move;
  int *table;                                 // the table before it is written: [B][width]
  int *need;                                  // [B] pages of the items before this one
  int *free;                                  // the pages given out; compact: where a page goes
  int *holders, *last;                        // [pages] where they do not fit into LDS (compact: no last)
};

struct StepArgs {
  int32_t *state;
  const int32_t *src, *len, *n_new;
  int32_t *granted;
  PlanWs ws;
  int B, width, pages, shift, n;
  Quot by_width;
};

// Sum of a number over the threads before this one (waves in order, lanes in order); total: over all.
// Waits for every thread before it writes wsum.
__device__ __forceinline__ int plan_scan(int x, int *wsum, int &total) {
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
  for (int i = 0; i < kPlanWaves; ++i) {
    if (i < w) base += wsum[i];
    total += wsum[i];
  }
  return base + inc - x;
}

// What an item asks of a step.
struct Want {
  int rows, m, kept, more, tail;              // rows kept and to come, their pages, the last kept page (-1: none)
  bool open;                                  // new rows go into the last kept page
};

// One workgroup, as each part of a plan needs the one before it: nine passes with a barrier between, over the
// table, the items and the pages.  Bound by their latency: 5.6 us for one item, 7.6 for 16 items that
// fork (a pool of 161 pages), 10.7 for 16 that take over others' rows (280 pages); grid-wide passes would
// be a launch each, 3.6 us.
template <bool LDS>
__global__ __launch_bounds__(kPlanThreads) void k_pstep(StepArgs a) {
  extern __shared__ int sm[];
  __shared__ int wsum[kPlanWaves], found;
  const int tid = threadIdx.x, R = 1 << a.shift;
  int *table = a.state, *holders_out = a.state + table_numbers(a.B, a.width);
  int *holders = LDS ? sm : a.ws.holders, *last = LDS ? sm + a.pages : a.ws.last;
  const int size = a.B * a.width;             // up to 2^28
  // (a capacity is up to 2^30 rows, so no sum here leaves 32 bits)
  auto want = [&](int b) {
    Want w;
    const int cap = a.width << a.shift;
    w.rows = min(max(a.len[b], 0), cap);
    if (a.src && (unsigned)a.src[b] >= (unsigned)a.B) w.rows = 0;
    w.m = min(a.n_new ? min(max(a.n_new[b], 0), a.n) : a.n, cap - w.rows);
    w.kept = (w.rows + R - 1) >> a.shift;
    w.more = ((w.rows + w.m + R - 1) >> a.shift) - w.kept;
    w.open = (w.rows & (R - 1)) && w.m > 0;
    w.tail = w.kept ? table[(long)b * a.width + w.kept - 1] : -1;   // (once the table is the new one)
    return w;
  };
  for (int p = tid; p < a.pages; p += kPlanThreads) holders[p] = 0, last[p] = -1;
  if (tid == 0) found = 0;
  // the rows kept, of the table as it was
  auto entry = [&](int x) {
    const int b = a.by_width(x), i = x - b * a.width, s = a.src ? a.src[b] : b;
    if ((unsigned)s >= (unsigned)a.B || i >= (min(max(a.len[b], 0), a.width << a.shift) + R - 1) >> a.shift) return -1;
    const int p = table[(long)s * a.width + i];
    return (unsigned)p < (unsigned)a.pages ? p : -1;
  };
  if (a.src) {
    for (int x = tid; x < size; x += kPlanThreads) a.ws.table[x] = entry(x);
    __syncthreads();
  }
  __syncthreads();
  for (int x = tid; x < size; x += kPlanThreads) {
    const int p = a.src ? a.ws.table[x] : entry(x);
    table[x] = p;
    if (p >= 0) atomicAdd(&holders[p], 1);
  }
  __syncthreads();
  // Pages that several entries hold and some items are about to write: holders - writers, 0 where all write,
  // and the last writer, which then keeps the page
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const Want w = want(b);
    if (w.open && w.tail >= 0) atomicMax(&last[w.tail], b), atomicSub(&holders[w.tail], 1);
  }
  __syncthreads();
  // pages needed, before each item
  int all = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int need = 0;
    bool copy = false;
    if (b < a.B) {
      const Want w = want(b);
      if (w.open && w.tail < 0) {
        need = 0;                                       // nothing to write in
      } else {
        copy = w.open && !(holders[w.tail] == 0 && last[w.tail] == b);
        need = w.more + copy;
      }
    }
    int total;
    const int before = plan_scan(need, wsum, total);
    if (b < a.B) a.ws.need[b] = (all + before) << 1 | copy;
    all += total;
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const Want w = want(b);
    if (w.open && w.tail >= 0) atomicAdd(&holders[w.tail], 1);
  }
  __syncthreads();
  // as many free pages as are needed, in order
  int got = 0;
  for (int p0 = 0; p0 < a.pages && got < all; p0 += kPlanThreads) {
    const int p = p0 + tid, is = p < a.pages && holders[p] == 0;
    int total;
    const int before = plan_scan(is, wsum, total);
    if (is && got + before < all) a.ws.free[got + before] = p;
    got = min(got + total, all);
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const Want w = want(b);
    const int off = a.ws.need[b] >> 1, copy = a.ws.need[b] & 1;
    const int need = w.open && w.tail < 0 ? 0 : w.more + copy, mine = min(max(got - off, 0), need);
    int give = 0;
    if (copy && mine) {
      const int to = a.ws.free[off];
      a.ws.move[atomicAdd(&found, 1)] = PageMove{w.tail, to, ((w.rows & (R - 1)) + kPTile - 1) / kPTile};
      table[(long)b * a.width + w.kept - 1] = to;
      atomicSub(&holders[w.tail], 1);
      atomicAdd(&holders[to], 1);
    }
    for (int i = 0; i < mine - copy; ++i) {
      const int p = a.ws.free[off + copy + i];
      table[(long)b * a.width + w.kept + i] = p;
      atomicAdd(&holders[p], 1);
    }
    if (!(w.open && w.tail < 0) && !(copy && !mine)) give = min(w.m, ((w.kept + mine - copy) << a.shift) - w.rows);
    a.granted[b] = give;
  }
  __syncthreads();
  // (a page whose copy found no free one has kept its holders, the last writer among them)
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const Want w = want(b);
    if (w.open && !(a.ws.need[b] & 1) && w.tail >= 0 && holders[w.tail] > 1) a.granted[b] = 0;
  }
  for (int p = tid; p < a.pages; p += kPlanThreads) holders_out[p] = holders[p];
  if (tid == 0) *a.ws.count = found;
}

struct CompactArgs {
  int32_t *state, *live;
  PlanWs ws;                                  // free: where the page of each number goes
  int B, width, pages, shift;
};

// As k_pstep: 3.9 us for a pool of 33 pages, 5.0 for 280.  Holders are counted anew here too (0.4 us of
// it), so that a page that the table names is never written over: what they were before may be older
// than the table.
template <bool LDS>
__global__ __launch_bounds__(kPlanThreads) void k_pcompact(CompactArgs a) {
  extern __shared__ int sm[];
  __shared__ int wsum[kPlanWaves];
  const int tid = threadIdx.x;
  int *table = a.state, *holders_out = a.state + table_numbers(a.B, a.width);
  int *holders = LDS ? sm : a.ws.holders;
  const int size = a.B * a.width;
  int mine = 0, L;
  for (int p = tid; p < a.pages; p += kPlanThreads) holders[p] = 0;
  __syncthreads();
  for (int x = tid; x < size; x += kPlanThreads) {
    const int p = table[x];
    if ((unsigned)p < (unsigned)a.pages) atomicAdd(&holders[p], 1);
  }
  __syncthreads();
  for (int p = tid; p < a.pages; p += kPlanThreads) mine += holders[p] > 0;
  plan_scan(mine, wsum, L);
  // both ends of the k-th move; as many live pages lie behind the end as free ones before it
  int low = 0, high = 0;
  for (int p0 = 0; p0 < a.pages; p0 += kPlanThreads) {
    const int p = p0 + tid;
    const bool in = p < a.pages, lives = in && holders[p] > 0;
    const int is = in && (p < L) != lives;    // a free page below L, or a live one from L on
    int total, before;
    const int lows = p0 < L ? min(L - p0, kPlanThreads) : 0;   // pages of this stretch below L
    before = plan_scan(is && p < L, wsum, total);
    if (is && p < L) a.ws.move[low + before].to = p;
    low += total;
    if (lows < kPlanThreads) {
      before = plan_scan(is && p >= L, wsum, total);
      if (is && p >= L) a.ws.move[high + before].from = p;
      high += total;
    }
  }
  __syncthreads();
  for (int i = tid; i < high; i += kPlanThreads) {
    const PageMove mv = a.ws.move[i];
    a.ws.move[i].tiles = (1 << a.shift) / kPTile;
    a.ws.free[mv.from] = mv.to;
    holders[mv.to] = holders[mv.from];
    holders[mv.from] = 0;
  }
  __syncthreads();
  // every page from L on that an entry names has moved
  for (int x = tid; x < size; x += kPlanThreads) {
    const int p = table[x];
    if (p >= L && p < a.pages) table[x] = a.ws.free[p];
  }
  for (int p = tid; p < a.pages; p += kPlanThreads) holders_out[p] = holders[p];
  if (tid == 0) {
    *a.ws.count = high;
    if (a.live) *a.live = L;
  }
}

constexpr int kMoveLayers = 64;               // of one launch
struct MoveArgs {
  uint16_t *pool[2 * kMoveLayers];            // each layer's keys, then its values
  const PageMove *move;
  const int *count;
  int pools, KV, tile;                        // elements of a tile
  int shift, chunk;                           // pieces of a head's page for one workgroup, in tiles
};

// The rows of a plan's moves, in every layer.  Rows lie together head by head, keys and values alike, so
// that a move is runs of memory, cut into chunks of 64 rows of a head.  How many there are is known on the
// device only: a fixed grid goes round them (2.3 us where there are none).  28 layers' copies for 16
// forks (61 MB): 9.0 us; 1.0 GB of a compaction: 199 us, 5.0 TB/s, a plain copy's rate.
__global__ __launch_bounds__(256) void k_pmove(MoveArgs a) {
  const int moves = *a.count;
  const int chunks = ((1 << a.shift) / kPTile + a.chunk - 1) / a.chunk;
  const long all = (long)moves * a.pools * a.KV * chunks;
  for (long x = blockIdx.x; x < all; x += gridDim.x) {
    const int c = (int)(x % chunks), h = (int)(x / chunks % a.KV);
    const int pool = (int)(x / chunks / a.KV % a.pools);
    const PageMove mv = a.move[x / chunks / a.KV / a.pools];
    const int t0 = c * a.chunk, t1 = min(t0 + a.chunk, mv.tiles);
    const long step = (long)a.tile << a.shift, per = step / kPTile;   // elements of a head's page
    u32x4 *to = reinterpret_cast<u32x4 *>(a.pool[pool] + ((long)mv.to * a.KV + h) * per + (long)t0 * a.tile);
    const u32x4 *from = reinterpret_cast<const u32x4 *>(a.pool[pool] + ((long)mv.from * a.KV + h) * per + (long)t0 * a.tile);
    const int n = (t1 - t0) * a.tile / 8;
    for (int i = threadIdx.x; i < n; i += 4 * 256) {
      u32x4 r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) r[u] = from[min(i + 256 * u, n - 1)];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + 256 * u < n) to[i + 256 * u] = r[u];
    }
  }
}

__global__ __launch_bounds__(256) void k_pinit(int32_t *state, long entries, long numbers, long all) {
  for (long x = blockIdx.x * 256L + threadIdx.x; x < all; x += gridDim.x * 256L) state[x] = x < entries ? -1 : 0;
}

// Floats of the workspace that a plan takes, and its parts.
long plan_numbers(long B, long width, long pages) { return 8 + B * width + B + 3 * std::max(B, pages) + 3 * pages; }
PlanWs plan_at(float *part, long B, long width, long pages) {
  int *at = reinterpret_cast<int *>(part);
  PlanWs w;
  w.count = at, at += 8;
  w.move = reinterpret_cast<PageMove *>(at), at += 3 * std::max(B, pages);
  w.table = at, at += B * width;
  w.need = at, at += B;
  w.free = at, at += pages;
  w.holders = at, at += pages;
  w.last = at;
  return w;
}

fc_status run_moves(fc_ctx *ctx, const fc_pcache *c, int n_layers, const PlanWs &ws, const char *what, hipStream_t st) {
  MoveArgs a{};
  a.move = ws.move, a.count = ws.count;
  a.KV = c->n_kv_heads, a.tile = kPTile * c->head_dim, a.shift = log2_of(c->page_rows), a.chunk = 8;
  for (int l0 = 0; l0 < n_layers; l0 += kMoveLayers) {
    const int layers = std::min(kMoveLayers, n_layers - l0);
    for (int l = 0; l < layers; ++l) a.pool[2 * l] = c[l0 + l].k, a.pool[2 * l + 1] = c[l0 + l].v;
    a.pools = 2 * layers;
    hipLaunchKernelGGL(k_pmove, dim3((unsigned)(8 * ctx->num_cus)), dim3(256), 0, st, a);
    FC_LAUNCH_OK(st, what);
  }
  return FC_OK;
}

}  // namespace

size_t pcache_state_bytes(long B, long width, long pages) {
  return (size_t)(table_numbers(B, width) + pages) * sizeof(int32_t);
}
long pcache_plan_numbers(long B, long width, long pages) { return plan_numbers(B, width, pages); }

fc_status launch_pcache_init(fc_ctx *ctx, const fc_pcache &c, int B, hipStream_t st) {
  const long entries = (long)B * c.max_pages, all = table_numbers(B, c.max_pages) + c.n_pages;
  ProfScope ps(ctx, st, "fc_pinit");
  hipLaunchKernelGGL(k_pinit, dim3((unsigned)std::min<long>((all + 255) / 256, 4096)), dim3(256), 0, st, c.state, entries, entries, all);
  FC_LAUNCH_OK(st, "k_pinit");
  return FC_OK;
}

fc_status launch_pcache_append(fc_ctx *ctx, const fc_pcache &c, const fc_rope_axes &rope,
                               const fc_qkv_rows &x, const int32_t *pos, const int32_t *len,
                               const int32_t *n_new, uint16_t *q_out, int B, int n, hipStream_t st) {
  PAppendArgs a{};
  a.q = x.q, a.k = x.k, a.v = x.v;
  a.q_row = x.q_row, a.k_row = x.k_row, a.v_row = x.v_row;
  a.q_item = x.q_item, a.k_item = x.k_item, a.v_item = x.v_item;
  a.pos = pos, a.len = len, a.n_new = n_new, a.pos_axis = (long)B * n;
  a.q_out = q_out, a.kc = c.k, a.vc = c.v;
  a.t = page_table(c);
  a.n = n, a.H = x.n_heads, a.KV = c.n_kv_heads, a.cap = c.max_pages * c.page_rows;
  const int half = c.head_dim / 2;
  const bool one = !(rope.section[0] || rope.section[1] || rope.section[2]);
  a.sec0 = one ? half : rope.section[0];
  a.sec1 = one ? half : rope.section[0] + rope.section[1];
  // two powers and products of them, as in launch_qcache_append
  const double r = std::pow(rope.theta, -2.0 / c.head_dim), r8 = std::pow(rope.theta, -16.0 / c.head_dim);
  a.lo[0] = 1.0 / (2.0 * M_PI), a.hi[0] = 1.0;
  for (int i = 1; i < 8; ++i) a.lo[i] = a.lo[i - 1] * r, a.hi[i] = a.hi[i - 1] * r8;
  // the new rows start inside a group, so one more may be touched than they fill
  const dim3 grid((unsigned)((n + 2 * kPTile - 2) / kPTile), (unsigned)B);
  ProfScope ps(ctx, st, "fc_pappend");
  if (c.head_dim == 128) hipLaunchKernelGGL(k_pappend<128>, grid, dim3(kPThreads), 0, st, a);
  else hipLaunchKernelGGL(k_pappend<64>, grid, dim3(kPThreads), 0, st, a);
  FC_LAUNCH_OK(st, "k_pappend");
  return FC_OK;
}

fc_status launch_pcache_step(fc_ctx *ctx, const fc_pcache *c, int n_layers, const int32_t *src,
                             const int32_t *len, const int32_t *n_new, int n, int32_t *granted, int B,
                             hipStream_t st) {
  StepArgs a{};
  a.state = c->state, a.src = src, a.len = len, a.n_new = n_new, a.granted = granted;
  a.ws = plan_at(ctx->part, B, c->max_pages, c->n_pages);
  a.B = B, a.width = c->max_pages, a.pages = c->n_pages, a.shift = log2_of(c->page_rows), a.n = n;
  a.by_width = quot_by(c->max_pages);
  {
    ProfScope ps(ctx, st, "fc_pstep");
    if (c->n_pages <= kPlanPages)
      hipLaunchKernelGGL(k_pstep<true>, dim3(1), dim3(kPlanThreads), 2 * c->n_pages * sizeof(int), st, a);
    else
      hipLaunchKernelGGL(k_pstep<false>, dim3(1), dim3(kPlanThreads), 0, st, a);
    FC_LAUNCH_OK(st, "k_pstep");
  }
  ProfScope ps(ctx, st, "fc_pstep_copy");
  return run_moves(ctx, c, n_layers, a.ws, "k_pmove", st);
}

fc_status launch_pcache_compact(fc_ctx *ctx, const fc_pcache *c, int n_layers, int32_t *live, int B, hipStream_t st) {
  CompactArgs a{};
  a.state = c->state, a.live = live;
  a.ws = plan_at(ctx->part, B, c->max_pages, c->n_pages);
  a.B = B, a.width = c->max_pages, a.pages = c->n_pages, a.shift = log2_of(c->page_rows);
  {
    ProfScope ps(ctx, st, "fc_pcompact");
    if (c->n_pages <= kPlanPages)
      hipLaunchKernelGGL(k_pcompact<true>, dim3(1), dim3(kPlanThreads), c->n_pages * sizeof(int), st, a);
    else
      hipLaunchKernelGGL(k_pcompact<false>, dim3(1), dim3(kPlanThreads), 0, st, a);
    FC_LAUNCH_OK(st, "k_pcompact");
  }
  ProfScope ps(ctx, st, "fc_pcompact_move");
  return run_moves(ctx, c, n_layers, a.ws, "k_pmove", st);
}

}  // namespace fc
