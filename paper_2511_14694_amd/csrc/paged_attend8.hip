// Attention of the newest tokens of every sequence over a paged cache of 8 bits
// (focus_paged_attend8).
//
//   attend8_attend  one workgroup per (chunk of a sequence's rows, one to four KV heads, up
//                   to 16 columns of each: a column is a new token and a query head); writes
//                   o and lse where the chunk is the whole sequence, else an unnormalised
//                   partial (running max, sum, output)
//   attend8_join    merges the partials of a sequence's chunks by log-sum-exp
//   attend8_plan    before both for more than 128 sequences: the chunks
//
// Every cached byte is read once for up to 16 columns.  A wave takes 32 rows at a time; each
// lane's loads become operands of bf16 matrix products as they arrive, without LDS (e4m3
// numbers are bf16 numbers, so nothing is rounded):
//     S^T = K Q^T     row m of product t is cached row 8 (m / 4) + 4 t + m % 4, so lane
//                     (column q = lane % 16, group x = lane / 16) gets the scores of
//                     rows 8 x .. 8 x + 7 of column q
//     O^T += V^T P^T  contraction index 8 x + j is row 8 x + j: the lane's own weights;
//                     lane i of group x loaded elements D/16 i .. of rows 8 x .. 8 x + 7,
//                     of which product t takes element D/16 i + t
// so maximum, sum and rescaling of a column stay in its lanes.  The eight rows of a lane lie
// in one block, whose scales it multiplies its scores and weights with.
#include "paged_split.h"

#include <algorithm>
#include <type_traits>

namespace {

using focus::bf16x8;
using focus::f32x4;
using focus::kMinit;
using focus::u32x4;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kMaxGrid = focus::kSplitGrid;
constexpr int kCols = 16;       // columns of a workgroup
constexpr int kPages = 1024;    // pages held in LDS at a time
constexpr int kWhole = 256;     // rows of a table that is not split
constexpr int kUnit = 128;      // rows of a chunk times KV heads of a workgroup: a multiple of this
constexpr int kRows = 32;       // rows of a wave at a time
constexpr int kMost = 512;      // columns of a KV head
// Rows that a chunk's beginning and end cost (focus::Split::each), twice those of a bf16 cache.
constexpr int kStart = 144;

// What a lane reads in the place of eight rows that begin past their sequence's end or
// lie in a page outside the pool.
__device__ __align__(16) const uint32_t kZeros[64] = {};

// Workspace: int4 info[batch]; for more than focus::kWave sequences int owner[slots]; then the
// partials of `slots` chunks: float2 ml[slots][columns], float o[slots][columns][D].
struct Plan {
  int64_t slots, target, cap;
  int64_t owner, ml, o; // byte offsets
  size_t bytes;
  int tiles;            // workgroups a KV head's columns take
  int wide, unit;       // KV heads of a workgroup; chunks are multiples of `unit` rows
  int64_t groups;       // workgroups of a chunk
  int columns;          // of all heads
  bool single, planned;
};

// Workgroups of attend8_attend that a compute unit holds (by their registers).
constexpr int resident(int head_dim) { return head_dim == 64 ? 4 : 2; }

Plan make_plan(const focus_paged_attend8_desc* d) {
  const focus_paged_kv& c = d->cache.kv;
  Plan p = {};
  p.cap = (int64_t)c.max_pages * c.page_rows;
  const int per_head = d->n_heads / c.n_kv_heads * d->max_rows;
  p.columns = per_head * c.n_kv_heads;
  p.tiles = (int)focus::ceil_div(per_head, kCols);
  // neighbouring heads' rows read together, where they lie side by side
  p.wide = c.head_stride > c.row_stride ? 1 : c.n_kv_heads % 4 == 0 ? 4 : c.n_kv_heads % 2 == 0 ? 2 : 1;
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads * p.tiles;
  p.single = d->split_keys == 0 && (p.cap <= kWhole || (p.cap <= 2 * kWhole && heads >= 128));
  if (p.single && heads <= 1024) p.wide = 1;
  p.planned = !p.single && c.batch > focus::kWave;
  p.unit = kUnit / p.wide;
  p.groups = (int64_t)c.n_kv_heads / p.wide * p.tiles;
  if (p.single) {
    p.slots = c.batch;
  } else if (d->split_keys > 0) {
    p.slots = c.batch * std::max<int64_t>(1, focus::ceil_div(p.cap, d->split_keys));
  } else {
    p.target = std::max<int64_t>(1, resident(c.head_dim) * focus::device_cus() / p.groups);
    // a chunk has at least half of the rows of the batch over the target; a sequence at
    // least one
    p.slots = std::min(c.batch + 2 * p.target, c.batch * std::max<int64_t>(1, focus::ceil_div(p.cap, p.unit)));
  }
  const int64_t partials = p.slots * p.columns;
  p.owner = 16 * (int64_t)c.batch;
  p.ml = p.owner + (p.planned ? focus::ceil_div(4 * p.slots, 16) * 16 : 0);
  p.o = p.ml + focus::ceil_div(8 * partials, 16) * 16;
  p.bytes = p.single ? 0 : (size_t)(p.o + 4 * partials * c.head_dim);
  return p;
}

struct Args {
  focus_paged_attend8_desc d;
  focus::Split split;
  float sc;             // softmax scale in log2 units
  int shift, scale_shift;  // log2 page_rows, scale_rows
  int tiles, wide_shift;
  int units;            // workgroups of a chunk and 16 columns each
  int group;            // query heads of a KV head
  int per_head, columns;   // columns of a KV head at most, of all heads
  int parts;            // workgroups of a KV head in attend8_join
  float2* ml;
  float* o;
};

// The rows of q of sequence b: [first, first + count); count -1 if they are not to be touched.
struct Tokens {
  int64_t first;
  int count;
};
__device__ inline Tokens tokens_of(const Args& a, int b, int32_t& bits) {
  if (!a.d.cu_rows) return {b, 1};
  const int r0 = a.d.cu_rows[b], r1 = a.d.cu_rows[b + 1];
  if (r0 < 0 || r1 < r0 || r1 > a.d.n_rows) {
    bits |= FOCUS_ERR_BOUNDS;
    return {0, -1};
  }
  if (r1 - r0 > a.d.max_rows) {
    bits |= FOCUS_ERR_CAPACITY;
    return {0, -1};
  }
  return {r0, r1 - r0};
}

__global__ __launch_bounds__(focus::kPlan) void attend8_plan(Args a) { focus::plan_chunks(a.split, a.d.cache.kv); }

// Eight e4m3 numbers in bf16; a pair of them.
__device__ inline uint32_t widen(uint32_t w, bool high) {
  const bf16x2 r = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, false);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ inline bf16x8 widen8(uint32_t w0, uint32_t w1) {
  const u32x4 r = {widen(w0, false), widen(w0, true), widen(w1, false), widen(w1, true)};
  return __builtin_bit_cast(bf16x8, r);
}

// Load from global memory, past the caches unless other workgroups read the same rows.
template <typename V, bool SHARED>
__device__ __forceinline__ V load_row(const void* p) {
  const auto* from = reinterpret_cast<const __attribute__((address_space(1))) V*>(reinterpret_cast<uintptr_t>(p));
  if constexpr (SHARED) return *from;
  else return __builtin_nontemporal_load(from);
}

template <int D> struct Tile {
  static constexpr int kPer = D / 16;               // elements of a V row a lane holds
  static constexpr int kWords = kPer / 4;
  static constexpr int kPieces = D / 64;            // 16-byte pieces of a K row a lane holds
  using V = typename std::conditional<kWords == 2, u32x2, uint32_t>::type;
  u32x4 k[2][kPieces];
  V v[8];
  float ks, vs;         // the scales of the rows of the lane's scores
  __device__ uint32_t word(int j, int i) const {
    if constexpr (kWords == 2) return v[j][i];
    else return v[j];
  }
};

// Bytes of w that are NaN (0x7f or 0xff) as 1, others 0; and w with zeros in their place.
__device__ inline uint32_t nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

// SHARED: a KV head has more than 16 columns, whose workgroups read the same rows.
// T: of q and o.  float32 queries enter in three bf16 parts, weights in two (17 bits; their
// rounding is far below that of a bf16 output) or, for float32 outputs, three.
template <typename T, int D, bool SHARED>
__global__ __launch_bounds__(kThreads, resident(D)) void attend8_attend(Args a) {
  using L = Tile<D>;
  constexpr int kPitch = D + 4, kSteps = D / 32;
  constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kWeightParts = sizeof(T) == 2 ? 2 : 3;
  __shared__ int64_t s_page[kPages + 1];  // (a chunk may begin inside a page)
  __shared__ int s_id[kPages + 1];
  __shared__ float s_o[kWaves][kCols][kPitch];
  __shared__ float2 s_ml[kWaves][kCols];
  const focus_paged_kv& c = a.d.cache.kv;
  const int H = a.d.n_heads, G = a.group;
  // (a wave's number in a scalar register: its loops are branches then, not masks)
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int lane = tid % 64, col = lane % 16, x = lane / 16;
  int slot_id = blockIdx.z * kMaxGrid + blockIdx.y, tile_id = 0, g0 = blockIdx.x;
  if constexpr (SHARED) {
    // Workgroups are dealt over the XCDs in turn: those that read the same rows to one XCD,
    // one after another, so that its L2 reads them once.
    const int id = blockIdx.x, among = id % (focus::kXcds * a.tiles);
    const int unit = id / (focus::kXcds * a.tiles) * focus::kXcds + among % focus::kXcds;
    tile_id = among / focus::kXcds;
    slot_id = unit / a.units;
    g0 = unit % a.units;
  }
  g0 <<= a.wide_shift;
  // waves of a KV head; this wave's head, and which of its waves it is
  const int by = kWaves >> a.wide_shift, at_head = wave >> (2 - a.wide_shift), g = g0 + at_head, among = wave & (by - 1);
  const focus::Chunk ch = focus::find_chunk(a.split, c, slot_id);
  if (ch.chunks == 0) return;
  const int b = ch.b, r0 = ch.c * ch.rows, r1 = min(ch.n, r0 + ch.rows);
  const bool first = g0 == 0 && tile_id == 0;
  int32_t bits = 0;
  const Tokens tok = tokens_of(a, b, bits);
  if (first && ch.c == 0 && tid == 0) {
    if (a.split.info && !a.split.owner) a.split.info[b] = make_int4(ch.slot0, ch.chunks, ch.n, ch.rows);
    if (ch.n != c.length[b]) bits |= FOCUS_ERR_CAPACITY;
    if (bits) focus::raise_err(a.d.err, bits);
  }
  // columns of this workgroup; this lane's: token and head of the KV head, and the rows it sees
  const int cols = min(kCols, tok.count * G - tile_id * kCols);
  if (cols <= 0) return;
  const int cc = tile_id * kCols + min(col, cols - 1), token = cc / G, head = cc - token * G;
  const int sees = max(0, ch.n - (tok.count - 1 - token)), sees_all = max(0, ch.n - (tok.count - 1));

  bf16x8 q[kParts][kSteps];  // column col, elements as the K rows' pieces
  {
    const T* src = reinterpret_cast<const T*>(a.d.q) + (tok.first + token) * a.d.q_row + (int64_t)(g * G + head) * a.d.q_head;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int e = (i / 2 * 4 + x) * 16 + i % 2 * 8;
      if constexpr (sizeof(T) == 2) {
        q[0][i] = *reinterpret_cast<const bf16x8*>(src + e);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float f = src[e + k];
#pragma unroll
          for (int part = 0; part < kParts; ++part) {
            q[part][i][k] = (__bf16)f;
            f -= (float)q[part][i][k];
          }
        }
      }
    }
  }

  const uint8_t* kbase = reinterpret_cast<const uint8_t*>(c.k) + (int64_t)g * c.head_stride;
  const uint8_t* vbase = reinterpret_cast<const uint8_t*>(c.v) + (int64_t)g * c.head_stride;
  const uint8_t* zeros = reinterpret_cast<const uint8_t*>(kZeros);
  const int per_page = c.page_rows >> a.scale_shift;            // blocks of a page
  const uint32_t page_scales = (uint32_t)(c.n_kv_heads * per_page);
  const float* ks_base = a.d.cache.k_scale + g * per_page;
  const float* vs_base = a.d.cache.v_scale + g * per_page;
  const int mask = c.page_rows - 1;
  // rows of eight from which this lane reads K and V; the offset of its K row in them
  const int k8 = col / 4 * 8, k_in = col % 4, v8 = x * 8;

  float m = kMinit, l = 0.f;
  f32x4 o[L::kPer];
#pragma unroll
  for (int t = 0; t < L::kPer; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int seg = r0; seg < r1; seg += kPages << a.shift) {
    const int seg_end = min(r1, seg + (kPages << a.shift)), page0 = seg >> a.shift;
    __syncthreads();
    for (int i = tid; i + page0 <= (seg_end - 1) >> a.shift; i += kThreads) {
      const int64_t p = focus::page_of(c, b, (i + page0) << a.shift, a.shift);
      if (p < 0 && first) focus::raise_err(a.d.err, FOCUS_ERR_BOUNDS);
      s_page[i] = p < 0 ? -1 : p * c.page_stride;
      s_id[i] = (int)p;
    }
    __syncthreads();
    // tiles that are whole and seen by all columns end here
    const int clean = max(seg, min(seg_end, sees_all));
    const int full_end = clean - (clean - seg) % kRows;
    // offset of the page that holds the eight rows at r (negative: none, or past end)
    auto page = [&](int r, int end) { return r < end ? s_page[(r >> a.shift) - page0] : -1; };
    // Rows of eight lie in one page, so all of them can be read where the first is cached.
    auto load = [&](L& w, int r, int end) {
      const int64_t pk = page(r + k8, end), pv = page(r + v8, end);
      const uint32_t step = (uint32_t)c.row_stride;
      const uint64_t ks = pk >= 0 ? step : 0, vs = pv >= 0 ? step : 0;
      const uint8_t* kp = (pk >= 0 ? kbase + pk + (uint64_t)(uint32_t)((r + k8) & mask) * step : zeros) + k_in * ks + x * 16;
      const uint8_t* vp = (pv >= 0 ? vbase + pv + (uint64_t)(uint32_t)((r + v8) & mask) * step : zeros) + col * L::kPer;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < L::kPieces; ++i) w.k[t][i] = load_row<u32x4, SHARED>(kp + 4 * t * ks + i * 64);
#pragma unroll
      for (int j = 0; j < 8; ++j) w.v[j] = load_row<typename L::V, SHARED>(vp + j * vs);
      const uint64_t at = pv >= 0 ? (uint64_t)(uint32_t)s_id[((r + v8) >> a.shift) - page0] * page_scales +
                                        (uint32_t)(((r + v8) & mask) >> a.scale_shift)
                                  : 0;
      const float* kz = reinterpret_cast<const float*>(kZeros);
      w.ks = *(pv >= 0 ? ks_base + at : kz);
      w.vs = *(pv >= 0 ? vs_base + at : kz);
    };
    auto compute = [&](L& w, int r, auto whole) {
      constexpr bool kWholeTile = decltype(whole)::value;
      f32x4 s[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const bf16x8 k = widen8(w.k[t][i / 2][i % 2 * 2], w.k[t][i / 2][i % 2 * 2 + 1]);
#pragma unroll
          for (int part = kParts - 1; part >= 0; --part)
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[part][i], s[t], 0, 0, 0);
        }
      }
      const int row = r + v8;  // of the lane's first score
      // of the lane's rows, those that count: the first `live`
      int live = page(row, seg_end) >= 0 ? 8 : 0;
      uint32_t bad = 0;
      if constexpr (!kWholeTile) {
        // Rows past the end may hold anything, and those that only later tokens see a NaN,
        // and zero times a NaN is a NaN: the first are cleared, the NaN of the others
        // taken out and put into the sums of the columns that see them.
        const int in = min(live, seg_end - row);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (j >= in) w.v[j] = typename L::V{};
#pragma unroll
          for (int i = 0; i < L::kWords; ++i) bad |= nan_bytes(w.word(j, i));
        }
        live = min(live, min(seg_end, sees) - row);
      }
      float y[8], mx = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = j < live ? s[j / 4][j % 4] * w.ks : -INFINITY;
        mx = fmaxf(mx, y[j]);
      }
      mx = focus::max_column(mx);
      // (scaled after the difference: scaled before, a score of 4096 would be rounded to
      // 2^-12, and so would the weight)
      const float alpha = __builtin_amdgcn_exp2f((m - mx) * a.sc);
      m = mx;
      l *= alpha;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = __builtin_amdgcn_exp2f((y[j] - m) * a.sc);
        l += y[j];
        y[j] = kWholeTile || j < live ? y[j] * w.vs : 0.f;
      }
#pragma unroll
      for (int t = 0; t < L::kPer; ++t) o[t] *= alpha;
      if constexpr (!kWholeTile) {
        if (__ballot(bad != 0)) {
          bf16x8 seen;
#pragma unroll
          for (int j = 0; j < 8; ++j) seen[j] = (__bf16)(j < live ? 1.f : 0.f);
#pragma unroll
          for (int t = 0; t < L::kPer; ++t) {
            bf16x8 mark;
#pragma unroll
            for (int j = 0; j < 8; ++j)
              mark[j] = (__bf16)(nan_bytes(w.word(j, t / 4)) >> (t % 4 * 8) & 1 ? 1.f : 0.f);
            const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mark, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (n[e] != 0.f) o[t][e] = NAN;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < L::kWords; ++i) {
              const uint32_t keep = ~(nan_bytes(w.word(j, i)) * 0xffu);
              if constexpr (L::kWords == 2) w.v[j][i] &= keep;
              else w.v[j] &= keep;
            }
        }
      }
      // product t's rows of V^T: pairs of rows by a byte permutation, then widened
      u32x4 z[L::kPer];
#pragma unroll
      for (int i = 0; i < L::kWords; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo = __builtin_amdgcn_perm(w.word(2 * e + 1, i), w.word(2 * e, i), 0x05010400);
          const uint32_t hi = __builtin_amdgcn_perm(w.word(2 * e + 1, i), w.word(2 * e, i), 0x07030602);
          z[4 * i][e] = widen(lo, false), z[4 * i + 1][e] = widen(lo, true);
          z[4 * i + 2][e] = widen(hi, false), z[4 * i + 3][e] = widen(hi, true);
        }
#pragma unroll
      for (int part = 0; part < kWeightParts; ++part) {
        bf16x8 p;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          p[j] = (__bf16)y[j];
          y[j] -= (float)p[j];
        }
#pragma unroll
        for (int t = 0; t < L::kPer; ++t)
          o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, z[t]), p, o[t], 0, 0, 0);
      }
    };
    // A wave's whole tiles, two a round, the next one's loads in flight while one is
    // computed; then the tiles that the chunk ends in or that not all columns see.  One way
    // out of the loop, loads past the end taken from kZeros and the last of them waited for
    // behind it: otherwise the compiler cannot tell which loads are in flight at a round's
    // start and waits for half of them.
    const int stride = by * kRows;
    int r = seg + among * kRows;
    if (r < full_end) {
      L w0, w1;
      load(w0, r, full_end);
      for (; r + stride < full_end; r += 2 * stride) {
        load(w1, r + stride, full_end);
        compute(w0, r, std::true_type{});
        load(w0, r + 2 * stride, full_end);
        compute(w1, r + stride, std::true_type{});
      }
      if (r < full_end) {
        compute(w0, r, std::true_type{});
        r += stride;
      }
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    }
    for (; r < seg_end; r += stride) {
      L w;
      load(w, r, seg_end);
      compute(w, r, std::false_type{});
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int t = 0; t < L::kPer; t += 4)
      *reinterpret_cast<float4*>(&s_o[wave][col][(x * 4 + e) * L::kPer + t]) =
          make_float4(o[t][e], o[t + 1][e], o[t + 2][e], o[t + 3][e]);
  // the waves' parts of each column, joined
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (x == 0) s_ml[wave][col] = make_float2(m, l);
  __syncthreads();
  constexpr int kLanes = D / 4;  // threads of a column, four elements each
  const int e = tid % kLanes * 4;
  for (int h = tid / kLanes, w0 = 0; w0 < kWaves; h += kThreads / kLanes) {
    while (h >= cols && w0 < kWaves) h -= cols, w0 += by;
    if (w0 >= kWaves) break;
    float2 ml = s_ml[w0][h];
    f32x4 y = *reinterpret_cast<const f32x4*>(&s_o[w0][h][e]);
    for (int w = w0 + 1; w < w0 + by; ++w) {
      const float2 other = s_ml[w][h];
      const float M = fmaxf(ml.x, other.x);
      const float f = __builtin_amdgcn_exp2f((ml.x - M) * a.sc), f2 = __builtin_amdgcn_exp2f((other.x - M) * a.sc);
      ml = make_float2(M, fmaf(ml.y, f, other.y * f2));
      y = y * f + *reinterpret_cast<const f32x4*>(&s_o[w][h][e]) * f2;
    }
    const int kv = g0 + (w0 >> (2 - a.wide_shift)), at_col = tile_id * kCols + h;
    if (ch.chunks == 1) {
      const int i = at_col / G;
      const int64_t at = (tok.first + i) * H + kv * G + (at_col - i * G);
      y = ml.y == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : y * (1.f / ml.y);
      T* to = reinterpret_cast<T*>(a.d.o) + at * D + e;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x2*>(to) = u32x2{focus::pack_bf16x2(y[0], y[1]), focus::pack_bf16x2(y[2], y[3])};
      else *reinterpret_cast<f32x4*>(to) = y;
      if (e == 0 && a.d.lse) a.d.lse[at] = focus::lse_of(a.sc, ml);
    } else {
      const int64_t slot = (int64_t)(ch.slot0 + ch.c) * a.columns + kv * a.per_head + at_col;
      *reinterpret_cast<f32x4*>(a.o + slot * D + e) = y;
      if (e == 0) a.ml[slot] = ml;
    }
  }
}

// One of `parts` workgroups of a (sequence, KV head): merges the partials of every parts-th
// of its columns (D / 4 threads over the output, the other groups of them over the chunks).
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void attend8_join(Args a) {
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes, kFlight = 8;
  __shared__ float4 s_o[kGroups][kLanes];
  __shared__ float2 s_ml;
  const focus_paged_kv& c = a.d.cache.kv;
  const int H = a.d.n_heads, G = a.group, tid = threadIdx.x, parts = a.parts, g = blockIdx.x;
  const int part = c.batch <= kMaxGrid ? blockIdx.z : blockIdx.z % parts;
  const int b = blockIdx.y + (c.batch <= kMaxGrid ? 0 : blockIdx.z / parts * kMaxGrid);
  if (b >= c.batch) return;
  const int4 info = a.split.info[b];
  if (info.y <= 1) return;
  int32_t bits = 0;
  const Tokens tok = tokens_of(a, b, bits);
  const int e = tid % kLanes, grp = tid / kLanes;
  const float4* o = reinterpret_cast<const float4*>(a.o);
  for (int cc = part; cc < tok.count * G; cc += parts) {
    const int column = g * a.per_head + cc;
    if (tid < 64) {
      const float2 ml = focus::joined(a.ml, a.sc, info, a.columns, column);
      if (tid == 0) s_ml = ml;
    }
    __syncthreads();
    const float2 ml = s_ml;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = grp; i0 < info.y; i0 += kGroups * kFlight) {
      float4 y[kFlight];
      float m[kFlight];
#pragma unroll
      for (int k = 0; k < kFlight; ++k) {
        const int64_t slot = (int64_t)(info.x + min(i0 + k * kGroups, info.y - 1)) * a.columns + column;
        y[k] = o[slot * kLanes + e];
        m[k] = a.ml[slot].x;
      }
#pragma unroll
      for (int k = 0; k < kFlight; ++k) {
        if (i0 + k * kGroups < info.y) {
          const float f = __builtin_amdgcn_exp2f((m[k] - ml.x) * a.sc);
          sum.x = fmaf(y[k].x, f, sum.x), sum.y = fmaf(y[k].y, f, sum.y);
          sum.z = fmaf(y[k].z, f, sum.z), sum.w = fmaf(y[k].w, f, sum.w);
        }
      }
    }
    s_o[grp][e] = sum;
    __syncthreads();
    if (tid < D) {
      float z = 0.f;
#pragma unroll
      for (int k = 0; k < kGroups; ++k) z += reinterpret_cast<const float*>(s_o[k])[tid];
      const int i = cc / G;
      const int64_t at = (tok.first + i) * H + g * G + (cc - i * G);
      reinterpret_cast<T*>(a.d.o)[at * D + tid] = (T)(ml.y == 0.f ? 0.f : z / ml.y);
      if (tid == 0 && a.d.lse) a.d.lse[at] = focus::lse_of(a.sc, ml);
    }
    __syncthreads();
  }
}

focus_status validate(const focus_paged_attend8_desc* d) {
  const focus_paged_kv& c = d->cache.kv;
  const focus_status st = focus::check_paged8(d->cache);
  if (st != FOCUS_OK) return st;
  const int64_t es = focus::elt_bytes(d->dtype);
  if (es == 0) return FOCUS_E_DTYPE;
  if (c.head_dim != 64 && c.head_dim != 128) return FOCUS_E_UNSUPPORTED;
  if (d->n_heads <= 0 || d->max_rows <= 0 || d->n_rows < 0 || d->split_keys < 0 || d->split_keys % kUnit ||
      !(d->softmax_scale == d->softmax_scale))
    return FOCUS_E_ARG;
  if (d->n_heads % c.n_kv_heads) return FOCUS_E_SHAPE;
  if ((int64_t)(d->n_heads / c.n_kv_heads) * d->max_rows > kMost || d->n_rows > INT32_MAX ||
      (!d->cu_rows && d->n_rows != c.batch))
    return FOCUS_E_SHAPE;
  if ((int64_t)c.batch * d->n_heads * d->max_rows > INT32_MAX / kThreads) return FOCUS_E_SHAPE;
  // (chunks are counted in 32 bits, in units of 32 rows at least)
  if ((int64_t)c.batch * focus::ceil_div((int64_t)c.max_pages * c.page_rows, 32) > INT32_MAX) return FOCUS_E_SHAPE;
  if (d->q_row < 0 || d->q_head < 0 || !focus::pieces16(d->q_row, es) || !focus::pieces16(d->q_head, es))
    return FOCUS_E_ARG;
  return FOCUS_OK;
}

template <typename T, int D>
focus_status launch(Args a, const Plan& p, hipStream_t s) {
  const focus_paged_kv& c = a.d.cache.kv;
  // workgroups of a (sequence, KV head) in the second launch: one per column, but not many
  // more than the device holds
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads;
  a.parts = (int)std::min<int64_t>(focus::ceil_div(8 * focus::device_cus(), heads), a.per_head);
  const int64_t slots = focus::ceil_div(p.slots, kMaxGrid), batches = focus::ceil_div(c.batch, kMaxGrid);
  if (p.groups * p.slots > INT32_MAX / kThreads - focus::kXcds * kMost || heads * a.parts > INT32_MAX / kThreads ||
      slots > kMaxGrid || batches * a.parts > kMaxGrid)
    return FOCUS_E_SHAPE;
  if (p.planned) {
    hipLaunchKernelGGL(attend8_plan, dim3(1), dim3(focus::kPlan), 0, s, a);
    const focus_status st = focus::launch_status();
    if (st != FOCUS_OK) return st;
  }
  const dim3 grid = p.tiles > 1 ? dim3((uint32_t)(focus::ceil_div(a.units * p.slots, focus::kXcds) * focus::kXcds * p.tiles))
                                : dim3((uint32_t)p.groups, (uint32_t)std::min<int64_t>(p.slots, kMaxGrid), (uint32_t)slots);
  if (p.tiles > 1) hipLaunchKernelGGL((attend8_attend<T, D, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((attend8_attend<T, D, false>), grid, dim3(kThreads), 0, s, a);
  const focus_status st = focus::launch_status();
  if (st != FOCUS_OK || p.single) return st;
  hipLaunchKernelGGL((attend8_join<T, D>),
                     dim3((uint32_t)c.n_kv_heads, (uint32_t)std::min(c.batch, kMaxGrid), (uint32_t)(batches * a.parts)),
                     dim3(kThreads), 0, s, a);
  return focus::launch_status();
}

}  // namespace

extern "C" size_t focus_paged_attend8_workspace(const focus_paged_attend8_desc* d) {
  if (!d || validate(d) != FOCUS_OK) return 0;
  return make_plan(d).bytes;
}

extern "C" focus_status focus_paged_attend8(const focus_paged_attend8_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  const focus_status st = validate(d);
  if (st != FOCUS_OK) return st;
  const focus_paged_kv& c = d->cache.kv;
  if (c.batch == 0 || d->n_rows == 0) return FOCUS_OK;
  if (!d->q || !d->o) return FOCUS_E_NULL;
  if (!focus::aligned16(d->q) || !focus::aligned16(d->o)) return FOCUS_E_ARG;
  for (const void* p : {(const void*)d->lse, (const void*)d->cu_rows, (const void*)d->err})
    if (reinterpret_cast<uintptr_t>(p) & 3u) return FOCUS_E_ARG;
  const Plan p = make_plan(d);
  if (p.bytes > 0 && (!d->workspace || d->workspace_bytes < p.bytes)) return FOCUS_E_WORKSPACE;
  if (!focus::aligned16(d->workspace)) return FOCUS_E_ARG;
  char* ws = reinterpret_cast<char*>(d->workspace);
  Args a = {};
  a.d = *d;
  a.shift = focus::page_shift(c), a.scale_shift = __builtin_ctz((unsigned)d->cache.scale_rows);
  a.tiles = p.tiles, a.wide_shift = __builtin_ctz((unsigned)p.wide), a.units = (int)(p.groups / p.tiles);
  a.group = d->n_heads / c.n_kv_heads, a.per_head = a.group * d->max_rows, a.columns = p.columns;
  focus::Split& s = a.split;
  s.split_keys = d->split_keys, s.unit_shift = __builtin_ctz((unsigned)p.unit), s.target = (int)p.target;
  s.each = (float)(kStart >> a.wide_shift) + 8.f * a.per_head;
  s.cap = p.cap, s.single = p.single, s.slots = p.slots;
  if (p.bytes > 0) {
    s.info = reinterpret_cast<int4*>(ws), a.ml = reinterpret_cast<float2*>(ws + p.ml);
    a.o = reinterpret_cast<float*>(ws + p.o);
  }
  if (p.planned) s.owner = reinterpret_cast<int*>(ws + p.owner);
  const float scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / sqrtf((float)c.head_dim);
  a.sc = scale * focus::kLog2e;
  hipStream_t on = reinterpret_cast<hipStream_t>(stream);
  if (d->dtype == FOCUS_BF16) return c.head_dim == 128 ? launch<__bf16, 128>(a, p, on) : launch<__bf16, 64>(a, p, on);
  return c.head_dim == 128 ? launch<float, 128>(a, p, on) : launch<float, 64>(a, p, on);
}
