// Attention of one new token over a paged K/V cache (focus_paged_decode).
//
//   paged_attend   one workgroup per (chunk of a sequence's rows, one to four KV heads, up
//                  to 16 query heads of each); writes o and lse where the chunk is the whole
//                  sequence, else an unnormalised partial (running max, sum, output)
//   paged_join     merges the partials of a sequence's chunks by log-sum-exp and, where
//                  weights are accumulated, turns the scores that paged_attend stored into
//                  weights of every row
//   paged_plan     before both for more than 128 sequences: the chunks' size and the sequence
//                  of each; of up to 128, a wave of paged_attend finds its chunk by itself
//
// Every cached byte is read once, for all query heads of its KV head, so the kernel is
// HBM bound as long as the products keep up: they run on the matrix cores at every
// group size (a group of one wastes 15 of 16 columns and still needs a tenth of the
// time its bytes take).  No operand goes through LDS: the products are arranged so that
// each lane's loads are operands as they arrive.  For bf16, a wave takes 32 rows:
//     S^T = K Q^T     row m of product t is cached row 8 (m / 4) + 4 t + m % 4, so lane
//                     (column q = lane % 16, group x = lane / 16) gets the scores of
//                     rows 8 x .. 8 x + 7 of query q
//     O^T += V^T P^T  contraction index 8 x + j is row 8 x + j: the lane's own weights;
//                     lane i of group x loaded elements D/16 i .. of rows 8 x .. 8 x + 7
//                     (whole rows, 16 lanes each), of which product t takes element
//                     D/16 i + t, one byte permutation per register
// so maximum, sum and rescaling of a query stay in the lanes of its column.  float32
// takes 16 rows a tile on the 16x16x4 products, which need no permutation at all.
//
// 16 sequences of 10 000 rows of 32 heads of 128 (bf16, 2.62 GB) take 403 us, 6.5 TB/s; one
// of 262 144 rows of 8 heads (1.07 GB) 170, 6.3 TB/s; 16 of 5 000 rows of 32 heads of 128 in
// float32 (2.62 GB) 458, 5.7 TB/s.  Where there is less to read the start
// and the second launch count: 64 sequences of 1 to 8 192 rows of 8 heads (0.26 GB), with
// weights, 71 us, of which 61 in paged_attend and 10 in paged_join.  The first form, one
// workgroup a (sequence, head) on the vector units, took 2754, 62 241 and 2061.
#include "paged.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace {

using focus::bf16x8;
using focus::f32x4;
using focus::u32x4;
using focus::wave_max;
using focus::wave_scan;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kMinit = -3.40282347e38f; // the least finite score still counts
constexpr int kThreads = 256, kWaves = 4;
constexpr int kMaxGrid = 32768; // workgroups in a grid's second and third dimension
constexpr int kCols = 16;       // query heads of a workgroup: columns of a product
constexpr int kPages = 1024;    // page offsets held in LDS at a time
constexpr int kWhole = 256;     // rows of a table that is not split
constexpr int kWave = 128;      // sequences whose lengths a wave holds, two a lane
constexpr int kPlan = 1024;     // threads of paged_plan
constexpr int kUnit = 128;      // rows of a chunk times KV heads of a workgroup: a multiple of this

// What a lane reads in the place of eight rows that begin past their sequence's end or
// lie in a page outside the pool.
__device__ __align__(16) const uint32_t kZeros[256] = {};

// Workspace: int4 info[batch] {first slot, chunks, rows, rows of a chunk}; for more than
// kWave sequences int owner[slots]; then the partials of `slots` chunks: float2
// ml[slots][H], float o[slots][H][D]; then, where weights are accumulated, float
// score[batch][H][cap] (unscaled).  None where nothing is handed on.
struct Plan {
  int64_t slots;        // upper bound of the chunks of all sequences
  int64_t target;       // chunks resident at a time (split_keys 0)
  int64_t cap;          // rows of a sequence's table
  int64_t owner, ml, o, score; // byte offsets
  size_t bytes;
  int tiles;            // workgroups a KV head's query heads take
  int wide, unit;       // KV heads of a workgroup; chunks are multiples of `unit` rows
  int64_t groups;       // workgroups of a chunk: n_kv_heads / wide * tiles
  bool single;          // a sequence is one chunk
  bool planned;         // by paged_plan
};

// Workgroups of paged_attend that a compute unit holds (by their registers).
constexpr int resident(int head_dim) { return head_dim == 64 ? 4 : 2; }

Plan make_plan(const focus_paged_decode_desc* d) {
  const focus_paged_kv& c = d->cache;
  Plan p = {};
  p.cap = (int64_t)c.max_pages * c.page_rows;
  p.tiles = (int)focus::ceil_div(d->n_heads / c.n_kv_heads, kCols);
  // Where the heads of a row lie side by side, the waves of a workgroup take one KV head
  // each (or two waves each of two): four neighbouring rows read together come faster than
  // by workgroups on their own.  8 KV heads, 268 MB: rows of 128 bytes at 5.5 TB/s together,
  // 4.5 apart; of 256 bytes 5.9, 5.3; 16 x 10 000 rows of 32 KV heads 6.5, 5.6.  Where a
  // head's rows follow one another (5.9) there is nothing to gain.
  p.wide = c.head_stride > c.row_stride ? 1 : c.n_kv_heads % 4 == 0 ? 4 : c.n_kv_heads % 2 == 0 ? 2 : 1;
  // Short tables are not split, so that without weights nothing is left for a second launch;
  // up to twice as long where their heads alone fill half of the device.  With few heads
  // the waves then share each.  us, split / not:
  //   sequences, KV heads, group     128 rows      256          500          1000
  //     1,  8, 4 (D 128, bf16)      9.2 /  5.8   9.2 /  7.6   9.4 /  9.8  10.0 / 17.8
  //    32,  8, 4                   11.4 /  6.9  15.3 / 10.1  22.4 / 15.5  31.8 / 27.5
  //    32,  4, 16 (f32)            18.8 / 10.2  23.1 / 15.5  30.1 / 26.1  40.9 / 46.7
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads * p.tiles;
  p.single = d->split_keys == 0 && (p.cap <= kWhole || (p.cap <= 2 * kWhole && heads >= 128));
  if (p.single && heads <= 1024) p.wide = 1;
  p.planned = !p.single && c.batch > kWave;
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
  const int64_t partials = p.slots * d->n_heads;
  p.owner = 16 * (int64_t)c.batch;
  p.ml = p.owner + (p.planned ? focus::ceil_div(4 * p.slots, 16) * 16 : 0);
  p.o = p.ml + focus::ceil_div(8 * partials, 16) * 16;
  p.score = p.o + 4 * partials * c.head_dim;
  p.bytes = (size_t)(p.score + (d->accumulate ? 4 * (int64_t)c.batch * d->n_heads * p.cap : 0));
  if (p.single && !d->accumulate) p.bytes = 0;  // nothing is handed on
  return p;
}

struct Args {
  focus_paged_decode_desc d;
  float sc;             // softmax scale in log2 units
  int shift;            // log2 page_rows
  int tiles, wide_shift, unit_shift, target;   // wide and unit are powers of two
  int units;            // workgroups of a chunk and 16 query heads each
  int group, parts;     // query heads of a KV head; workgroups of one in the second launch
  int64_t cap;
  bool single;
  int64_t slots;
  int4* info;
  int* owner;           // sequence of each slot (-1: none); null unless planned
  float2* ml;
  float* o;
  float* score;
};

// Maximum over the lanes 16 and 32 apart.
__device__ inline float max_column(float x) {
  const uint32_t u = __float_as_uint(x);
  auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])));
  y = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// Rows of a chunk when they are to be chosen, for `target` chunks resident at a time: the
// least estimate of the time among
//   the rows of the whole batch spread over `target` chunks, rounded up to units, or over
//   half or twice as many;
//   the least size at which the chunks of all sequences are resident at once (up to kWave
//   sequences; it needs 16 steps of a search);
//   no split at all.
// The estimate, in rows a resident workgroup streams while all of them do: what there is
// to read, and for each chunk kStart rows' worth of beginning and end and its partials
// written and read, over the target; where not all are resident at once kLate of the
// longest more, which may begin late; at least the longest at kAlone times the rate, as
// fast as one gets when the others have ended.  us, before twice as many were tried (kStart
// 100, all of the longest more) / now: 64 sequences of 4096 rows, 5 KV heads, 152 / 120; 48
// with 7 heads 152 / 121; 16 of 10 000, 32 heads, 417 / 409; 200 of 1000 to 2000, 8 heads,
// 272 / 246; 400 of 600 to 1200, 4 heads, 165 / 184; over 104 such batches 0.8 % less.
constexpr int kStart = 72;
constexpr float kLate = 0.3f, kAlone = 1.1f;

__device__ inline float estimate(const Args& a, uint32_t units, int chunks, int rows, int longest) {
  const float each = (float)(kStart >> a.wide_shift) + (a.d.cache.dtype == FOCUS_BF16 ? 4.f : 2.f) * a.group;
  const float even = ((float)units * (1 << a.unit_shift) + each * (float)chunks) / (float)a.target;
  const float last = (float)min(rows, longest);
  return fmaxf(chunks > a.target ? even + kLate * last : even, last / kAlone);
}

// Sum and maximum of f(rows) over the sequences: of a wave, two sequences a lane, or of
// paged_plan's workgroup.  The results are the same in all threads.
struct OverWave {
  int n0, n1;  // rows of the lane's sequences; -1 for none
  template <typename F> __device__ uint32_t total(F f) const {
    return (uint32_t)__builtin_amdgcn_readlane(wave_scan((int)(f(n0) + f(n1))), 63);
  }
  template <typename F> __device__ uint32_t most(F f) const { return (uint32_t)wave_max((int)max(f(n0), f(n1))); }
};
struct OverGroup {
  const focus_paged_kv& c;
  int* s_part;  // one per wave
  template <typename F> __device__ uint32_t total(F f) const {
    uint32_t x = 0;
    for (int b = threadIdx.x; b < c.batch; b += kPlan) x += f(focus::paged_length(c, b));
    return join(wave_scan((int)x), [](int x, int y) { return x + y; });
  }
  template <typename F> __device__ uint32_t most(F f) const {
    uint32_t x = 0;
    for (int b = threadIdx.x; b < c.batch; b += kPlan) x = max(x, f(focus::paged_length(c, b)));
    return join(wave_max((int)x), [](int x, int y) { return max(x, y); });
  }
  template <typename Op> __device__ uint32_t join(int x, Op op) const {
    __syncthreads();
    if (threadIdx.x % 64 == 63) s_part[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int w = 0; w < kPlan / 64; ++w) x = op(x, s_part[w]);
    return (uint32_t)x;
  }
};

// (Counted in units: the host has checked that all tables together hold fewer than 2^31.)
template <typename Over> __device__ int chunk_rows(const Args& a, const Over& over) {
  const int batch = a.d.cache.batch, shift = a.unit_shift, unit = 1 << shift;
  const uint32_t target = (uint32_t)a.target;
  // units of a sequence; its chunks of so many units
  auto units_of = [&](int n) { return (uint32_t)(max(n, 0) + unit - 1) >> shift; };
  auto chunks = [&](uint32_t units) {
    return over.total([&](int n) { return n < 0 ? 0u : max(1u, (units_of(n) + units - 1) / units); });
  };
  const uint32_t total = over.total(units_of);
  if (total + batch <= target) return unit;
  const uint32_t one = (total + target - 1) / target, two = min(2 * one, 1u << 30 >> shift);
  const uint32_t whole = max(1u, over.most(units_of));
  if (one >= whole) return (int)(whole << shift);
  const int longest = (int)(whole << shift);
  const uint32_t count1 = chunks(one), count2 = chunks(two);
  uint32_t units = one;
  float best = estimate(a, total, count1, one << shift, longest);
  auto better = [&](uint32_t count, uint32_t with) {
    const float e = estimate(a, total, count, with << shift, longest);
    if (e < best) best = e, units = with;
  };
  better(count2, two);
  const uint32_t half = (one + 1) / 2;
  better(chunks(half), half);
  if (count1 > target && batch <= kWave && (uint32_t)batch <= target) {
    uint32_t lo = one, hi = whole;  // too many chunks at lo, few enough at hi
    for (int k = 0; k < 16 && hi - lo > 1; ++k) {
      const uint32_t mid = (lo + hi) / 2;
      const bool many = chunks(mid) > target;
      lo = many ? mid : lo, hi = many ? hi : mid;
    }
    better(chunks(hi), hi);
  }
  better(batch, whole);
  return (int)(units << shift);
}

// The chunk of slot i (chunks 0: none), in scalar registers: all of a wave's lanes ask for
// the same.
__device__ inline int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
struct Chunk {
  int b, c, n, slot0, chunks, rows;
};
__device__ __forceinline__ Chunk find_chunk(const Args& a, int i) {
  const focus_paged_kv& c = a.d.cache;
  int b = 0, n = 0, slot0 = i, chunks = 0, rows = (int)a.cap;
  if (a.single) {
    if (i < c.batch) b = i, n = focus::paged_length(c, i), chunks = 1;
  } else if (a.owner) {
    const int own = i < a.slots ? scalar(a.owner[i]) : -1;
    if (own >= 0) {
      const int4 info = a.info[own];
      b = own, slot0 = info.x, chunks = info.y, n = info.z, rows = info.w;
    }
  } else {
    const int two = threadIdx.x % 64 * 2;
    const int n0 = two < c.batch ? focus::paged_length(c, two) : -1;
    const int n1 = two + 1 < c.batch ? focus::paged_length(c, two + 1) : -1;
    rows = scalar(a.d.split_keys ? a.d.split_keys : chunk_rows(a, OverWave{n0, n1}));
    auto chunks_of = [&](int n) { return n < 0 ? 0 : max(1, (n - 1) / rows + 1); };
    const int own0 = chunks_of(n0), own1 = chunks_of(n1), upto = wave_scan(own0 + own1);
    if (i < __builtin_amdgcn_readlane(upto, 63)) {
      const int lane = __ffsll((unsigned long long)__ballot(i < upto)) - 1;
      const int end = __builtin_amdgcn_readlane(upto, lane), last = __builtin_amdgcn_readlane(own1, lane);
      const bool second = i >= end - last;
      b = 2 * lane + second;
      n = __builtin_amdgcn_readlane(second ? n1 : n0, lane);
      chunks = __builtin_amdgcn_readlane(second ? own1 : own0, lane);
      slot0 = end - last - (second ? 0 : chunks);
    }
  }
  slot0 = scalar(slot0);
  return {scalar(b), i - slot0, scalar(n), slot0, scalar(chunks), scalar(rows)};
}

// The chunks of more than kWave sequences, by one workgroup.  (With every wave going through
// all lengths by itself 4096 sequences of 200 to 400 rows, 8 KV heads of 128, took 1570 us,
// now 900; of 128 sequences the launch would cost as much as it saves.)
__global__ __launch_bounds__(kPlan) void paged_plan(Args a) {
  __shared__ int s_part[kPlan / 64];
  const focus_paged_kv& c = a.d.cache;
  const int tid = threadIdx.x;
  const int rows = a.d.split_keys ? a.d.split_keys : chunk_rows(a, OverGroup{c, s_part});
  int before = 0;
  for (int b0 = 0; b0 < c.batch; b0 += kPlan) {
    const int b = b0 + tid, n = b < c.batch ? focus::paged_length(c, b) : 0;
    const int own = b < c.batch ? max(1, (n - 1) / rows + 1) : 0, upto = wave_scan(own);
    __syncthreads();  // the last round's sums are read
    if (tid % 64 == 63) s_part[tid / 64] = upto;
    __syncthreads();
    int slot = before + upto - own;
#pragma unroll
    for (int w = 0; w < kPlan / 64; ++w) {
      if (w < tid / 64) slot += s_part[w];
      before += s_part[w];
    }
    if (b < c.batch) a.info[b] = make_int4(slot, own, n, rows);
    for (int k = 0; k < own && slot + k < a.slots; ++k) a.owner[slot + k] = b;
  }
  for (int64_t i = before + tid; i < a.slots; i += kPlan) a.owner[i] = -1;
}

template <typename T, int D> struct Tile {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int kRows = kBf16 ? 32 : 16;     // rows a wave takes at a time
  static constexpr int kScores = kRows / 4;         // scores of a lane: rows kScores x ..
  static constexpr int kPer = D / 16;               // elements of a V row a lane holds
  static constexpr int kWords = kPer * sizeof(T) / 4;
  static constexpr int kPiece = 16 / sizeof(T);     // elements of a 16-byte load
  static constexpr int kSteps = D / (4 * kPiece);   // 16-byte pieces of a K row a lane holds
  static constexpr int kProducts = kBf16 ? 2 : 1;   // K rows a lane holds
  // pieces of 16 bytes (8 where a lane's share of a V row is that): whole vectors, which
  // stay where their load puts them
  using V = typename std::conditional<kWords == 2, u32x2, u32x4>::type;
  static constexpr int kVSize = sizeof(V) / 4, kVs = kWords / kVSize;
  u32x4 k[kProducts][kSteps];
  V v[kScores][kVs];
  __device__ uint32_t word(int j, int i) const { return v[j][i / kVSize][i % kVSize]; }
};

// Load from global memory: the compiler takes a choice between a page and kZeros for an
// address of any kind, whose loads it can only wait for all together.  Past the caches,
// unless other workgroups read the same rows: 64 sequences of 16 000 rows of one head of 128
// (bf16) in 90 us, 97 through them (of tables that the last-level cache could hold between
// calls, 102 MB: 35.7 and 33.6 if nothing comes between, 35.7 and 36.8 if something does).
template <typename V, bool SHARED>
__device__ __forceinline__ V load_row(const void* p) {
  const auto* from = reinterpret_cast<const __attribute__((address_space(1))) V*>(reinterpret_cast<uintptr_t>(p));
  if constexpr (SHARED) return *from;
  else return __builtin_nontemporal_load(from);
}

__device__ inline float lse_of(const Args& a, float2 ml) {
  return ml.y == 0.f ? -INFINITY : fmaf(ml.x, a.sc, log2f(ml.y)) * kLn2;
}

// SHARED: a KV head has more than 16 query heads, whose workgroups read the same rows.
template <typename T, int D, bool SHARED>
__global__ __launch_bounds__(kThreads, resident(D)) void paged_attend(Args a) {
  using L = Tile<T, D>;
  constexpr int kPitch = D + 4;
  __shared__ int64_t s_page[kPages + 1];  // (a chunk may begin inside a page)
  __shared__ float s_o[kWaves][kCols][kPitch];
  __shared__ float2 s_ml[kWaves][kCols];
  const focus_paged_kv& c = a.d.cache;
  const int H = a.d.n_heads, G = a.group;
  // (a wave's number in a scalar register: its loops are branches then, not masks)
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int lane = tid % 64, col = lane % 16, x = lane / 16;
  int slot_id = blockIdx.z * kMaxGrid + blockIdx.y, tile_id = 0, g0 = blockIdx.x;
  if constexpr (SHARED) {
    // Workgroups are dealt over the XCDs in turn: those that read the same rows to one XCD,
    // one after another, so that its L2 reads them once.  64 sequences of 16 000 rows of one
    // head of 128 (bf16), 32 query heads: 117 us; loaded past the caches 146, in the order of
    // the grid's indices as well 180.
    const int id = blockIdx.x, among = id % (focus::kXcds * a.tiles);
    const int unit = id / (focus::kXcds * a.tiles) * focus::kXcds + among % focus::kXcds;
    tile_id = among / focus::kXcds;
    slot_id = unit / a.units;
    g0 = unit % a.units;
  }
  g0 <<= a.wide_shift;
  // waves of a KV head; this wave's head, and which of its waves it is
  const int by = kWaves >> a.wide_shift, at_head = wave >> (2 - a.wide_shift), g = g0 + at_head, among = wave & (by - 1);
  const Chunk ch = find_chunk(a, slot_id);
  if (ch.chunks == 0) return;
  const int b = ch.b, r0 = ch.c * ch.rows, r1 = min(ch.n, r0 + ch.rows);
  const bool first = g0 == 0 && tile_id == 0;
  const int h0 = g * G + tile_id * kCols, heads = min(kCols, G - tile_id * kCols);

  // Q: column col, elements as the K rows' pieces
  u32x4 q[L::kSteps];
  {
    const T* src = reinterpret_cast<const T*>(a.d.q) + (int64_t)b * a.d.q_row + (int64_t)(h0 + col) * a.d.q_head;
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i)
      q[i] = col < heads ? *reinterpret_cast<const u32x4*>(src + (i * 4 + x) * L::kPiece) : u32x4{0, 0, 0, 0};
  }

  const T* kbase = reinterpret_cast<const T*>(c.k) + (int64_t)g * c.head_stride;
  const T* vbase = reinterpret_cast<const T*>(c.v) + (int64_t)g * c.head_stride;
  const T* zeros = reinterpret_cast<const T*>(kZeros);
  const int mask = c.page_rows - 1;
  // rows of eight from which this lane reads K and V; the offsets of its rows in them
  const int k8 = L::kBf16 ? col / 4 * 8 : col / 8 * 8, k_in = L::kBf16 ? col % 4 : col % 8;
  const int v8 = L::kBf16 ? x * 8 : x / 2 * 8, v_in = L::kBf16 ? 0 : x % 2 * 4;
  float* score = a.d.accumulate && col < heads ? a.score + ((int64_t)b * H + h0 + col) * a.cap : nullptr;

  float m, l;
  f32x4 o[L::kPer];
  // The lower parts of the weights (below) turn an infinity in V into a NaN: sums that are
  // NaN are taken again without them (the others keep what they are).
  auto pass = [&](auto with_low) {
    constexpr bool low = decltype(with_low)::value;
    m = kMinit;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < L::kPer; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int seg = r0; seg < r1; seg += kPages << a.shift) {
      const int seg_end = min(r1, seg + (kPages << a.shift)), page0 = seg >> a.shift;
      __syncthreads();
      for (int i = tid; i + page0 <= (seg_end - 1) >> a.shift; i += kThreads) {
        const int64_t p = focus::page_of(c, b, (i + page0) << a.shift, a.shift);
        if (p < 0 && first) focus::raise_err(a.d.err, FOCUS_ERR_BOUNDS);
        s_page[i] = p < 0 ? -1 : p * c.page_stride;
      }
      __syncthreads();
      // whole tiles end here
      const int full_end = seg_end - (seg_end - seg) % L::kRows;
      // offset of the page that holds the eight rows at r (negative: none, or past end)
      auto page = [&](int r, int end) { return r < end ? s_page[(r >> a.shift) - page0] : -1; };
      // Rows of eight lie in one page, so all of them can be read where the first is cached.
      auto load = [&](L& w, int r, int end) {
        const int64_t pk = page(r + k8, end), pv = page(r + v8, end);
        const uint32_t step = (uint32_t)c.row_stride;
        const uint64_t ks = pk >= 0 ? step : 0, vs = pv >= 0 ? step : 0;
        const T* kp = (pk >= 0 ? kbase + pk + (uint64_t)(uint32_t)((r + k8) & mask) * step : zeros) + k_in * ks + x * L::kPiece;
        const T* vp = (pv >= 0 ? vbase + pv + (uint64_t)(uint32_t)((r + v8) & mask) * step : zeros) + v_in * vs + col * L::kPer;
#pragma unroll
        for (int t = 0; t < L::kProducts; ++t)
#pragma unroll
          for (int i = 0; i < L::kSteps; ++i) w.k[t][i] = load_row<u32x4, SHARED>(kp + 4 * t * ks + i * 4 * L::kPiece);
#pragma unroll
        for (int j = 0; j < L::kScores; ++j)
#pragma unroll
          for (int i = 0; i < L::kVs; ++i) w.v[j][i] = load_row<typename L::V, SHARED>(vp + j * vs + i * L::kPiece);
      };
      auto compute = [&](L& w, int r, auto whole) {
        f32x4 s[L::kProducts];
#pragma unroll
        for (int t = 0; t < L::kProducts; ++t) {
          s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < L::kSteps; ++i) {
            if constexpr (L::kBf16) {
              s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.k[t][i]),
                                                             __builtin_bit_cast(bf16x8, q[i]), s[t], 0, 0, 0);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.k[t][i][e]), __uint_as_float(q[i][e]), s[t],
                                                            0, 0, 0);
            }
          }
        }
        const int row = r + v8 + v_in;  // of the lane's first score
        // of the lane's rows, those that count: the first `live`
        int live = page(r + v8, seg_end) >= 0 ? L::kScores : 0;
        if constexpr (!decltype(whole)::value) {
          live = min(live, seg_end - row);
          // rows past the end may hold anything, and zero times a NaN is a NaN
#pragma unroll
          for (int j = 0; j < L::kScores; ++j)
#pragma unroll
            for (int i = 0; i < L::kVs; ++i)
              if (j >= live) w.v[j][i] = typename L::V{};
        }
        float y[L::kScores], mx = m;
#pragma unroll
        for (int j = 0; j < L::kScores; ++j) {
          y[j] = j < live ? s[j / 4][j % 4] : -INFINITY;
          mx = fmaxf(mx, y[j]);
        }
        if (score && (decltype(whole)::value || row < seg_end)) {
#pragma unroll
          for (int j = 0; j < L::kScores; j += 4)
            *reinterpret_cast<float4*>(score + row + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
        }
        mx = max_column(mx);
        // (scaled after the difference: scaled before, a score of 4096 would be rounded to
        // 2^-12, and so would the weight)
        const float alpha = __builtin_amdgcn_exp2f((m - mx) * a.sc);
        m = mx;
        l *= alpha;
#pragma unroll
        for (int j = 0; j < L::kScores; ++j) {
          y[j] = __builtin_amdgcn_exp2f((y[j] - m) * a.sc);
          l += y[j];
        }
#pragma unroll
        for (int t = 0; t < L::kPer; ++t) o[t] *= alpha;
        if constexpr (L::kBf16) {
          // product t's rows of V^T, in the place of what was loaded
          u32x4 z[L::kPer];
#pragma unroll
          for (int t = 0; t < L::kPer; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              z[t][e] = __builtin_amdgcn_perm(w.word(2 * e + 1, t / 2), w.word(2 * e, t / 2), t % 2 ? 0x07060302 : 0x05040100);
          // The weights in three bf16 parts, which hold all 24 bits of a float32, one part
          // after another: by products instead, all parts of each, D = 64 spills and takes 2 to
          // 6 % longer.  (Two parts, 17 bits, round twice as many elements of o the other way
          // and take as long within 2 %: 16 x 10 000 rows of 32 heads of 128 400 and 400 us, of
          // 64 208 and 208, 64 x 16 000 rows of one head of 128 for 128 query heads 307 and 305.)
#pragma unroll
          for (int part = 0; part < (low ? 3 : 1); ++part) {
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
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int t = 0; t < L::kPer; ++t)
              o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.word(j, t)), y[j], o[t], 0, 0, 0);
        }
      };
      // A wave's whole tiles, two a round, the next one's loads in flight while one is
      // computed; then, for one wave, the tile that the chunk ends in.  One way out of the
      // loop, loads past the end taken from kZeros and the last of them waited for behind
      // it: otherwise the compiler cannot tell which loads are in flight at a round's start
      // and waits for half of them.
      const int stride = by * L::kRows;
      int r = seg + among * L::kRows;
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
      if (r < seg_end && r == full_end) {
        L w;
        load(w, r, seg_end);
        compute(w, r, std::false_type{});
      }
    }
    bool nan = false;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int t = 0; t < L::kPer; t += 4) {
        float4* to = reinterpret_cast<float4*>(&s_o[wave][col][(x * 4 + e) * L::kPer + t]);
        float4 y = make_float4(o[t][e], o[t + 1][e], o[t + 2][e], o[t + 3][e]);
        if (L::kBf16 && !low) {
          const float4 was = *to;
          y = make_float4(was.x == was.x ? was.x : y.x, was.y == was.y ? was.y : y.y, was.z == was.z ? was.z : y.z,
                          was.w == was.w ? was.w : y.w);
        }
        *to = y;
        nan |= y.x != y.x || y.y != y.y || y.z != y.z || y.w != y.w;
      }
    return nan;
  };
  const bool nan = pass(std::integral_constant<bool, L::kBf16>{});
  if constexpr (L::kBf16) {
    if (__syncthreads_or(nan)) pass(std::false_type{});
  }

  // (not at the start, where it would leave b in vector registers during the loops)
  if (first && ch.c == 0 && tid == 0) {
    if (a.info && !a.owner) a.info[b] = make_int4(ch.slot0, ch.chunks, ch.n, ch.rows);
    if (ch.n != c.length[b]) focus::raise_err(a.d.err, FOCUS_ERR_CAPACITY);
  }
  // the waves' parts of each query head, joined
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (x == 0) s_ml[wave][col] = make_float2(m, l);
  __syncthreads();
  constexpr int kLanes = D / 4;  // threads of a head, four elements each
  const int e = tid % kLanes * 4;
  for (int h = tid / kLanes, w0 = 0; w0 < kWaves; h += kThreads / kLanes) {
    while (h >= heads && w0 < kWaves) h -= heads, w0 += by;
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
    const int head = (g0 + (w0 >> (2 - a.wide_shift))) * G + tile_id * kCols + h;
    const int64_t at = (int64_t)b * H + head, slot = (int64_t)(ch.slot0 + ch.c) * H + head;
    if (ch.chunks == 1) {
      y = ml.y == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : y * (1.f / ml.y);
      T* o_at = reinterpret_cast<T*>(a.d.o) + at * D + e;
      if constexpr (L::kBf16)
        *reinterpret_cast<u32x2*>(o_at) = u32x2{focus::pack_bf16x2(y[0], y[1]), focus::pack_bf16x2(y[2], y[3])};
      else *reinterpret_cast<f32x4*>(o_at) = y;
      if (e == 0 && a.d.lse) a.d.lse[at] = lse_of(a, ml);
    } else {
      *reinterpret_cast<f32x4*>(a.o + slot * D + e) = y;
    }
    if (e == 0 && a.ml) a.ml[slot] = ml;
  }
}

// Maximum and sum over a sequence's chunks of head h, by one wave.
__device__ float2 joined(const Args& a, const int4& info, int h) {
  const int H = a.d.n_heads, lane = threadIdx.x % 64;
  float M = kMinit, L = 0.f;
  for (int i = lane; i < info.y; i += 64) {
    const float2 y = a.ml[(int64_t)(info.x + i) * H + h];
    const float m = fmaxf(M, y.x);
    L = L * __builtin_amdgcn_exp2f((M - m) * a.sc) + y.y * __builtin_amdgcn_exp2f((y.x - m) * a.sc);
    M = m;
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    const float m2 = __shfl_xor(M, k), l2 = __shfl_xor(L, k), m = fmaxf(M, m2);
    L = L * __builtin_amdgcn_exp2f((M - m) * a.sc) + l2 * __builtin_amdgcn_exp2f((m2 - m) * a.sc);
    M = m;
  }
  return make_float2(M, L);
}

constexpr int kWeightRows = 4 * kThreads;   // rows whose weights a workgroup writes at a time
constexpr int kMaxGroup = 512;              // query heads of a KV head

// One of `parts` workgroups of a (sequence, KV head): merges the partials of every
// parts-th of its query heads (D / 4 threads over the output, the other groups of them
// over the chunks, eight loads in flight each) and, where weights are accumulated, writes
// those of every parts-th block of rows.  Maxima and sums come first, a wave a head; the
// first partials, scores and old weights are in flight meanwhile.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_join(Args a) {
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes, kFlight = 8, kHeads = 2;
  __shared__ float4 s_o[kGroups][kLanes];
  __shared__ float2 s_ml[kMaxGroup];  // a head's maximum and sum
  __shared__ float s_inv[kMaxGroup];  // 1 / the sum
  const focus_paged_kv& c = a.d.cache;
  const int K = c.n_kv_heads, H = a.d.n_heads, G = a.group, tid = threadIdx.x, parts = a.parts;
  // (part 0 of all first: the later ones have nothing to do where sequences are short, and
  // with parts side by side those that do would all lie on a few of the XCDs)
  const int part = c.batch <= kMaxGrid ? blockIdx.z : blockIdx.z % parts, g = blockIdx.x;
  const int b = blockIdx.y + (c.batch <= kMaxGrid ? 0 : blockIdx.z / parts * kMaxGrid);
  if (b >= c.batch) return;
  const int4 info = a.info[b];
  const int n = info.z;
  const bool merges = info.y > 1 && part < G, weighs = a.d.accumulate && part * kWeightRows < n;
  if (!merges && !weighs) return;
  const int e = tid % kLanes, grp = tid / kLanes;
  const float4* o = reinterpret_cast<const float4*>(a.o);
  float4 y[kFlight];
  float m[kFlight];
  auto load_partials = [&](int h, int i0) {
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int64_t slot = (int64_t)(info.x + min(i0 + k * kGroups, info.y - 1)) * H + g * G + h;
      y[k] = o[slot * kLanes + e];
      m[k] = a.ml[slot].x;
    }
  };
  float* w = c.weight + ((int64_t)b * K + g) * c.weight_rows;
  float4 sc[kHeads];
  float old[4];
  const float* score = a.score + ((int64_t)b * H + g * G) * a.cap;
  auto load_scores = [&](int r, int h0) {
#pragma unroll
    for (int k = 0; k < kHeads; ++k)
      if (r < n && h0 + k < G) sc[k] = *reinterpret_cast<const float4*>(score + (h0 + k) * a.cap + r);
  };
  auto load_weights = [&](int r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) old[i] = r + i < n && a.d.weight_decay != 0.f ? w[r + i] : 0.f;
  };
  if (merges) load_partials(part, grp);
  if (weighs) load_scores(part * kWeightRows + 4 * tid, 0), load_weights(part * kWeightRows + 4 * tid);
  // of all heads for the weights, else of those to be merged
  const int first = weighs ? 0 : part, step = weighs ? 1 : parts;
  for (int h = first + tid / 64 * step; h < G; h += kWaves * step) {
    const float2 ml = joined(a, info, g * G + h);
    if (tid % 64 == 0) s_ml[h] = ml, s_inv[h] = ml.y == 0.f ? 0.f : 1.f / ml.y;
  }
  __syncthreads();
  if (merges) {
    for (int h = part; h < G; h += parts) {
      const float2 ml = s_ml[h];
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i0 = grp; i0 < info.y; i0 += kGroups * kFlight) {
        if (h > part || i0 > grp) load_partials(h, i0);
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
        const int64_t at = (int64_t)b * H + g * G + h;
        reinterpret_cast<T*>(a.d.o)[at * D + tid] = (T)(ml.y == 0.f ? 0.f : z / ml.y);
        if (tid == 0 && a.d.lse) a.d.lse[at] = lse_of(a, ml);
      }
      __syncthreads();
    }
  }
  if (!weighs) return;
  // weights, four rows a thread
  for (int r0 = part * kWeightRows; r0 < n; r0 += parts * kWeightRows) {
    const int r = r0 + 4 * tid;
    if (r0 > part * kWeightRows) load_weights(r);
    float x[4] = {};
    for (int h0 = 0; h0 < G; h0 += kHeads) {
      if (r0 > part * kWeightRows || h0 > 0) load_scores(r, h0);
#pragma unroll
      for (int k = 0; k < kHeads; ++k) {
        if (r < n && h0 + k < G) {
          const float top = s_ml[h0 + k].x, inv = s_inv[h0 + k];
          auto add = [&](float& to, float s) { to = fmaf(__builtin_amdgcn_exp2f((s - top) * a.sc), inv, to); };
          add(x[0], sc[k].x), add(x[1], sc[k].y), add(x[2], sc[k].z), add(x[3], sc[k].w);
        }
      }
    }
    // (scores are stored up to the next multiple of four rows; weights end at n)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (r + i < n) w[r + i] = a.d.weight_decay == 0.f ? x[i] : fmaf(a.d.weight_decay, old[i], x[i]);
  }
}

focus_status validate(const focus_paged_decode_desc* d) {
  const focus_paged_kv& c = d->cache;
  const focus_status st = focus::check_paged(c);
  if (st != FOCUS_OK) return st;
  if (c.head_dim != 64 && c.head_dim != 128) return FOCUS_E_UNSUPPORTED;
  if (d->n_heads <= 0 || d->split_keys < 0 || d->split_keys % kUnit || !(d->softmax_scale == d->softmax_scale) ||
      !isfinite(d->weight_decay))
    return FOCUS_E_ARG;
  if (d->n_heads % c.n_kv_heads) return FOCUS_E_SHAPE;
  if ((int64_t)c.batch * d->n_heads > INT32_MAX / kThreads || d->n_heads / c.n_kv_heads > kMaxGroup) return FOCUS_E_SHAPE;
  // (chunks are counted in 32 bits, in units of 32 rows at least)
  if ((int64_t)c.batch * focus::ceil_div((int64_t)c.max_pages * c.page_rows, 32) > INT32_MAX) return FOCUS_E_SHAPE;
  const int64_t es = focus::elt_bytes(c.dtype);
  if (d->q_row < 0 || d->q_head < 0 || !focus::pieces16(d->q_row, es) || !focus::pieces16(d->q_head, es))
    return FOCUS_E_ARG;
  return FOCUS_OK;
}

template <typename T, int D>
focus_status launch(Args a, const Plan& p, hipStream_t s) {
  const focus_paged_kv& c = a.d.cache;
  // workgroups of a (sequence, KV head) in the second launch: one per query head, or, for
  // weights, per block of the table's rows, but not many more than the device holds
  const int64_t per = focus::ceil_div(std::max<int64_t>(p.cap, 1), kWeightRows), heads = (int64_t)c.batch * c.n_kv_heads;
  const int64_t most = focus::ceil_div(8 * focus::device_cus(), heads);
  a.parts = (int)std::min(most, a.d.accumulate ? std::max(per, std::min<int64_t>(a.group, 4)) : a.group);
  const int64_t slots = focus::ceil_div(p.slots, kMaxGrid), batches = focus::ceil_div(c.batch, kMaxGrid);
  if (p.groups * p.slots > INT32_MAX / kThreads - focus::kXcds * kMaxGroup ||
      heads * a.parts > INT32_MAX / kThreads || slots > kMaxGrid || batches * a.parts > kMaxGrid)
    return FOCUS_E_SHAPE;
  if (p.planned) {
    hipLaunchKernelGGL(paged_plan, dim3(1), dim3(kPlan), 0, s, a);
    const focus_status st = focus::launch_status();
    if (st != FOCUS_OK) return st;
  }
  const dim3 grid = p.tiles > 1 ? dim3((uint32_t)(focus::ceil_div(a.units * p.slots, focus::kXcds) * focus::kXcds * p.tiles))
                                : dim3((uint32_t)p.groups, (uint32_t)std::min<int64_t>(p.slots, kMaxGrid), (uint32_t)slots);
  if (p.tiles > 1) hipLaunchKernelGGL((paged_attend<T, D, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((paged_attend<T, D, false>), grid, dim3(kThreads), 0, s, a);
  const focus_status st = focus::launch_status();
  if (st != FOCUS_OK || (p.single && !a.d.accumulate)) return st;
  hipLaunchKernelGGL((paged_join<T, D>),
                     dim3((uint32_t)c.n_kv_heads, (uint32_t)std::min(c.batch, kMaxGrid), (uint32_t)(batches * a.parts)),
                     dim3(kThreads), 0, s, a);
  return focus::launch_status();
}

}  // namespace

extern "C" size_t focus_paged_decode_workspace(const focus_paged_decode_desc* d) {
  if (!d || validate(d) != FOCUS_OK) return 0;
  return make_plan(d).bytes;
}

extern "C" focus_status focus_paged_decode(const focus_paged_decode_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  const focus_status st = validate(d);
  if (st != FOCUS_OK) return st;
  const focus_paged_kv& c = d->cache;
  if (c.batch == 0) return FOCUS_OK;
  if (!d->q || !d->o || (d->accumulate && !c.weight)) return FOCUS_E_NULL;
  if (!focus::aligned16(d->q) || !focus::aligned16(d->o) || (reinterpret_cast<uintptr_t>(d->lse) & 3u)) return FOCUS_E_ARG;
  const Plan p = make_plan(d);
  if (p.bytes > 0 && (!d->workspace || d->workspace_bytes < p.bytes)) return FOCUS_E_WORKSPACE;
  if (!focus::aligned16(d->workspace)) return FOCUS_E_ARG;
  char* ws = reinterpret_cast<char*>(d->workspace);
  Args a = {};
  a.d = *d;
  a.shift = focus::page_shift(c);
  a.tiles = p.tiles, a.wide_shift = __builtin_ctz((unsigned)p.wide), a.unit_shift = __builtin_ctz((unsigned)p.unit);
  a.target = (int)p.target, a.units = (int)(p.groups / p.tiles);
  a.group = d->n_heads / c.n_kv_heads;
  a.cap = p.cap, a.single = p.single, a.slots = p.slots;
  if (p.bytes > 0) {
    a.info = reinterpret_cast<int4*>(ws), a.ml = reinterpret_cast<float2*>(ws + p.ml);
    a.o = reinterpret_cast<float*>(ws + p.o), a.score = reinterpret_cast<float*>(ws + p.score);
  }
  if (p.planned) a.owner = reinterpret_cast<int*>(ws + p.owner);
  const float scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / sqrtf((float)c.head_dim);
  a.sc = scale * kLog2e;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (c.dtype == FOCUS_BF16) return c.head_dim == 128 ? launch<__bf16, 128>(a, p, s) : launch<__bf16, 64>(a, p, s);
  return c.head_dim == 128 ? launch<float, 128>(a, p, s) : launch<float, 64>(a, p, s);
}
