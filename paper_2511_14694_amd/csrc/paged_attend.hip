// Attention of the newest tokens of every sequence over a paged cache of 8 bits
// (focus_paged_attend).
//
//   attend_rows   the rows of the whole batch, laid end to end, are dealt in equal shares: one
//                 workgroup takes a share (parts of one sequence or of several) for one to
//                 eight KV heads and up to 16 or 32 columns of each (a column is a new token
//                 and a query head); it writes o and lse where a sequence lies in its share,
//                 else an unnormalised partial (running max, sum, output)
//   attend_join   merges the partials of a sequence by log-sum-exp
//   attend_plan   before both for more than 128 sequences: where each begins
//
// Every cached byte is read once for up to 32 columns.  A wave takes 32 rows at a time; each
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
//
// HBM bound where there is much to read: 16 sequences of 10 000 rows of 32 heads of 128 (1.31
// GB) take 208 us, 6.3 TB/s, the vector units busy for 39 % of the cycles and the matrix cores
// for 13 %; one of 262 144 rows of 8 heads (0.54 GB) 94, 5.7 TB/s.  Where there is less the
// latencies of the beginning (lengths, page table, first rows: 6 us) and the second launch
// (5 us and the gap before it) count: 64 sequences of 1 to 8 192 rows of 8 heads (0.13 GB) 35;
// up to five tokens of 32 sequences of up to 16 384 rows (0.15 GB, 20 columns) 45.  The first
// form, in equal chunks of each sequence found by a search and 16 columns at a time, took 227,
// 106, 44 and 69.
#include "paged_softmax.h"

#include <algorithm>
#include <type_traits>

namespace {

using focus::bf16x8;
using focus::f32x4;
using focus::kMinit;
using focus::scalar;
using focus::u32x4;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kPages = 1024;    // pages held in LDS at a time
constexpr int kWhole = 256;     // rows of a table that is not split
constexpr int kUnit = 128;      // rows of a share's units times sets of KV heads of a workgroup
constexpr int kRows = 32;       // rows of a wave at a time
constexpr int kMost = 512;      // columns of a KV head
// Units that a sequence's beginning and end in a share cost: its queries, pages and first rows
// arrive one after another, some 5 us, in which a workgroup could stream two units, and its
// outputs leave.  1 / 2 / 3 / 4 units: 64 sequences of 1 to 8 192 rows 46.4 / 41.8 / 41.5 / 41.2
// us, up to five tokens of 32 sequences 61.1 / 60.0 / 56.3 / 56.2.
constexpr int kEnds = 4;

// What a lane reads in the place of eight rows that begin past their sequence's end or
// lie in a page outside the pool.
__device__ __align__(16) const uint32_t kZeros[64] = {};

// Workspace: int2 info[batch] {first share, shares}; for more than focus::kWave sequences int
// ends[1 + batch] {units of a share, units up to each sequence's end}; then two partials of a
// share, of the sequence that goes on from the share before and of the one that goes on behind it:
// float2 ml[2 shares][columns], float o[2 shares][columns][D].
struct Plan {
  int64_t shares, cap;
  int64_t ends, ml, o;  // byte offsets
  size_t bytes;
  int cols, tiles;      // columns of a workgroup; workgroups a KV head's columns take
  int heads;            // KV heads of a wave
  int wide, unit;       // sets of these of a workgroup; rows of a unit
  int64_t groups;       // workgroups of a share
  int columns;          // of all heads
  bool single, planned; // a share is a sequence; attend_plan runs
};

// Workgroups of attend_rows that a compute unit holds (by their registers).
constexpr int resident(int head_dim, int tiles, int heads) { return head_dim == 64 && tiles * heads == 1 ? 3 : 2; }

Plan make_plan(const focus_paged_attend_desc* d) {
  const focus_paged_kv& c = d->cache.kv;
  Plan p = {};
  p.cap = (int64_t)c.max_pages * c.page_rows;
  const int per_head = d->n_heads / c.n_kv_heads * d->max_rows;
  p.columns = per_head * c.n_kv_heads;
  // (float32 queries take three times the registers)
  p.cols = per_head > 16 && d->dtype == FOCUS_BF16 ? 32 : 16;
  p.tiles = (int)focus::ceil_div(per_head, p.cols);
  // Neighbouring heads' rows read together, where they lie side by side; two heads of 64
  // bytes, which share a cache line, by the same wave.  (By waves of their own half of the lines
  // came twice: 16 x 10 000 rows of 32 such heads 165 us, now 136.  With two tiles of columns
  // besides, the registers do not suffice.)
  const bool beside = c.head_stride < c.row_stride;
  const bool pairs = c.head_dim == 64 && beside && c.n_kv_heads % 2 == 0;
  p.heads = pairs && p.cols == 16 ? 2 : 1;
  const int sets = c.n_kv_heads / p.heads;
  // (a given split fixes which waves share a head's rows too, however many columns there are)
  const int alike = d->split_keys > 0 && pairs ? c.n_kv_heads / 2 : sets;
  auto wide = [&](int most) { return most >= 4 && alike % 4 == 0 ? 4 : most >= 2 && alike % 2 == 0 ? 2 : 1; };
  p.wide = wide(beside ? 4 : 1);
  const int64_t heads = (int64_t)c.batch * c.n_kv_heads * p.tiles;
  p.single = d->split_keys == 0 && (p.cap <= kWhole || (p.cap <= 2 * kWhole && heads >= 128));
  // (short tables: no more waves for a head than there are tiles; 108 sequences of 32 float32
  // heads in tables of 16 rows 51 us with four, now 22)
  if (p.single) p.wide = std::max(heads <= 1024 ? 1 : p.wide, wide(p.cap <= kRows ? 4 : p.cap <= 2 * kRows ? 2 : 1));
  p.planned = !p.single && c.batch > focus::kWave;
  // as many shares as run together, but no more than there may be units
  auto shares = [&](int wide) {
    return std::min(std::max<int64_t>(1, resident(c.head_dim, p.cols / 16, p.heads) * focus::device_cus() / (sets / wide * p.tiles)),
                    c.batch * (std::max<int64_t>(1, focus::ceil_div(p.cap, kUnit / wide)) + kEnds));
  };
  // Neighbouring heads by one workgroup are read faster, but leave each head as many times more
  // partials, of all columns: not where a share has few rows for its columns (the tables' rows:
  // the lengths are not known here).  By 4 / 2 / 1 heads a workgroup: 16 sequences of 10 000 rows of 32
  // heads 215 / 224 / 244 us, 20 columns of 32 of up to 16 384 rows 52.8 / 52.5 / 55.2, of two of up
  // to 10 064 38.5 / 32.8 / 30.8; 240 shapes 32.9 / 31.9 / 32.4 in the geometric mean, by this rule 31.7.
  if (!p.single && d->split_keys == 0)
    while (p.wide > 1 && c.batch * p.cap < (p.wide == 4 ? 128 : 32) * per_head * shares(p.wide)) p.wide /= 2;
  p.groups = (int64_t)sets / p.wide * p.tiles;
  if (p.single) {
    p.unit = (int)std::max<int64_t>(p.cap, 1), p.shares = c.batch;
  } else if (d->split_keys > 0) {
    p.unit = d->split_keys, p.shares = c.batch * std::max<int64_t>(1, focus::ceil_div(p.cap, p.unit));
  } else {
    p.unit = kUnit / p.wide, p.shares = shares(p.wide);
  }
  const int64_t partials = 2 * p.shares * p.columns;
  p.ends = focus::ceil_div(8 * (int64_t)c.batch, 16) * 16;
  p.ml = p.ends + (p.planned ? focus::ceil_div(4 * ((int64_t)c.batch + 1), 16) * 16 : 0);
  p.o = p.ml + focus::ceil_div(8 * partials, 16) * 16;
  p.bytes = p.single ? 0 : (size_t)(p.o + 4 * partials * c.head_dim);
  return p;
}

struct Args {
  focus_paged_attend_desc d;
  float sc;             // softmax scale in log2 units
  float less, more;     // what weights are multiplied by; its inverse, what sums are
  int shift, scale_shift;  // log2 page_rows, scale_rows
  int tiles, wide_shift;
  int units;            // workgroups of a share, tiles aside
  int around;           // shares' workgroups that run together once on every compute unit
  int group;            // query heads of a KV head
  int per_head, columns;   // columns of a KV head at most, of all heads
  int unit, shares, over;  // rows of a unit; shares; units that a sequence costs besides
  bool single, fixed;   // a share is a sequence; a unit
  int wide_from;        // shares of a sequence from which on a workgroup joins its columns
  int2* info;
  int* ends;            // null unless planned
  float2* ml;
  float* o;
};

// The rows of q of a sequence: [first, first + count); count -1 if they are not to be touched.
struct Tokens {
  int64_t first;
  int count;
};
__device__ inline Tokens tokens_of(const Args& a, int r0, int r1, int32_t& bits) {
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

// Units of a sequence of n rows, its ends included; of a share, of so many in all.
__device__ inline int units_of(const Args& a, int n) { return max((n - 1) / a.unit + 1, 1) + a.over; }
__device__ inline int units_of_share(const Args& a, int total) { return a.fixed ? 1 : max(1, (total - 1) / a.shares + 1); }

constexpr int kPlan = 1024;

__global__ __launch_bounds__(kPlan) void attend_plan(Args a) {
  __shared__ int s_part[kPlan / 64];
  const focus_paged_kv& c = a.d.cache.kv;
  const int tid = threadIdx.x;
  int before = 0;
  for (int b0 = 0; b0 < c.batch; b0 += kPlan) {
    const int b = b0 + tid;
    int upto = focus::wave_scan(b < c.batch ? units_of(a, focus::paged_length(c, b)) : 0);
    __syncthreads();  // the last round's sums are read
    if (tid % 64 == 63) s_part[tid / 64] = upto;
    __syncthreads();
    upto += before;
#pragma unroll
    for (int w = 0; w < kPlan / 64; ++w) {
      if (w < tid / 64) upto += s_part[w];
      before += s_part[w];
    }
    if (b < c.batch) a.ends[1 + b] = upto;
  }
  if (tid == 0) a.ends[0] = units_of_share(a, before);
}

// The sequences of a share, in scalar registers: all lanes of a wave walk along together.
struct Walk {
  int b, n;             // the sequence and its rows
  int begin, units;     // where its units begin; how many they are
  int share;            // units of a share
  int c0, c1;           // its rows of q begin and end there
  int n0, n1;           // rows of the lane's two sequences, where a wave holds all
  int e0, e1, e2;       // and where their rows of q begin and end

  __device__ __forceinline__ void at(const Args& a, int seq) {
    const focus_paged_kv& c = a.d.cache.kv;
    b = seq;
    if (b >= c.batch) return;
    if (a.single || a.ends) {
      const int rows = focus::paged_length(c, b);
      const int from = a.d.cu_rows ? a.d.cu_rows[b] : b, to = a.d.cu_rows ? a.d.cu_rows[b + 1] : b + 1;
      n = scalar(rows), c0 = scalar(from), c1 = scalar(to);
    } else {
      const bool odd = b % 2;
      n = __builtin_amdgcn_readlane(odd ? n1 : n0, b / 2);
      c0 = __builtin_amdgcn_readlane(odd ? e1 : e0, b / 2), c1 = __builtin_amdgcn_readlane(odd ? e2 : e1, b / 2);
    }
    units = units_of(a, n);
  }
  // The first sequence of share i.
  __device__ __forceinline__ Walk(const Args& a, int i) {
    const focus_paged_kv& c = a.d.cache.kv;
    const int lane = threadIdx.x % 64;
    n0 = n1 = e0 = e1 = e2 = 0;
    if (a.single) {
      share = 1, begin = i;
      at(a, i);
    } else if (a.ends) {
      share = scalar(a.ends[0]);
      const int from = i * share;
      const int* ends = a.ends + 1;
      int lo = 0, len = c.batch;
      while (len > 0) {  // the first that ends behind `from`, 64 looked at together
        const int step = (len + 63) / 64, last = lo + (lane + 1) * step - 1;
        const int parts = __popcll(__ballot(last < lo + len && ends[last] <= from));
        lo += parts * step;
        len = min(step - 1, len - parts * step);
      }
      begin = lo > 0 && lo < c.batch ? scalar(ends[lo - 1]) : 0;
      at(a, lo);
    } else {
      const int two = lane * 2;
      n0 = two < c.batch ? focus::paged_length(c, two) : 0;
      n1 = two + 1 < c.batch ? focus::paged_length(c, two + 1) : 0;
      const int last = min(two + 2, c.batch);
      e0 = a.d.cu_rows ? a.d.cu_rows[min(two, last)] : two;
      e1 = a.d.cu_rows ? a.d.cu_rows[min(two + 1, last)] : two + 1;
      e2 = a.d.cu_rows ? a.d.cu_rows[last] : two + 2;
      const int u0 = two < c.batch ? units_of(a, n0) : 0, u1 = two + 1 < c.batch ? units_of(a, n1) : 0;
      const int upto = focus::wave_scan(u0 + u1);
      share = scalar(units_of_share(a, __builtin_amdgcn_readlane(upto, 63)));
      const int from = i * share;
      const unsigned long long behind = __ballot(upto > from);
      if (!behind) {
        b = c.batch;
        return;
      }
      const int l = __ffsll(behind) - 1;
      const int end = __builtin_amdgcn_readlane(upto, l), second = end - __builtin_amdgcn_readlane(u1, l);
      const bool odd = from >= second;
      begin = odd ? second : second - __builtin_amdgcn_readlane(u0, l);
      at(a, 2 * l + odd);
    }
  }
  __device__ __forceinline__ void next(const Args& a) {
    begin += units;
    at(a, b + 1);
  }
};

// Slot of the partial of part `chunk` of a sequence whose first share is `first`.
__device__ inline int64_t slot_of(int first, int chunk) { return chunk == 0 ? 2 * (int64_t)first + 1 : 2 * ((int64_t)first + chunk); }

// A pair of e4m3 numbers in bf16; eight.
__device__ inline uint32_t widen(uint32_t w, bool high) {
  const bf16x2 r = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, false);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ inline bf16x8 widen8(uint32_t w0, uint32_t w1) {
  const u32x4 r = {widen(w0, false), widen(w0, true), widen(w1, false), widen(w1, true)};
  return __builtin_bit_cast(bf16x8, r);
}

// Load from global memory, past the caches unless other workgroups read the same rows.  (Said
// to be global: the compiler takes a choice between a page and kZeros for an address of any
// kind, whose loads it can only wait for all together.)
template <typename V, bool SHARED>
__device__ __forceinline__ V load_row(const void* p) {
  const auto* from = reinterpret_cast<const __attribute__((address_space(1))) V*>(reinterpret_cast<uintptr_t>(p));
  if constexpr (SHARED) return *from;
  else return __builtin_nontemporal_load(from);
}

template <int D, int HEADS> struct Tile {
  static constexpr int kPer = D / 16;               // elements of a V row a lane holds
  static constexpr int kWords = kPer / 4;
  static constexpr int kPieces = D / 64;            // 16-byte pieces of a K row a lane holds
  using V = typename std::conditional<kWords == 2, u32x2, uint32_t>::type;
  u32x4 k[HEADS][2][kPieces];
  V v[HEADS][8];
  float ks[HEADS], vs[HEADS];  // the scales of the rows of the lane's scores
  __device__ uint32_t word(int h, int j, int i) const {
    if constexpr (kWords == 2) return v[h][j][i];
    else return v[h][j];
  }
};

// Bytes of w that are NaN (0x7f or 0xff) as 1, others 0.
__device__ inline uint32_t nan_bytes(uint32_t w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u; }

// SHARED: a KV head has more columns than a workgroup takes, whose workgroups read the same
// rows.  TILES: 16 columns each, all of which use a wave's rows as they are loaded.  HEADS: KV
// heads of a wave, whose rows lie side by side.
// T: of q and o.  float32 queries enter in three bf16 parts, weights in two (17 bits; their
// rounding is far below that of a bf16 output) or, for float32 outputs, three.
template <typename T, int D, int TILES, int HEADS, bool SHARED>
__global__ __launch_bounds__(kThreads, resident(D, TILES, HEADS)) void attend_rows(Args a) {
  using L = Tile<D, HEADS>;
  constexpr int kPitch = D + 4, kSteps = D / 32, kCols = 16 * TILES, kStates = TILES * HEADS;
  constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kWeightParts = sizeof(T) == 2 ? 2 : 3;
  __shared__ int s_page[kPages + 1];  // (rows may begin inside a page)
  __shared__ float s_o[kWaves][HEADS * kCols][kPitch];
  __shared__ float2 s_ml[kWaves][HEADS * kCols];
  __shared__ __align__(16) uint8_t s_nan[kWaves][kRows][16];  // NaN among a row's elements, a bit each
  const focus_paged_kv& c = a.d.cache.kv;
  const int H = a.d.n_heads, G = a.group;
  // (a wave's number in a scalar register: its loops are branches then, not masks)
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int lane = tid % 64, col = lane % 16, x = lane / 16;
  int share, tile_id = 0, g0;
  if constexpr (SHARED) {
    // Workgroups are dealt over the XCDs in turn: those that read the same rows to one XCD,
    // one after another, so that its L2 reads them once.
    const int id = blockIdx.x, among = id % (focus::kXcds * a.tiles);
    const int unit = id / (focus::kXcds * a.tiles) * focus::kXcds + among % focus::kXcds;
    tile_id = among / focus::kXcds;
    share = unit / a.units, g0 = unit % a.units;
    if (share >= a.shares) return;
  } else {
    // The two workgroups of a compute unit take different heads: those whose heads begin at
    // even multiples of 512 bytes are 15 % slower than the others, and with the same heads on
    // every unit of an XCD half of the XCDs would end late.
    share = blockIdx.x / a.units, g0 = (blockIdx.x + share / a.around) % a.units;
  }
  g0 *= HEADS << a.wide_shift;
  // waves of a set of KV heads; this wave's first head, and which of the set's waves it is
  const int by = kWaves >> a.wide_shift, at_set = wave >> (2 - a.wide_shift), g = g0 + HEADS * at_set, among = wave & (by - 1);
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
  const bool reports = g0 == 0 && tile_id == 0;

  // (a vector register: the scalar ones are all taken, and with this one more in a lane of a spilled
  // one two tiles of columns were 1.5 to 2 % slower)
  float less = a.less;
  asm("" : "+v"(less));

  Walk walk(a, share);
  const int from = share * walk.share, upto = from + walk.share;
  for (; walk.b < c.batch && walk.begin < upto; walk.next(a)) {
    // this share's rows of the sequence: its units behind the first `over`
    const int data = walk.begin + a.over, b = walk.b, n = walk.n;
    const int u0 = max(from - data, 0), u1 = min(upto, walk.begin + walk.units) - data;
    if (u0 >= u1) continue;
    const int last = walk.begin + walk.units - 1;
    const int first = walk.share == 1 ? data : data / walk.share, chunk = share - first;
    const int chunks = (walk.share == 1 ? last : last / walk.share) - first + 1;
    const int r0 = (int)min((int64_t)u0 * a.unit, (int64_t)n), r1 = (int)min((int64_t)u1 * a.unit, (int64_t)n);
    int32_t bits = 0;
    const Tokens tok = tokens_of(a, walk.c0, walk.c1, bits);
    if (reports && chunk == 0 && tid == 0) {
      if (a.info) a.info[b] = make_int2(first, chunks);
      if (n != c.length[b]) bits |= FOCUS_ERR_CAPACITY;
      if (bits) focus::raise_err(a.d.err, bits);
    }
    // columns of this workgroup; this lane's: token and head of the KV head, the rows it sees
    const int cols = min(kCols, tok.count * G - tile_id * kCols);
    if (cols <= 0) continue;
    const int sees_all = max(0, n - (tok.count - 1));
    int sees[TILES];
    bf16x8 q[kStates][kParts][kSteps];  // column col, elements as the K rows' pieces
#pragma unroll
    for (int state = 0; state < kStates; ++state) {
      const int tile = state % TILES, cc = tile_id * kCols + min(16 * tile + col, cols - 1), token = cc / G;
      const int head = (g + state / TILES) * G + cc - token * G;
      sees[tile] = max(0, n - (tok.count - 1 - token));
      const T* src = reinterpret_cast<const T*>(a.d.q) + (tok.first + token) * a.d.q_row + (int64_t)head * a.d.q_head;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int e = (i / 2 * 4 + x) * 16 + i % 2 * 8;
        if constexpr (sizeof(T) == 2) {
          q[state][0][i] = *reinterpret_cast<const bf16x8*>(src + e);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            // (cut off, not rounded: the largest numbers would become infinities)
            float f = src[e + k];
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
              const float high = __uint_as_float(__float_as_uint(f) & 0xffff0000u);
              q[state][part][i][k] = (__bf16)high;
              f -= high;
            }
          }
        }
      }
    }

    float m[kStates], l[kStates];
    f32x4 o[kStates][L::kPer];
#pragma unroll
    for (int state = 0; state < kStates; ++state) {
      m[state] = kMinit, l[state] = 0.f;
#pragma unroll
      for (int t = 0; t < L::kPer; ++t) o[state][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int seg = r0; seg < r1; seg += kPages << a.shift) {
      const int seg_end = min(r1, seg + (kPages << a.shift)), page0 = seg >> a.shift;
      __syncthreads();
      for (int i = tid; i + page0 <= (seg_end - 1) >> a.shift; i += kThreads) {
        const int64_t p = focus::page_of(c, b, (i + page0) << a.shift, a.shift);
        if (p < 0 && reports) focus::raise_err(a.d.err, FOCUS_ERR_BOUNDS);
        s_page[i] = (int)p;
      }
      __syncthreads();
      const int clean = min(seg_end, sees_all);  // tiles up to here are whole and seen by all columns
      // the page that holds the eight rows at r (negative: none, or past end)
      auto page = [&](int r, int end) { return r < end ? s_page[(r >> a.shift) - page0] : -1; };
      // Rows of eight lie in one page, so all of them can be read where the first is cached.
      // Heads that share a cache line are read in turn, so that it comes once.
      auto load = [&](L& w, int r, int end) {
        const int pk = page(r + k8, end), pv = page(r + v8, end);
        const uint32_t step = (uint32_t)c.row_stride, far = (uint32_t)c.page_stride;
        const uint32_t ks = pk >= 0 ? step : 0, vs = pv >= 0 ? step : 0;
        auto at = [&](const uint8_t* base, int p, int row) {
          return base + (uint64_t)(uint32_t)p * far + (uint64_t)(uint32_t)(row & mask) * step;
        };
        const uint8_t* kp = (pk >= 0 ? at(kbase, pk, r + k8) : zeros) + (uint64_t)(uint32_t)k_in * ks + x * 16;
        const uint8_t* vp = (pv >= 0 ? at(vbase, pv, r + v8) : zeros) + col * L::kPer;
        const uint64_t k_next = pk >= 0 ? c.head_stride : 0, v_next = pv >= 0 ? c.head_stride : 0;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < L::kPieces; ++i)
#pragma unroll
            for (int h = 0; h < HEADS; ++h)
              w.k[h][t][i] = load_row<u32x4, SHARED>(kp + 4 * t * (uint64_t)ks + i * 64 + h * k_next);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int h = 0; h < HEADS; ++h) w.v[h][j] = load_row<typename L::V, SHARED>(vp + j * (uint64_t)vs + h * v_next);
        const uint64_t sc = (uint64_t)(uint32_t)pv * page_scales + (uint32_t)(((r + v8) & mask) >> a.scale_shift);
        const float* none = reinterpret_cast<const float*>(kZeros);
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
          w.ks[h] = load_row<float, true>(pv >= 0 ? ks_base + h * per_page + sc : none);
          w.vs[h] = load_row<float, true>(pv >= 0 ? vs_base + h * per_page + sc : none);
        }
      };
      auto compute = [&](L& w, int r) {
        const int row = r + v8;  // of the lane's first score
        // of the lane's rows, those that count: the first `live`
        const int live = page(row, seg_end) >= 0 ? 8 : 0;
        const bool tail = r + kRows > clean;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
          const int at0 = h * TILES;  // the head's first state
          uint32_t bad = 0;
          if (tail) {
            // Rows past the end may hold anything, and those that only later tokens see a NaN,
            // and zero times a NaN is a NaN: the first are cleared, the NaN of the others
            // taken out and put into the sums of the columns that see them.
            const int in = min(live, seg_end - row);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              if (j >= in) w.v[h][j] = typename L::V{};
#pragma unroll
              for (int i = 0; i < L::kWords; ++i) bad |= nan_bytes(w.word(h, j, i));
            }
          }
          const float vs = w.vs[h] * less;
          float y[TILES][8];
#pragma unroll
          for (int tile = 0; tile < TILES; ++tile) {
            f32x4 s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int i = 0; i < kSteps; ++i) {
                const bf16x8 k = widen8(w.k[h][t][i / 2][i % 2 * 2], w.k[h][t][i / 2][i % 2 * 2 + 1]);
#pragma unroll
                for (int part = kParts - 1; part >= 0; --part)
                  s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[at0 + tile][part][i], s[t], 0, 0, 0);
              }
            }
            const int lives = tail ? min(live, min(seg_end, sees[tile]) - row) : live;
            float mx = m[at0 + tile];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              y[tile][j] = j < lives ? s[j / 4][j % 4] * w.ks[h] : -INFINITY;
              mx = fmaxf(mx, y[tile][j]);
            }
            mx = focus::max_column(mx);
            // (scaled after the difference: scaled before, a score of 4096 would be rounded to
            // 2^-12, and so would the weight)
            if (__ballot(mx > m[at0 + tile])) {  // rare once a few rows are seen
              const float alpha = __builtin_amdgcn_exp2f((m[at0 + tile] - mx) * a.sc);
              m[at0 + tile] = mx;
              l[at0 + tile] *= alpha;
#pragma unroll
              for (int t = 0; t < L::kPer; ++t) o[at0 + tile][t] *= alpha;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              y[tile][j] = __builtin_amdgcn_exp2f((y[tile][j] - m[at0 + tile]) * a.sc);
              l[at0 + tile] += y[tile][j];
              y[tile][j] *= vs;
            }
            if (tail) {  // (of rows that do not count the scale may be anything)
#pragma unroll
              for (int j = 0; j < 8; ++j) y[tile][j] = j < lives ? y[tile][j] : 0.f;
            }
          }
          if (tail && __ballot(bad != 0)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t bits = 0;
#pragma unroll
              for (int i = 0; i < L::kWords; ++i) {
                const uint32_t is = nan_bytes(w.word(h, j, i)), keep = ~(is * 0xffu);
                bits |= (is * 0x10204080u >> 28) << 4 * i;  // the bytes' bits side by side
                if constexpr (L::kWords == 2) w.v[h][j][i] &= keep;
                else w.v[h][j] &= keep;
              }
              s_nan[wave][v8 + j][col] = (uint8_t)bits;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile) {
              uint32_t any = 0;  // byte e: elements (4 x + e) kPer + t
              const int end = min(seg_end, sees[tile]) - r;
#pragma unroll 1
              for (int i = 0; i < kRows; ++i) {
                const uint32_t of_row = *reinterpret_cast<const uint32_t*>(&s_nan[wave][i][4 * x]);
                any |= i < end ? of_row : 0u;
              }
#pragma unroll
              for (int t = 0; t < L::kPer; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (any >> (8 * e + t) & 1) o[at0 + tile][t][e] = NAN;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          }
          // product t's rows of V^T: pairs of rows by a byte permutation, then widened; four
          // products at a time
          bf16x8 p[TILES][kWeightParts];
#pragma unroll
          for (int tile = 0; tile < TILES; ++tile)
#pragma unroll
            for (int part = 0; part < kWeightParts; ++part)
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                p[tile][part][j] = (__bf16)y[tile][j];
                y[tile][j] -= (float)p[tile][part][j];
              }
#pragma unroll
          for (int i = 0; i < L::kWords; ++i) {
            u32x4 z[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t lo = __builtin_amdgcn_perm(w.word(h, 2 * e + 1, i), w.word(h, 2 * e, i), 0x05010400);
              const uint32_t hi = __builtin_amdgcn_perm(w.word(h, 2 * e + 1, i), w.word(h, 2 * e, i), 0x07030602);
              z[0][e] = widen(lo, false), z[1][e] = widen(lo, true);
              z[2][e] = widen(hi, false), z[3][e] = widen(hi, true);
            }
#pragma unroll
            for (int tile = 0; tile < TILES; ++tile)
#pragma unroll
              for (int part = 0; part < kWeightParts; ++part)
#pragma unroll
                for (int t = 0; t < 4; ++t)
                  o[at0 + tile][4 * i + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, z[t]), p[tile][part],
                                                                               o[at0 + tile][4 * i + t], 0, 0, 0);
          }
        }
      };
      // A wave's tiles, two a round, the next one's loads in flight while one is computed.
      // One way out of the loop, loads past the end taken from kZeros and the last of them
      // waited for behind it: otherwise the compiler cannot tell which loads are in flight
      // at a round's start and waits for half of them.
      const int stride = by * kRows;
      int r = seg + among * kRows;
      if (r < seg_end) {
        L w0, w1;
        load(w0, r, seg_end);
        for (; r + stride < seg_end; r += 2 * stride) {
          load(w1, r + stride, seg_end);
          compute(w0, r);
          load(w0, r + 2 * stride, seg_end);
          compute(w1, r + stride);
        }
        if (r < seg_end) compute(w0, r);
        __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
      }
    }
    __syncthreads();  // the last sequence's outputs are read
#pragma unroll
    for (int state = 0; state < kStates; ++state) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < L::kPer; t += 4)
          *reinterpret_cast<float4*>(&s_o[wave][16 * state + col][(x * 4 + e) * L::kPer + t]) =
              make_float4(o[state][t][e], o[state][t + 1][e], o[state][t + 2][e], o[state][t + 3][e]);
      // the waves' parts of each column, joined
      l[state] += __shfl_xor(l[state], 16);
      l[state] += __shfl_xor(l[state], 32);
      if (x == 0) s_ml[wave][16 * state + col] = make_float2(m[state], l[state]);
    }
    __syncthreads();
    constexpr int kLanes = D / 4;  // threads of a column, four elements each
    const int e = tid % kLanes * 4;
    // over the columns `h` of each head of the sets, which begin at waves w0
    for (int h = tid / kLanes, w0 = 0, second = 0; w0 < kWaves; h += kThreads / kLanes) {
      while (h >= cols && w0 < kWaves) {
        h -= cols, ++second;
        if (second == HEADS) second = 0, w0 += by;
      }
      if (w0 >= kWaves) break;
      const int at_lds = second * kCols + h;
      float2 ml = s_ml[w0][at_lds];
      f32x4 y = *reinterpret_cast<const f32x4*>(&s_o[w0][at_lds][e]);
      for (int w = w0 + 1; w < w0 + by; ++w) {
        const float2 other = s_ml[w][at_lds];
        const float M = fmaxf(ml.x, other.x);
        const float f = __builtin_amdgcn_exp2f((ml.x - M) * a.sc), f2 = __builtin_amdgcn_exp2f((other.x - M) * a.sc);
        ml = make_float2(M, fmaf(ml.y, f, other.y * f2));
        y = y * f + *reinterpret_cast<const f32x4*>(&s_o[w][at_lds][e]) * f2;
      }
      const int kv = g0 + HEADS * (w0 >> (2 - a.wide_shift)) + second, at_col = tile_id * kCols + h;
      if (chunks == 1) {
        const int i = at_col / G;
        const int64_t at = (tok.first + i) * H + kv * G + (at_col - i * G);
        y = ml.y == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : y * (a.more / ml.y);
        T* to = reinterpret_cast<T*>(a.d.o) + at * D + e;
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<u32x2*>(to) = u32x2{focus::pack_bf16x2(y[0], y[1]), focus::pack_bf16x2(y[2], y[3])};
        else *reinterpret_cast<f32x4*>(to) = y;
        if (e == 0 && a.d.lse) a.d.lse[at] = focus::lse_of(a.sc, ml);
      } else {
        const int64_t slot = slot_of(first, chunk) * a.columns + kv * a.per_head + at_col;
        *reinterpret_cast<f32x4*>(a.o + slot * D + e) = y;
        if (e == 0) a.ml[slot] = ml;
      }
    }
  }
}

// Merges a column's partials: by a wave, or, where a sequence has many shares (WIDE), by a
// workgroup for every 32 elements of it.  Lanes lie over the elements, four each, and groups of
// them over the shares; the first partials are in flight while the maxima and sums are merged,
// by every wave for itself.
//
// (A wave has 16 shares of 128 elements in flight.  WIDE for few columns, two to a compute unit,
// of many shares each: by waves and so one sequence of 100 000 rows, four columns of 512 shares, 47
// and 22 us; 16 of up to 7 629 rows, 512 of 16 or fewer, 25.5 and 23.8, but 32 of up to 30 517, 2 048
// of 8, 34.3 and 37.5; eight tokens of 16 of 8 000 rows, 4 096 of 16, 9.3 and 33.6 in the join alone.  Few shares are not
// worth the workgroups: three sequences of up to 2 021 rows, 60 shares, 14.7 and 15.6.)
//
// The two add the partials in different orders, and the rule follows from the batch and the
// tables: with a given split_keys, which fixes a sequence's bits, its own shares alone say which,
// 128 or more a workgroup, and both are launched where tables hold so many.  (One sequence of 262 144
// rows in 512 shares 144 us by waves, by workgroups 113.)
constexpr int kJoin = 256, kManyShares = 16, kWideFrom = 128, kFewColumns = 512;
template <typename T, int D, bool WIDE>
__global__ __launch_bounds__(kJoin) void attend_join(Args a) {
  constexpr int kFlight = 8, kThreadsOf = WIDE ? kJoin : 64, kSlices = WIDE ? D / 32 : 1;
  constexpr int kLanes = D / 4 / kSlices, kGroups = kThreadsOf / kLanes;
  __shared__ float4 s_o[WIDE ? kJoin : 1];
  const focus_paged_kv& c = a.d.cache.kv;
  const int G = a.group, tid = threadIdx.x % kThreadsOf, lane = threadIdx.x % 64;
  const int64_t id = WIDE ? blockIdx.x / kSlices : (int64_t)blockIdx.x * (kJoin / 64) + scalar(threadIdx.x / 64);
  const int b = (int)(id / a.columns), column = (int)(id % a.columns), g = column / a.per_head, cc = column % a.per_head;
  if (b >= c.batch) return;
  const int2 info = a.info[b];
  int32_t bits = 0;
  const Tokens tok = a.d.cu_rows ? tokens_of(a, a.d.cu_rows[b], a.d.cu_rows[b + 1], bits) : Tokens{b, 1};
  if (info.y <= 1 || (info.y >= a.wide_from) != WIDE || cc >= tok.count * G) return;
  const int e = (WIDE ? blockIdx.x % kSlices * kLanes : 0) + tid % kLanes, grp = tid / kLanes;
  const float4* o = reinterpret_cast<const float4*>(a.o);
  float4 y[kFlight], sum = make_float4(0.f, 0.f, 0.f, 0.f);
  float m[kFlight];
  auto load = [&](int i0) {
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int64_t slot = slot_of(info.x, min(i0 + k * kGroups, info.y - 1)) * a.columns + column;
      y[k] = o[slot * (D / 4) + e];
      m[k] = a.ml[slot].x;
    }
  };
  load(grp);
  // maximum and sum over the shares
  float M = kMinit, S = 0.f;
  for (int i = lane; i < info.y; i += 64) {
    const float2 z = a.ml[slot_of(info.x, i) * a.columns + column];
    const float top = fmaxf(M, z.x);
    S = S * __builtin_amdgcn_exp2f((M - top) * a.sc) + z.y * __builtin_amdgcn_exp2f((z.x - top) * a.sc);
    M = top;
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) {
    const float m2 = __shfl_xor(M, k), l2 = __shfl_xor(S, k), top = fmaxf(M, m2);
    S = S * __builtin_amdgcn_exp2f((M - top) * a.sc) + l2 * __builtin_amdgcn_exp2f((m2 - top) * a.sc);
    M = top;
  }
  for (int i0 = grp; i0 < info.y; i0 += kGroups * kFlight) {
    if (i0 > grp) load(i0);
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      if (i0 + k * kGroups < info.y) {
        const float f = __builtin_amdgcn_exp2f((m[k] - M) * a.sc);
        sum.x = fmaf(y[k].x, f, sum.x), sum.y = fmaf(y[k].y, f, sum.y);
        sum.z = fmaf(y[k].z, f, sum.z), sum.w = fmaf(y[k].w, f, sum.w);
      }
    }
  }
  if constexpr (WIDE) {
    s_o[tid] = sum;
    __syncthreads();
    if (tid >= kLanes) return;
    sum = s_o[tid];
    for (int k = 1; k < kGroups; ++k) {
      const float4 z = s_o[k * kLanes + tid];
      sum.x += z.x, sum.y += z.y, sum.z += z.z, sum.w += z.w;
    }
  } else {
#pragma unroll
    for (int k = kLanes; k < 64; k <<= 1)
      sum.x += __shfl_xor(sum.x, k), sum.y += __shfl_xor(sum.y, k), sum.z += __shfl_xor(sum.z, k), sum.w += __shfl_xor(sum.w, k);
    if (tid >= kLanes) return;
  }
  const float inv = S == 0.f ? 0.f : a.more / S;  // (the sum is zero too)
  const int i = cc / G;
  const int64_t at = (tok.first + i) * a.d.n_heads + g * G + (cc - i * G);
  T* to = reinterpret_cast<T*>(a.d.o) + at * D + 4 * e;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x2*>(to) = u32x2{focus::pack_bf16x2(sum.x * inv, sum.y * inv), focus::pack_bf16x2(sum.z * inv, sum.w * inv)};
  else *reinterpret_cast<float4*>(to) = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
  if (e == 0 && a.d.lse) a.d.lse[at] = focus::lse_of(a.sc, make_float2(M, S));
}

focus_status validate(const focus_paged_attend_desc* d) {
  const focus_paged_kv& c = d->cache.kv;
  const focus_status st = focus::check_paged8(d->cache);
  if (st != FOCUS_OK) return st;
  const int64_t es = focus::elt_bytes(d->dtype);
  if (es == 0) return FOCUS_E_DTYPE;
  if (c.head_dim != 64 && c.head_dim != 128) return FOCUS_E_UNSUPPORTED;
  if (d->n_heads <= 0 || d->max_rows <= 0 || d->n_rows < 0 || d->split_keys < 0 || d->split_keys % 128 ||
      !(d->softmax_scale == d->softmax_scale))
    return FOCUS_E_ARG;
  if (d->n_heads % c.n_kv_heads || c.page_stride > UINT32_MAX) return FOCUS_E_SHAPE;
  if ((int64_t)(d->n_heads / c.n_kv_heads) * d->max_rows > kMost || d->n_rows > INT32_MAX ||
      (!d->cu_rows && d->n_rows != c.batch))
    return FOCUS_E_SHAPE;
  if ((int64_t)c.batch * d->n_heads * d->max_rows > INT32_MAX / 4 / kThreads) return FOCUS_E_SHAPE;
  // (units, of 32 rows at least, are counted in 32 bits)
  if ((int64_t)c.batch * (focus::ceil_div((int64_t)c.max_pages * c.page_rows, 32) + 1 + kEnds) > INT32_MAX / 2)
    return FOCUS_E_SHAPE;
  if (d->q_row < 0 || d->q_head < 0 || !focus::pieces16(d->q_row, es) || !focus::pieces16(d->q_head, es))
    return FOCUS_E_ARG;
  return FOCUS_OK;
}

// The plan of a call that has something to do, if a launch holds its workgroups; of one that has
// not, an empty one (with no sequences there may be any number of heads).
focus_status checked_plan(const focus_paged_attend_desc* d, Plan& p) {
  p = {};
  const focus_status st = validate(d);
  if (st != FOCUS_OK || d->cache.kv.batch == 0 || d->n_rows == 0) return st;
  p = make_plan(d);
  return p.groups * p.shares > INT32_MAX / kThreads - focus::kXcds * kMost ? FOCUS_E_SHAPE : FOCUS_OK;
}

template <typename T, int D>
focus_status launch(Args a, const Plan& p, hipStream_t s) {
  const focus_paged_kv& c = a.d.cache.kv;
  const int64_t columns = (int64_t)c.batch * p.columns;
  if (p.planned) {
    hipLaunchKernelGGL(attend_plan, dim3(1), dim3(kPlan), 0, s, a);
    const focus_status st = focus::launch_status();
    if (st != FOCUS_OK) return st;
  }
  const dim3 grid((uint32_t)(p.tiles > 1 ? focus::ceil_div(a.units * p.shares, focus::kXcds) * focus::kXcds * p.tiles
                                         : p.groups * p.shares));
  auto attend = [&](auto tiles, auto heads, auto shared) {
    constexpr int kTiles = decltype(tiles)::value, kHeads = decltype(heads)::value;
    constexpr bool kShared = decltype(shared)::value;
    hipLaunchKernelGGL((attend_rows<T, D, kTiles, kHeads, kShared>), grid, dim3(kThreads), 0, s, a);
  };
  auto of_heads = [&](auto tiles, auto shared) {
    if constexpr (D == 64 && decltype(tiles)::value == 1) {
      if (p.heads == 2) return attend(tiles, std::integral_constant<int, 2>{}, shared);
    }
    attend(tiles, std::integral_constant<int, 1>{}, shared);
  };
  constexpr std::integral_constant<int, sizeof(T) == 2 ? 2 : 1> kMore;  // tiles of more than 16 columns
  constexpr std::integral_constant<int, 1> kOne;
  if (p.tiles > 1) of_heads(kMore, std::true_type{});
  else if (p.cols == 32) of_heads(kMore, std::false_type{});
  else of_heads(kOne, std::false_type{});
  const focus_status st = focus::launch_status();
  if (st != FOCUS_OK || p.single) return st;
  const bool given = a.d.split_keys > 0;
  const bool wide = given ? focus::ceil_div(p.cap, p.unit) >= kWideFrom
                          : columns <= kFewColumns && p.shares >= std::max<int64_t>((int64_t)kManyShares * c.batch, kWideFrom);
  a.wide_from = given ? kWideFrom : wide ? 0 : INT32_MAX;
  if (wide)
    hipLaunchKernelGGL((attend_join<T, D, true>), dim3((uint32_t)(columns * (D / 32))), dim3(kJoin), 0, s, a);
  if (given || !wide)
    hipLaunchKernelGGL((attend_join<T, D, false>), dim3((uint32_t)focus::ceil_div(columns, kJoin / 64)), dim3(kJoin), 0, s, a);
  return focus::launch_status();
}

}  // namespace

extern "C" size_t focus_paged_attend_workspace(const focus_paged_attend_desc* d) {
  Plan p;
  return d && checked_plan(d, p) == FOCUS_OK ? p.bytes : 0;
}

extern "C" focus_status focus_paged_attend(const focus_paged_attend_desc* d, focus_stream_t stream) {
  if (!d) return FOCUS_E_NULL;
  Plan p;
  const focus_status st = checked_plan(d, p);
  const focus_paged_kv& c = d->cache.kv;
  if (st != FOCUS_OK || c.batch == 0 || d->n_rows == 0) return st;
  if (!d->q || !d->o) return FOCUS_E_NULL;
  if (!focus::aligned16(d->q) || !focus::aligned16(d->o)) return FOCUS_E_ARG;
  for (const void* p : {(const void*)d->lse, (const void*)d->cu_rows, (const void*)d->err})
    if (reinterpret_cast<uintptr_t>(p) & 3u) return FOCUS_E_ARG;
  if (p.bytes > 0 && (!d->workspace || d->workspace_bytes < p.bytes)) return FOCUS_E_WORKSPACE;
  if (!focus::aligned16(d->workspace)) return FOCUS_E_ARG;
  char* ws = reinterpret_cast<char*>(d->workspace);
  Args a = {};
  a.d = *d;
  a.shift = focus::page_shift(c), a.scale_shift = __builtin_ctz((unsigned)d->cache.scale_rows);
  a.tiles = p.tiles, a.wide_shift = __builtin_ctz((unsigned)p.wide), a.units = (int)(p.groups / p.tiles);
  a.around = std::max(1, focus::device_cus() / a.units);
  a.group = d->n_heads / c.n_kv_heads, a.per_head = a.group * d->max_rows, a.columns = p.columns;
  a.single = p.single, a.fixed = p.single || d->split_keys > 0;
  a.unit = p.unit, a.shares = (int)p.shares, a.over = a.fixed ? 0 : kEnds;
  if (p.bytes > 0) {
    a.info = reinterpret_cast<int2*>(ws), a.ml = reinterpret_cast<float2*>(ws + p.ml);
    a.o = reinterpret_cast<float*>(ws + p.o);
  }
  if (p.planned) a.ends = reinterpret_cast<int*>(ws + p.ends);
  const float scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / sqrtf((float)c.head_dim);
  a.sc = scale * focus::kLog2e;
  // Where the mean of values is a float32 number, their sum need not be one: weights are multiplied
  // by a power of two below half of one over a table's rows, which is exact, and the mean by its inverse.
  // (What it costs is at the other end: a weight times its scale has the least step of bf16, 2^-133,
  // times that inverse.)
  const int bits = 33 - __builtin_clz((unsigned)std::max<int64_t>(p.cap, 1));
  a.less = ldexpf(1.f, -bits), a.more = ldexpf(1.f, bits);
  hipStream_t on = reinterpret_cast<hipStream_t>(stream);
  if (d->dtype == FOCUS_BF16) return c.head_dim == 128 ? launch<__bf16, 128>(a, p, on) : launch<__bf16, 64>(a, p, on);
  return c.head_dim == 128 ? launch<float, 128>(a, p, on) : launch<float, 64>(a, p, on);
}
