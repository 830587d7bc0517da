// Attention of single tokens to a paged cache:
//   out = sum_j p_j v_j,  p = softmax_j(scale * q . k_j)
// over the keys of a row's sequence, in one pass with the running maximum and sum of
// the softmax.  The query heads that share a head of the cache are the columns of the
// matrix instructions, so keys and values are read once for up to 16 of them.
//
// Bound by HBM: 4 dim bytes per key and head of the cache, for 4 dim operations per query
// head.  Measured: 64 rows of 4096 to 8192 keys, 32 heads on 8 of 128 dims, 1.6 GB in 282 + 7 us (5.7 TB/s where a kernel
// that only reads reaches 6.2); 2 rows of 131072, 16 heads on 2 of 256, 537 MB in 92 + 7; one row of 4095 keys,
// 32 on 8 of 128, 5.7 + 3.6, which is three dependent trips to memory (table, keys and values,
// results) and a second launch; 37 rows of up to 3001 keys, 16 heads of 64, a window of 2048 and three of ten places
// closed, 129 MB in 39 + 4: its 5000 workgroups are short, and all their places' scores are looked over.
//
// A tile is 32 keys of one head.  Scores are K Q^T: row i of the first matrix
// instruction of two is key 8 (i / 4) + i % 4 of the tile, of the second 4 more, so a lane's
// eight scores are eight consecutive keys, an octet, which never leaves a page; and they
// lie as the second product, V^T P^T, takes its right operand: the softmax's weights go from
// one product to the other in registers.  A lane loads eight (four, for heads of 64)
// neighbouring values of its octet's eight rows, whole rows per 16 lanes, and turns that square around
// in registers for the left operand.  Neither keys nor values pass LDS.
//
// The four waves of a workgroup take a tile each (or two): a part, whose four results are joined through LDS.
// The parts of 512 keys in order are a run, four runs in order a stretch, and the stretches are joined in order:
// always the same steps.  How much of that a workgroup does by itself follows from the number of
// workgroups that there would be: a stretch, requests running ahead of the products; a run; or
// one part, the quickest.  A second kernel does the rest.  So a row's bits do not depend on the number of
// rows.
#include "decode_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kThreads = 256, kWaves = 4, kTile = 32, kColumns = 16;
constexpr float kNone = -__builtin_inff(), kLog2e = 1.44269504088896340736f;

// Heads of up to 64 dims take two tiles at once: what is done per tile and part is half the work there.
template <int DP>
struct Shape {
  static constexpr int kTiles = DP <= 64 ? 2 : 1;                  // per wave of a part
  static constexpr int kPart = kWaves * kTiles * kTile;            // keys of a part
  static constexpr int kRun = 512 / kPart;                         // parts of a run
};
constexpr int kRunKeys = 512, kStretchKeys = 2048, kFour = 4;

// How the keys are divided; the same for all rows.
struct Parts {
  int keys;                      // that a workgroup takes (a piece): a part, a run or a stretch
  uint32_t pieces;               // of the longest row (and head)
  uint32_t blocks;               // of kColumns query heads that share a head
  float* sums;                   // [row][query head][piece][dim], null where one piece is all
  float2* state;                 // [row][query head][piece]: maximum (of scores in base 2), sum
};

// the keys that a row sees: [lo, hi), and the first key of its first part
struct Span {
  int64_t lo, hi, begin;
};

__device__ __forceinline__ Span span_of(const AttendArgs& p, int64_t row) {
  Span s;
  s.hi = max(int64_t(0), min(static_cast<int64_t>(p.lengths[row]), p.max_length));
  s.lo = p.window ? max(int64_t(0), s.hi - p.window) : 0;
  s.begin = s.lo / kTile * kTile;
  return s;
}

// which of the eight keys from `key` on a row sees
__device__ __forceinline__ uint32_t octet_of(const Span& s, int64_t key) {
  const int hi = static_cast<int>(max(int64_t(0), min(int64_t(8), s.hi - key)));
  const int lo = static_cast<int>(max(int64_t(0), min(int64_t(8), s.lo - key)));
  return ((1u << hi) - 1) & ~((1u << lo) - 1);
}

// which of the eight places from `key` on of a mask row of `width` are open
__device__ __forceinline__ uint32_t open_of(const uint8_t* mask, int64_t key, int64_t width) {
  typedef uint32_t words __attribute__((ext_vector_type(2), aligned(1)));
  uint32_t open = 0;
  if (key + 8 <= width) {
    const words w = *reinterpret_cast<const words*>(mask + key);
#pragma unroll
    for (int j = 0; j < 8; ++j) open |= (w[j / 4] >> 8 * (j % 4) & 0xff ? 1u : 0u) << j;
  } else {
    for (int j = 0; key + j < width; ++j) open |= (mask[key + j] ? 1u : 0u) << j;
  }
  return open;
}

// Four values' weighted sums over some keys: of exp2(score - top) * value, scaled as the row's weights are, and of the weights alone.
struct Sum {
  float4 v;
  float top, total;
};

// a and b joined; the same operations wherever it is called
__device__ __forceinline__ Sum join(const Sum& a, const Sum& b) {
  Sum r;
  r.top = fmaxf(a.top, b.top);
  const float base = r.top == kNone ? 0.f : r.top;
  const float f = __builtin_amdgcn_exp2f(a.top - base), e = __builtin_amdgcn_exp2f(b.top - base);
  r.v.x = __builtin_fmaf(a.v.x, f, e * b.v.x);
  r.v.y = __builtin_fmaf(a.v.y, f, e * b.v.y);
  r.v.z = __builtin_fmaf(a.v.z, f, e * b.v.z);
  r.v.w = __builtin_fmaf(a.v.w, f, e * b.v.w);
  r.total = __builtin_fmaf(a.total, f, e * b.total);
  return r;
}

__device__ __forceinline__ void finish(uint16_t* out, const Sum& s) {
  const float inv = s.total == 0.f ? 0.f : 1.f / s.total, f[4] = {s.v.x * inv, s.v.y * inv, s.v.z * inv, s.v.w * inv};
  put_values<false, 4>(out, f);
}

__device__ __forceinline__ float other_rows_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// Dims of the heads padded to DP; EXACT: they are DP.  HOLES: there is a mask, and keys that it closes are not read.
// MANY: a workgroup takes more than one part.
template <int DP, bool EXACT, bool HOLES, bool MANY>
__global__ __launch_bounds__(kThreads, MANY && DP <= 128 ? 3 : 2) void attend_kernel(AttendArgs p, Parts d, uint32_t base) {
  using S = Shape<DP>;
  constexpr int U = S::kTiles;
  constexpr int KC = DP / 32;                          // steps of 32 dims of the first product
  constexpr int VW = DP >= 128 ? 8 : 4, VH = DP / (16 * VW);   // a lane's neighbouring values, and how many such
  constexpr bool QL = MANY && DP >= 128;               // queries in LDS: in registers they are too many
  extern __shared__ float4 shared[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  const PagedArgs& cache = p.cache;
  const int dim = EXACT ? DP : cache.dim;
  const int group = p.q_heads / cache.heads;
  const int64_t page_mask = (int64_t(1) << cache.page_shift) - 1;
  const uint32_t item = base + blockIdx.x;
  uint32_t rest = item / d.pieces;
  const int64_t piece = item - rest * d.pieces;
  const int block = static_cast<int>(rest % d.blocks);
  rest /= d.blocks;
  const int head = static_cast<int>(rest % cache.heads);
  const int64_t row = rest / cache.heads;
  const int columns = min(kColumns, group - block * kColumns);
  const int q_head = head * group + block * kColumns;
  // LDS: the waves' results, the queries, the sums of the run and of the stretch so far
  const int live = min(kColumns, group);
  constexpr int STRIDE = DP + 4;
  float* joint = reinterpret_cast<float*>(shared);                                     // [wave][column][STRIDE]
  float2* joint_state = reinterpret_cast<float2*>(joint + kWaves * live * STRIDE);     // [wave][column]
  uint4* queries = reinterpret_cast<uint4*>(joint_state + kWaves * live);              // [KC][64]
  float4* so_far = reinterpret_cast<float4*>(queries + (QL ? KC * 64 : 0));            // [run, stretch][column][DP / 4]
  float2* so_far_state = reinterpret_cast<float2*>(so_far + 2 * live * (DP / 4));
  // queries: the first product's right operand, a column per lane's head
  constexpr int QN = QL ? (KC + kWaves - 1) / kWaves : KC;
  uint4 q[QN];
#pragma unroll
  for (int i = 0; i < QN; ++i) {
    const int c = QL ? i * kWaves + wave : i, at = 32 * c + 8 * g;
    q[i] = make_uint4(0, 0, 0, 0);
    if (c < KC && c16 < columns && at < dim) q[i] = load16(p.q + row * p.ldq + static_cast<int64_t>(q_head + c16) * dim + at);
  }
  // The pages and the open places of this wave's octets, an octet per lane; requested before the
  // row's length is known, unless a window hangs on it.
  const bool in_time = p.window == 0;
  Span span;
  if (!in_time) span = span_of(p, row);
  const int64_t first = (in_time ? 0 : span.begin) + piece * d.keys;
  const int take = MANY ? d.keys / S::kPart : 1;
  // the first key of this wave's tiles of part t, and of a lane's octet
  auto tile_key = [&](int t) { return first + (t * kWaves + wave) * (U * kTile); };
  const int octet_lane = min(lane, 4 * U * take - 1);
  const int64_t key_lane = tile_key(octet_lane / (4 * U)) + 8 * (octet_lane % (4 * U));
  int page_lane = -1;
  uint32_t here_lane = 0xff;
  if (cache.sequences > 0) {
    const int64_t sequence = p.sequence ? p.sequence[row] : row, place = key_lane >> cache.page_shift;
    const int32_t page = cache.tables[max(int64_t(0), min(sequence, cache.sequences - 1)) * cache.ldt +
                                      min(place, static_cast<int64_t>(cache.max_pages) - 1)];
    const bool there = sequence >= 0 && sequence < cache.sequences && place < cache.max_pages;
    page_lane = there && page >= 0 && page < cache.pages ? page : -1;
  }
  if (HOLES) here_lane = open_of(p.mask + row * p.ldm, key_lane, p.max_length);
  if (in_time) span = span_of(p, row);
  if (d.pieces > 1 && first >= span.hi) return;       // (the same for the whole workgroup)
  here_lane &= page_lane < 0 ? 0u : octet_of(span, key_lane);
  page_lane = max(page_lane, 0);                     // (read, if at all, and not used)

  // Weights are scaled by a power of two that keeps their sum, over all keys of the row, below 1: sums of values then stay within the
  // largest of them, and what follows is divided by the weights' sum anyway.
  const int bits = 64 - __clzll(static_cast<unsigned long long>(max(int64_t(0), span.hi - span.lo)));
  const float down = __uint_as_float(static_cast<uint32_t>(127 - bits) << 23);

  const int parts = MANY ? static_cast<int>(max(int64_t(1), min(static_cast<int64_t>(take), (span.hi - first + S::kPart - 1) / S::kPart))) : 1;
  // (a tile without keys of its row has none behind it)
  auto there = [&](int t) { return t < parts && tile_key(t) < span.hi; };
  uint4 kr[U][2][KC];
  uint32_t vr[U][8][VH][VW / 2];
  // A tile's keys and values.  Where there is no further tile, and at closed places, the address is the cache's first: it
  // stays in the L1, and there are no branches between the loads, around which the compiler would wait for all of them.
  auto load_keys = [&](int t) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int octet = 4 * (t * U + u) + (c16 >> 2);
      const int64_t key = tile_key(t) + u * kTile + 8 * (c16 >> 2) + (c16 & 3);
      const uint16_t* from = cache.keys + (there(t) ? token_at(cache, __shfl(page_lane, octet), head, key & page_mask) : 0);
      const uint32_t here = HOLES ? __shfl(here_lane, octet) : 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint16_t* row_from = from + 4 * h * dim;
        if (HOLES) row_from = here >> (4 * h + (c16 & 3)) & 1 ? row_from : cache.keys;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          int at = 32 * c + 8 * g;
          if (!EXACT && at >= dim) at = 0;             // (made 0 before it is used)
          kr[u][h][c] = *reinterpret_cast<const uint4*>(row_from + at);
        }
      }
    }
  };
  auto load_values = [&](int t) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int octet = 4 * (t * U + u) + g;
      const int64_t key = tile_key(t) + u * kTile + 8 * g;
      const uint16_t* from = cache.values + (there(t) ? token_at(cache, __shfl(page_lane, octet), head, key & page_mask) : 0);
      const uint32_t here = HOLES ? __shfl(here_lane, octet) : 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint16_t* row_from = from + j * dim;
        if (HOLES) row_from = here >> j & 1 ? row_from : cache.values;
#pragma unroll
        for (int h = 0; h < VH; ++h) {
          int at = 16 * VW * h + VW * c16;
          if (!EXACT && at >= dim) at = 0;             // (columns that are not stored)
          if constexpr (VW == 8) {
            const uint4 v = *reinterpret_cast<const uint4*>(row_from + at);
            vr[u][j][h][0] = v.x, vr[u][j][h][1] = v.y, vr[u][j][h][2] = v.z, vr[u][j][h][3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(row_from + at);
            vr[u][j][h][0] = v.x, vr[u][j][h][1] = v.y;
          }
        }
      }
    }
  };

  if (MANY) {
    load_keys(0);
    load_values(0);
  }
  if (QL) {
#pragma unroll
    for (int i = 0; i < QN; ++i)
      if (i * kWaves + wave < KC) queries[(i * kWaves + wave) * 64 + lane] = q[i];
    lds_barrier();                       // (the tile's requests go on)
  }
  for (int t = 0; t < parts; ++t) {
    float m = kNone, l = 0.f;
    f32x4 o[VH * VW];
#pragma unroll
    for (int i = 0; i < VH * VW; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (there(t)) {
    if (!MANY) {
      load_keys(t);
      load_values(t);
    }
    float s[U][8];
    f32x4 score[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) score[u][0] = score[u][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bf16x8 q_c = __builtin_bit_cast(bf16x8, QL ? queries[c * 64 + lane] : q[QL ? 0 : c]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 k = kr[u][h][c];
          if (!EXACT && 32 * c + 8 * g >= dim) k = make_uint4(0, 0, 0, 0);
          score[u][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), q_c, score[u][h], 0, 0, 0);
        }
      if (QL) __builtin_amdgcn_sched_barrier(0);       // (else all of the queries are in registers at once)
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[u][j] = score[u][j / 4][j % 4] * (p.scale * kLog2e);
    if (MANY) {
      load_keys(t + 1);
      asm volatile("" ::: "memory");     // (the requests stay where they are)
    }
    // What turns two keys' values into a pair of the left operand; of a key that does not count a 0 (whatever the cache holds).
    uint32_t pick[U][2][4];
    float top = kNone;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int j = 0; j < 4; ++j) pick[u][0][j] = 0x05040100u, pick[u][1][j] = 0x07060302u;
      const uint32_t here = __shfl(here_lane, 4 * (t * U + u) + g);
      if (!__all(here == 0xff)) {
        auto choose = [](uint32_t bits, uint32_t a, uint32_t b) { return (bits & a) | (~bits & b); };
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t a = static_cast<uint32_t>(static_cast<int32_t>(here << (31 - 2 * j)) >> 31);      // all bits the key's
          const uint32_t b = static_cast<uint32_t>(static_cast<int32_t>(here << (30 - 2 * j)) >> 31);
          s[u][2 * j] = __uint_as_float(choose(a, __float_as_uint(s[u][2 * j]), __float_as_uint(kNone)));
          s[u][2 * j + 1] = __uint_as_float(choose(b, __float_as_uint(s[u][2 * j + 1]), __float_as_uint(kNone)));
          const uint32_t both = __builtin_amdgcn_perm(b, a, 0x05040100u);
          pick[u][0][j] = choose(both, 0x05040100u, 0x0c0c0c0cu);
          pick[u][1][j] = choose(both, 0x07060302u, 0x0c0c0c0cu);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, s[u][j]);
    }
    m = other_rows_max(top);
    const float all = m == kNone ? 0.f : m;
    // The weights in three terms, each the next 8 bits cut off: together float32's 24.  (Two would be off by up to 2^-17 of each weight, one
    // by 2^-8.)  The second and third are at least 2^-30 of the weight and so not 0 where it is not (from 2^-64 of the largest on), so that a
    // seen key's infinite value stays one where 0 times it would be NaN; a weight of 0 adds nothing, however large the value.
    constexpr float kLeast = 9.31322574615478515625e-10f;
    auto high = [](float a) { return __uint_as_float(__float_as_uint(a) & 0xffff0000u); };
    auto pair = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); };
    bf16x8 weights[3][U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t bits[3][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a = __builtin_amdgcn_exp2f(s[u][2 * j] - all) * down, b = __builtin_amdgcn_exp2f(s[u][2 * j + 1] - all) * down;
        l += a;
        l += b;
        const float a_least = a * kLeast, b_least = b * kLeast;
        const float a1 = fmaxf(a - high(a), a_least), b1 = fmaxf(b - high(b), b_least);
        bits[0][j] = pair(a, b);
        bits[1][j] = pair(a1, b1);
        bits[2][j] = pair(fmaxf(a1 - high(a1), a_least), fmaxf(b1 - high(b1), b_least));
      }
#pragma unroll
      for (int w = 0; w < 3; ++w) weights[w][u] = __builtin_bit_cast(bf16x8, make_uint4(bits[w][0], bits[w][1], bits[w][2], bits[w][3]));
    }
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
      for (int i = 0; i < VW; ++i) {
        f32x4& acc = o[h * VW + i];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          uint32_t a[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) a[j] = __builtin_amdgcn_perm(vr[u][2 * j + 1][h][i / 2], vr[u][2 * j][h][i / 2], pick[u][i & 1][j]);
          const bf16x8 v = __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3]));
#pragma unroll
          for (int w = 0; w < 3; ++w) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, weights[w][u], acc, 0, 0, 0);
        }
        if (i & 1) __builtin_amdgcn_sched_barrier(0);      // (else all operands are made first, in registers that there are not)
      }
    if (MANY) {
      load_values(t + 1);
      asm volatile("" ::: "memory");
    }
    }

    // the waves' results joined in order, the part to its run, the run to its stretch
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (MANY && t > 0) lds_barrier();    // (the part before has been read)
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));     // (what follows from it is made here, not kept in registers through the loop)
    const int col_here = thread & 15, g_here = thread >> 4 & 3;
    if (col_here < columns) {
      if (g_here == 0) joint_state[wave * live + col_here] = make_float2(m, l);
      float* to = joint + (wave * live + col_here) * STRIDE + 4 * VW * g_here;
#pragma unroll
      for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < VW; i += 4)
            *reinterpret_cast<float4*>(to + 16 * VW * h + VW * r + i) =
                make_float4(o[h * VW + i][r], o[h * VW + i + 1][r], o[h * VW + i + 2][r], o[h * VW + i + 3][r]);
    }
    lds_barrier();
    const bool last = t + 1 == parts;
    const int items = live * (DP / 4);
    for (int e = thread; e < columns * (DP / 4); e += kThreads) {
      const int col = e / (DP / 4), at = e % (DP / 4) * 4;
      Sum sum;
      sum.top = kNone, sum.total = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum.top = fmaxf(sum.top, joint_state[w * live + col].x);
      const float all = sum.top == kNone ? 0.f : sum.top;
      sum.v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 state = joint_state[w * live + col];
        const float f = __builtin_amdgcn_exp2f(state.x - all);
        const float4 v = *reinterpret_cast<const float4*>(joint + (w * live + col) * STRIDE + at);
        sum.v.x = __builtin_fmaf(f, v.x, sum.v.x), sum.v.y = __builtin_fmaf(f, v.y, sum.v.y);
        sum.v.z = __builtin_fmaf(f, v.z, sum.v.z), sum.v.w = __builtin_fmaf(f, v.w, sum.v.w);
        sum.total = __builtin_fmaf(f, state.y, sum.total);
      }
      if (MANY) {
        auto before = [&](int i) { return Sum{so_far[i], so_far_state[i].x, so_far_state[i].y}; };
        auto keep = [&](int i) { so_far[i] = sum.v, so_far_state[i] = make_float2(sum.top, sum.total); };
        if (t % S::kRun) sum = join(before(e), sum);
        if (!last && (t + 1) % S::kRun) {
          keep(e);
          continue;
        }
        if (t >= S::kRun) sum = join(before(items + e), sum);
        if (!last) {
          keep(items + e);
          continue;
        }
      }
      if (at >= dim) continue;
      if (d.sums) {
        const int64_t slot = (row * p.q_heads + q_head + col) * d.pieces + piece;
        *reinterpret_cast<float4*>(d.sums + slot * dim + at) = sum.v;
        if (at == 0) d.state[slot] = make_float2(sum.top, sum.total);
      } else {
        finish(p.out + row * p.ldo + static_cast<int64_t>(q_head + col) * dim + at, sum);
      }
    }
  }
}

// The pieces of one row and query head joined, 64 values of the head per workgroup: 16 threads of
// four values by 16 slices.  A slice joins PER pieces (the parts of a run, the runs of a stretch, or one stretch);
// then the runs of each stretch (RUNS), then the stretches, in order.
template <int PER, bool RUNS>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendArgs p, Parts d, uint32_t base) {
  constexpr int COLS = 16, SLICES = kThreads / COLS, STEP = SLICES * PER;
  __shared__ float4 sums[2][SLICES][COLS];
  __shared__ float2 states[2][SLICES];
  const int col = threadIdx.x % COLS, slice = threadIdx.x / COLS;
  const uint32_t chunks = (p.cache.dim + 63) / 64;
  const uint32_t item = base + blockIdx.x;
  const uint32_t of = item / chunks;
  const int at = static_cast<int>(item - of * chunks) * 64 + 4 * col;
  const int64_t row = of / p.q_heads;
  const bool live = at < p.cache.dim;
  const int last = static_cast<int>(d.pieces) - 1;
  const float2* state = d.state + static_cast<int64_t>(of) * d.pieces;
  const float* from = d.sums + static_cast<int64_t>(of) * d.pieces * p.cache.dim + (live ? at : 0);
  float2 s[PER];
  float4 v[PER];
  // (requested before the row's length is known, and ahead: past it the workspace holds anything, which is not used)
  auto request = [&](int i0) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = min(i0 + slice * PER + j, last);
      s[j] = state[i];
      v[j] = *reinterpret_cast<const float4*>(from + static_cast<int64_t>(i) * p.cache.dim);
    }
  };
  request(0);
  const Span span = span_of(p, row);
  const int pieces = span.hi > span.lo ? static_cast<int>((span.hi - span.begin + d.keys - 1) / d.keys) : 0;
  Sum all{make_float4(0.f, 0.f, 0.f, 0.f), kNone, 0.f};
  for (int i0 = 0, turn = 0; i0 < pieces; i0 += STEP, turn ^= 1) {
    Sum own{v[0], s[0].x, s[0].y};
#pragma unroll
    for (int j = 1; j < PER; ++j)
      if (i0 + slice * PER + j < pieces) own = join(own, Sum{v[j], s[j].x, s[j].y});
    const int units = min((pieces - i0 + PER - 1) / PER, SLICES);     // that there are
    auto put = [&] {
      sums[turn][slice][col] = own.v;
      if (col == 0) states[turn][slice] = make_float2(own.top, own.total);
    };
    auto get = [&](int i) { return Sum{sums[turn][i][col], states[turn][i].x, states[turn][i].y}; };
    put();
    if (i0 + STEP < pieces) request(i0 + STEP);
    lds_barrier();
    if constexpr (RUNS) {
      if (slice % kFour == 0 && slice < units) {
        for (int i = slice + 1; i < min(slice + kFour, units); ++i) own = join(own, get(i));
        put();
      }
      lds_barrier();
    }
    if (slice == 0) {
      all = i0 == 0 ? own : join(all, own);
      for (int i = RUNS ? kFour : 1; i < units; i += RUNS ? kFour : 1) all = join(all, get(i));
    }
  }
  if (slice == 0 && live) finish(p.out + row * p.ldo + static_cast<int64_t>(of - row * p.q_heads) * p.cache.dim + at, all);
}

// workgroups of a launch (a grid counts fewer than 2^32 threads)
constexpr uint32_t kMaxGrid = 1u << 23;

int part_keys(int dim) { return dim <= 64 ? Shape<64>::kPart : Shape<128>::kPart; }

// What a workgroup takes, by the stretches that there are (heads of the cache x rows x capacity): a whole one from three per CU on
// (768 of 128 dims: 144 us, in runs 150, in parts 158; 1024: 190, 197, 208), but from one per CU on if rows are of 16 or
// more, whose unequal lengths then leave little idle (256 of 256 dims: 108 us, 115 in runs); fewer leave CUs idle
// and each takes 20 to 60 us by itself (64 of 128 dims: 36 us, 17 in runs or parts).  Runs from one stretch per CU on
// (384 of 128 dims: 79 us, in parts 83), for 64 dims never (384: 47 in parts and 56, with a mask 34 and 38).  Stretches of 64 dims are as
// fast as parts where lengths are unequal and masked (768: 61 and 62 us), up to 15 % slower where they are equal (1024: 131, 114).
// The capacity stands for the lengths, which the host does not know: far above them few workgroups have all the work (one row of
// 4095 keys, 32 heads on 8 of 128: 10 us, with a table for 32768 tokens 15, for 131072 49).
Parts parts_of(int64_t n, int q_heads, int heads, int dim, int64_t max_length, int64_t window, void* workspace) {
  Parts d;
  const int64_t longest = window ? std::min(max_length, window + kTile - 1) : max_length;
  const int group = q_heads / heads;
  d.blocks = static_cast<uint32_t>((group + kColumns - 1) / kColumns);
  auto pieces = [&](int keys) { return std::max<int64_t>(1, (longest + keys - 1) / keys); };
  const int64_t groups = n * heads * d.blocks;
  const int64_t stretches = groups * longest / kStretchKeys;
  d.keys = stretches >= (longest >= 16 * kStretchKeys ? 256 : 768) ? kStretchKeys : stretches >= 256 && dim > 64 ? kRunKeys : part_keys(dim);
  d.pieces = static_cast<uint32_t>(pieces(d.keys));
  d.sums = d.pieces > 1 ? static_cast<float*>(workspace) : nullptr;
  d.state = d.sums ? reinterpret_cast<float2*>(d.sums + n * q_heads * d.pieces * dim) : nullptr;
  return d;
}

template <int DP, bool EXACT, bool HOLES, bool MANY>
void launch(const AttendArgs& a, const Parts& d, uint32_t items, hipStream_t stream) {
  const int live = std::min(kColumns, a.q_heads / a.cache.heads);
  const size_t lds = static_cast<size_t>(kWaves) * live * (4 * (DP + 4) + 8) + (MANY && DP >= 128 ? DP / 32 * 1024 : 0) +
                     (MANY ? static_cast<size_t>(2 * live) * (DP / 4) * 24 : 0);
  for (uint32_t base = 0; base < items; base += kMaxGrid) {
    hipLaunchKernelGGL((attend_kernel<DP, EXACT, HOLES, MANY>), dim3(std::min(items - base, kMaxGrid)), dim3(kThreads), lds, stream, a, d, base);
    launched("attention");
  }
}

template <int DP, bool EXACT, bool HOLES>
void launch(const AttendArgs& a, const Parts& d, uint32_t items, hipStream_t stream) {
  if (d.keys > Shape<DP>::kPart)
    launch<DP, EXACT, HOLES, true>(a, d, items, stream);
  else
    launch<DP, EXACT, HOLES, false>(a, d, items, stream);
}

template <int DP>
void launch(const AttendArgs& a, const Parts& d, uint32_t items, hipStream_t stream) {
  if (a.cache.dim == DP && !a.mask)
    launch<DP, true, false>(a, d, items, stream);
  else if (a.cache.dim == DP)
    launch<DP, true, true>(a, d, items, stream);
  else if (!a.mask)
    launch<DP, false, false>(a, d, items, stream);
  else
    launch<DP, false, true>(a, d, items, stream);
}

}  // namespace

size_t decode_attend_workspace(int64_t n, int q_heads, int heads, int dim, int64_t max_length, int64_t window) {
  const Parts d = parts_of(n, q_heads, heads, dim, max_length, window, nullptr);
  return d.pieces > 1 ? static_cast<size_t>(n) * q_heads * d.pieces * (static_cast<size_t>(dim) * 4 + 8) : 0;
}

bool decode_attend(const AttendArgs& a, hipStream_t stream) {
  const Parts d = parts_of(a.n, a.q_heads, a.cache.heads, a.cache.dim, a.max_length, a.window, a.workspace);
  const int64_t groups = a.n * a.cache.heads * d.blocks;        // (n * q_heads fits 32 bits, so do these)
  if (groups * d.pieces >= int64_t(1) << 31 || a.n * a.q_heads * ((a.cache.dim + 63) / 64) >= int64_t(1) << 31) return false;
  const uint32_t items = static_cast<uint32_t>(groups * d.pieces);
  if (a.cache.dim <= 64)
    launch<64>(a, d, items, stream);
  else if (a.cache.dim <= 128)
    launch<128>(a, d, items, stream);
  else
    launch<256>(a, d, items, stream);
  if (!d.sums) return true;
  const uint32_t joins = static_cast<uint32_t>(a.n * a.q_heads) * ((a.cache.dim + 63) / 64);
  for (uint32_t base = 0; base < joins; base += kMaxGrid) {
    const dim3 grid(std::min(joins - base, kMaxGrid));
    const dim3 threads(kThreads);
    if (d.keys == kStretchKeys)
      hipLaunchKernelGGL((join_kernel<1, false>), grid, threads, 0, stream, a, d, base);
    else if (d.keys == kRunKeys)
      hipLaunchKernelGGL((join_kernel<kFour, false>), grid, threads, 0, stream, a, d, base);
    else if (d.keys == 256)
      hipLaunchKernelGGL((join_kernel<2, true>), grid, threads, 0, stream, a, d, base);
    else
      hipLaunchKernelGGL((join_kernel<4, true>), grid, threads, 0, stream, a, d, base);
    launched("attention's join");
  }
  return true;
}

}  // namespace k
}  // namespace dycl
