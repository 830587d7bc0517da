// Attention of single tokens to a paged cache:
//   out = sum_j p_j v_j,  p = softmax_j(scale * q . k_j)
// over the keys of a row's sequence, in one pass with the running maximum and sum of
// the softmax.  The query heads that share a head of the cache are the columns of the
// matrix instructions, so keys and values are read once for up to 16 of them.
//
// Bound by HBM: 4 dim bytes per key and head of the cache, for 4 dim operations per query
// head.
//
// A tile is 32 keys of one head.  Scores are K Q^T: row i of the first matrix
// instruction of two is key 8 (i / 4) + i % 4 of the tile, of the second 4 more, so a lane's
// eight scores are eight consecutive keys, an octet, which never leaves a page; and they
// lie as the second product, V^T P^T, takes its right operand: the softmax's weights go from
// one product to the other in registers.  A lane loads eight (four, for heads of 64)
// neighbouring values of its octet's eight rows, whole rows per 16 lanes, and turns that square around
// in registers for the left operand.  Nothing passes LDS until the end.
//
// A workgroup of four waves takes a part, `tiles` tiles per wave; waves join
// through LDS, parts through the workspace and a second kernel, each in order.
// The size of a part follows from the capacity, not from the number of rows: a row's bits
// do not depend on its company.
#include "decode_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kThreads = 256, kWaves = 4, kTile = 32, kColumns = 16;
constexpr float kNone = -__builtin_inff(), kLog2e = 1.44269504088896340736f;

// How the keys are divided; the same for all rows.
struct Parts {
  int tiles;                     // per wave
  int keys;                      // of a part
  uint32_t parts;                // of the longest row
  uint32_t blocks;                  // of kColumns query heads that share a head
  float* sums;                   // [row][query head][part][dim], null where one part is all
  float2* state;                 // [row][query head][part]: maximum (of scores in base 2), sum
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

__device__ __forceinline__ float other_rows_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// Dims of the heads padded to DP; EXACT: they are DP.
template <int DP, bool EXACT>
__global__ __launch_bounds__(kThreads) void attend_kernel(AttendArgs p, Parts d, uint32_t items) {
  constexpr int KC = DP / 32;                          // steps of 32 dims of the first product
  constexpr int VW = DP >= 128 ? 8 : 4, VH = DP / (16 * VW);   // a lane's neighbouring values, and how many such
  constexpr int STRIDE = DP + 4;
  __shared__ float joint[kWaves][kColumns][STRIDE];
  __shared__ float2 joint_state[kWaves][kColumns];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c16 = lane & 15, g = lane >> 4;
  const PagedArgs& cache = p.cache;
  const int dim = EXACT ? DP : cache.dim;
  const int group = p.q_heads / cache.heads;
  const int64_t page_mask = (int64_t(1) << cache.page_shift) - 1;
  for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
    uint32_t rest = item / d.parts;
    const int64_t part = item - rest * d.parts;
    const int block = static_cast<int>(rest % d.blocks);
    rest /= d.blocks;
    const int head = static_cast<int>(rest % cache.heads);
    const int64_t row = rest / cache.heads;
    const Span span = span_of(p, row);
    const int64_t first = span.begin + part * d.keys;
    if (d.parts > 1 && first >= span.hi) continue;     // (the same for the whole workgroup)
    const int columns = min(kColumns, group - block * kColumns);
    const int q_head = head * group + block * kColumns;

    // queries: the right operand, a column per lane's head
    bf16x8 q[KC];
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      uint4 v = make_uint4(0, 0, 0, 0);
      const int at = 32 * c + 8 * g;
      if (c16 < columns && at < dim) v = load16(p.q + row * p.ldq + static_cast<int64_t>(q_head + c16) * dim + at);
      q[c] = __builtin_bit_cast(bf16x8, v);
    }

    // this wave's octets' pages, one per lane
    const int64_t begin = first + static_cast<int64_t>(wave) * d.tiles * kTile;
    const int64_t sequence = p.sequence ? p.sequence[row] : row;
    int page_lane = -1;
    if (lane < 4 * d.tiles && begin + 8 * lane < span.hi) page_lane = static_cast<int>(page_of(cache, sequence, begin + 8 * lane));

    float m = kNone, l = 0.f;
    f32x4 o[VH * VW];
#pragma unroll
    for (int i = 0; i < VH * VW; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int tiles = static_cast<int>(max(int64_t(0), min(static_cast<int64_t>(d.tiles), (span.hi - begin + kTile - 1) / kTile)));
    for (int t = 0; t < tiles; ++t) {
      const int64_t key = begin + t * kTile;
      const int page_k = __shfl(page_lane, 4 * t + (c16 >> 2)), page_v = __shfl(page_lane, 4 * t + g);
      const int64_t key_k = key + 8 * (c16 >> 2) + (c16 & 3), key_v = key + 8 * g;
      const uint16_t* kp = cache.keys + token_at(cache, max(page_k, 0), head, key_k & page_mask);
      const uint16_t* vp = cache.values + token_at(cache, max(page_v, 0), head, key_v & page_mask);
      uint4 kr[2][KC];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const int at = 32 * c + 8 * g;
          kr[h][c] = make_uint4(0, 0, 0, 0);
          if (EXACT || at < dim) kr[h][c] = *reinterpret_cast<const uint4*>(kp + 4 * h * dim + at);
        }
      uint32_t vr[8][VH][VW / 2];
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int h = 0; h < VH; ++h) {
          int at = 16 * VW * h + VW * c16;
          if (!EXACT && at >= dim) at = 0;             // (columns that are not stored)
          if constexpr (VW == 8) {
            const uint4 v = *reinterpret_cast<const uint4*>(vp + j * dim + at);
            vr[j][h][0] = v.x, vr[j][h][1] = v.y, vr[j][h][2] = v.z, vr[j][h][3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(vp + j * dim + at);
            vr[j][h][0] = v.x, vr[j][h][1] = v.y;
          }
        }

      // which keys of the lane's octet count
      uint32_t here = 0;
      if (page_v >= 0) {
        const int hi = static_cast<int>(max(int64_t(0), min(int64_t(8), span.hi - key_v)));
        const int lo = static_cast<int>(max(int64_t(0), min(int64_t(8), span.lo - key_v)));
        here = ((1u << hi) - 1) & ~((1u << lo) - 1);
        if (p.mask) {
          const uint8_t* mask = p.mask + row * p.ldm + key_v;
          uint32_t open = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (here >> j & 1) open |= (mask[j] != 0 ? 1u : 0u) << j;
          here = open;
        }
      }

      float s[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[h][c]), q[c], acc, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[4 * h + r] = acc[r] * (p.scale * kLog2e);
      }
      if (!__all(here == 0xff)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool on = here >> j & 1;
          s[j] = on ? s[j] : kNone;
#pragma unroll
          for (int h = 0; h < VH; ++h)
#pragma unroll
            for (int w = 0; w < VW / 2; ++w) vr[j][h][w] = on ? vr[j][h][w] : 0u;
        }
      }
      float top = s[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
      const float now = fmaxf(m, other_rows_max(top));
      const float base = now == kNone ? 0.f : now;
      const float scale = __builtin_amdgcn_exp2f(m - base);
      m = now;
      l *= scale;
      if (!__all(scale == 1.f)) {
#pragma unroll
        for (int i = 0; i < VH * VW; ++i) o[i] *= scale;
      }
      // The weights in two terms (a single bf16 would be off by up to 2^-8 of each): the first is
      // the weight cut off after 8 bits, the second the rest, never 0, so that a seen key's infinite value
      // stays one where 0 times it would be NaN; 2^-126 of a value is below its sum's rounding.
      constexpr float kLeast = 1.17549435e-38f;
      uint32_t ph[4], pl[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a = __builtin_amdgcn_exp2f(s[2 * j] - base), b = __builtin_amdgcn_exp2f(s[2 * j + 1] - base);
        l += a;
        l += b;
        ph[j] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
        pl[j] = pack_bf16(fmaxf(a - __uint_as_float(ph[j] << 16), kLeast), fmaxf(b - __uint_as_float(ph[j] & 0xffff0000u), kLeast));
      }
      const bf16x8 p_hi = __builtin_bit_cast(bf16x8, make_uint4(ph[0], ph[1], ph[2], ph[3]));
      const bf16x8 p_lo = __builtin_bit_cast(bf16x8, make_uint4(pl[0], pl[1], pl[2], pl[3]));
#pragma unroll
      for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int i = 0; i < VW; ++i) {
          uint32_t a[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            a[j] = __builtin_amdgcn_perm(vr[2 * j + 1][h][i / 2], vr[2 * j][h][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
          const bf16x8 v = __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3]));
          f32x4& acc = o[h * VW + i];
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p_hi, acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p_lo, acc, 0, 0, 0);
        }
    }

    // the waves' results, joined in order
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (c16 < columns) {
      if (g == 0) joint_state[wave][c16] = make_float2(m, l);
#pragma unroll
      for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < VW; i += 4) {
            const int at = 16 * VW * h + VW * (4 * g + r) + i;
            *reinterpret_cast<float4*>(&joint[wave][c16][at]) =
                make_float4(o[h * VW + i][r], o[h * VW + i + 1][r], o[h * VW + i + 2][r], o[h * VW + i + 3][r]);
          }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < columns * (DP / 4); e += kThreads) {
      const int col = e / (DP / 4), at = e % (DP / 4) * 4;
      float top = kNone;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, joint_state[w][col].x);
      const float base = top == kNone ? 0.f : top;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(joint_state[w][col].x - base);
        const float4 v = *reinterpret_cast<const float4*>(&joint[w][col][at]);
        sum.x += f * v.x, sum.y += f * v.y, sum.z += f * v.z, sum.w += f * v.w;
        total += f * joint_state[w][col].y;
      }
      if (at >= dim) continue;
      if (d.sums) {
        const int64_t slot = (row * p.q_heads + q_head + col) * d.parts + part;
        *reinterpret_cast<float4*>(d.sums + slot * dim + at) = sum;
        if (at == 0) d.state[slot] = make_float2(top, total);
      } else {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        uint16_t* out = p.out + row * p.ldo + static_cast<int64_t>(q_head + col) * dim + at;
        out[0] = f2bf(sum.x * inv), out[1] = f2bf(sum.y * inv), out[2] = f2bf(sum.z * inv), out[3] = f2bf(sum.w * inv);
      }
    }
    __syncthreads();             // (the next item's results)
  }
}

// The parts' sums of one row and query head: threads of DP / 4 columns by slices of parts.
template <int DP>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendArgs p, Parts d, int64_t items) {
  constexpr int COLS = DP / 4, SLICES = kThreads / COLS;
  __shared__ float tops[kWaves];
  __shared__ float4 sums[SLICES][COLS];
  __shared__ float totals[SLICES];
  const int col = threadIdx.x % COLS, slice = threadIdx.x / COLS;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row = item / p.q_heads;
    const Span span = span_of(p, row);
    const int64_t parts = span.hi > span.lo ? (span.hi - span.begin + d.keys - 1) / d.keys : 0;
    const float2* state = d.state + item * d.parts;
    const float* from = d.sums + item * d.parts * p.cache.dim;
    float top = kNone;
    for (int64_t i = threadIdx.x; i < parts; i += kThreads) top = fmaxf(top, state[i].x);
#pragma unroll
    for (int w = 1; w < 64; w *= 2) top = fmaxf(top, __shfl_xor(top, w));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float base = top == kNone ? 0.f : top;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    float total = 0.f;
    if (4 * col < p.cache.dim)
#pragma unroll 4
      for (int64_t i = slice; i < parts; i += SLICES) {
        const float2 s = state[i];
        const float4 v = *reinterpret_cast<const float4*>(from + i * p.cache.dim + 4 * col);
        const float f = __builtin_amdgcn_exp2f(s.x - base);
        sum.x += f * v.x, sum.y += f * v.y, sum.z += f * v.z, sum.w += f * v.w;
        total += f * s.y;
      }
    sums[slice][col] = sum;
    if (col == 0) totals[slice] = total;
    __syncthreads();
    if (slice == 0 && 4 * col < p.cache.dim) {
#pragma unroll
      for (int i = 1; i < SLICES; ++i) {
        const float4 v = sums[i][col];
        sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
        total += totals[i];
      }
      const float inv = total == 0.f ? 0.f : 1.f / total;
      uint16_t* out = p.out + row * p.ldo + (item - row * p.q_heads) * p.cache.dim + 4 * col;
      out[0] = f2bf(sum.x * inv), out[1] = f2bf(sum.y * inv), out[2] = f2bf(sum.z * inv), out[3] = f2bf(sum.w * inv);
    }
    __syncthreads();
  }
}

constexpr int64_t kMaxGrid = int64_t(1) << 22;

Parts parts_of(int64_t n, int q_heads, int heads, int dim, int64_t max_length, int64_t window, void* workspace) {
  Parts d;
  const int64_t longest = window ? std::min(max_length, window + kTile - 1) : max_length;
  const int group = q_heads / heads;
  d.tiles = longest <= 4096 ? 1 : 4;
  d.keys = kWaves * kTile * d.tiles;
  d.parts = static_cast<uint32_t>(std::max<int64_t>(1, (longest + d.keys - 1) / d.keys));
  d.blocks = static_cast<uint32_t>((group + kColumns - 1) / kColumns);
  d.sums = d.parts > 1 ? static_cast<float*>(workspace) : nullptr;
  d.state = d.sums ? reinterpret_cast<float2*>(d.sums + n * q_heads * d.parts * dim) : nullptr;
  return d;
}

template <int DP>
void launch(const AttendArgs& a, const Parts& d, uint32_t items, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(items, kMaxGrid)));
  if (a.cache.dim == DP)
    hipLaunchKernelGGL((attend_kernel<DP, true>), grid, dim3(kThreads), 0, stream, a, d, items);
  else
    hipLaunchKernelGGL((attend_kernel<DP, false>), grid, dim3(kThreads), 0, stream, a, d, items);
  launched("attention");
  if (!d.sums) return;
  const int64_t rows = a.n * a.q_heads;
  hipLaunchKernelGGL(join_kernel<DP>, dim3(static_cast<unsigned>(std::min(rows, kMaxGrid))), dim3(kThreads), 0, stream, a, d, rows);
  launched("attention's join");
}

}  // namespace

size_t decode_attend_workspace(int64_t n, int q_heads, int heads, int dim, int64_t max_length, int64_t window) {
  const Parts d = parts_of(n, q_heads, heads, dim, max_length, window, nullptr);
  return d.parts > 1 ? static_cast<size_t>(n) * q_heads * d.parts * (static_cast<size_t>(dim) * 4 + 8) : 0;
}

bool decode_attend(const AttendArgs& a, hipStream_t stream) {
  const Parts d = parts_of(a.n, a.q_heads, a.cache.heads, a.cache.dim, a.max_length, a.window, a.workspace);
  const int64_t groups = a.n * a.cache.heads * d.blocks;        // (n * q_heads fits 32 bits, so do these)
  if (groups * d.parts >= int64_t(1) << 31) return false;
  const uint32_t items = static_cast<uint32_t>(groups * d.parts);
  if (a.cache.dim <= 64)
    launch<64>(a, d, items, stream);
  else if (a.cache.dim <= 128)
    launch<128>(a, d, items, stream);
  else
    launch<256>(a, d, items, stream);
  return true;
}

}  // namespace k
}  // namespace dycl
