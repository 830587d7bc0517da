// Heads turned by their positions, alone or on the way into the paged cache, and the
// cache's reordering behind a choice of beams.
//
// Rotation of the pair (a, b) by t = position * frequency: a cos t - b sin t,
// b cos t + a sin t.  t in float32 loses 0.06 at position 10^6, so it is float64 until
// it is reduced to an eighth of a turn around the nearest quarter; sine and cosine of
// that are Taylor polynomials in float32 (remainders below 2^-28 at pi / 4).
//
// Bound by HBM: every value is read and written once.  A workgroup takes a tile of rows;
// their cosines and sines are made once into LDS for all of a row's heads, then a lane
// takes eight pairs (16 bytes of each half in bf16, at any alignment) or eight
// neighbours.
#include "decode_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kThreads = 256, kMaxRows = 64, kTableSize = 2048;

// (cos, sin) of position * frequency
__device__ __forceinline__ float2 turn(int32_t position, double frequency) {
  double t = static_cast<double>(position) * frequency * 0.15915494309189533577;   // in turns
  t -= rint(t);
  const double quarter = rint(t * 4.0);
  const float x = static_cast<float>((t - quarter * 0.25) * 6.283185307179586477);
  const float x2 = x * x;
  float s = __builtin_fmaf(x2, 1.f / 362880.f, -1.f / 5040.f);
  s = __builtin_fmaf(x2, s, 1.f / 120.f);
  s = __builtin_fmaf(x2, s, -1.f / 6.f);
  s = __builtin_fmaf(x2 * x, s, x);
  float c = __builtin_fmaf(x2, -1.f / 3628800.f, 1.f / 40320.f);
  c = __builtin_fmaf(x2, c, -1.f / 720.f);
  c = __builtin_fmaf(x2, c, 1.f / 24.f);
  c = __builtin_fmaf(x2, c, -0.5f);
  c = __builtin_fmaf(x2, c, 1.f);
  const int n = static_cast<int>(quarter) & 3;
  const float cc = n & 1 ? s : c, ss = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -cc : cc, n >= 2 ? -ss : ss);
}

// x / d for x * d < 2^32, m = ceil(2^32 / d) (d > 1; 0 stands for d = 1)
struct Divide {
  uint32_t m;
  explicit Divide(int d) : m(d > 1 ? static_cast<uint32_t>(((uint64_t(1) << 32) + d - 1) / d) : 0) {}
  __device__ int operator()(int x) const { return m ? static_cast<int>(__umulhi(static_cast<uint32_t>(x), m)) : x; }
};

struct Units {
  int rows;                      // of a tile
  int turned, copied, plain;     // units of a head's turned and other values, of a head of v
  int of_q, of_row;              // units of q's heads, of a whole row
  Divide row, head, v_head;
};

template <bool F32>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs p, Units u) {
  __shared__ float2 table[kTableSize];
  __shared__ int64_t pages[kMaxRows];          // page of the row's token, -1: none
  __shared__ int32_t places[kMaxRows];
  const int t = threadIdx.x, per_head = u.turned + u.copied;
  const size_t size = F32 ? 4 : 2;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * u.rows; r0 < p.n; r0 += static_cast<int64_t>(gridDim.x) * u.rows) {
    const int rows = static_cast<int>(min(p.n - r0, static_cast<int64_t>(u.rows)));
    for (int r = t; r < rows; r += kThreads) {
      const int32_t at = p.positions[r0 + r];
      places[r] = at;
      pages[r] = p.k ? page_of(p.cache, p.sequence ? p.sequence[r0 + r] : r0 + r, at) : -1;
    }
    for (int i = t; i < rows * p.pairs; i += kThreads) {
      const int r = i / p.pairs;
      float2 cs = turn(p.positions[r0 + r], p.frequencies[i - r * p.pairs]);
      cs.x *= p.magnitude;
      cs.y *= p.magnitude * p.sign;
      table[i] = cs;
    }
    __syncthreads();
    for (int i = t; i < rows * u.of_row; i += kThreads) {
      const int r = u.row(i);
      int w = i - r * u.of_row;
      const char* from;
      char* to;
      bool to_cache = true, turned;
      int first, count, head;
      if (w < u.of_q) {
        head = u.head(w);
        w -= head * per_head;
        from = static_cast<const char*>(p.q) + (static_cast<size_t>(r0 + r) * p.ldq + static_cast<size_t>(head) * p.dim) * size;
        to = static_cast<char*>(p.q_out) + (static_cast<size_t>(r0 + r) * p.ldo + static_cast<size_t>(head) * p.dim) * size;
        to_cache = false;
        turned = w < u.turned;
      } else {
        if (pages[r] < 0) continue;
        w -= u.of_q;
        const bool is_v = w >= p.cache.heads * per_head;
        if (is_v) {
          w -= p.cache.heads * per_head;
          head = u.v_head(w);
          w -= head * u.plain;
        } else {
          head = u.head(w);
          w -= head * per_head;
        }
        from = static_cast<const char*>(is_v ? p.v : p.k) +
               (static_cast<size_t>(r0 + r) * (is_v ? p.ldv : p.ldk) + static_cast<size_t>(head) * p.dim) * size;
        const int64_t slot = places[r] & ((1 << p.cache.page_shift) - 1);
        to = reinterpret_cast<char*>((is_v ? p.cache.values : p.cache.keys) + token_at(p.cache, pages[r], head, slot));
        turned = !is_v && w < u.turned;
        if (is_v) w += u.turned;               // (counted as copied from the head's first value)
        first = is_v ? 0 : 2 * p.pairs;
        first += 8 * (w - u.turned);
      }
      if (!to_cache) first = 2 * p.pairs + 8 * (w - u.turned);
      float a[8], b[8];
      if (!turned) {
        count = min(8, p.dim - first);
        read8<F32>(from + first * size, count, a);
        if (to_cache)
          write8<false>(to + first * 2, count, a);
        else {
          if (p.padding && places[r] < 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) a[j] = 0.f;
          write8<F32>(to + first * size, count, a);
        }
        continue;
      }
      const bool none = !to_cache && p.padding && places[r] < 0;
      const float2* cs = table + r * p.pairs;
      if (p.interleaved) {
        first = 8 * w;
        count = min(8, 2 * p.pairs - first);
        read8<F32>(from + first * size, count, a);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 c = cs[min(4 * w + j, p.pairs - 1)];
          b[2 * j] = none ? 0.f : a[2 * j] * c.x - a[2 * j + 1] * c.y;
          b[2 * j + 1] = none ? 0.f : a[2 * j + 1] * c.x + a[2 * j] * c.y;
        }
        if (to_cache)
          write8<false>(to + first * 2, count, b);
        else
          write8<F32>(to + first * size, count, b);
      } else {
        first = 8 * w;
        count = min(8, p.pairs - first);
        read8<F32>(from + first * size, count, a);
        read8<F32>(from + (p.pairs + first) * size, count, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 c = cs[min(first + j, p.pairs - 1)];
          const float y = a[j] * c.x - b[j] * c.y;
          b[j] = none ? 0.f : b[j] * c.x + a[j] * c.y;
          a[j] = none ? 0.f : y;
        }
        if (to_cache) {
          write8<false>(to + first * 2, count, a);
          write8<false>(to + (p.pairs + first) * 2, count, b);
        } else {
          write8<F32>(to + first * size, count, a);
          write8<F32>(to + (p.pairs + first) * size, count, b);
        }
      }
    }
    __syncthreads();             // (the next tile's table)
  }
}

// A row's table and length, and the begun page's tokens: one workgroup per row and head.
__global__ __launch_bounds__(kThreads) void fork_kernel(ForkArgs p) {
  const int heads = p.cache.keys ? p.cache.heads : 1;
  for (int64_t i = blockIdx.x; i < p.n * heads; i += gridDim.x) {
    const int64_t row = i / heads;
    const int head = static_cast<int>(i - row * heads);
    const int64_t parent = p.parents[row];
    const bool live = parent >= 0 && parent < p.cache.sequences;
    int64_t length = live ? p.lengths[parent] : 0;
    length = max(int64_t(0), min(length, static_cast<int64_t>(p.cache.max_pages) << p.cache.page_shift));
    const int64_t begun = length >> p.cache.page_shift;
    const int used = static_cast<int>(length & ((1 << p.cache.page_shift) - 1));
    if (head == 0 && p.new_tables) {
      if (threadIdx.x == 0) p.new_lengths[row] = static_cast<int32_t>(length);
      for (int j = threadIdx.x; j < p.cache.max_pages; j += kThreads)
        p.new_tables[row * p.ldn + j] = !live ? -1 : j == begun ? p.fresh[row] : p.cache.tables[parent * p.cache.ldt + j];
    }
    if (!p.cache.keys || !used) continue;
    const int64_t from = page_of(p.cache, parent, length), to = p.fresh[row];
    if (from < 0 || to < 0 || to >= p.cache.pages || to == from) continue;
    const int64_t a = token_at(p.cache, from, head, 0), b = token_at(p.cache, to, head, 0);
    const int vectors = used * (p.cache.dim / 8);
    for (int j = threadIdx.x; j < 2 * vectors; j += kThreads) {
      uint16_t* t = j < vectors ? p.cache.keys : p.cache.values;
      const int64_t at = 8 * static_cast<int64_t>(j < vectors ? j : j - vectors);
      *reinterpret_cast<uint4*>(t + b + at) = *reinterpret_cast<const uint4*>(t + a + at);
    }
  }
}

constexpr int64_t kMaxGrid = 1 << 16;

}  // namespace

void decode_rotate(const RotateArgs& a, hipStream_t stream) {
  const int turned = a.interleaved ? (2 * a.pairs + 7) / 8 : (a.pairs + 7) / 8, copied = (a.dim - 2 * a.pairs + 7) / 8;
  const int plain = (a.dim + 7) / 8, q_heads = a.q ? a.q_heads : 0, heads = a.k ? a.cache.heads : 0;
  const int of_q = q_heads * (turned + copied), of_row = of_q + heads * (turned + copied + plain);
  // Tiles of about 1024 units (4 a lane), fewer where the rows would not fill the CUs.
  int64_t rows = 1024 / of_row;
  if (a.pairs) rows = std::min<int64_t>(rows, kTableSize / a.pairs);
  rows = std::max<int64_t>(1, std::min<int64_t>({rows, kMaxRows, a.n / 1024}));
  const Units u{static_cast<int>(rows), turned, copied, plain, of_q, of_row, Divide(of_row), Divide(turned + copied), Divide(plain)};
  const dim3 grid(static_cast<unsigned>(std::min((a.n + rows - 1) / rows, kMaxGrid)));
  if (a.f32)
    hipLaunchKernelGGL(rotate_kernel<true>, grid, dim3(kThreads), 0, stream, a, u);
  else
    hipLaunchKernelGGL(rotate_kernel<false>, grid, dim3(kThreads), 0, stream, a, u);
  launched("rotation");
}

void decode_fork(const ForkArgs& a, hipStream_t stream) {
  const int64_t blocks = a.n * (a.cache.keys ? a.cache.heads : 1);
  hipLaunchKernelGGL(fork_kernel, dim3(static_cast<unsigned>(std::min(blocks, kMaxGrid))), dim3(kThreads), 0, stream, a);
  launched("reordering of the cache");
}

}  // namespace k
}  // namespace dycl
