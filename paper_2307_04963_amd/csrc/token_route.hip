// The choice of k of E experts for every row, and the stable partition of the
// (row, expert) pairs by expert.
//
// One wave takes a row.  A group's experts lie in 64 / G neighbouring lanes (G: the
// number of groups, rounded up to a power of two), V consecutive ones in each, so
// lanes and an expert's place in its lane keep the experts' order.  Up to four a lane
// sorts its values once and a round of the choice looks at the lanes' best; a round is
// a maximum over the wave (six DPP steps), a ballot for the lowest lane that has it,
// and that lane's next best.  Bound by instruction issue: 467 vector instructions for
// a row of 256 experts in 8 groups, eight of them chosen, the rounds half of that.
//
// Measured: 65536 rows of 256 experts, 8 chosen in 4 of 8 groups: choice 60 us, sums
// 5, places 9 (the bytes would take 14); 32768 rows of 64, 14 + 4 + 4 us; 24 rows of
// 256, one launch, 8.5 us: up to 64 rows are one workgroup of 16 waves, so eight of them
// take two rows one after the other, 16 rounds of dependent steps at 0.4 us.
//
// The partition works on blocks of 64 rows: an expert's rows in a block are one
// 64-bit mask in LDS, so a pair's rank among the block's is a bit count and
// the order of the atomics that set the bits changes nothing.  Blocks' counts
// are summed per expert by a second kernel, and a third places the pairs; up
// to 64 rows are one block and one launch.
#include "token_dev.hpp"

namespace dycl {
namespace k {

namespace {

// Rows of a block: 64 in one block for few rows, then few enough that the
// blocks fill the CUs (4096 rows in blocks of 64 took 27 us of 64 experts' 8 rounds, on
// a quarter of the CUs), 64 for many, whose counts per block are the fewest.
int block_rows_of(int64_t n) { return n <= 64 || n >= 32768 ? 64 : n >= 16384 ? 32 : 16; }
constexpr float kClosed = -__builtin_inff();

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}

// The maximum over the wave, the same in every lane: a lane without a source keeps
// its value, so lane 63 ends up with all.  (From the builtins the compiler makes four
// instructions of each step.)
__device__ __forceinline__ float wave_max(float v) {
  asm("s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:1 row_mask:0xf bank_mask:0xf\n\t"
      "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:2 row_mask:0xf bank_mask:0xf\n\t"
      "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:4 row_mask:0xf bank_mask:0xf\n\t"
      "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_shr:8 row_mask:0xf bank_mask:0xf\n\t"
      "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_bcast:15 row_mask:0xa bank_mask:0xf\n\t"
      "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_bcast:31 row_mask:0xc bank_mask:0xf\n\ts_nop 1"
      : "+v"(v));
  return lane_value(v, 63);
}

// exp(x): relative error 2^-24 |x| + one unit, which for the scores that take part in
// a choice is the rounding of the logit
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

__device__ __forceinline__ float sigmoid_of(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-x)); }

// exclusive prefix sums of `count(e)` over the experts into base[0 .. E], by one wave
template <class F>
__device__ __forceinline__ void scan_experts(int E, int* base, F count) {
  const int lane = threadIdx.x & 63;
  int total = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int e = e0 + lane;
    const int c = e < E ? count(e) : 0;
    const int incl = scan_lanes(c);
    if (e < E) base[e] = total + incl - c;
    total += __builtin_amdgcn_readlane(incl, 63);
  }
  if (lane == 0) base[E] = total;
}

// How a wave holds a row's experts.
struct Layout {
  int size;                // experts of a group
  int lanes;               // lanes of a group, a power of two
  int first, count;        // this lane's experts [first, first + count)
  int group;               // its group (>= groups: none)
};

template <int V>
__device__ __forceinline__ Layout layout_of(const RouteArgs& p) {
  const int lane = threadIdx.x & 63;
  Layout l;
  int g = 1;
  while (g < p.groups) g <<= 1;
  l.size = p.experts / p.groups;
  l.lanes = 64 / g;
  l.group = lane / l.lanes;
  const int in = (lane - l.group * l.lanes) * V;    // place of the first in its group
  l.first = l.group * l.size + in;
  const int left = l.group < p.groups ? l.size - in : 0;
  l.count = left < 0 ? 0 : left < V ? left : V;
  return l;
}

// a loaded logit's bits to its value (NaN: closed)
__device__ __forceinline__ float logit_of(const RouteArgs& p, uint32_t bits) {
  const float z = __uint_as_float(p.logits_f32 ? bits : bits << 16);
  return z > kClosed ? fminf(z, 3.402823466e38f) : kClosed;
}

// the two largest of two descending pairs
__device__ __forceinline__ void merge2(float& a, float& b, float c, float d) {
  const float low = fminf(a, c);
  a = fmaxf(a, c);
  b = fmaxf(low, fmaxf(b, d));
}

// The row's choice by one wave: lane j < k returns the j-th choice (id, and its
// weight).  v: this lane's logits, bias: its experts' (-infinity past its count);
// scores [experts]: the wave's own LDS.
template <int V>
__device__ __forceinline__ void choose(const RouteArgs& p, const Layout& l, const float (&bias)[V], float (&v)[V], float* scores, int& id, float& weight) {
  const int lane = threadIdx.x & 63;
  id = -1;
  weight = 0.f;
  float top = 0.f, inv = 1.f;
  if (!p.sigmoid) {
    top = v[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, v[i]);
    top = wave_max(top);
    if (top == kClosed) return;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) sum += exp_of(v[i] - top);
    inv = 1.0f / wave_sum(sum);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float prob = p.sigmoid ? sigmoid_of(v[i]) : exp_of(v[i] - top) * inv;
    if (i < l.count) scores[l.first + i] = prob;
    const float s = prob + bias[i];
    v[i] = v[i] > kClosed && s > kClosed ? s : kClosed;
  }

  // V <= 4: descending, with each value's place in a byte of `places`
  uint32_t places = 0x03020100u;
  if constexpr (V == 2 || V == 4) {
    int at[V];
#pragma unroll
    for (int i = 0; i < V; ++i) at[i] = i;
    // (of equals the lower place stays first: only neighbours are compared)
    auto order = [&](int i) __attribute__((always_inline)) {
      const bool swap = v[i + 1] > v[i];
      const float x = swap ? v[i + 1] : v[i], y = swap ? v[i] : v[i + 1];
      const int c = swap ? at[i + 1] : at[i], d = swap ? at[i] : at[i + 1];
      v[i] = x;
      v[i + 1] = y;
      at[i] = c;
      at[i + 1] = d;
    };
#pragma unroll
    for (int pass = V - 1; pass > 0; --pass)
#pragma unroll
      for (int i = 0; i < pass; ++i) order(i);
    places = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) places |= static_cast<uint32_t>(at[i]) << (8 * i);
  }

  if (p.groups > 1) {
    // each group's two largest, in all its lanes
    float a = v[0], b = kClosed;
    if constexpr (V == 2 || V == 4) {
      b = v[1];
    } else {
#pragma unroll
      for (int i = 1; i < V; ++i) merge2(a, b, v[i], kClosed);
    }
    if (l.lanes > 1) merge2(a, b, dpp<0xb1>(a), dpp<0xb1>(b));          // the neighbour
    if (l.lanes > 2) merge2(a, b, dpp<0x4e>(a), dpp<0x4e>(b));          // the other pair of four
    if (l.lanes > 4) merge2(a, b, dpp<0x141>(a), dpp<0x141>(b));        // the other four of eight
    if (l.lanes > 8) merge2(a, b, dpp<0x140>(a), dpp<0x140>(b));        // the other eight of 16
    if (l.lanes > 16) merge2(a, b, __shfl_xor(a, 16), __shfl_xor(b, 16));
    // half the sum: that of two lowest values is finite, above a group with none open
    const float score = b == kClosed ? 0.5f * a : 0.5f * a + 0.5f * b;
    int better = 0;
    for (int g = 0; g < p.groups; ++g) {
      const float o = lane_value(score, g * l.lanes);
      better += o > score || (o == score && g < l.group);
    }
    if (better >= p.top_groups) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = kClosed;
    }
  }

  for (int j = 0; j < p.k; ++j) {
    float best = v[0];
    int at = places & 0xff;
    if constexpr (V > 4) {
      at = 0;
#pragma unroll
      for (int i = 1; i < V; ++i) {
        at = v[i] > best ? i : at;
        best = fmaxf(best, v[i]);
      }
    }
    const float most = wave_max(best);
    if (most == kClosed) break;
    const int from = __ffsll(static_cast<unsigned long long>(__ballot(best == most))) - 1;
    const int e = __builtin_amdgcn_readlane(l.first + at, from);
    id = lane == j ? e : id;
    const bool mine = lane == from;
    if constexpr (V <= 4) {
#pragma unroll
      for (int i = 0; i < V - 1; ++i) v[i] = mine ? v[i + 1] : v[i];
      v[V - 1] = mine ? kClosed : v[V - 1];
      places = mine ? places >> 8 : places;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = mine && i == at ? kClosed : v[i];
    }
  }
  __builtin_amdgcn_wave_barrier();
  if (id >= 0) weight = scores[id];
  __builtin_amdgcn_wave_barrier();
  if (p.renormalise) {
    const float total = wave_sum(weight);
    weight = total > 0.f ? weight / total : 0.f;
  }
  weight *= p.scale;
}

// Places the pairs of rows [row0, row0 + rows), whose choices are `ids`: masks[e] has
// a bit for each of them that chose e, base[e] is the position of the first.
__device__ __forceinline__ void place(const RouteArgs& p, const int32_t* ids, int64_t row0, int rows, const unsigned long long* masks, const int* base) {
  for (int q = threadIdx.x; q < rows * p.k; q += blockDim.x) {
    const int64_t pair = row0 * p.k + q;
    const int e = ids[q];
    int pos = -1;
    if (e >= 0) {
      const int r = q / p.k;
      pos = base[e] + __popcll(masks[e] & ((1ull << r) - 1));
      p.order[pos] = static_cast<int32_t>(pair);
    }
    p.slots[pair] = pos;
  }
}

// counts [E][blocks] in the workspace, then totals [E]
__device__ __forceinline__ int32_t* counts_of(const RouteArgs& p) { return static_cast<int32_t*>(p.workspace); }

// (V of 16 and more take more registers than 16 waves leave)
template <int V>
__global__ __launch_bounds__(V < 16 ? 1024 : 512) void route_choose_kernel(RouteArgs p, int blocks, int block_rows, int block0) {
  extern __shared__ __align__(16) char lds[];
  unsigned long long* masks = reinterpret_cast<unsigned long long*>(lds);
  int* base = reinterpret_cast<int*>(masks + p.experts);
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float* scores = reinterpret_cast<float*>(base + p.experts + 1) + wave * p.experts;
  int32_t* chosen = reinterpret_cast<int32_t*>(base + p.experts + 1) + waves * p.experts;     // one block: [64][k]
  const Layout l = layout_of<V>(p);
  float bias[V];
  uint32_t next[V];
#pragma unroll
  for (int i = 0; i < V; ++i) bias[i] = i < l.count ? (p.bias ? p.bias[l.first + i] : 0.f) : kClosed;
  const int block = block0 + static_cast<int>(blockIdx.x);
  const int64_t row0 = static_cast<int64_t>(block) * block_rows;
  const int rows = p.n - row0 < block_rows ? static_cast<int>(p.n - row0) : block_rows;
  // a row's logits are requested a row ahead
  auto request = [&](int r) __attribute__((always_inline)) {
    const int64_t at = (row0 + r) * p.ldl + l.first;
    if (p.logits_f32) {
#pragma unroll
      for (int i = 0; i < V; ++i) next[i] = i < l.count ? static_cast<const uint32_t*>(p.logits)[at + i] : 0xff800000u;
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) next[i] = i < l.count ? static_cast<const uint16_t*>(p.logits)[at + i] : 0xff80u;
    }
  };
  if (wave < rows) request(wave);
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) masks[e] = 0;
  __syncthreads();
  for (int r = wave; r < rows; r += waves) {
    const int64_t row = row0 + r;
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = logit_of(p, next[i]);
    const bool in = !p.mask || p.mask[row] != 0;
    if (r + waves < rows) request(r + waves);
    int id = -1;
    float w = 0.f;
    if (in) choose<V>(p, l, bias, v, scores, id, w);
    if (lane < p.k) {
      p.ids[row * p.k + lane] = id;
      p.weights[row * p.k + lane] = w;
      if (blocks == 1) chosen[r * p.k + lane] = id;
      if (id >= 0) atomicOr(&masks[id], 1ull << r);
    }
  }
  if (!p.offsets) return;
  __syncthreads();
  if (blocks > 1) {
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x)
      counts_of(p)[static_cast<size_t>(e) * blocks + block] = __popcll(masks[e]);
    return;
  }
  if (wave == 0) scan_experts(p.experts, base, [&](int e) { return __popcll(masks[e]); });
  __syncthreads();
  for (int e = threadIdx.x; e <= p.experts; e += blockDim.x) p.offsets[e] = base[e];
  place(p, chosen, 0, rows, masks, base);
  for (int64_t q = base[p.experts] + threadIdx.x; q < p.n * p.k; q += blockDim.x) p.order[q] = -1;
}

// an expert's counts to the pairs in the blocks before, and its total
__global__ __launch_bounds__(256) void route_sum_kernel(RouteArgs p, int blocks) {
  __shared__ int part[4];
  int32_t* c = counts_of(p) + static_cast<size_t>(blockIdx.x) * blocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int total = 0;
  for (int b0 = 0; b0 < blocks; b0 += 256) {
    const int b = b0 + threadIdx.x;
    const int v = b < blocks ? c[b] : 0;
    const int incl = scan_lanes(v);
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    int before = total;
    for (int w = 0; w < 4; ++w) {
      before += w < wave ? part[w] : 0;
      total += part[w];
    }
    if (b < blocks) c[b] = before + incl - v;
    __syncthreads();
  }
  if (threadIdx.x == 0) counts_of(p)[static_cast<size_t>(p.experts) * blocks + blockIdx.x] = total;
}

__global__ __launch_bounds__(256) void route_place_kernel(RouteArgs p, int blocks, int block_rows, int block0) {
  extern __shared__ __align__(16) char lds[];
  unsigned long long* masks = reinterpret_cast<unsigned long long*>(lds);
  int* base = reinterpret_cast<int*>(masks + p.experts);
  const int block = block0 + static_cast<int>(blockIdx.x);
  const int64_t row0 = static_cast<int64_t>(block) * block_rows;
  const int rows = p.n - row0 < block_rows ? static_cast<int>(p.n - row0) : block_rows;
  const int32_t* totals = counts_of(p) + static_cast<size_t>(p.experts) * blocks;
  for (int e = threadIdx.x; e < p.experts; e += 256) masks[e] = 0;
  if (threadIdx.x < 64) scan_experts(p.experts, base, [&](int e) { return totals[e]; });
  __syncthreads();
  for (int q = threadIdx.x; q < rows * p.k; q += 256) {
    const int e = p.ids[row0 * p.k + q];
    if (e >= 0) atomicOr(&masks[e], 1ull << (q / p.k));
  }
  if (block == 0)
    for (int e = threadIdx.x; e <= p.experts; e += 256) p.offsets[e] = base[e];
  const int64_t all = base[p.experts];
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += 256) base[e] += counts_of(p)[static_cast<size_t>(e) * blocks + block];
  __syncthreads();
  place(p, p.ids + row0 * p.k, row0, rows, masks, base);
  for (int64_t q = all + static_cast<int64_t>(block) * 256 + threadIdx.x; q < p.n * p.k; q += blocks * 256L) p.order[q] = -1;
}

__global__ void route_empty_kernel(int32_t* offsets, int experts) {
  for (int e = threadIdx.x; e <= experts; e += blockDim.x) offsets[e] = 0;
}

// Blocks of one launch.  A launch holds less than 2^32 threads, which 512 threads for
// every 64 rows pass at 2^29 rows: more blocks take more launches.
constexpr int kLaunchBlocks = 1 << 22;

template <int V>
void launch_choose(const RouteArgs& a, int blocks, int block_rows, hipStream_t s) {
  const int waves = blocks > 1 || V >= 16 ? 8 : 16;
  const size_t lds = a.experts * 8 + (a.experts + 1) * 4 + waves * a.experts * 4 + (blocks == 1 ? 64 * a.k * 4 : 0);
  for (int b = 0; b < blocks; b += kLaunchBlocks) {
    const int here = blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks;
    route_choose_kernel<V><<<here, 64 * waves, lds, s>>>(a, blocks, block_rows, b);
    launched("choice of experts");
  }
}

}  // namespace

size_t token_route_workspace(int64_t n, int experts, int k) {
  const int64_t blocks = (n + block_rows_of(n) - 1) / block_rows_of(n);
  return blocks <= 1 ? 0 : (static_cast<size_t>(blocks) + 1) * experts * sizeof(int32_t);
}

void token_route(const RouteArgs& a, hipStream_t s) {
  const int block_rows = block_rows_of(a.n);
  const int blocks = static_cast<int>((a.n + block_rows - 1) / block_rows);
  int g = 1;
  while (g < a.groups) g <<= 1;
  const int per_lane = (a.experts / a.groups + 64 / g - 1) / (64 / g);
  if (per_lane <= 1)
    launch_choose<1>(a, blocks, block_rows, s);
  else if (per_lane <= 2)
    launch_choose<2>(a, blocks, block_rows, s);
  else if (per_lane <= 4)
    launch_choose<4>(a, blocks, block_rows, s);
  else if (per_lane <= 8)
    launch_choose<8>(a, blocks, block_rows, s);
  else if (per_lane <= 16)
    launch_choose<16>(a, blocks, block_rows, s);
  else
    launch_choose<32>(a, blocks, block_rows, s);
  if (!a.offsets || blocks == 1) return;
  route_sum_kernel<<<a.experts, 256, 0, s>>>(a, blocks);
  launched("sums of a partition");
  for (int b = 0; b < blocks; b += kLaunchBlocks) {
    const int here = blocks - b < kLaunchBlocks ? blocks - b : kLaunchBlocks;
    route_place_kernel<<<here, 256, a.experts * 8 + (a.experts + 1) * 4, s>>>(a, blocks, block_rows, b);
    launched("places of a partition");
  }
}

void token_route_empty(int32_t* offsets, int experts, hipStream_t s) {
  route_empty_kernel<<<1, 256, 0, s>>>(offsets, experts);
  launched("empty partition");
}

}  // namespace k
}  // namespace dycl
