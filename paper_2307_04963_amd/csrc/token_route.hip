// The choice of k of E experts for every row, and the stable partition of the
// (row, expert) pairs by expert.
//
// One wave takes a row: lane l holds experts l V to l V + V - 1.  A round of
// the choice is a maximum over the wave and a ballot for the lowest lane that
// has it.
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

constexpr int kBlockRows = 64;
constexpr float kClosed = -__builtin_inff();

__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, rotate16<8>(v));
  v = fmaxf(v, rotate16<4>(v));
  v = fmaxf(v, rotate16<2>(v));
  v = fmaxf(v, rotate16<1>(v));
  return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

// inclusive prefix sum over the lanes of a wave
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// exclusive prefix sums of `count(e)` over the experts into base[0 .. E], by one wave
template <class F>
__device__ __forceinline__ void scan_experts(int E, int* base, F count) {
  const int lane = threadIdx.x & 63;
  int total = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int e = e0 + lane;
    const int c = e < E ? count(e) : 0;
    const int incl = wave_scan(c);
    if (e < E) base[e] = total + incl - c;
    total += __shfl(incl, 63);
  }
  if (lane == 0) base[E] = total;
}

// LDS index of expert e's value: a lane that walks over a group starts in a bank of its own
__device__ __forceinline__ int spread(int e) { return e + (e >> 5); }

// The row's choice by one wave: lane j < k returns the j-th choice (id, and p as weight).
template <int V>
__device__ __forceinline__ void choose(const RouteArgs& p, int64_t row, float* values, int& id, float& weight) {
  const int lane = threadIdx.x & 63;
  const int E = p.experts;
  id = -1;
  weight = 0.f;
  if (p.mask && p.mask[row] == 0) return;
  float prob[V], v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane * V + i;
    float z = kClosed;
    if (e < E)
      z = p.logits_f32 ? static_cast<const float*>(p.logits)[row * p.ldl + e]
                       : bf2f(static_cast<const uint16_t*>(p.logits)[row * p.ldl + e]);
    z = z > kClosed ? fminf(z, 3.402823466e38f) : kClosed;
    prob[i] = z;
  }
  if (p.sigmoid) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = prob[i];
      prob[i] = 1.0f / (1.0f + expf(-prob[i]));
    }
  } else {
    float top = kClosed, sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) top = fmaxf(top, prob[i]);
    top = wave_max(top);
    if (top == kClosed) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = prob[i];
      prob[i] = expf(prob[i] - top);
      sum += prob[i];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < V; ++i) prob[i] /= sum;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane * V + i;
    float s = prob[i];
    if (p.bias && e < E) s += p.bias[e];
    v[i] = v[i] > kClosed && s > kClosed ? s : kClosed;
  }

  if (p.groups > 1) {
    // lane g scores group g; a group stays if fewer than top_groups are better
#pragma unroll
    for (int i = 0; i < V; ++i) values[spread(lane * V + i)] = v[i];
    __builtin_amdgcn_wave_barrier();
    const int size = E / p.groups;
    float a = kClosed, b = kClosed;
    if (lane < p.groups)
      for (int i = 0; i < size; ++i) {
        const float c = values[spread(lane * size + i)];
        b = fmaxf(b, fminf(a, c));
        a = fmaxf(a, c);
      }
    __builtin_amdgcn_wave_barrier();
    const float score = b == kClosed ? a : a + b;
    int better = 0;
    for (int g = 0; g < p.groups; ++g) {
      const float o = __shfl(score, g);
      better += o > score || (o == score && g < lane);
    }
    const uint64_t keep = __ballot(lane < p.groups && better < p.top_groups);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = lane * V + i;
      if (e < E && !(keep >> (e / size) & 1)) v[i] = kClosed;
    }
  }

  float total = 0.f;
  for (int j = 0; j < p.k; ++j) {
    float best = v[0], bp = prob[0];
    int bi = 0;
#pragma unroll
    for (int i = 1; i < V; ++i)
      if (v[i] > best) {
        best = v[i];
        bp = prob[i];
        bi = i;
      }
    const float top = wave_max(best);
    if (top == kClosed) break;
    const int from = __ffsll(static_cast<unsigned long long>(__ballot(best == top))) - 1;
    const float w = lane_value(bp, from);
    const int e = from * V + __builtin_amdgcn_readlane(bi, from);
    total += w;
    if (lane == j) {
      id = e;
      weight = w;
    }
    if (lane == from) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i == bi) v[i] = kClosed;
    }
  }
  if (p.renormalise) weight = total > 0.f ? weight / total : 0.f;
  weight *= p.scale;
}

// Places the pairs of rows [row0, row0 + 64): masks[e] has a bit for each of
// them that chose e, base[e] is the position of the first.
__device__ __forceinline__ void place(const RouteArgs& p, int64_t row0, const unsigned long long* masks, const int* base) {
  const int64_t rows = p.n - row0 < kBlockRows ? p.n - row0 : kBlockRows;
  for (int q = threadIdx.x; q < rows * p.k; q += blockDim.x) {
    const int64_t pair = row0 * p.k + q;
    const int e = p.ids[pair];
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

template <int V>
__global__ __launch_bounds__(1024) void route_choose_kernel(RouteArgs p, int blocks) {
  extern __shared__ __align__(16) char lds[];
  unsigned long long* masks = reinterpret_cast<unsigned long long*>(lds);
  int* base = reinterpret_cast<int*>(masks + p.experts);
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float* values = reinterpret_cast<float*>(base + p.experts + 1) + wave * (V * 66);
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kBlockRows;
  for (int e = threadIdx.x; e < p.experts; e += blockDim.x) masks[e] = 0;
  __syncthreads();
  for (int r = wave; r < kBlockRows && row0 + r < p.n; r += waves) {
    const int64_t row = row0 + r;
    int id;
    float w;
    choose<V>(p, row, values, id, w);
    if (lane < p.k) {
      p.ids[row * p.k + lane] = id;
      p.weights[row * p.k + lane] = w;
      if (id >= 0) atomicOr(&masks[id], 1ull << r);
    }
  }
  if (!p.offsets) return;
  __syncthreads();
  if (blocks > 1) {
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x)
      counts_of(p)[static_cast<size_t>(e) * blocks + blockIdx.x] = __popcll(masks[e]);
    return;
  }
  if (wave == 0) scan_experts(p.experts, base, [&](int e) { return __popcll(masks[e]); });
  __threadfence_block();
  __syncthreads();
  for (int e = threadIdx.x; e <= p.experts; e += blockDim.x) p.offsets[e] = base[e];
  place(p, 0, masks, base);
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
    const int incl = wave_scan(v);
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

__global__ __launch_bounds__(256) void route_place_kernel(RouteArgs p, int blocks) {
  extern __shared__ __align__(16) char lds[];
  unsigned long long* masks = reinterpret_cast<unsigned long long*>(lds);
  int* base = reinterpret_cast<int*>(masks + p.experts);
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kBlockRows;
  const int32_t* totals = counts_of(p) + static_cast<size_t>(p.experts) * blocks;
  for (int e = threadIdx.x; e < p.experts; e += 256) masks[e] = 0;
  if (threadIdx.x < 64) scan_experts(p.experts, base, [&](int e) { return totals[e]; });
  __syncthreads();
  const int64_t rows = p.n - row0 < kBlockRows ? p.n - row0 : kBlockRows;
  for (int q = threadIdx.x; q < rows * p.k; q += 256) {
    const int e = p.ids[row0 * p.k + q];
    if (e >= 0) atomicOr(&masks[e], 1ull << (q / p.k));
  }
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= p.experts; e += 256) p.offsets[e] = base[e];
  const int64_t all = base[p.experts];
  __syncthreads();
  for (int e = threadIdx.x; e < p.experts; e += 256) base[e] += counts_of(p)[static_cast<size_t>(e) * blocks + blockIdx.x];
  __syncthreads();
  place(p, row0, masks, base);
  for (int64_t q = all + static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; q < p.n * p.k; q += gridDim.x * 256L) p.order[q] = -1;
}

__global__ void route_empty_kernel(int32_t* offsets, int experts) {
  for (int e = threadIdx.x; e <= experts; e += blockDim.x) offsets[e] = 0;
}

template <int V>
void launch_choose(const RouteArgs& a, int blocks, hipStream_t s) {
  const int waves = blocks > 1 || V == 16 ? 8 : 16;
  const size_t lds = a.experts * 8 + (a.experts + 1) * 4 + (a.groups > 1 ? waves * V * 66 * 4 : 0);
  route_choose_kernel<V><<<blocks, waves * 64, lds, s>>>(a, blocks);
}

}  // namespace

size_t token_route_workspace(int64_t n, int experts, int k) {
  const int64_t blocks = (n + kBlockRows - 1) / kBlockRows;
  return blocks <= 1 ? 0 : (static_cast<size_t>(blocks) + 1) * experts * sizeof(int32_t);
}

void token_route(const RouteArgs& a, hipStream_t s) {
  const int blocks = static_cast<int>((a.n + kBlockRows - 1) / kBlockRows);
  if (a.experts <= 64)
    launch_choose<1>(a, blocks, s);
  else if (a.experts <= 128)
    launch_choose<2>(a, blocks, s);
  else if (a.experts <= 256)
    launch_choose<4>(a, blocks, s);
  else if (a.experts <= 512)
    launch_choose<8>(a, blocks, s);
  else
    launch_choose<16>(a, blocks, s);
  if (!a.offsets || blocks == 1) return;
  route_sum_kernel<<<a.experts, 256, 0, s>>>(a, blocks);
  route_place_kernel<<<blocks, 256, a.experts * 8 + (a.experts + 1) * 4, s>>>(a, blocks);
}

void token_route_empty(int32_t* offsets, int experts, hipStream_t s) {
  route_empty_kernel<<<1, 256, 0, s>>>(offsets, experts);
}

}  // namespace k
}  // namespace dycl
