// The choice of the next tokens: the k largest of scores[w] + log softmax(logits[w])[t]
// over a sequence's beams w and words t, the lowest w * words + t among equals.
//
// log softmax only shifts a beam's logits, so a beam's best candidates are those of its
// logits.  A workgroup takes a segment of a row into registers: sum of exponentials
// around its maximum, and its k largest.  The least of the four waves' ceil(k / 4)-th largest of
// their lanes' maxima (to 16 bits, rounded down) is a bound that k values reach and few others; those that
// reach it go to LDS and are ranked by counting the larger ones.  Where more reach it than LDS
// holds (a row of equal values) the k are taken one after the other.  A second kernel sums a beam's segments, in order, and
// takes the k largest of the segments' lists the same way.
//
// Bound by HBM (a logit is read once) and close behind by instruction issue: about 8 vector
// instructions per logit, the exponential 4 of them.
#include "decode_dev.hpp"

namespace dycl {
namespace k {

namespace {

constexpr int kThreads = 256, kWaves = 4, kRoom = 512;
constexpr float kClosed = -__builtin_inff(), kLog2e = 1.44269504088896340736f, kLargest = 3.402823466e38f;

// a value and an index as one number: larger values first, then lower indices; 0 is none
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);       // (-0 becomes 0: they are equal)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) {
  return v == kClosed ? 0 : static_cast<uint64_t>(ordered(v)) << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return 0xffffffffu - static_cast<uint32_t>(key); }

// a bound that at least k of the wave's 64 values reach, within 2^-7 below the k-th largest; -inf where fewer are open
__device__ __forceinline__ float bound_of(float v, int k) {
  const uint32_t o = ordered(v) >> 16;
  uint32_t t = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t with = t | 1u << bit;
    if (__popcll(__ballot(o >= with)) >= k) t = with;
  }
  return t <= (ordered(kClosed) >> 16) ? kClosed : value_of(t << 16);
}

struct Chosen {                        // in LDS
  uint64_t keys[kRoom];
  uint64_t best[kWaves];
  float bounds[2][kWaves];
  int count;
};

// A bound that k of the workgroup's values reach if v is each lane's largest; -inf where fewer lanes are
// open.  All threads call it; what was written to LDS before is visible after it.
__device__ __forceinline__ float bound_of_all(Chosen& s, float v, int k) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float own = bound_of(v, (k + kWaves - 1) / kWaves);
  if (lane == 0) s.bounds[0][wave] = own;
  __syncthreads();
  const float least = fminf(fminf(s.bounds[0][0], s.bounds[0][1]), fminf(s.bounds[0][2], s.bounds[0][3]));
  if (least > kClosed) return least;
  // a wave with fewer open lanes than its share: the best wave's k-th
  const float single = bound_of(v, k);
  if (lane == 0) s.bounds[1][wave] = single;
  __syncthreads();
  return fmaxf(fmaxf(s.bounds[1][0], s.bounds[1][1]), fmaxf(s.bounds[1][2], s.bounds[1][3]));
}

// The k largest of the candidates in `s`: rank r's key to put(r, key), r below the number of them and k.
template <class PUT>
__device__ __forceinline__ void rank_all(const Chosen& s, int k, PUT&& put) {
  const int n = s.count;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t key = s.keys[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += s.keys[j] > key;
    if (rank < k) put(rank, key);
  }
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const uint64_t o = static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(v), w));
    v = o > v ? o : v;
  }
  return v;
}

struct Segments {
  int count;                           // of a row
  float2* state;                       // [row][segment]: maximum, sum of exponentials around it
  uint64_t* lists;                     // [row][segment][k] keys, largest first, 0 past the last
};

// V: groups of 8 values per lane
template <bool F32, int V>
__global__ __launch_bounds__(kThreads) void segment_kernel(BeamArgs p, Segments g, int64_t items) {
  __shared__ Chosen s;
  __shared__ float2 waves[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t row = item / g.count;
    const int segment = static_cast<int>(item - row * g.count);
    // beams without candidates of their own are not read
    const float score = p.scores[row];
    if ((p.ended && p.ended[row]) || !(score > kClosed)) continue;        // (the same for the whole workgroup; the second kernel skips them too)
    if (threadIdx.x == 0) s.count = 0;
    const char* base = static_cast<const char*>(p.logits) + row * p.ldl * (F32 ? 4 : 2);
    const int first = segment * (kThreads * 8 * V) + 8 * threadIdx.x;
    float v[8 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = first + i * kThreads * 8;
      read8<F32>(base + static_cast<int64_t>(at) * (F32 ? 4 : 2), min(8, max(0, p.words - at)), v + 8 * i);
#pragma unroll
      for (int j = 0; j < 8; ++j)                    // NaN is closed, +infinity the largest finite value
        v[8 * i + j] = at + j < p.words ? fminf(fmaxf(v[8 * i + j], kClosed), kLargest) : kClosed;
    }
    float top = v[0];
#pragma unroll
    for (int i = 1; i < 8 * V; ++i) top = fmaxf(top, v[i]);
    float m = top;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) m = fmaxf(m, __shfl_xor(m, w));
    const float around = m == kClosed ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8 * V; ++i) sum += __builtin_amdgcn_exp2f((v[i] - around) * kLog2e);
    sum = wave_sum(sum);
    if (lane == 0) waves[wave] = make_float2(m, sum);
    const float bound = bound_of_all(s, top, p.k);
    if (threadIdx.x == 0) {
      const float all = fmaxf(fmaxf(waves[0].x, waves[1].x), fmaxf(waves[2].x, waves[3].x)), base2 = all == kClosed ? 0.f : all;
      float total = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) total += __builtin_amdgcn_exp2f((waves[w].x - base2) * kLog2e) * waves[w].y;
      g.state[item] = make_float2(all, total);
    }
    if (top >= bound) {
#pragma unroll
      for (int i = 0; i < 8 * V; ++i)
        if (v[i] >= bound && v[i] > kClosed) {
          const int at = atomicAdd(&s.count, 1);
          if (at < kRoom) s.keys[at] = key_of(v[i], first + i / 8 * (kThreads * 8) + i % 8);
        }
    }
    __syncthreads();
    uint64_t* list = g.lists + item * p.k;
    if (s.count <= kRoom) {
      rank_all(s, p.k, [&](int rank, uint64_t key) { list[rank] = key; });
      for (int i = s.count + threadIdx.x; i < p.k; i += kThreads) list[i] = 0;
    } else {
      uint64_t before = ~uint64_t(0);
      for (int round = 0; round < p.k; ++round) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < 8 * V; ++i) {
          const uint64_t key = key_of(v[i], first + i / 8 * (kThreads * 8) + i % 8);
          best = key < before && key > best ? key : best;
        }
        best = wave_max(best);
        if (lane == 0) s.best[wave] = best;
        __syncthreads();
        best = max(max(s.best[0], s.best[1]), max(s.best[2], s.best[3]));
        if (threadIdx.x == 0) list[round] = best;
        before = best;
        __syncthreads();
      }
    }
    __syncthreads();
  }
}

// One sequence: its beams' sums, then the k largest of all lists.
__global__ __launch_bounds__(kThreads) void choose_kernel(BeamArgs p, Segments g) {
  __shared__ Chosen s;
  __shared__ float2 shift[kBeamMaxBeams];      // a beam's largest logit, and the value of that one; -inf: none of its logits
  __shared__ float kept[kBeamMaxBeams];        // an ended beam's score, -inf: it has not ended
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t b = blockIdx.x; b < p.sequences; b += gridDim.x) {
    if (threadIdx.x == 0) s.count = 0;
    for (int w = wave; w < p.beams; w += kWaves) {
      const int64_t row = b * p.beams + w;
      const float given = p.scores[row], score = fminf(given, kLargest);
      const bool open = given > kClosed, over = p.ended && p.ended[row];
      float m = kClosed, total = 0.f;
      if (open && !over) {
        const float2* state = g.state + row * g.count;
        for (int i = lane; i < g.count; i += 64) m = fmaxf(m, state[i].x);
#pragma unroll
        for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
        if (m > kClosed)
          for (int i = lane; i < g.count; i += 64) total += __builtin_amdgcn_exp2f((state[i].x - m) * kLog2e) * state[i].y;
        total = wave_sum(total);
      }
      if (lane == 0) {
        shift[w] = make_float2(m, score - logf(total));
        kept[w] = open && over ? score : kClosed;
      }
    }
    __syncthreads();
    // candidates' keys: a thread's lists are threadIdx.x, + 256, ...
    const int lists = p.beams * g.count;
    const uint64_t* all = g.lists + b * lists * p.k;
    auto key_at = [&](int list, int i) -> uint64_t {
      const int w = list / g.count;
      if (shift[w].x == kClosed) return 0;
      const uint64_t key = all[static_cast<int64_t>(list) * p.k + i];
      // (a sum past the least finite value is closed, as -infinity is)
      return key ? key_of((value_of(static_cast<uint32_t>(key >> 32)) - shift[w].x) + shift[w].y, w * p.words + index_of(key)) : 0;
    };
    uint64_t head = 0;
    for (int i = threadIdx.x; i < lists; i += kThreads) head = max(head, key_at(i, 0));
    if (threadIdx.x < p.beams && kept[threadIdx.x] > kClosed)
      head = max(head, key_of(kept[threadIdx.x], threadIdx.x * p.words + p.end));
    const float bound = bound_of_all(s, head ? value_of(static_cast<uint32_t>(head >> 32)) : kClosed, p.k);
    auto each = [&](auto&& f) {                      // the thread's candidates that reach the bound
      for (int i = threadIdx.x; i < lists; i += kThreads)
        for (int j = 0; j < p.k; ++j) {
          const uint64_t key = key_at(i, j);
          if (!key || value_of(static_cast<uint32_t>(key >> 32)) < bound) break;
          f(key);
        }
      if (threadIdx.x < p.beams && kept[threadIdx.x] > kClosed) f(key_of(kept[threadIdx.x], threadIdx.x * p.words + p.end));
    };
    each([&](uint64_t key) {
      const int at = atomicAdd(&s.count, 1);
      if (at < kRoom) s.keys[at] = key;
    });
    __syncthreads();
    auto put = [&](int rank, uint64_t key) {
      const int64_t at = b * p.k + rank;
      if (!key) {
        p.parents[at] = p.tokens[at] = -1;
        p.new_scores[at] = kClosed;
        p.new_ended[at] = 0;
        return;
      }
      const uint32_t index = index_of(key);
      const int w = static_cast<int>(index / p.words), word = static_cast<int>(index - w * p.words);
      p.parents[at] = static_cast<int32_t>(b * p.beams + w);
      p.tokens[at] = word;
      p.new_scores[at] = value_of(static_cast<uint32_t>(key >> 32));
      p.new_ended[at] = word == p.end || kept[w] > kClosed;
    };
    if (s.count <= kRoom) {
      rank_all(s, p.k, put);
      for (int i = s.count + threadIdx.x; i < p.k; i += kThreads) put(i, 0);
    } else {
      uint64_t before = ~uint64_t(0);
      for (int round = 0; round < p.k; ++round) {
        uint64_t best = 0;
        each([&](uint64_t key) { best = key < before && key > best ? key : best; });
        best = wave_max(best);
        if (lane == 0) s.best[wave] = best;
        __syncthreads();
        best = max(max(s.best[0], s.best[1]), max(s.best[2], s.best[3]));
        if (threadIdx.x == 0) put(round, best);
        before = best;
        __syncthreads();
      }
    }
    __syncthreads();
  }
}

// Values of a segment follow from the words alone, so a row's sum does too.
int groups_of(int words) { return words <= 65536 ? 2 : 4; }
int segments_of(int words) { return (words + kThreads * 8 * groups_of(words) - 1) / (kThreads * 8 * groups_of(words)); }

constexpr int64_t kMaxGrid = int64_t(1) << 22;

}  // namespace

size_t decode_beam_workspace(int64_t sequences, int beams, int words, int k) {
  return static_cast<size_t>(sequences) * beams * segments_of(words) * (8 + static_cast<size_t>(k) * 8);
}

void decode_beam(const BeamArgs& a, hipStream_t stream) {
  Segments g;
  g.count = segments_of(a.words);
  const int64_t items = a.sequences * a.beams * g.count;
  g.lists = static_cast<uint64_t*>(a.workspace);
  g.state = reinterpret_cast<float2*>(g.lists + items * a.k);
  const dim3 grid(static_cast<unsigned>(std::min(items, kMaxGrid))), threads(kThreads);
  const bool four = groups_of(a.words) == 4;
  if (a.f32 && four)
    hipLaunchKernelGGL((segment_kernel<true, 4>), grid, threads, 0, stream, a, g, items);
  else if (a.f32)
    hipLaunchKernelGGL((segment_kernel<true, 2>), grid, threads, 0, stream, a, g, items);
  else if (four)
    hipLaunchKernelGGL((segment_kernel<false, 4>), grid, threads, 0, stream, a, g, items);
  else
    hipLaunchKernelGGL((segment_kernel<false, 2>), grid, threads, 0, stream, a, g, items);
  launched("choice of tokens, segments");
  hipLaunchKernelGGL(choose_kernel, dim3(static_cast<unsigned>(std::min(a.sequences, kMaxGrid))), threads, 0, stream, a, g);
  launched("choice of tokens");
}

}  // namespace k
}  // namespace dycl
