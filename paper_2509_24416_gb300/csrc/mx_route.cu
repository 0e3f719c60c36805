// Routing of tokens to experts, the rows that a routing gives them, and the weighted
// sum of what comes back.
#include "clq_device.cuh"
#include "mx_kernels.h"

#include <cfloat>

namespace clq {
namespace mx {
namespace {

constexpr uint32_t kAll = 0xffffffffu;
constexpr int ROUTE_WARPS = 8;

// Order-preserving bits of a float (no NaN); -0 as +0.
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t u = __float_as_uint(__fadd_rn(f, 0.f));
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
constexpr uint32_t kMasked = 0x007FFFFFu;  // ordered(-infinity)

template <typename T>
__device__ __forceinline__ float load_logit(const void* p, size_t i) {
  return Num<T>::to_f(__ldg(static_cast<const uint16_t*>(p) + i));
}
template <>
__device__ __forceinline__ float load_logit<float>(const void* p, size_t i) {
  return __ldg(static_cast<const float*>(p) + i);
}

// Largest key of the warp; key[i] belongs to expert 32 i + lane, 0 to none.
template <int C>
__device__ __forceinline__ uint32_t warp_max(const uint32_t (&key)[C]) {
  uint32_t m = key[0];
#pragma unroll
  for (int i = 1; i < C; ++i) m = max(m, key[i]);
  return __reduce_max_sync(kAll, m);
}

// From each lane's two largest keys of a group: the sum of the group's two largest (or
// the largest) as ordered bits.
__device__ __forceinline__ uint32_t group_sum(uint32_t a, uint32_t b, int lane, bool two) {
  const uint32_t first = __reduce_max_sync(kAll, a);
  if (!two) return first;
  // the lane that holds it (one of them) offers its second
  const int owner = __ffs(__ballot_sync(kAll, a == first)) - 1;
  const uint32_t second = __reduce_max_sync(kAll, lane == owner ? b : a);
  return ordered(__fadd_rn(unordered(first), unordered(second)));
}

// The eighth largest of the lanes' values: eights sorted in turn down and up; the larger ones of
// the pairs of two such neighbours are the eight largest of both.
__device__ __forceinline__ uint32_t eighth_largest(uint32_t v, int lane) {
  auto step = [&](int stride, int size) {
    const uint32_t o = __shfl_xor_sync(kAll, v, stride);
    v = ((lane & stride) == 0) == ((lane & size) == 0) ? max(v, o) : min(v, o);
  };
  step(1, 2);
  step(2, 4), step(1, 4);
  step(4, 8), step(2, 8), step(1, 8);
  v = max(v, __shfl_xor_sync(kAll, v, 8));
  step(4, 16), step(2, 16), step(1, 16);
  v = max(v, __shfl_xor_sync(kAll, v, 16));
  return __reduce_min_sync(kAll, v);
}

// The experts of the k largest keys above kMasked, in descending order, ties to the
// lowest expert: the j-th in lane j with its p in score, -1 and 0 in the other lanes.
//
// The k-th largest of the 32 lanes' own largest keys is a bound that the k largest keys
// reach, and few others do: those are brought together, one a lane, and each counts how
// many are in front of it.  Where more than 32 reach it (many equal scores), the largest
// is taken k times.  32768 tokens of 256 experts, k = 8: 41 us with the second way alone.
template <int C>
__device__ __forceinline__ int choose(uint32_t (&key)[C], const float (&p)[C], int lane, int k,
                                      uint4* slots, float& score) {
  uint32_t top = key[0];
#pragma unroll
  for (int i = 1; i < C; ++i) top = max(top, key[i]);
  uint32_t bound = 0;
  if (k > 4 && k <= 8) {
    bound = eighth_largest(top, lane);
  } else {
    uint32_t rest = top;
    for (int j = 0; j < k; ++j) {
      bound = __reduce_max_sync(kAll, rest);
      if (bound <= kMasked) break;
      if (lane == __ffs(__ballot_sync(kAll, rest == bound)) - 1) rest = 0;
    }
  }
  bound = max(bound, kMasked + 1);
  uint32_t have[C];
  int n = 0;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    have[i] = __ballot_sync(kAll, key[i] >= bound);
    n += __popc(have[i]);
  }
  int mine = -1;
  score = 0.f;
  if (n <= 32) {
    // lane l takes the l-th of them in the order of the experts
    int before = 0;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      if (key[i] >= bound)
        slots[before + __popc(have[i] & ((1u << lane) - 1u))] =
            make_uint4(key[i], 32 * i + lane, __float_as_uint(p[i]), 0);
      before += __popc(have[i]);
    }
    __syncwarp();
    const uint4 my = slots[lane];
    int rank = 0;
    for (int j = 0; j < n; ++j) {
      const uint32_t o = __shfl_sync(kAll, my.x, j);
      rank += o > my.x || (o == my.x && j < lane) ? 1 : 0;
    }
    __syncwarp();
    if (lane < n && rank < k) slots[rank] = my;
    __syncwarp();
    if (lane < min(k, n)) {
      const uint4 s = slots[lane];
      mine = static_cast<int>(s.y);
      score = __uint_as_float(s.z);
    }
    return mine;
  }
  for (int j = 0; j < k; ++j) {
    const uint32_t best = warp_max<C>(key);
    if (best <= kMasked) break;
    uint32_t e = 0x7FFFFFFFu;
#pragma unroll
    for (int i = C - 1; i >= 0; --i)
      if (key[i] == best) e = 32 * i + lane;
    const int at = static_cast<int>(__reduce_min_sync(kAll, e));
#pragma unroll
    for (int i = 0; i < C; ++i)
      if (32 * i + lane == at) key[i] = 0u;
    if (lane == j) mine = at;
  }
  // the scores from the lanes that have them
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const float v = __shfl_sync(kAll, p[i], mine & 31);
    if (mine >> 5 == i) score = v;
  }
  return mine;
}

// Two largest of two pairs of them: max(a, a'), max(min(a, a'), b, b').
__device__ __forceinline__ void two_largest(uint32_t& a, uint32_t& b, uint32_t a2, uint32_t b2) {
  b = max(min(a, a2), max(b, b2));
  a = max(a, a2);
}

// The same for groups of 32 regs neighbours, regs a power of two: lane g ends with group
// g's, the others with 0.  Each of the first stages halves the registers that a lane looks
// after, so that 9 exchanges of two words do what C = 8 groups by themselves take 16
// reductions and 8 ballots for.
template <int C>
__device__ __forceinline__ uint32_t group_keys_wide(const uint32_t (&key)[C], int lane, int regs,
                                                    int groups, bool two) {
  uint32_t x[C], y[C];
#pragma unroll
  for (int i = 0; i < C; ++i) x[i] = key[i], y[i] = 0;
  int m = 16;
#pragma unroll
  for (int h = C / 2; h >= 1; h /= 2, m /= 2) {
    const bool up = lane & m;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const uint32_t x2 = __shfl_xor_sync(kAll, up ? x[i] : x[i + h], m);
      const uint32_t y2 = h == C / 2 ? 0 : __shfl_xor_sync(kAll, up ? y[i] : y[i + h], m);
      x[i] = up ? x[i + h] : x[i];
      y[i] = up ? y[i + h] : y[i];
      two_largest(x[i], y[i], x2, y2);
    }
  }
#pragma unroll
  for (; m >= 1; m /= 2)
    two_largest(x[0], y[0], __shfl_xor_sync(kAll, x[0], m), __shfl_xor_sync(kAll, y[0], m));
  constexpr int LANES = 32 / C;  // that hold one register's
  for (m = LANES; m < LANES * regs; m *= 2)
    two_largest(x[0], y[0], __shfl_xor_sync(kAll, x[0], m), __shfl_xor_sync(kAll, y[0], m));
  const uint32_t g = two ? ordered(__fadd_rn(unordered(x[0]), unordered(y[0]))) : x[0];
  const uint32_t mine = __shfl_sync(kAll, g, lane * LANES * regs);
  return lane < groups ? mine : 0u;
}

// The same for groups of 32 / 2^n neighbours: each lane ends with its group's, in
// every register.
template <int C>
__device__ __forceinline__ void group_keys_narrow(const uint32_t (&key)[C], int size, bool two,
                                                  uint32_t (&g)[C]) {
#pragma unroll
  for (int i = 0; i < C; ++i) {
    uint32_t a = key[i], b = 0;
    for (int m = 1; m < size; m *= 2) {
      const uint32_t a2 = __shfl_xor_sync(kAll, a, m), b2 = __shfl_xor_sync(kAll, b, m);
      two_largest(a, b, a2, b2);
    }
    g[i] = two ? ordered(__fadd_rn(unordered(a), unordered(b))) : a;
  }
}

// One warp a token, 32 C >= E; keys in registers.  Bound by instructions: 32768 tokens of 256
// experts, k = 8, sigmoid, 4 of 8 groups kept, 902 a token, 81 % of the issue slots, 30.1 us;
// without groups 671, 84 %, 23.8.  Five blocks a SM cover the chains of exchanges best (four,
// six: 3 % slower).
template <typename T, int C>
__global__ void __launch_bounds__(32 * ROUTE_WARPS, C <= 8 ? 5 : 3) route_kernel(RouteArgs a) {
  const int lane = threadIdx.x & 31;
  const int t = blockIdx.x * ROUTE_WARPS + (threadIdx.x >> 5);
  pdl_wait();
  pdl_launch_dependents();
  if (t >= a.T) return;
  float p[C];
  uint32_t key[C];
  bool masked[C];
  float most = -INFINITY;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int e = 32 * i + lane;
    const float x = e < a.E ? load_logit<T>(a.logits, static_cast<size_t>(t) * a.ld + e) : -INFINITY;
    masked[i] = !(x > -INFINITY);  // a NaN too
    p[i] = fminf(x, FLT_MAX);
    if (!masked[i]) most = fmaxf(most, p[i]);
  }
  if (a.scoring == 0) {
    // (a float's order is that of its ordered bits)
    most = unordered(__reduce_max_sync(kAll, ordered(most)));
    float s[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      p[i] = masked[i] ? 0.f : expf(__fsub_rn(p[i], most));
      s[i] = p[i];
    }
    // by halves: C is a power of two, and halves beyond E add zeros
#pragma unroll
    for (int h = C / 2; h >= 1; h /= 2)
#pragma unroll
      for (int i = 0; i < h; ++i) s[i] = __fadd_rn(s[i], s[i + h]);
#pragma unroll
    for (int h = 16; h >= 1; h /= 2) s[0] = __fadd_rn(s[0], __shfl_xor_sync(kAll, s[0], h));
#pragma unroll
    for (int i = 0; i < C; ++i) p[i] = __fdiv_rn(p[i], s[0]);
  } else {
#pragma unroll
    for (int i = 0; i < C; ++i) p[i] = __frcp_rn(__fadd_rn(1.f, expf(-p[i])));
  }
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int e = 32 * i + lane;
    float c = p[i];
    if (a.balance != nullptr && e < a.E) c = __fadd_rn(c, __ldg(a.balance + e));
    key[i] = masked[i] || c != c ? kMasked : ordered(c);
  }
  if (a.groups > 1) {
    const int size = a.E / a.groups;
    const bool two = a.group_top == 2 && size > 1;
    uint32_t gkey = 0;  // lane g: group g (at most 32)
    if (size % 32 == 0 && (size & (size - 1)) == 0) {
      gkey = group_keys_wide<C>(key, lane, size / 32, a.groups, two);
    } else if (size % 32 == 0) {
      const int regs = size / 32;  // registers of a group
      uint32_t x = 0, y = 0;       // this lane's two largest of the group
      int g = 0, left = regs;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        y = max(y, min(x, key[i]));
        x = max(x, key[i]);
        if (--left == 0) {
          const uint32_t k = group_sum(x, y, lane, two);
          if (lane == g) gkey = k;
          ++g;
          left = regs;
          x = y = 0;
        }
      }
      if (lane >= a.groups) gkey = 0;
    } else if (size < 32 && (size & (size - 1)) == 0) {
      uint32_t g[C];
      group_keys_narrow<C>(key, size, two, g);
      const int per = 32 / size;  // groups of a register
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const uint32_t k = __shfl_sync(kAll, g[i], (lane % per) * size);
        if (lane / per == i && lane < a.groups) gkey = k;
      }
    } else {
      for (int g = 0; g < a.groups; ++g) {
        uint32_t x = 0, y = 0;
#pragma unroll
        for (int i = 0; i < C; ++i) {
          const int e = 32 * i + lane;
          const uint32_t k = e >= g * size && e < (g + 1) * size ? key[i] : 0u;
          y = max(y, min(x, k));
          x = max(x, k);
        }
        const uint32_t k = group_sum(x, y, lane, two);
        if (lane == g) gkey = k;
      }
    }
    uint32_t keep = 0;
    for (int j = 0; j < a.top_groups; ++j) {
      const uint32_t best = __reduce_max_sync(kAll, gkey);
      const int g = __ffs(__ballot_sync(kAll, gkey == best)) - 1;
      keep |= 1u << g;
      if (lane == g) gkey = 0;
    }
    // e / size: the factor's error times 512 stays below 1 / 512
    const uint32_t inv = ((1u << 20) + size - 1) / size;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const uint32_t e = 32 * i + lane;
      if (!((keep >> ((e * inv) >> 20)) & 1u)) key[i] = kMasked;
    }
  }
  __shared__ uint4 slots[ROUTE_WARPS][32];
  float w;
  const int mine = choose<C>(key, p, lane, a.k, slots[threadIdx.x >> 5], w);
  float total = w;
#pragma unroll
  for (int o = 16; o >= 1; o /= 2) total = __fadd_rn(total, __shfl_xor_sync(kAll, total, o));
  if (a.renormalize) w = total > 0.f ? __fdiv_rn(w, total) : 0.f;
  if (lane < a.k) {
    a.experts[static_cast<size_t>(t) * a.k + lane] = mine;
    a.weights[static_cast<size_t>(t) * a.k + lane] = w * a.scale;
  }
}

// ------------------------------------------------------------------- plan ---
constexpr int CHUNK = 32;  // tokens a bit mask holds
constexpr int WORDS = 4;   // masks a block of the histogram and of the rows looks after
constexpr int PLAN_THREADS = 512;

// Rows of experts e = threadIdx.x .. < E with counts[e] rows each: where each starts,
// and the tiles that cover them.  One block; E <= blockDim.x.
__device__ void plan_tiles(int count, int E, int32_t* start, int32_t* counts, RowTile* t128,
                           RowTile* t256) {
  __shared__ int32_t sum[3][PLAN_THREADS / 32];
  const int e = threadIdx.x, lane = e & 31, warp = e >> 5;
  const int n128 = (count + 127) / 128, n256 = (count + 255) / 256;
  int a = n128, b = n256;  // inclusive sums over the experts
  for (int o = 1; o < 32; o *= 2) {
    const int x = __shfl_up_sync(kAll, a, o), y = __shfl_up_sync(kAll, b, o);
    if (lane >= o) {
      a += x;
      b += y;
    }
  }
  if (lane == 31) {
    sum[0][warp] = a;
    sum[1][warp] = b;
  }
  __syncthreads();
  for (int w = 0; w < warp; ++w) {
    a += sum[0][w];
    b += sum[1][w];
  }
  if (e < E) {
    const int at = a - n128;
    start[e] = at * kRowBlock;
    for (int i = 0; i < n128; ++i)
      t128[at + i] = RowTile{e, (at + i) * kRowBlock, min(128, count - 128 * i), 0};
    for (int i = 0; i < n256; ++i)
      t256[b - n256 + i] = RowTile{e, (at + 2 * i) * kRowBlock, min(256, count - 256 * i), 0};
    if (e == E - 1) {
      counts[0] = a;
      counts[1] = b;
    }
  }
}

// mask[w][e]: which of the CHUNK tokens from t0 + w CHUNK name expert e.
__device__ void expert_masks(const int32_t* __restrict__ experts, int t0, int T, int k, int E,
                             uint32_t* mask) {
  for (int i = threadIdx.x; i < WORDS * E; i += blockDim.x) mask[i] = 0;
  __syncthreads();
  const int n = min(WORDS * CHUNK, T - t0) * k;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int e = __ldg(experts + static_cast<size_t>(t0) * k + i), t = i / k;
    if (e >= 0 && e < E) atomicOr(&mask[t / CHUNK * E + e], 1u << (t % CHUNK));
  }
  __syncthreads();
}

// Block c: hist[e][c] = tokens of its WORDS CHUNK that name expert e; rows of `pitch` bytes,
// zeros behind the last block's.
__global__ void __launch_bounds__(PLAN_THREADS)
    plan_hist_kernel(const int32_t* __restrict__ experts, int T, int k, int E, int pitch,
                     uint8_t* __restrict__ hist) {
  extern __shared__ uint32_t mask[];  // [WORDS][E]
  pdl_wait();
  pdl_launch_dependents();
  const int c = blockIdx.x;
  expert_masks(experts, c * WORDS * CHUNK, T, k, E, mask);
  for (int e = threadIdx.x; e < E; e += blockDim.x) {
    int n = 0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) n += __popc(mask[w * E + e]);
    uint8_t* h = hist + static_cast<size_t>(e) * pitch;
    h[c] = static_cast<uint8_t>(n);
    if (c == static_cast<int>(gridDim.x) - 1)
      for (int i = c + 1; i < pitch; ++i) h[i] = 0;
  }
}

// One warp an expert, four blocks' counts a lane: prefix[e][c] = rows of e in the blocks before
// c, count[e].  (With one count a lane and 32 tokens a block, 32768 tokens of 256 experts, k = 8,
// took 20.6 us for 16.7; with this inside plan_start_kernel's one block 24.6, and 9.2 for 8.7 at
// 8192 tokens of 64.)
__global__ void __launch_bounds__(256)
    plan_prefix_kernel(const uint8_t* __restrict__ hist, int E, int pitch,
                       int32_t* __restrict__ prefix, int32_t* __restrict__ count) {
  const int e = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  if (e >= E) return;
  const uint32_t* h = reinterpret_cast<const uint32_t*>(hist + static_cast<size_t>(e) * pitch);
  int4* out = reinterpret_cast<int4*>(prefix + static_cast<size_t>(e) * pitch);
  const int words = pitch / 4;
  int carry = 0;
  uint32_t next = lane < words ? h[lane] : 0;
  for (int c = lane; c - lane < words; c += 32) {
    const uint32_t n = next;
    next = c + 32 < words ? h[c + 32] : 0;
    const int n0 = n & 0xFF, n1 = n >> 8 & 0xFF, n2 = n >> 16 & 0xFF, n3 = n >> 24;
    int s = n0 + n1 + n2 + n3;
    const int own = s;
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(kAll, s, o);
      if (lane >= o) s += x;
    }
    const int before = carry + s - own;
    if (c < words) out[c] = make_int4(before, before + n0, before + n0 + n1, before + n0 + n1 + n2);
    carry += __shfl_sync(kAll, s, 31);
  }
  if (lane == 0) count[e] = carry;
}

__global__ void __launch_bounds__(PLAN_THREADS)
    plan_start_kernel(const int32_t* __restrict__ count, int E, int32_t* start, int32_t* counts,
                      RowTile* t128, RowTile* t256) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = static_cast<int>(threadIdx.x) < E ? count[threadIdx.x] : 0;
  plan_tiles(n, E, start, counts, t128, t256);
}

__global__ void __launch_bounds__(PLAN_THREADS)
    plan_rows_kernel(const int32_t* __restrict__ experts, int T, int k, int E, int pitch,
                     const int32_t* __restrict__ prefix, const int32_t* __restrict__ start,
                     int32_t* __restrict__ rows) {
  extern __shared__ uint32_t mask[];  // [WORDS][E]
  pdl_wait();
  pdl_launch_dependents();
  const int c = blockIdx.x, t0 = c * WORDS * CHUNK;
  expert_masks(experts, t0, T, k, E, mask);
  const int n = min(WORDS * CHUNK, T - t0) * k;
  const size_t at = static_cast<size_t>(t0) * k;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int e = __ldg(experts + at + i), t = i / k;
    int r = -1;
    if (e >= 0 && e < E) {
      r = start[e] + prefix[static_cast<size_t>(e) * pitch + c];
#pragma unroll
      for (int w = 0; w < WORDS; ++w) {  // the tokens before t
        const int bits = min(max(t - w * CHUNK, 0), 32);
        r += __popc(mask[w * E + e] & static_cast<uint32_t>((1ull << bits) - 1ull));
      }
    }
    rows[at + i] = r;
  }
}

// All of it in one block, for up to SMALL_CHUNKS chunks of tokens: masks [chunks][E].
constexpr int SMALL_CHUNKS = 16;
__global__ void __launch_bounds__(PLAN_THREADS)
    plan_small_kernel(const int32_t* __restrict__ experts, int T, int k, int E, int chunks,
                      int32_t* start, int32_t* counts, RowTile* t128, RowTile* t256,
                      int32_t* __restrict__ rows) {
  extern __shared__ uint32_t mask[];  // [chunks][E]; then first[E], starts
  __shared__ int32_t first[PLAN_THREADS];
  pdl_wait();
  pdl_launch_dependents();
  for (int i = threadIdx.x; i < chunks * E; i += blockDim.x) mask[i] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < T * k; i += blockDim.x) {
    const int e = __ldg(experts + i), t = i / k;
    if (e >= 0 && e < E) atomicOr(&mask[(t / CHUNK) * E + e], 1u << (t % CHUNK));
  }
  __syncthreads();
  int n = 0;
  if (static_cast<int>(threadIdx.x) < E)
    for (int c = 0; c < chunks; ++c) n += __popc(mask[c * E + threadIdx.x]);
  plan_tiles(n, E, first, counts, t128, t256);
  __syncthreads();
  for (int i = threadIdx.x; i < T * k; i += blockDim.x) {
    const int e = __ldg(experts + i), t = i / k;
    int r = -1;
    if (e >= 0 && e < E) {
      r = first[e] + __popc(mask[(t / CHUNK) * E + e] & ((1u << (t % CHUNK)) - 1u));
      for (int c = 0; c < t / CHUNK; ++c) r += __popc(mask[c * E + e]);
    }
    rows[i] = r;
  }
}

// ---------------------------------------------------------------- combine ---
// One thread eight columns of a token; blockIdx.y a share of the columns.
template <typename T>
__global__ void __launch_bounds__(256)
    combine_kernel(const uint4* __restrict__ Y, const int32_t* __restrict__ rows,
                   const float* __restrict__ weights, int tokens, int k, int D, int R, uint4* out,
                   int32_t* status) {
  const int units = D / 8;
  const int u = blockIdx.y * blockDim.x + threadIdx.x;
  const int t = blockIdx.x * blockDim.y + threadIdx.y;
  pdl_wait();
  pdl_launch_dependents();
  if (u >= units || t >= tokens) return;
  float s[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] = 0.f;
  const int32_t* tr = rows + static_cast<size_t>(t) * k;
  const float* tw = weights + static_cast<size_t>(t) * k;
  for (int j0 = 0; j0 < k; j0 += 4) {  // four rows' loads at a time
    uint4 p[4];
    float w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int r = j0 + j < k ? __ldg(tr + j0 + j) : -1;
      if (r >= R) {
        record_status(status, CLQ_ERR_DEVICE_INDEX);
        r = -1;
      }
      w[j] = r < 0 ? 0.f : __ldg(tw + j0 + j);
      p[j] = r < 0 ? make_uint4(0, 0, 0, 0) : __ldg(Y + static_cast<size_t>(r) * units + u);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t q[4] = {p[j].x, p[j].y, p[j].z, p[j].w};
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        s[2 * h] = fmaf(w[j], Num<T>::to_f(static_cast<uint16_t>(q[h])), s[2 * h]);
        s[2 * h + 1] = fmaf(w[j], Num<T>::to_f(static_cast<uint16_t>(q[h] >> 16)), s[2 * h + 1]);
      }
    }
  }
  out[static_cast<size_t>(t) * units + u] =
      make_uint4(Num<T>::pack2(s[0], s[1]), Num<T>::pack2(s[2], s[3]), Num<T>::pack2(s[4], s[5]),
                 Num<T>::pack2(s[6], s[7]));
}

template <typename T>
cudaError_t route_t(const RouteArgs& a, cudaStream_t st) {
  const int grid = (a.T + ROUTE_WARPS - 1) / ROUTE_WARPS;
  const int threads = 32 * ROUTE_WARPS;
  if (a.E <= 32) return launch_pdl(route_kernel<T, 1>, grid, threads, 0, st, a);
  if (a.E <= 64) return launch_pdl(route_kernel<T, 2>, grid, threads, 0, st, a);
  if (a.E <= 128) return launch_pdl(route_kernel<T, 4>, grid, threads, 0, st, a);
  if (a.E <= 256) return launch_pdl(route_kernel<T, 8>, grid, threads, 0, st, a);
  return launch_pdl(route_kernel<T, 16>, grid, threads, 0, st, a);
}

}  // namespace

PlanLayout plan_layout(int T, int k, int E) {
  PlanLayout p{};
  const int64_t n = static_cast<int64_t>(T) * k;
  const int64_t used = std::min<int64_t>(E, n);
  const int masks = (T + CHUNK - 1) / CHUNK;
  p.chunks = masks <= SMALL_CHUNKS ? masks : (masks + WORDS - 1) / WORDS;
  p.pitch = (p.chunks + 3) / 4 * 4;
  p.max128 = plan_rows(T, k, E) / kRowBlock;
  p.max256 = static_cast<int>((n + 255 * used) / 256);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) & ~static_cast<size_t>(255);
    return at;
  };
  p.counts_off = take(16);
  p.tiles128_off = take(static_cast<size_t>(p.max128) * sizeof(RowTile));
  p.tiles256_off = take(static_cast<size_t>(p.max256) * sizeof(RowTile));
  p.start_off = take(static_cast<size_t>(2 * E) * 4);  // starts, then row counts
  if (masks > SMALL_CHUNKS) {
    p.hist_off = take(static_cast<size_t>(E) * p.pitch);
    p.prefix_off = take(static_cast<size_t>(E) * p.pitch * 4);
  }
  p.bytes = off;
  return p;
}

cudaError_t launch_route(const RouteArgs& a, int dtype, cudaStream_t st) {
  return dtype == CLQ_F32   ? route_t<float>(a, st)
         : dtype == CLQ_F16 ? route_t<__half>(a, st)
                            : route_t<__nv_bfloat16>(a, st);
}

cudaError_t launch_plan(const int32_t* experts, int T, int k, int E, int32_t* out_rows, void* plan,
                        const PlanLayout& pl, cudaStream_t st) {
  uint8_t* p = static_cast<uint8_t*>(plan);
  int32_t* counts = reinterpret_cast<int32_t*>(p + pl.counts_off);
  int32_t* start = reinterpret_cast<int32_t*>(p + pl.start_off);
  RowTile* t128 = reinterpret_cast<RowTile*>(p + pl.tiles128_off);
  RowTile* t256 = reinterpret_cast<RowTile*>(p + pl.tiles256_off);
  if (pl.hist_off == 0)  // at most 16 * 512 masks of 4 bytes: 32 KB
    return launch_pdl(plan_small_kernel, 1, PLAN_THREADS,
                      static_cast<size_t>(pl.chunks) * E * 4, st, experts, T, k, E, pl.chunks,
                      start, counts, t128, t256, out_rows);
  uint8_t* hist = p + pl.hist_off;
  int32_t* prefix = reinterpret_cast<int32_t*>(p + pl.prefix_off);
  const size_t smem = static_cast<size_t>(WORDS) * E * 4;
  cudaError_t e = launch_pdl(plan_hist_kernel, pl.chunks, PLAN_THREADS, smem, st, experts, T, k,
                             E, pl.pitch, hist);
  if (e != cudaSuccess) return e;
  e = launch_pdl(plan_prefix_kernel, (E + 7) / 8, 256, 0, st, const_cast<const uint8_t*>(hist), E,
                 pl.pitch, prefix, start + E);
  if (e != cudaSuccess) return e;
  e = launch_pdl(plan_start_kernel, 1, PLAN_THREADS, 0, st, const_cast<const int32_t*>(start + E),
                 E, start, counts, t128, t256);
  if (e != cudaSuccess) return e;
  return launch_pdl(plan_rows_kernel, pl.chunks, PLAN_THREADS, smem, st, experts, T, k, E, pl.pitch,
                    const_cast<const int32_t*>(prefix), const_cast<const int32_t*>(start),
                    out_rows);
}

cudaError_t launch_combine(const void* Y, int dtype, const int32_t* rows, const float* weights,
                           int T, int k, int D, int R, void* out, int32_t* status,
                           cudaStream_t st) {
  const int units = D / 8;
  const int tx = std::min(256, (units + 31) / 32 * 32), ty = 256 / tx;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((T + ty - 1) / ty), static_cast<unsigned>((units + tx - 1) / tx));
  cfg.blockDim = dim3(static_cast<unsigned>(tx), static_cast<unsigned>(ty));
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  auto f16 = combine_kernel<__half>;
  auto bf16 = combine_kernel<__nv_bfloat16>;
  return cudaLaunchKernelEx(&cfg, dtype == CLQ_F16 ? f16 : bf16, static_cast<const uint4*>(Y), rows,
                            weights, T, k, D, R, static_cast<uint4*>(out), status);
}

}  // namespace mx
}  // namespace clq
