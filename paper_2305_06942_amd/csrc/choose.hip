// The router of a mixture-of-experts layer (ebag_a2a_moe_choose of
// include/ebag_a2a.h): every token's experts and their weights, the experts'
// totals with the two losses made of them, and the gradients of all of it.
#include <hip/hip_runtime.h>

#include "common.h"
#include "ebag_a2a.h"
#include "lanes.h"
#include "moe.h"
#include "vec16.h"

using namespace ebag;

namespace {

// L lanes (4 to 64) have a token, V of its logits each, four neighbouring ones at
// a time: logit (u * L + lane) * 4 + c in place 4 u + c.
constexpr int kMostParts = 256;   // workgroups whose totals are joined
constexpr int kMostGroups = 1 << 22;  // of a launch, whose threads are numbered in 32 bits
constexpr int kJoinColumns = 32;  // of a workgroup that joins them
constexpr int kMostJoins = (kMaxExperts + kJoinColumns) / kJoinColumns;

struct ChooseArgs {
  const char* logits;
  char* dlogits;
  const float* bias;        // nullptr: none
  const uint8_t* live;      // nullptr: every token counts
  int32_t* ids;
  float* weights;
  const float* dweights;    // nullptr: none
  const float* dlosses;     // nullptr: none
  int32_t* counts;          // nullptr: no totals
  float* sums;
  float* losses;
  float* work;              // of the joining workgroups: how many are done, their parts of the balance; then sums
                            // [workgroups][experts + 1], then counts
  int64_t ld, ld_out;       // bytes
  int64_t tokens;
  int32_t E, k;
  int32_t turns;            // tokens of a group of lanes
  int32_t dtype;
  int32_t normalise;
  float coef;               // experts / choices
};

__device__ __forceinline__ float* parts_of(float* work) { return work + 32; }
static_assert(1 + kMostJoins <= 32, "");

__device__ __forceinline__ double join(uint32_t lo, uint32_t hi) { return __hiloint2double((int)hi, (int)lo); }

template <int CTRL>
__device__ __forceinline__ double move_dpp(double v) {
  return join(__builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, true),
              __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, true));
}

// What a lane of the other half of 2 * D lanes has, the same lane in both halves of what
// follows: lanes of a group hold the same before and after steps 1, 2, ... up to D.
template <int D>
__device__ __forceinline__ double other(double v, int lane) {
  if constexpr (D == 1) return move_dpp<0xB1>(v);    // quad_perm 1 0 3 2
  if constexpr (D == 2) return move_dpp<0x4E>(v);    // quad_perm 2 3 0 1
  if constexpr (D == 4) return move_dpp<0x141>(v);   // row_half_mirror
  if constexpr (D == 8) return move_dpp<0x140>(v);   // row_mirror
  if constexpr (D == 16) {
    const u32x2 lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
    const u32x2 hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
    return lane & 16 ? join(lo[0], hi[0]) : join(lo[1], hi[1]);
  }
  const u32x2 lo = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
  const u32x2 hi = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
  return lane & 32 ? join(lo[0], hi[0]) : join(lo[1], hi[1]);
}

// The largest over L neighbouring lanes, in each of them.
template <int L>
__device__ __forceinline__ double largest(double v) {
  v = __builtin_fmax(v, move_dpp<0xB1>(v));
  v = __builtin_fmax(v, move_dpp<0x4E>(v));
  if constexpr (L >= 8) v = __builtin_fmax(v, move_dpp<0x141>(v));
  if constexpr (L >= 16) v = __builtin_fmax(v, move_dpp<0x140>(v));
  if constexpr (L >= 32) {
    const u32x2 lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
    const u32x2 hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
    v = __builtin_fmax(join(lo[0], hi[0]), join(lo[1], hi[1]));
  }
  if constexpr (L >= 64) {
    const u32x2 lo = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
    const u32x2 hi = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
    v = __builtin_fmax(join(lo[0], hi[0]), join(lo[1], hi[1]));
  }
  return v;
}

// A score and its expert's number as one double, so that the larger of two is the
// one to choose: fp32 widened leaves the lowest 29 bits of the mantissa free for the
// number, counted down where larger bits are a larger double (scores from 0 on) and
// up where they are a smaller one.  -0 is made 0, +inf 2^128; -inf and NaN are no
// choice at all.  Comparing takes one instruction (v_max_f64, at fp32's own rate).
constexpr uint32_t kNumber = 511;
__device__ __forceinline__ double none() { return join(0xffffffffu, 0xffefffffu); }  // -DBL_MAX
__device__ __forceinline__ bool is_none(double key) { return (uint32_t)__double2hiint(key) == 0xffefffffu; }

__device__ __forceinline__ double key_of(float score, int e) {
  const double d = (double)(score + 0.f);
  const int hi = __double2hiint(d);
  const int lo = __double2loint(d) | (e ^ (~(hi >> 31) & (int)kNumber));
  return score > -__builtin_inff() ? join((uint32_t)lo, (uint32_t)(hi < 0x47f00000 ? hi : 0x47f00000)) : none();
}
__device__ __forceinline__ int number_of(double key) {
  const uint32_t at = (uint32_t)__double2loint(key) & kNumber;
  return is_none(key) ? -1 : (int)(__double2hiint(key) < 0 ? at : kNumber - at);
}
__device__ __forceinline__ float score_of(double key) {
  return (float)join((uint32_t)__double2loint(key) & ~kNumber, (uint32_t)__double2hiint(key));
}

__device__ __forceinline__ void order(double& a, double& b) {
  const double x = a, y = b;
  a = __builtin_fmax(x, y);
  b = __builtin_fmin(x, y);
}

// Sorts V keys downwards (Batcher's odd-even merge sort).
template <int V>
__device__ __forceinline__ void sort_down(double* key) {
#pragma unroll
  for (int p = 1; p < V; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < V; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < V && (i + j) / (2 * p) == (i + j + q) / (2 * p)) order(key[i + j], key[i + j + q]);
}

// The K largest of two lists of K sorted downwards, sorted: the larger of one's first and the
// other's last and so on are those K in an order that rises once and falls once.
template <int K>
__device__ __forceinline__ void merge_down(double* a, const double* b) {
#pragma unroll
  for (int i = 0; i < K; ++i) a[i] = __builtin_fmax(a[i], b[K - 1 - i]);
#pragma unroll
  for (int d = K / 2; d >= 1; d /= 2)
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (!(i & d)) order(a[i], a[i + d]);
}

template <int D, int K>
__device__ __forceinline__ void merge_lanes(double* key, int lane) {
  double theirs[K];
#pragma unroll
  for (int i = 0; i < K; ++i) theirs[i] = other<D>(key[i], lane);
  merge_down<K>(key, theirs);
}

__device__ __forceinline__ float logit_at(const ChooseArgs& a, const char* row, int e) {
  if (a.dtype == EBAG_F32) return reinterpret_cast<const float*>(row)[e];
  const uint16_t v = reinterpret_cast<const uint16_t*>(row)[e];
  return a.dtype == EBAG_F16 ? (float)__builtin_bit_cast(_Float16, v) : __uint_as_float((uint32_t)v << 16);
}

typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// A lane's V logits; -inf behind the last expert.
template <int V, int L>
__device__ __forceinline__ void load_logits(int dtype, int E, const char* row, int lane, float* x) {
  uint32_t raw[V];
  if (dtype == EBAG_F32) {
#pragma unroll
    for (int u = 0; u < V / 4; ++u) {
      const int e = (u * L + lane) * 4;
      if (e + 4 <= E) {
        const vec16 v = load16(row + e * 4);
#pragma unroll
        for (int c = 0; c < 4; ++c) raw[4 * u + c] = v[c];
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) raw[4 * u + c] = e + c < E ? reinterpret_cast<const uint32_t*>(row)[e + c] : 0xff800000u;
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = __uint_as_float(raw[i]);
    return;
  }
  const uint32_t below = dtype == EBAG_F16 ? 0xfc00u : 0xff80u;
#pragma unroll
  for (int u = 0; u < V / 4; ++u) {
    const int e = (u * L + lane) * 4;
    if (e + 4 <= E) {
      const u32x2_any two = *reinterpret_cast<const u32x2_any*>(row + e * 2);
#pragma unroll
      for (int c = 0; c < 4; ++c) raw[4 * u + c] = c & 1 ? two[c / 2] >> 16 : two[c / 2] & 0xffffu;
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) raw[4 * u + c] = e + c < E ? reinterpret_cast<const uint16_t*>(row)[e + c] : below;
    }
  }
  if (dtype == EBAG_F16) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)raw[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = __uint_as_float(raw[i] << 16);
  }
}

// exp(x - top) of a lane's logits in place of them; their sum over the token's lanes.
template <int V, int L>
__device__ __forceinline__ float exponentials(float* x, float top) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    x[i] = __expf(x[i] - top);
    sum += x[i];
  }
  return sum_lanes(sum, L);
}

template <int V, int L>
__device__ __forceinline__ float top_of(const float* x) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < V; ++i) top = fmaxf(top, x[i]);
  return max_lanes(top, L);
}

// The k largest scores of a token.  K (8 or 16, k up to that): every lane sorts its keys and keeps
// K, and the lanes' lists become one in log2(L) merges, which every lane then has
// whole.  K = 0: the largest of the lanes' first keys is taken off k times (16384 tokens of 256 fp32 logits,
// 16 choices, 21.4 us, in lists of sixteen 11.2).
//
// TOTALS: the probabilities are summed over a workgroup's tokens, in registers, then
// over its waves in LDS, always in the same order; the choices are counted there
// with atomics on whole numbers.  One workgroup finishes by itself, several leave
// their parts to a second launch.
//
// Bound by vector instructions, not by bytes: 16384 tokens of 256 fp32 logits, eight choices, 9.0 us without totals (2.6
// of them the read), 18 with: 12 the first launch, 5 the second.  Its 965 instructions a wave keep the SIMDs busy 63 %
// of the time; sorting and merging take a third of them.  32 logits of a lane instead of 16 need fewer (two merges less for a token), but
// half the waves hide less: 9.3 and 19.  Parts laid out for the second launch, 16 bytes of every workgroup for two columns, cost
// the first more than they save there: 21.  With few tokens the chain is what counts: 32 tokens of 128 5.1 us.
template <int V, int L, int K, bool TOTALS>
__global__ __launch_bounds__(TOTALS ? 1024 : 256) void choose_kernel(const ChooseArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x % L, own = threadIdx.x / L, groups = blockDim.x / L;
  const int E = a.E, k = a.k;
  double* chosen = reinterpret_cast<double*>(lds) + own * k;
  int32_t* counts = reinterpret_cast<int32_t*>(lds + (size_t)groups * k * 8);  // [E + 1]
  float* parts = reinterpret_cast<float*>(counts + E + 1);                     // [waves][E + 1]
  if (TOTALS) {
    for (int e = threadIdx.x; e <= E; e += blockDim.x) counts[e] = 0;
    __syncthreads();
  }
  float total[V];
  float squares = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) total[i] = 0.f;
  for (int turn = 0; turn < a.turns; ++turn) {
    const int64_t n = ((int64_t)turn * gridDim.x + blockIdx.x) * groups + own;
    const bool here = n < a.tokens;
    const bool live = here && (!a.live || a.live[n]);
    const char* row = a.logits + n * a.ld;
    // The compiler keeps a comparison with E for each logit in scalar registers, and spills them, unless E is new here.
    int E = a.E;
    asm("" : "+s"(E));
    float x[V];
    double key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
    if (live) load_logits<V, L>(a.dtype, E, row, lane, x);
    if (a.bias) {
      float score[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = (i / 4 * L + lane) * 4 + i % 4;
        score[i] = x[i] + a.bias[e < E ? e : E - 1];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) key[i] = key_of(score[i], (i / 4 * L + lane) * 4 + i % 4);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) key[i] = key_of(x[i], (i / 4 * L + lane) * 4 + i % 4);
    }
    const float top = top_of<V, L>(x);
    const bool counted = top > -__builtin_inff();
    const float sum = exponentials<V, L>(x, counted ? top : 0.f);
    if (TOTALS && counted) {
      const float inv = 1.f / sum;
#pragma unroll
      for (int i = 0; i < V; ++i) total[i] = __builtin_fmaf(x[i], inv, total[i]);
      const float lse = top + logf(sum);
      squares = __builtin_fmaf(lse, lse, squares);
    }
    if (TOTALS) {
      const uint64_t some = __ballot(counted && lane == 0);
      if ((threadIdx.x & 63) == 0) atomicAdd(&counts[E], (int)__popcll(some));
    }
    if constexpr (K > 0) {
      sort_down<K>(key);
      if constexpr (V > K) {
        sort_down<K>(key + K);
        merge_down<K>(key, key + K);
      }
      merge_lanes<1, K>(key, lane);
      merge_lanes<2, K>(key, lane);
      if constexpr (L >= 8) merge_lanes<4, K>(key, lane);
      if constexpr (L >= 16) merge_lanes<8, K>(key, lane);
      if constexpr (L >= 32) merge_lanes<16, K>(key, threadIdx.x);
      if constexpr (L >= 64) merge_lanes<32, K>(key, threadIdx.x);
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (lane == j % L && j < k) chosen[j] = key[j];
    } else {
      sort_down<V>(key);
#pragma unroll 1
      for (int j = 0; j < k; ++j) {
        const double best = largest<L>(key[0]);
        const bool mine = key[0] == best;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          double next = i + 1 < V ? key[i + 1] : none();
          asm("" : "+v"(next));  // a value, not an index to select by
          key[i] = mine ? next : key[i];
        }
        if (lane == 0) chosen[j] = best;
      }
    }
    __builtin_amdgcn_wave_barrier();
    auto logit = [&](double c, int id) {  // of a choice, without the bias
      return a.bias ? logit_at(a, row, id) : score_of(c);
    };
    float from = top, over = sum;
    if (a.normalise) {
      from = -__builtin_inff();
      for (int j = lane; j < k; j += L) {
        const int id = number_of(chosen[j]);
        if (id >= 0) from = fmaxf(from, logit(chosen[j], id));
      }
      from = max_lanes(from, L);
      over = 0.f;
      for (int j = lane; j < k; j += L) {
        const int id = number_of(chosen[j]);
        if (id >= 0) over += __expf(logit(chosen[j], id) - from);
      }
      over = sum_lanes(over, L);
    }
    for (int j = lane; j < k; j += L) {
      const int id = counted ? number_of(chosen[j]) : -1;
      if (TOTALS && id >= 0) atomicAdd(&counts[id], 1);
      if (here) {
        a.ids[n * k + j] = id;
        a.weights[n * k + j] = id < 0 ? 0.f : __expf(logit(chosen[j], id) - from) / over;
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  if (!TOTALS) return;
  // Over the groups of a wave, then over the waves.
#pragma unroll
  for (int d = 32; d >= L; d /= 2) {
#pragma unroll
    for (int i = 0; i < V; ++i) total[i] += __shfl_xor(total[i], d);
    squares += __shfl_xor(squares, d);
  }
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) < L) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = (i / 4 * L + lane) * 4 + i % 4;
      if (e < E) parts[wave * (E + 1) + e] = total[i];
    }
    if (lane == 0) parts[wave * (E + 1) + E] = squares;
  }
  __syncthreads();
  const bool alone = gridDim.x == 1;
  float* sums = parts_of(a.work) + (size_t)blockIdx.x * (E + 1);
  int32_t* numbers = reinterpret_cast<int32_t*>(parts_of(a.work)) + ((size_t)gridDim.x + blockIdx.x) * (E + 1);
  for (int e = threadIdx.x; e <= E; e += blockDim.x) {
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += parts[w * (E + 1) + e];
    if (alone) {
      parts[e] = s;  // no other thread reads this column
      a.sums[e] = s;
      a.counts[e] = counts[e];
    } else {
      sums[e] = s;
      numbers[e] = counts[e];
    }
  }
  if (!alone) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<uint32_t*>(a.work) = 0;  // joining workgroups that are done
    return;
  }
  __syncthreads();
  if (wave > 0) return;
  float part = 0.f;
  for (int e = threadIdx.x; e < E; e += 64) part = __builtin_fmaf((float)counts[e], parts[e], part);
  part = sum_lanes(part, 64);
  const float per = counts[E] ? 1.f / (float)counts[E] : 0.f;
  if (threadIdx.x == 0) {
    a.losses[0] = a.coef * part * per * per;
    a.losses[1] = parts[E] * per;
  }
}

// The workgroups' totals, summed in their order: a workgroup has `columns` of them, eight threads or more each.  One
// workgroup that has all columns makes the losses of them; of several the last one to be done, whichever it is, adds up
// what all made of the balance loss, in their order.  (16384 tokens, 256 experts, 256 parts: nine workgroups of 32 columns
// and 256 threads 4.8 us, of 1024 threads 5.8, one workgroup alone 12; 60 experts, 141 parts: one of 1024 threads 3.3, two
// of 256 4.4.)
__global__ __launch_bounds__(1024) void choose_join_kernel(const ChooseArgs a, int parts, int columns) {
  __shared__ float sums[1024];
  __shared__ int32_t counts[1024];
  __shared__ float waves[16];
  const int E = a.E, column = threadIdx.x & (columns - 1), slices = blockDim.x / columns, slice = threadIdx.x / columns;
  const int e = blockIdx.x * columns + column;
  const float* work = parts_of(a.work);
  float s = 0.f;
  int32_t c = 0;
  if (e <= E) {
    const int32_t* numbers = reinterpret_cast<const int32_t*>(work) + (size_t)parts * (E + 1);
#pragma unroll 16
    for (int w = slice; w < parts; w += slices) {
      s += work[(size_t)w * (E + 1) + e];
      c += numbers[(size_t)w * (E + 1) + e];
    }
  }
  sums[threadIdx.x] = s;
  counts[threadIdx.x] = c;
  __syncthreads();
  const bool alone = gridDim.x == 1;
  float part = 0.f;
  if (slice == 0 && e <= E) {
    for (int i = 1; i < slices; ++i) {
      s += sums[i * columns + column];
      c += counts[i * columns + column];
    }
    // At device scope: another workgroup reads the last column's.
    __hip_atomic_store(&a.sums[e], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(&a.counts[e], c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (e < E) part = (float)c * s;
    if (alone && e == E) {
      sums[0] = s;  // column 0's own is in its thread's register
      counts[0] = c;
    }
  }
  part = sum_lanes(part, 64);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = part;
  __syncthreads();
  if (threadIdx.x) return;
  float all = 0.f;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) all += waves[w];
  float squares;
  int32_t T;
  if (alone) {
    squares = sums[0];
    T = counts[0];
  } else {
    __hip_atomic_store(&a.work[1 + blockIdx.x], all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // All 32 columns are this thread's wave's: its release waits for their stores.
    const uint32_t done = __hip_atomic_fetch_add(reinterpret_cast<uint32_t*>(a.work), 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    if (done + 1 != gridDim.x) return;
    all = 0.f;
    for (unsigned i = 0; i < gridDim.x; ++i)
      all += __hip_atomic_load(&a.work[1 + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    T = __hip_atomic_load(&a.counts[E], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    squares = __hip_atomic_load(&a.sums[E], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  const float per = T ? 1.f / (float)T : 0.f;
  a.losses[0] = a.coef * all * per * per;
  a.losses[1] = squares * per;
}

// With a_e = dlosses[0] E / (k T^2) counts[e], q = 2 dlosses[1] lse / T and p the
// softmax: dlogits[e] = p_e (a_e - <p, a> + q), and of the weights w with gradients d,
// in the chosen places w_j (d_j - <w, d>) where they are normalised, otherwise w_j d_j,
// and -p_e <w, d> everywhere.  The softmax is found anew: its row is read anyway.
//
// A chosen expert's logit is looked up in LDS, where the row lies until its places are
// needed for the chosen experts' part of the gradient.  16384 tokens of 256 fp32 logits, 34 MB: 12.1 us, 2.9 TB/s; bound by
// its chain (row, largest, sum, choices' sum, store) with every workgroup in it at a time.
template <int V, int L>
__global__ __launch_bounds__(256) void choose_backward_kernel(const ChooseArgs a) {
  __shared__ float places[256 / L][V * L];  // logit (u, lane, c) at ((u * 4 + c) * L + lane)
  const int lane = threadIdx.x % L, own = threadIdx.x / L;
  const int E = a.E, k = a.k;
  float* place = places[own];
  auto place_of = [&](int id) { return ((id >> 2) / L * 4 + (id & 3)) * L + (id >> 2) % L; };
  const int64_t n = (int64_t)blockIdx.x * (256 / L) + own;
  const bool here = n < a.tokens;
  const bool live = here && (!a.live || a.live[n]);
  const bool weighed = a.dweights != nullptr;
  // A lane's first choice stays in registers; further ones, where there are more than L, are read again.
  auto number = [&](int j) {
    const int id = live && j < k ? a.ids[n * k + j] : -1;
    return (uint32_t)id < (uint32_t)E ? id : -1;
  };
  const int id0 = weighed ? number(lane) : -1;
  const float d0 = id0 >= 0 ? a.dweights[n * k + lane] : 0.f;
  const char* row = a.logits + n * a.ld;
  float x[V];
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
  if (live) load_logits<V, L>(a.dtype, E, row, lane, x);
  float pull[V];
  float tokens = 0.f, balance = 0.f, squares = 0.f;
  if (a.dlosses) {
    tokens = (float)a.counts[E];
    balance = a.dlosses[0];
    squares = a.dlosses[1];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = (i / 4 * L + lane) * 4 + i % 4;
      pull[i] = (float)a.counts[e < E ? e : E - 1];
    }
  }
  float l0 = 0.f;
  if (weighed) {
#pragma unroll
    for (int i = 0; i < V; ++i) place[i * L + lane] = x[i];
    __builtin_amdgcn_wave_barrier();
    l0 = id0 >= 0 ? place[place_of(id0)] : -__builtin_inff();
  }
  const float top = top_of<V, L>(x);
  const bool counted = top > -__builtin_inff();
  const float sum = exponentials<V, L>(x, counted ? top : 0.f);
  const float inv = counted ? 1.f / sum : 0.f;
  float shift = 0.f;  // of all places, times p
  if (a.dlosses) {
    const float per = tokens > 0.f ? 1.f / tokens : 0.f, scale = balance * a.coef * per * per;
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      pull[i] *= scale;
      dot = __builtin_fmaf(x[i] * inv, pull[i], dot);
    }
    shift = 2.f * squares * per * (top + logf(sum)) - sum_lanes(dot, L);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) pull[i] = 0.f;
  }
  if (weighed) {
    float from = top, over = sum;
    if (a.normalise) {
      from = l0;
      for (int j = lane + L; j < k; j += L) {
        const int id = number(j);
        if (id >= 0) from = fmaxf(from, place[place_of(id)]);
      }
      from = max_lanes(from, L);
    }
    const float e0 = id0 >= 0 ? __expf(l0 - from) : 0.f;
    if (a.normalise) {
      over = e0;
      for (int j = lane + L; j < k; j += L) {
        const int id = number(j);
        if (id >= 0) over += __expf(place[place_of(id)] - from);
      }
      over = sum_lanes(over, L);
    }
    const float w0 = id0 >= 0 ? e0 / over : 0.f;
    float dot = w0 * d0;
    for (int j = lane + L; j < k; j += L) {
      const int id = number(j);
      if (id >= 0) dot = __builtin_fmaf(__expf(place[place_of(id)] - from) / over, a.dweights[n * k + j], dot);
    }
    dot = sum_lanes(dot, L);
    const float less = a.normalise ? dot : 0.f;
    if (!a.normalise) shift -= dot;
    // The row makes room.  Choices behind a lane's first are added from the logits in memory.
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < V; ++i) place[i * L + lane] = 0.f;
    __builtin_amdgcn_wave_barrier();
    if (id0 >= 0) atomicAdd(&place[place_of(id0)], w0 * (d0 - less));
    for (int j = lane + L; j < k; j += L) {
      const int id = number(j);
      if (id >= 0) atomicAdd(&place[place_of(id)], __expf(logit_at(a, row, id) - from) / over * (a.dweights[n * k + j] - less));
    }
    __builtin_amdgcn_wave_barrier();
  }
  if (!here) return;
  char* out = a.dlogits + n * a.ld_out;
#pragma unroll
  for (int u = 0; u < V / 4; ++u) {
    const int e = (u * L + lane) * 4;
    float d[8] = {};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int i = 4 * u + c;
      const float chosen = weighed ? place[i * L + lane] : 0.f;
      d[c] = counted ? __builtin_fmaf(x[i] * inv, pull[i] + shift, chosen) : 0.f;
    }
    if (a.dtype == EBAG_F32) {
      if (e + 4 <= E) {
        store16(out + e * 4, Type<0>::narrow(d));
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (e + c < E) reinterpret_cast<float*>(out)[e + c] = d[c];
      }
    } else {
      const vec16 v = a.dtype == EBAG_F16 ? Type<1>::narrow(d) : Type<2>::narrow(d);
      if (e + 4 <= E) {
        *reinterpret_cast<u32x2_any*>(out + e * 2) = u32x2_any{v[0], v[1]};
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (e + c < E) reinterpret_cast<uint16_t*>(out)[e + c] = (uint16_t)(c & 1 ? v[c / 2] >> 16 : v[c / 2] & 0xffffu);
      }
    }
  }
}

typedef void (*choose_fn)(const ChooseArgs);

// The instance for `lanes` lanes of `values` logits.
template <int K, bool TOTALS>
choose_fn pick_wide(int lanes) {
  switch (lanes) {
    case 4: return choose_kernel<16, 4, K, TOTALS>;
    case 8: return choose_kernel<16, 8, K, TOTALS>;
    case 16: return choose_kernel<16, 16, K, TOTALS>;
    default: return choose_kernel<16, 32, K, TOTALS>;
  }
}
template <bool TOTALS>
choose_fn pick_forward(int values, int lanes, int keep) {
  if (values == 16) return keep == 8 ? pick_wide<8, TOTALS>(lanes) : keep == 16 ? pick_wide<16, TOTALS>(lanes) : pick_wide<0, TOTALS>(lanes);
  if (values == 8) return choose_kernel<8, 64, 0, TOTALS>;
  switch (lanes) {
    case 4: return choose_kernel<4, 4, 0, TOTALS>;
    case 8: return choose_kernel<4, 8, 0, TOTALS>;
    case 16: return choose_kernel<4, 16, 0, TOTALS>;
    case 32: return choose_kernel<4, 32, 0, TOTALS>;
    default: return choose_kernel<4, 64, 0, TOTALS>;
  }
}
choose_fn pick_backward(int values, int lanes) {
  if (values == 16) {
    switch (lanes) {
      case 4: return choose_backward_kernel<16, 4>;
      case 8: return choose_backward_kernel<16, 8>;
      case 16: return choose_backward_kernel<16, 16>;
      default: return choose_backward_kernel<16, 32>;
    }
  }
  if (values == 8) return choose_backward_kernel<8, 64>;
  switch (lanes) {
    case 4: return choose_backward_kernel<4, 4>;
    case 8: return choose_backward_kernel<4, 8>;
    case 16: return choose_backward_kernel<4, 16>;
    case 32: return choose_backward_kernel<4, 32>;
    default: return choose_backward_kernel<4, 64>;
  }
}

int hipf(hipError_t e, const char* what) { return fail(EBAG_EHIP, "%s: %s", what, hipGetErrorString(e)); }

// Lanes of a token and logits of a lane.  Four logits where there are few tokens, so that the steps are short and
// spread over the card; 16, with fewer steps over the lanes, where the card is full with them.  fp32 with totals, in us
// by four (eight above 256 experts) and by 16:
//   8 choices: 16384 tokens of 64 11.7, 11.4; 32768 of 64 16.3, 12.7; 8192 of 128 13.4, 12.0; 16384 of 128 18.7, 13.3; 4096 of 256
//     14.2, 12.6; 8192 of 256 20.1, 13.6; 2048 of 512 15.2, 14.0; 4096 of 512 17.7, 15.1
//   16 choices: 8192 of 64 11.7, 14.9; 16384 of 64 14.0, 14.7; 4096 of 128 13.2, 15.5; 8192 of 128 16.4, 14.8; 2048 of 256 14.2, 15.9;
//     4096 of 256 17.5, 14.5; 1024 of 512 17.0, 17.5; 2048 of 512 18.4, 16.5
//   2 choices: 16384 of 64 10.1, 12.1; 65536 of 64 18.0, 18.2; 8192 of 128 11.6, 13.2; 32768 of 128 20.3, 19.6; 4096 of 256
//     12.1, 13.4; 8192 of 256 15.1, 14.9; 4096 of 512 14.9, 16.3
//   the gradient: 32768 of 64 6.4, 9.0; 8192 of 128 4.7, 5.3; 16384 of 128 6.7, 6.7; 8192 of 256 6.9, 7.3; 16384 of 256 11.1, 10.9;
//     4096 of 512 6.7, 7.2; 8192 of 512 10.6, 10.9
// Up to 32 experts 16 logits would leave lanes idle: 16384 of 32 with 2 choices 8.3, 12.6; 65536 of 32 11.2, 15.7, with 8 14.4, 14.3.
void shape_for(int64_t tokens, int E, int keep, int* values, int* lanes) {
  *lanes = 4;
  if (E > 32) {
    while (*lanes * 16 < E) *lanes *= 2;
    *values = 16;
    if (tokens * *lanes >= (keep == 16 ? 64 * 1024 : 64 * 2048)) return;
  }
  *values = E > 256 ? 8 : 4;
  while (*lanes * *values < E) *lanes *= 2;
}

int choose_args(ebag_a2a_moe_t h, const void* logits, int64_t ldl, int32_t dtype, int64_t tokens, const uint8_t* live,
                int32_t normalise, int keep, ChooseArgs* a, int* values, int* lanes) {
  if (int rc = check_moe_plan(h, tokens)) return rc;
  if (dtype != EBAG_F32 && dtype != EBAG_F16 && dtype != EBAG_BF16) return fail(EBAG_EINVAL, "bad dtype %d", (int)dtype);
  if (normalise != 0 && normalise != 1) return fail(EBAG_EINVAL, "normalise must be 0 or 1");
  const int elt = dtype == EBAG_F32 ? 4 : 2;
  if (tokens) {
    if (!logits) return fail(EBAG_EINVAL, "null logits");
    if (reinterpret_cast<uintptr_t>(logits) % elt) return fail(EBAG_EINVAL, "logits not aligned to its elements");
    if (ldl < h->experts || ldl > (int64_t)1 << 40)
      return fail(EBAG_EINVAL, "row step %lld of logits below the %d experts", (long long)ldl, h->experts);
  }
  *a = ChooseArgs{};
  a->logits = static_cast<const char*>(logits);
  a->ld = ldl * elt;
  a->live = live;
  a->tokens = tokens;
  a->E = h->experts;
  a->k = h->choices;
  a->dtype = dtype;
  a->normalise = normalise;
  a->coef = (float)((double)h->experts / h->choices);
  a->turns = 1;
  shape_for(tokens, a->E, keep, values, lanes);
  return EBAG_OK;
}

}  // namespace

extern "C" {

int64_t ebag_a2a_moe_choose_work(ebag_a2a_moe_t h) {
  return h ? 32 + (int64_t)kMostParts * 2 * (h->experts + 1) : 0;
}

int ebag_a2a_moe_choose(ebag_a2a_moe_t h, const void* logits, int64_t ldl, int32_t dtype, int64_t tokens,
                        const float* bias, const uint8_t* live, int32_t normalise, int32_t* ids, float* weights,
                        int32_t* counts, float* sums, float* losses, float* work, hipStream_t stream) {
  ChooseArgs a;
  int values, lanes;
  // Lists of eight or sixteen, or the largest taken off k times, where that is once or twice (fp32, in us by lists of eight and
  // taken off: 16384 tokens of 256, one choice 8.0, 7.6, with totals 17.0, 18.8; two 7.6, 8.1, 16.8, 19.5; three 7.6, 9.2, 16.9, 20.6;
  // eight 7.7, 14.1, 17.0, 24.3; 32768 of 64, one choice 4.8, 4.9, with totals 12.1, 13.2; two 4.8, 5.4, 12.0, 13.6): one and two
  // choices with totals lose 8 to 14 % by this rule.
  const int keep = !h || h->choices <= 2 || h->choices > 16 ? 0 : h->choices <= 8 ? 8 : 16;
  if (int rc = choose_args(h, logits, ldl, dtype, tokens, live, normalise, keep, &a, &values, &lanes)) return rc;
  if (tokens && (!ids || !weights)) return fail(EBAG_EINVAL, "null ids or weights");
  const bool totals = counts || sums || losses || work;
  if (totals && (!counts || !sums || !losses || !work))
    return fail(EBAG_EINVAL, "counts, sums, losses and work go together: all of them or none");
  if (!tokens && !totals) return EBAG_OK;
  a.bias = bias;
  a.ids = ids;
  a.weights = weights;
  a.counts = counts;
  a.sums = sums;
  a.losses = losses;
  a.work = work;
  // With totals large workgroups, as every one of them leaves a part to be joined, but not so large that they leave CUs
  // idle (8 choices, with 256, 512 and 1024 threads: 500 tokens of 256 15.0, 12.6 and 13.1 us, 1000 15.8, 15.0 and 14.6, 2000 18.8, 16.1
  // and 16.7, 4000 25.1, 19.2 and 17.9; 1000 of 128 13.9, 11.7 and 12.1, 4000 17.5, 14.6 and 16.0, 12000 28.9, 21.3 and 19.1; 4000 of 60 12.1, 10.0
  // and 10.1, 8000 15.1, 12.5 and 11.2, 16000 20.4, 15.4 and 14.0).
  int threads = 256;
  if (totals && tokens * lanes > 256 * 64) threads = tokens * lanes > kMostParts * 512 ? 1024 : 512;
  while (threads > 256 && threads / lanes * a.k > 6144) threads /= 2;  // 48 KiB of choices
  const int groups = threads / lanes;
  int64_t wgs = (tokens + groups - 1) / groups;
  if (wgs < 1) wgs = 1;
  const int64_t most = totals ? kMostParts : kMostGroups;
  if (wgs > most) {
    a.turns = (int32_t)((wgs + most - 1) / most);
    wgs = (wgs + a.turns - 1) / a.turns;
  }
  size_t lds = (size_t)groups * a.k * 8;
  if (totals) lds += (size_t)(a.E + 1) * 4 * (1 + threads / 64) + 64;
  const choose_fn fn = totals ? pick_forward<true>(values, lanes, keep) : pick_forward<false>(values, lanes, keep);
  hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(threads), lds, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hipf(e, "launch the choice");
  if (!totals || wgs == 1) return EBAG_OK;
  const int columns = a.E < 64 ? 64 : a.E < 128 ? 128 : kJoinColumns;
  hipLaunchKernelGGL(choose_join_kernel, dim3(a.E / columns + 1), dim3(columns == kJoinColumns ? 256 : 1024), 0, stream, a, (int)wgs, columns);
  e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the choice's totals");
}

int ebag_a2a_moe_choose_backward(ebag_a2a_moe_t h, const void* logits, int64_t ldl, int32_t dtype, int64_t tokens,
                                 const uint8_t* live, int32_t normalise, const int32_t* ids, const float* dweights,
                                 const int32_t* counts, const float* dlosses, void* dlogits, int64_t lddl,
                                 hipStream_t stream) {
  ChooseArgs a;
  int values, lanes;
  if (int rc = choose_args(h, logits, ldl, dtype, tokens, live, normalise, 0, &a, &values, &lanes)) return rc;
  if (!tokens) return EBAG_OK;
  if (!dlogits) return fail(EBAG_EINVAL, "null dlogits");
  if (dweights && !ids) return fail(EBAG_EINVAL, "null ids");
  if (dlosses && !counts) return fail(EBAG_EINVAL, "null counts");
  const int elt = dtype == EBAG_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(dlogits) % elt) return fail(EBAG_EINVAL, "dlogits not aligned to its elements");
  if (lddl < a.E || lddl > (int64_t)1 << 40)
    return fail(EBAG_EINVAL, "row step %lld of dlogits below the %d experts", (long long)lddl, a.E);
  a.ids = const_cast<int32_t*>(ids);
  a.dweights = dweights;
  a.counts = const_cast<int32_t*>(counts);
  a.dlosses = dlosses;
  a.dlogits = static_cast<char*>(dlogits);
  a.ld_out = lddl * elt;
  const int64_t groups = 256 / lanes, step = kMostGroups * groups;
  for (;;) {
    const int64_t wgs = (a.tokens + groups - 1) / groups;
    hipLaunchKernelGGL(pick_backward(values, lanes), dim3((unsigned)(wgs < kMostGroups ? wgs : kMostGroups)), dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hipf(e, "launch the choice's gradient");
    if (a.tokens <= step) return EBAG_OK;
    a.tokens -= step;
    a.logits += step * a.ld;
    a.dlogits += step * a.ld_out;
    if (a.live) a.live += step;
    if (a.ids) a.ids += step * a.k;
    if (a.dweights) a.dweights += step * a.k;
  }
}

}  // extern "C"
