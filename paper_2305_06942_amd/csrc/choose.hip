// The router of a mixture-of-experts layer (ebag_a2a_moe_choose of
// include/ebag_a2a.h): every token's experts and their weights, the experts'
// totals with the two losses made of them, and the gradients of all of it.
#include <hip/hip_runtime.h>

#include <climits>

#include "common.h"
#include "ebag_a2a.h"
#include "lanes.h"
#include "moe.h"
#include "vec16.h"

using namespace ebag;

namespace {

// 2^k lanes (4 to 64) have a token, V of its logits each, four neighbouring ones at
// a time: logit (u * lanes + lane) * 4 + c in place 4 u + c.
constexpr int kLeastLanes = 4;
constexpr int kMostParts = 256;   // workgroups whose totals are joined

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
  float* work;              // sums [workgroups][experts + 1], then counts
  int64_t ld, ld_out;       // bytes
  int64_t tokens;
  int32_t E, k;
  int32_t lanes, lanes_shift;
  int32_t turns;            // tokens of a group of lanes
  int32_t normalise;
  float coef;               // experts / choices
};

__device__ __forceinline__ double join(uint32_t lo, uint32_t hi) { return __hiloint2double((int)hi, (int)lo); }

template <int CTRL>
__device__ __forceinline__ double larger_dpp(double v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, true);
  return __builtin_fmax(v, join(lo, hi));
}

// The largest over 2^k neighbouring lanes, 4 at least, in each of them.
__device__ __forceinline__ double largest(double v, int lanes) {
  v = larger_dpp<0xB1>(v);
  v = larger_dpp<0x4E>(v);
  if (lanes >= 8) v = larger_dpp<0x141>(v);
  if (lanes >= 16) v = larger_dpp<0x140>(v);
  if (lanes >= 32) {
    const u32x2 lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
    const u32x2 hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
    v = __builtin_fmax(join(lo[0], hi[0]), join(lo[1], hi[1]));
  }
  if (lanes >= 64) {
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
  uint32_t hi = (uint32_t)__double2hiint(d), lo = (uint32_t)__double2loint(d);
  if (score == __builtin_inff()) hi = 0x47f00000u;
  lo |= (int32_t)hi < 0 ? (uint32_t)e : kNumber - (uint32_t)e;
  return score > -__builtin_inff() ? join(lo, hi) : none();
}
__device__ __forceinline__ int number_of(double key) {
  const uint32_t at = (uint32_t)__double2loint(key) & kNumber;
  return (int)(__double2hiint(key) < 0 ? at : kNumber - at);
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
          if (i + j + q < V && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const double a = key[i + j], b = key[i + j + q];
            key[i + j] = __builtin_fmax(a, b);
            key[i + j + q] = __builtin_fmin(a, b);
          }
}

template <int DT>
__device__ __forceinline__ float logit_at(const char* row, int e) {
  return Type<DT>::widen(reinterpret_cast<const typename Type<DT>::elt*>(row)[e]);
}

typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// A lane's V logits; -inf behind the last expert.
template <int DT, int V>
__device__ __forceinline__ void load_logits(const ChooseArgs& a, const char* row, int lane, float* x) {
#pragma unroll
  for (int u = 0; u < V / 4; ++u) {
    const int e = (u * a.lanes + lane) * 4;
    if (e + 4 <= a.E) {
      if constexpr (DT == 0) {
        Type<0>::widen(load16(row + e * 4), x + 4 * u);
      } else {
        const u32x2_any two = *reinterpret_cast<const u32x2_any*>(row + e * 2);
        float f[8];
        Type<DT>::widen(vec16{two[0], two[1], 0, 0}, f);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[4 * u + c] = f[c];
      }
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) x[4 * u + c] = e + c < a.E ? logit_at<DT>(row, e + c) : -__builtin_inff();
    }
  }
}

// exp(x - top) of a lane's logits in place of them; their sum over the token's lanes.
template <int V>
__device__ __forceinline__ float exponentials(float* x, float top, int lanes) {
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    x[i] = __expf(x[i] - top);
    sum += x[i];
  }
  return sum_lanes(sum, lanes);
}

template <int V>
__device__ __forceinline__ float top_of(const float* x, int lanes) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < V; ++i) top = fmaxf(top, x[i]);
  return max_lanes(top, lanes);
}

// Which lanes of a group and which token.
struct Group {
  int lane, own, groups;   // lane of the group; the group's number in the workgroup, of so many
  __device__ __forceinline__ Group(const ChooseArgs& a) {
    lane = threadIdx.x & (a.lanes - 1);
    own = threadIdx.x >> a.lanes_shift;
    groups = blockDim.x >> a.lanes_shift;
  }
};

// Losses of the totals in LDS (sums and counts of experts + 1 each), and the totals to where they belong.
__device__ void finish(const ChooseArgs& a, const float* sums, const int32_t* counts, float* waves) {
  const float T = (float)counts[a.E];
  float part = 0.f;
  for (int e = threadIdx.x; e <= a.E; e += blockDim.x) {
    a.sums[e] = sums[e];
    a.counts[e] = counts[e];
    if (e < a.E && T > 0.f) part += (float)counts[e] / T * (sums[e] / T);
  }
  part = sum_lanes(part, 64);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = part;
  __syncthreads();
  if (threadIdx.x == 0) {
    float all = 0.f;
    for (unsigned w = 0; w < blockDim.x / 64; ++w) all += waves[w];
    a.losses[0] = a.coef * all;
    a.losses[1] = T > 0.f ? sums[a.E] / T : 0.f;
  }
}

// The k largest scores of a token: every lane sorts its keys, then the largest of the
// lanes' first ones is taken off k times.
//
// TOTALS: the probabilities are summed over a workgroup's tokens, in registers, then
// over its waves in LDS, always in the same order; the choices are counted there
// with atomics on whole numbers.  One workgroup finishes by itself, several leave
// their parts to a second launch.
template <int DT, int V, bool TOTALS>
__global__ __launch_bounds__(TOTALS ? 1024 : 256) void choose_kernel(const ChooseArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Group g(a);
  const int E = a.E, k = a.k;
  int2* chosen = reinterpret_cast<int2*>(lds) + g.own * k;  // number and score of each choice
  int32_t* counts = reinterpret_cast<int32_t*>(lds + (size_t)g.groups * k * 8);  // [E + 1]
  float* parts = reinterpret_cast<float*>(counts + E + 1);                       // [waves][E + 1]
  if (TOTALS) {
    for (int e = threadIdx.x; e <= E; e += blockDim.x) counts[e] = 0;
    __syncthreads();
  }
  float bias[V], total[V];
  float squares = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = ((i / 4) * a.lanes + g.lane) * 4 + i % 4;
    bias[i] = a.bias && e < E ? a.bias[e] : 0.f;
    total[i] = 0.f;
  }
  for (int turn = 0; turn < a.turns; ++turn) {
    const int64_t n = ((int64_t)turn * gridDim.x + blockIdx.x) * g.groups + g.own;
    const bool here = n < a.tokens;
    const bool live = here && (!a.live || a.live[n]);
    const char* row = a.logits + n * a.ld;
    float x[V];
    if (live) {
      load_logits<DT, V>(a, row, g.lane, x);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
    }
    double key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = key_of(x[i] + bias[i], ((i / 4) * a.lanes + g.lane) * 4 + i % 4);
    const float top = top_of<V>(x, a.lanes);
    const bool counted = top > -__builtin_inff();
    const float sum = exponentials<V>(x, counted ? top : 0.f, a.lanes);
    if (TOTALS && counted) {
      const float inv = 1.f / sum;
#pragma unroll
      for (int i = 0; i < V; ++i) total[i] = __builtin_fmaf(x[i], inv, total[i]);
      const float lse = top + logf(sum);
      squares = __builtin_fmaf(lse, lse, squares);
      if (g.lane == 0) atomicAdd(&counts[E], 1);
    }
    sort_down<V>(key);
    for (int j = 0; j < k; ++j) {
      const double best = largest(key[0], a.lanes);
      const bool mine = key[0] == best;
#pragma unroll
      for (int i = 0; i + 1 < V; ++i) key[i] = mine ? key[i + 1] : key[i];
      key[V - 1] = mine ? none() : key[V - 1];
      if (g.lane == 0) {
        const uint32_t hi = (uint32_t)__double2hiint(best), lo = (uint32_t)__double2loint(best) & ~kNumber;
        chosen[j] = is_none(best) || !counted ? int2{-1, 0} : int2{number_of(best), (int)__float_as_uint((float)join(lo, hi))};
      }
    }
    __builtin_amdgcn_wave_barrier();
    auto logit = [&](const int2& c) {  // of a choice, without the bias
      return c.x < 0 ? -__builtin_inff() : a.bias ? logit_at<DT>(row, c.x) : __uint_as_float(c.y);
    };
    float from = top, over = sum;
    if (a.normalise) {
      from = -__builtin_inff();
      for (int j = g.lane; j < k; j += a.lanes) from = fmaxf(from, logit(chosen[j]));
      from = max_lanes(from, a.lanes);
      over = 0.f;
      for (int j = g.lane; j < k; j += a.lanes) {
        const int2 c = chosen[j];
        if (c.x >= 0) over += __expf(logit(c) - from);
      }
      over = sum_lanes(over, a.lanes);
    }
    for (int j = g.lane; j < k; j += a.lanes) {
      const int2 c = chosen[j];
      if (TOTALS && c.x >= 0) atomicAdd(&counts[c.x], 1);
      if (here) {
        a.ids[n * k + j] = c.x;
        a.weights[n * k + j] = c.x < 0 ? 0.f : __expf(logit(c) - from) / over;
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  if (!TOTALS) return;
  // Over the groups of a wave, then over the waves.
#pragma unroll
  for (int d = 32; d >= kLeastLanes; d /= 2) {
    if (d < a.lanes) break;
#pragma unroll
    for (int i = 0; i < V; ++i) total[i] += __shfl_xor(total[i], d);
    squares += __shfl_xor(squares, d);
  }
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) < a.lanes) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = ((i / 4) * a.lanes + g.lane) * 4 + i % 4;
      if (e < E) parts[wave * (E + 1) + e] = total[i];
    }
    if (g.lane == 0) parts[wave * (E + 1) + E] = squares;
  }
  __syncthreads();
  const bool alone = gridDim.x == 1;
  float* sums = a.work + (size_t)blockIdx.x * (E + 1);
  int32_t* numbers = reinterpret_cast<int32_t*>(a.work) + ((size_t)gridDim.x + blockIdx.x) * (E + 1);
  for (int e = threadIdx.x; e <= E; e += blockDim.x) {
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += parts[w * (E + 1) + e];
    if (alone) {
      parts[e] = s;  // no other thread reads this column
    } else {
      sums[e] = s;
      numbers[e] = counts[e];
    }
  }
  if (!alone) return;
  __syncthreads();
  finish(a, parts, counts, parts + (size_t)waves * (E + 1));
}

// The workgroups' totals, summed in their order.  Threads: `slices` times the columns, rounded up to whole waves.
__global__ __launch_bounds__(1024) void choose_join_kernel(const ChooseArgs a, int workgroups, int columns, int slices) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int E = a.E, e = threadIdx.x % columns, slice = threadIdx.x / columns;
  float* sums = reinterpret_cast<float*>(lds);                              // [slices][E + 1]
  int32_t* counts = reinterpret_cast<int32_t*>(sums + (size_t)slices * (E + 1));
  float* waves = reinterpret_cast<float*>(counts + (size_t)slices * (E + 1));
  if (e <= E && slice < slices) {
    const int32_t* numbers = reinterpret_cast<const int32_t*>(a.work) + (size_t)workgroups * (E + 1);
    float s = 0.f;
    int32_t c = 0;
#pragma unroll 16
    for (int w = slice; w < workgroups; w += slices) {
      s += a.work[(size_t)w * (E + 1) + e];
      c += numbers[(size_t)w * (E + 1) + e];
    }
    sums[slice * (E + 1) + e] = s;
    counts[slice * (E + 1) + e] = c;
  }
  __syncthreads();
  if (slice == 0 && e <= E) {
    float s = 0.f;
    int32_t c = 0;
    for (int i = 0; i < slices; ++i) {
      s += sums[i * (E + 1) + e];
      c += counts[i * (E + 1) + e];
    }
    sums[e] = s;
    counts[e] = c;
  }
  __syncthreads();
  finish(a, sums, counts, waves);
}

// With a_e = dlosses[0] E / (k T^2) counts[e], q = 2 dlosses[1] lse / T and p the
// softmax: dlogits[e] = p_e (a_e - <p, a> + q), and of the weights w with gradients d,
// in the chosen places w_j (d_j - <w, d>) where they are normalised, otherwise w_j d_j,
// and -p_e <w, d> everywhere.  The softmax is found anew: its row is read anyway.
template <int DT, int V>
__global__ __launch_bounds__(256) void choose_backward_kernel(const ChooseArgs a) {
  typedef Type<DT> T;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Group g(a);
  const int E = a.E, k = a.k;
  float* direct = reinterpret_cast<float*>(lds) + (size_t)g.own * a.lanes * V;  // of the chosen places, in the lanes' order
  const int64_t n = (int64_t)blockIdx.x * g.groups + g.own;
  const bool here = n < a.tokens;
  const bool live = here && (!a.live || a.live[n]);
  const char* row = a.logits + n * a.ld;
  float x[V];
  if (live) {
    load_logits<DT, V>(a, row, g.lane, x);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = -__builtin_inff();
  }
#pragma unroll
  for (int i = 0; i < V; ++i) direct[i * a.lanes + g.lane] = 0.f;
  const float top = top_of<V>(x, a.lanes);
  const bool counted = top > -__builtin_inff();
  const float sum = exponentials<V>(x, counted ? top : 0.f, a.lanes);
  const float inv = counted ? 1.f / sum : 0.f;
  float shift = 0.f;  // of all places, times p
  float pull[V];
  if (a.dlosses) {
    const float tokens = (float)a.counts[E], per = tokens > 0.f ? 1.f / tokens : 0.f;
    const float scale = a.dlosses[0] * a.coef * per * per;
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = ((i / 4) * a.lanes + g.lane) * 4 + i % 4;
      pull[i] = e < E ? scale * (float)a.counts[e] : 0.f;
      dot = __builtin_fmaf(x[i] * inv, pull[i], dot);
    }
    shift = 2.f * a.dlosses[1] * per * (top + logf(sum)) - sum_lanes(dot, a.lanes);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) pull[i] = 0.f;
  }
  if (a.dweights) {
    auto number = [&](int j) {
      const int id = counted ? a.ids[n * k + j] : -1;
      return (uint32_t)id < (uint32_t)E ? id : -1;
    };
    float from = top, over = sum;
    if (a.normalise) {
      from = -__builtin_inff();
      for (int j = g.lane; j < k; j += a.lanes) {
        const int id = number(j);
        if (id >= 0) from = fmaxf(from, logit_at<DT>(row, id));
      }
      from = max_lanes(from, a.lanes);
      over = 0.f;
      for (int j = g.lane; j < k; j += a.lanes) {
        const int id = number(j);
        if (id >= 0) over += __expf(logit_at<DT>(row, id) - from);
      }
      over = sum_lanes(over, a.lanes);
    }
    float dot = 0.f;
    for (int j = g.lane; j < k; j += a.lanes) {
      const int id = number(j);
      if (id >= 0) dot = __builtin_fmaf(__expf(logit_at<DT>(row, id) - from) / over, a.dweights[n * k + j], dot);
    }
    dot = sum_lanes(dot, a.lanes);
    __builtin_amdgcn_wave_barrier();
    for (int j = g.lane; j < k; j += a.lanes) {
      const int id = number(j);
      if (id < 0) continue;
      const float w = __expf(logit_at<DT>(row, id) - from) / over;
      const int quad = id >> 2;  // its place: number u * lanes + lane of the lanes' quads
      const int at = ((quad >> a.lanes_shift) * 4 + (id & 3)) * a.lanes + (quad & (a.lanes - 1));
      atomicAdd(&direct[at], w * (a.dweights[n * k + j] - (a.normalise ? dot : 0.f)));
    }
    __builtin_amdgcn_wave_barrier();
    if (!a.normalise) shift -= dot;
  }
  if (!here) return;
  char* out = a.dlogits + n * a.ld_out;
#pragma unroll
  for (int u = 0; u < V / 4; ++u) {
    const int e = (u * a.lanes + g.lane) * 4;
    float d[8] = {};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int i = 4 * u + c;
      d[c] = counted ? __builtin_fmaf(x[i] * inv, pull[i] + shift, direct[i * a.lanes + g.lane]) : 0.f;
    }
    if (e + 4 <= E) {
      if constexpr (DT == 0) {
        store16(out + e * 4, T::narrow(d));
      } else {
        const vec16 v = T::narrow(d);
        *reinterpret_cast<u32x2_any*>(out + e * 2) = u32x2_any{v[0], v[1]};
      }
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (e + c < E) reinterpret_cast<typename T::elt*>(out)[e + c] = T::narrow(d[c]);
    }
  }
}

typedef void (*choose_fn)(const ChooseArgs);

template <int DT>
choose_fn pick_forward(int values, bool totals) {
  if (totals) return values == 4 ? choose_kernel<DT, 4, true> : values == 8 ? choose_kernel<DT, 8, true> : choose_kernel<DT, 16, true>;
  return values == 4 ? choose_kernel<DT, 4, false> : values == 8 ? choose_kernel<DT, 8, false> : choose_kernel<DT, 16, false>;
}
template <int DT>
choose_fn pick_backward(int values) {
  return values == 4 ? choose_backward_kernel<DT, 4> : values == 8 ? choose_backward_kernel<DT, 8> : choose_backward_kernel<DT, 16>;
}

int hipf(hipError_t e, const char* what) { return fail(EBAG_EHIP, "%s: %s", what, hipGetErrorString(e)); }

// Logits of a lane: few where there are few tokens, so that their steps are short and spread over the card; many
// where the card is full anyway.
int values_for(int64_t tokens, int E) {
  for (int v = 16; v > 4; v /= 2) {
    int lanes = kLeastLanes;
    while (lanes * v < E) lanes *= 2;
    if (tokens * lanes >= 64 * 2048) return v;
  }
  return E > 256 ? 8 : 4;
}

int choose_args(ebag_a2a_moe_t h, const void* logits, int64_t ldl, int32_t dtype, int64_t tokens, const uint8_t* live,
                int32_t normalise, ChooseArgs* a, int* values) {
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
  a->normalise = normalise;
  a->coef = (float)((double)h->experts / h->choices);
  a->turns = 1;
  *values = values_for(tokens, a->E);
  a->lanes = kLeastLanes;
  a->lanes_shift = 2;
  while (a->lanes * *values < a->E) {
    a->lanes *= 2;
    ++a->lanes_shift;
  }
  return EBAG_OK;
}

}  // namespace

extern "C" {

int64_t ebag_a2a_moe_choose_work(ebag_a2a_moe_t h) {
  return h ? (int64_t)kMostParts * 2 * (h->experts + 1) : 0;
}

int ebag_a2a_moe_choose(ebag_a2a_moe_t h, const void* logits, int64_t ldl, int32_t dtype, int64_t tokens,
                        const float* bias, const uint8_t* live, int32_t normalise, int32_t* ids, float* weights,
                        int32_t* counts, float* sums, float* losses, float* work, hipStream_t stream) {
  ChooseArgs a;
  int values;
  if (int rc = choose_args(h, logits, ldl, dtype, tokens, live, normalise, &a, &values)) return rc;
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
  // With totals large workgroups, as every one of them leaves a part to be joined.
  int threads = 256;
  if (totals && tokens * a.lanes > 256 * 64) threads = 1024;
  while (threads > 256 && threads / a.lanes * a.k > 6144) threads /= 2;  // 48 KiB of choices
  const int groups = threads / a.lanes;
  int64_t wgs = (tokens + groups - 1) / groups;
  if (wgs < 1) wgs = 1;
  if (totals && wgs > kMostParts) {
    a.turns = (int32_t)((wgs + kMostParts - 1) / kMostParts);
    wgs = (wgs + a.turns - 1) / a.turns;
  }
  if (wgs > INT_MAX) return fail(EBAG_EINVAL, "too many tokens for one launch");
  size_t lds = (size_t)groups * a.k * 8;
  if (totals) lds += (size_t)(a.E + 1) * 4 * (1 + threads / 64) + 64;
  const choose_fn fn = dtype == EBAG_F32   ? pick_forward<0>(values, totals)
                       : dtype == EBAG_F16 ? pick_forward<1>(values, totals)
                                           : pick_forward<2>(values, totals);
  hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(threads), lds, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hipf(e, "launch the choice");
  if (!totals || wgs == 1) return EBAG_OK;
  const int columns = (a.E + 1 + 63) / 64 * 64, slices = 1024 / columns;
  hipLaunchKernelGGL(choose_join_kernel, dim3(1), dim3(columns * slices), (size_t)slices * (a.E + 1) * 8 + 64, stream, a,
                     (int)wgs, columns, slices);
  e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the choice's totals");
}

int ebag_a2a_moe_choose_backward(ebag_a2a_moe_t h, const void* logits, int64_t ldl, int32_t dtype, int64_t tokens,
                                 const uint8_t* live, int32_t normalise, const int32_t* ids, const float* dweights,
                                 const int32_t* counts, const float* dlosses, void* dlogits, int64_t lddl,
                                 hipStream_t stream) {
  ChooseArgs a;
  int values;
  if (int rc = choose_args(h, logits, ldl, dtype, tokens, live, normalise, &a, &values)) return rc;
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
  const int groups = 256 / a.lanes;
  const int64_t wgs = (tokens + groups - 1) / groups;
  if (wgs > INT_MAX) return fail(EBAG_EINVAL, "too many tokens for one launch");
  const choose_fn fn = dtype == EBAG_F32   ? pick_backward<0>(values)
                       : dtype == EBAG_F16 ? pick_backward<1>(values)
                                           : pick_backward<2>(values);
  hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(256), (size_t)256 * values * 4, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, "launch the choice's gradient");
}

}  // extern "C"
