// Tokens by expert (ebag_a2a_moe_* of include/ebag_a2a.h): the sort of the
// tokens' choices and the kernels that move and sum the tokens' rows.
#include <hip/hip_runtime.h>

#include <climits>
#include <new>

#include "common.h"
#include "ebag_a2a.h"
#include "in_flight.h"
#include "vec16.h"

using namespace ebag;

namespace {

constexpr int kMaxChoices = 64, kMaxExperts = 512;

// ------------------------------------------------------------------- sort
//
// A stable counting sort: pos(i) = choices of smaller keys + earlier choices of
// the same key, the key being the expert, or `experts` for a dropped choice.  A
// workgroup takes chunks of 4096 choices, 256 to a wave in four batches of a
// lane each.  Inside a batch a lane's rank is the number of lower lanes with
// its key, found with a ballot per bit of the key; a counter per (wave, key) in
// LDS carries it from batch to batch, and sums over the waves and over the
// chunks before place the rest.  No atomic decides an order.

constexpr int kSortWaves = 16, kSortBatches = 4, kSortThreads = 64 * kSortWaves;
constexpr int kSortChunk = kSortThreads * kSortBatches;
constexpr int kSortMaxWgs = 128;

struct SortArgs {
  const int32_t* experts_of;
  int32_t* offsets;
  int32_t* pos;
  int32_t* src;
  uint32_t* counts;  // [workgroups][experts + 1]
  uint32_t S;
  uint32_t chunks;         // of the whole sort
  uint32_t chunks_per_wg;
  int32_t experts;
  int32_t key_bits;        // bits of experts + 1
};

__device__ __forceinline__ uint32_t key_at(const SortArgs& a, uint32_t i) {
  if (i >= a.S) return a.experts + 1;  // no choice
  const uint32_t e = (uint32_t)a.experts_of[i];
  return e < (uint32_t)a.experts ? e : (uint32_t)a.experts;
}

// Choices of each key in this workgroup's chunks, into total[experts + 1].
__device__ void count_keys(const SortArgs& a, uint32_t first, uint32_t last, uint32_t* total) {
  for (int e = threadIdx.x; e <= a.experts; e += kSortThreads) total[e] = 0;
  __syncthreads();
  for (uint32_t c = first; c < last; ++c) {
#pragma unroll
    for (int b = 0; b < kSortBatches; ++b) {
      const uint32_t key = key_at(a, c * kSortChunk + b * kSortThreads + threadIdx.x);
      if (key <= (uint32_t)a.experts) atomicAdd(&total[key], 1u);
    }
  }
  __syncthreads();
}

__device__ __forceinline__ void wg_chunks(const SortArgs& a, uint32_t* first, uint32_t* last) {
  *first = blockIdx.x * a.chunks_per_wg;
  *last = *first + a.chunks_per_wg < a.chunks ? *first + a.chunks_per_wg : a.chunks;
}

__global__ __launch_bounds__(kSortThreads) void moe_count_kernel(const SortArgs a) {
  __shared__ uint32_t total[kMaxExperts + 1];
  uint32_t first, last;
  wg_chunks(a, &first, &last);
  count_keys(a, first, last, total);
  for (int e = threadIdx.x; e <= a.experts; e += kSortThreads) a.counts[blockIdx.x * (a.experts + 1) + e] = total[e];
}

// ALONE: one workgroup has all choices and counts them itself.
template <bool ALONE>
__global__ __launch_bounds__(kSortThreads) void moe_place_kernel(const SortArgs a) {
  __shared__ uint32_t base[kMaxExperts + 1];  // where the next choice of each key goes
  __shared__ uint32_t wave_sum[kSortWaves];
  __shared__ uint16_t seen[kSortWaves][kMaxExperts + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int e = threadIdx.x;  // the key this thread sums (experts + 1 <= 1024 keys)
  uint32_t first, last, total = 0, before = 0;
  wg_chunks(a, &first, &last);
  if (ALONE) {
    count_keys(a, first, last, base);
    if (e <= a.experts) total = base[e];
  } else if (e <= a.experts) {
    for (uint32_t g = 0; g < gridDim.x; ++g) {
      const uint32_t n = a.counts[g * (a.experts + 1) + e];
      total += n;
      if (g < blockIdx.x) before += n;
    }
  }
  // Exclusive sum of the totals over the keys.
  uint32_t upto = total;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += wave_sum[w];
  if (e <= a.experts) {
    base[e] = upto - total + before;
    if (blockIdx.x == 0) a.offsets[e] = (int32_t)(upto - total);
  }
  for (uint32_t c = first; c < last; ++c) {
    for (int k = lane; k <= a.experts; k += 64) seen[wave][k] = 0;
    __builtin_amdgcn_wave_barrier();
    uint32_t key[kSortBatches], rank[kSortBatches];
    const uint32_t i0 = c * kSortChunk + wave * (64 * kSortBatches) + lane;
#pragma unroll
    for (int b = 0; b < kSortBatches; ++b) key[b] = key_at(a, i0 + b * 64);
#pragma unroll
    for (int b = 0; b < kSortBatches; ++b) {
      uint64_t same = ~0ull;
      for (int bit = 0; bit < a.key_bits; ++bit) {
        const bool on = key[b] >> bit & 1;
        const uint64_t with = __ballot(on);
        same &= on ? with : ~with;
      }
      const uint32_t lower = __popcll(same & ((1ull << lane) - 1));
      rank[b] = 0;
      if (key[b] <= (uint32_t)a.experts) {
        // A wave's LDS accesses stay in order: every lane reads the counter before its first lane moves it on.
        const uint32_t n = seen[wave][key[b]];
        rank[b] = n + lower;
        __builtin_amdgcn_wave_barrier();
        if (lower == 0) seen[wave][key[b]] = (uint16_t)(n + __popcll(same));
      }
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    uint32_t in_chunk = 0;
    if (e <= a.experts) {
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t n = seen[w][e];
        seen[w][e] = (uint16_t)in_chunk;
        in_chunk += n;
      }
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kSortBatches; ++b) {
      if (key[b] > (uint32_t)a.experts) continue;
      const uint32_t i = i0 + b * 64, p = base[key[b]] + seen[wave][key[b]] + rank[b];
      a.pos[i] = (int32_t)p;
      a.src[p] = (int32_t)i;
    }
    __syncthreads();
    if (e <= a.experts) base[e] += in_chunk;
  }
}

// ------------------------------------------------------------------- rows

struct RowArgs {
  const char* in;          // dispatch: x; combine: ys; combine backward: dout
  const char* in2;         // combine backward: ys
  char* out;               // dispatch: xs; combine: out; combine backward: dys
  const int32_t* offsets;
  const int32_t* pos;
  const float* weights;    // nullptr: 1
  float* dweights;
  int64_t ld_in, ld_in2, ld_out;  // bytes
  int64_t tokens;
  uint32_t S;
  int32_t choices, experts;
  int32_t vecs;            // whole 16-byte vectors of a row
  int32_t tail;            // elements behind them
  int32_t lanes;           // lanes of a token: a power of two, 64 for rows of more than 32 vectors
};

// Rows of more than 32 vectors have a wave (or several) to themselves: the
// token and its places are the same for all lanes and sit in scalar registers.
// Shorter ones share a wave.
template <bool WHOLE>
struct Place {
  int64_t token;
  int lane, lanes;
  bool any;
  __device__ __forceinline__ Place(const RowArgs& a) {
    const int wave = threadIdx.x >> 6;
    if (WHOLE) {
      lanes = 64;
      lane = threadIdx.x & 63;
      token = (int64_t)blockIdx.x * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(wave);
    } else {
      lanes = a.lanes;
      lane = threadIdx.x & (lanes - 1);
      token = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / lanes;
    }
    any = token < a.tokens;
  }
};

// Places below `kept` hold an expert's row, those up to S a dropped one.
__device__ __forceinline__ uint32_t kept_rows(const RowArgs& a) {
  const uint32_t n = (uint32_t)a.offsets[a.experts];
  return n < a.S ? n : a.S;
}

constexpr int kRowThreads = 256, kAtOnce = 8;

// xs[pos[n, j]] = x[n]: every row is read once and written `choices` times.
template <int DT, bool WHOLE>
__global__ __launch_bounds__(kRowThreads) void moe_dispatch_kernel(const RowArgs a) {
  typedef Type<DT> T;
  const Place<WHOLE> at(a);
  if (!at.any) return;
  const uint32_t kept = kept_rows(a);
  const int32_t* pos = a.pos + at.token * a.choices;
  const char* row = a.in + at.token * a.ld_in;
  const vec16 zero = {0, 0, 0, 0};
  for (int v = at.lane + blockIdx.y * at.lanes; v < a.vecs; v += at.lanes * gridDim.y) {
    const vec16 r = load16(row + (int64_t)v * 16);
    for (int j = 0; j < a.choices; ++j) {
      const uint32_t p = (uint32_t)pos[j];
      if (p < a.S) store16(a.out + p * a.ld_out + (int64_t)v * 16, p < kept ? r : zero);
    }
  }
  if (blockIdx.y == 0) {
    for (int t = at.lane; t < a.tail; t += at.lanes) {
      const int64_t byte = (int64_t)a.vecs * 16 + t * (int)sizeof(typename T::elt);
      const typename T::elt r = *reinterpret_cast<const typename T::elt*>(row + byte);
      for (int j = 0; j < a.choices; ++j) {
        const uint32_t p = (uint32_t)pos[j];
        if (p < a.S) *reinterpret_cast<typename T::elt*>(a.out + p * a.ld_out + byte) = p < kept ? r : (typename T::elt)0;
      }
    }
  }
}

// out[n] = sum_j weights[n, j] * in[pos[n, j]].
template <int DT, bool WHOLE>
__global__ __launch_bounds__(kRowThreads) void moe_combine_kernel(const RowArgs a) {
  typedef Type<DT> T;
  const Place<WHOLE> at(a);
  if (!at.any) return;
  const uint32_t kept = kept_rows(a);
  const int32_t* pos = a.pos + at.token * a.choices;
  const float* weights = a.weights ? a.weights + at.token * a.choices : nullptr;
  char* row = a.out + at.token * a.ld_out;
  for (int v = at.lane + blockIdx.y * at.lanes; v < a.vecs; v += at.lanes * gridDim.y) {
    float sum[T::N] = {};
    for (int j0 = 0; j0 < a.choices; j0 += kAtOnce) {
      vec16 r[kAtOnce];
      float w[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        r[i] = vec16{0, 0, 0, 0};
        w[i] = 0.f;
        const int j = j0 + i;
        if (j >= a.choices) continue;
        const uint32_t p = (uint32_t)pos[j];
        if (p >= kept) continue;
        w[i] = weights ? weights[j] : 1.f;
        r[i] = load16(a.in + p * a.ld_in + (int64_t)v * 16);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        float f[T::N];
        T::widen(r[i], f);
#pragma unroll
        for (int n = 0; n < T::N; ++n) sum[n] = __builtin_fmaf(w[i], f[n], sum[n]);
      }
    }
    store16(row + (int64_t)v * 16, T::narrow(sum));
  }
  if (blockIdx.y == 0) {
    for (int t = at.lane; t < a.tail; t += at.lanes) {
      const int64_t byte = (int64_t)a.vecs * 16 + t * (int)sizeof(typename T::elt);
      float sum = 0.f;
      for (int j = 0; j < a.choices; ++j) {
        const uint32_t p = (uint32_t)pos[j];
        if (p < kept)
          sum = __builtin_fmaf(weights ? weights[j] : 1.f,
                               T::widen(*reinterpret_cast<const typename T::elt*>(a.in + p * a.ld_in + byte)), sum);
      }
      *reinterpret_cast<typename T::elt*>(row + byte) = T::narrow(sum);
    }
  }
}

// dys[pos[n, j]] = weights[n, j] * dout[n] and dweights[n, j] = <dout[n],
// ys[pos[n, j]]>: one pass over dout and ys.
template <int DT, bool WHOLE>
__global__ __launch_bounds__(kRowThreads) void moe_combine_backward_kernel(const RowArgs a) {
  typedef Type<DT> T;
  const Place<WHOLE> at(a);
  if (!at.any) return;
  const uint32_t kept = kept_rows(a);
  const int32_t* pos = a.pos + at.token * a.choices;
  const float* weights = a.weights + at.token * a.choices;
  const char* row = a.in + at.token * a.ld_in;
  for (int j0 = 0; j0 < a.choices; j0 += kAtOnce) {
    float dot[kAtOnce] = {};
    for (int v = at.lane; v < a.vecs; v += at.lanes) {
      float d[T::N];
      T::widen(load16(row + (int64_t)v * 16), d);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int j = j0 + i;
        if (j >= a.choices) continue;
        const uint32_t p = (uint32_t)pos[j];
        float y[T::N] = {}, s[T::N] = {};
        if (p < kept) {
          T::widen(load16(a.in2 + p * a.ld_in2 + (int64_t)v * 16), y);
          const float w = weights[j];
#pragma unroll
          for (int n = 0; n < T::N; ++n) {
            s[n] = w * d[n];
            dot[i] = __builtin_fmaf(d[n], y[n], dot[i]);
          }
        }
        if (p < a.S) store16(a.out + p * a.ld_out + (int64_t)v * 16, T::narrow(s));
      }
    }
    for (int t = at.lane; t < a.tail; t += at.lanes) {
      const int64_t byte = (int64_t)a.vecs * 16 + t * (int)sizeof(typename T::elt);
      const float d = T::widen(*reinterpret_cast<const typename T::elt*>(row + byte));
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int j = j0 + i;
        if (j >= a.choices) continue;
        const uint32_t p = (uint32_t)pos[j];
        float s = 0.f;
        if (p < kept) {
          s = weights[j] * d;
          dot[i] = __builtin_fmaf(d, T::widen(*reinterpret_cast<const typename T::elt*>(a.in2 + p * a.ld_in2 + byte)), dot[i]);
        }
        if (p < a.S) *reinterpret_cast<typename T::elt*>(a.out + p * a.ld_out + byte) = T::narrow(s);
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      for (int d = at.lanes / 2; d; d /= 2) dot[i] += __shfl_xor(dot[i], d);
      if (at.lane == 0 && j0 + i < a.choices) a.dweights[at.token * a.choices + j0 + i] = dot[i];
    }
  }
}

typedef void (*row_fn)(const RowArgs);

template <bool WHOLE>
row_fn pick_dispatch(int dt) {
  return dt == EBAG_F32 ? moe_dispatch_kernel<0, WHOLE> : dt == EBAG_F16 ? moe_dispatch_kernel<1, WHOLE> : moe_dispatch_kernel<2, WHOLE>;
}
template <bool WHOLE>
row_fn pick_combine(int dt) {
  return dt == EBAG_F32 ? moe_combine_kernel<0, WHOLE> : dt == EBAG_F16 ? moe_combine_kernel<1, WHOLE> : moe_combine_kernel<2, WHOLE>;
}
template <bool WHOLE>
row_fn pick_backward(int dt) {
  return dt == EBAG_F32   ? moe_combine_backward_kernel<0, WHOLE>
         : dt == EBAG_F16 ? moe_combine_backward_kernel<1, WHOLE>
                          : moe_combine_backward_kernel<2, WHOLE>;
}

int hipf(hipError_t e, const char* what) { return fail(EBAG_EHIP, "%s: %s", what, hipGetErrorString(e)); }

}  // namespace

struct ebag_a2a_moe_plan {
  int device = 0;
  int64_t max_tokens = 0;
  int32_t choices = 0, experts = 0;
  uint32_t* d_counts = nullptr;
  InFlight sort;
};

namespace {

void free_moe(ebag_a2a_moe_plan* h) {
  if (!h) return;
  if (h->sort.done) (void)hipEventDestroy(h->sort.done);
  (void)hipFree(h->d_counts);
  delete h;
}

int check_plan(ebag_a2a_moe_plan* h, int64_t tokens) {
  if (!h) return fail(EBAG_EINVAL, "null plan");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != h->device)
    return fail(EBAG_EINVAL, "the plan belongs to device %d, but device %d is current", h->device, dev);
  if (tokens < 0 || tokens > h->max_tokens)
    return fail(EBAG_EINVAL, "tokens=%lld outside [0, max_tokens=%lld]", (long long)tokens, (long long)h->max_tokens);
  return EBAG_OK;
}

// Checks a row call's shape and fills what all of them share.
int row_args(ebag_a2a_moe_plan* h, int64_t dim, int32_t dtype, int64_t tokens, const int32_t* offsets,
             const int32_t* pos, RowArgs* a) {
  if (int rc = check_plan(h, tokens)) return rc;
  if (dtype != EBAG_F32 && dtype != EBAG_F16 && dtype != EBAG_BF16) return fail(EBAG_EINVAL, "bad dtype %d", (int)dtype);
  if (dim < 1 || dim > INT_MAX / 4) return fail(EBAG_EINVAL, "dim=%lld outside [1, 2^29)", (long long)dim);
  if (tokens && (!offsets || !pos)) return fail(EBAG_EINVAL, "null offsets or pos");
  const int elt = dtype == EBAG_F32 ? 4 : 2;
  *a = RowArgs{};
  a->offsets = offsets;
  a->pos = pos;
  a->tokens = tokens;
  a->S = (uint32_t)(tokens * h->choices);
  a->choices = h->choices;
  a->experts = h->experts;
  a->vecs = (int32_t)(dim * elt / 16);
  a->tail = (int32_t)(dim - (int64_t)a->vecs * (16 / elt));
  a->lanes = 1;
  while (a->lanes < 64 && a->lanes < a->vecs) a->lanes *= 2;
  return EBAG_OK;
}

int row_matrix(const char* what, const void* p, int64_t ld, int64_t dim, int32_t dtype, int64_t* ld_bytes) {
  const int elt = dtype == EBAG_F32 ? 4 : 2;
  if (!p) return fail(EBAG_EINVAL, "null %s", what);
  if (reinterpret_cast<uintptr_t>(p) % elt) return fail(EBAG_EINVAL, "%s is not aligned to its elements", what);
  if (ld < dim || ld > (int64_t)1 << 40) return fail(EBAG_EINVAL, "row step %lld of %s below dim=%lld", (long long)ld, what, (long long)dim);
  *ld_bytes = ld * elt;
  return EBAG_OK;
}

int launch_rows(row_fn whole, row_fn part, const RowArgs& a, bool split, const char* what, hipStream_t stream) {
  const int64_t per_wg = kRowThreads / a.lanes;
  const int64_t wgs = (a.tokens + per_wg - 1) / per_wg;
  if (wgs > INT_MAX) return fail(EBAG_EINVAL, "too many tokens for one launch");
  unsigned y = 1;
  if (split && a.lanes == 64) {
    while (y < 64 && (int)(y * 128) < a.vecs) y *= 2;
  }
  hipLaunchKernelGGL(a.lanes == 64 ? whole : part, dim3((unsigned)wgs, y), dim3(kRowThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EBAG_OK : hipf(e, what);
}

}  // namespace

extern "C" {

int ebag_a2a_moe_create(ebag_a2a_moe_t* out, int64_t max_tokens, int32_t choices, int32_t experts) {
  if (!out) return fail(EBAG_EINVAL, "null output handle");
  *out = nullptr;
  if (choices < 1 || choices > kMaxChoices) return fail(EBAG_EINVAL, "choices=%d outside [1, %d]", choices, kMaxChoices);
  if (experts < 1 || experts > kMaxExperts) return fail(EBAG_EINVAL, "experts=%d outside [1, %d]", experts, kMaxExperts);
  if (max_tokens < 0 || max_tokens > (INT_MAX - kSortChunk) / choices)
    return fail(EBAG_EINVAL, "max_tokens=%lld: max_tokens * choices must be below 2^31", (long long)max_tokens);
  ebag_a2a_moe_plan* h = new (std::nothrow) ebag_a2a_moe_plan();
  if (!h) return fail(EBAG_ENOMEM, "host allocation failed");
  h->max_tokens = max_tokens;
  h->choices = choices;
  h->experts = experts;
  hipError_t e = hipGetDevice(&h->device);
  if (e == hipSuccess) e = hipMalloc((void**)&h->d_counts, sizeof(uint32_t) * kSortMaxWgs * (experts + 1));
  if (e == hipSuccess) e = hipEventCreateWithFlags(&h->sort.done, hipEventDisableTiming);
  if (e != hipSuccess) {
    free_moe(h);
    return hipf(e, "create the plan");
  }
  *out = h;
  clear_error();
  return EBAG_OK;
}

int ebag_a2a_moe_sort(ebag_a2a_moe_t h, const int32_t* experts_of, int64_t tokens, int32_t* offsets, int32_t* pos,
                      int32_t* src, hipStream_t stream) {
  if (int rc = check_plan(h, tokens)) return rc;
  if (!offsets || (tokens && (!experts_of || !pos || !src))) return fail(EBAG_EINVAL, "null experts_of, offsets, pos or src");
  SortArgs a{};
  a.experts_of = experts_of;
  a.offsets = offsets;
  a.pos = pos;
  a.src = src;
  a.counts = h->d_counts;
  a.S = (uint32_t)(tokens * h->choices);
  a.chunks = (a.S + kSortChunk - 1) / kSortChunk;
  a.experts = h->experts;
  while (1 << a.key_bits < a.experts + 2) ++a.key_bits;
  // One workgroup alone has no second launch, but its chunks follow each other.
  if (a.chunks <= 4) {
    a.chunks_per_wg = a.chunks;
    hipLaunchKernelGGL(moe_place_kernel<true>, dim3(1), dim3(kSortThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? EBAG_OK : hipf(e, "launch the sort");
  }
  if (int rc = check_busy(h->sort, stream, "sort")) return rc;
  a.chunks_per_wg = (a.chunks + kSortMaxWgs - 1) / kSortMaxWgs;
  const unsigned wgs = (a.chunks + a.chunks_per_wg - 1) / a.chunks_per_wg;
  hipLaunchKernelGGL(moe_count_kernel, dim3(wgs), dim3(kSortThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return hipf(e, "launch the sort's count");
  hipLaunchKernelGGL(moe_place_kernel<false>, dim3(wgs), dim3(kSortThreads), 0, stream, a);
  e = hipGetLastError();
  if (e != hipSuccess) return hipf(e, "launch the sort");
  return note_call(h->sort, stream);
}

int ebag_a2a_moe_dispatch(ebag_a2a_moe_t h, const void* x, int64_t ldx, int64_t dim, int32_t dtype, int64_t tokens,
                          const int32_t* offsets, const int32_t* pos, void* xs, int64_t ldxs, hipStream_t stream) {
  RowArgs a;
  if (int rc = row_args(h, dim, dtype, tokens, offsets, pos, &a)) return rc;
  if (!tokens) return EBAG_OK;
  if (int rc = row_matrix("x", x, ldx, dim, dtype, &a.ld_in)) return rc;
  if (int rc = row_matrix("xs", xs, ldxs, dim, dtype, &a.ld_out)) return rc;
  a.in = static_cast<const char*>(x);
  a.out = static_cast<char*>(xs);
  return launch_rows(pick_dispatch<true>(dtype), pick_dispatch<false>(dtype), a, true, "launch dispatch", stream);
}

int ebag_a2a_moe_dispatch_backward(ebag_a2a_moe_t h, const void* dxs, int64_t lddxs, int64_t dim, int32_t dtype,
                                   int64_t tokens, const int32_t* offsets, const int32_t* pos, void* dx, int64_t lddx,
                                   hipStream_t stream) {
  RowArgs a;
  if (int rc = row_args(h, dim, dtype, tokens, offsets, pos, &a)) return rc;
  if (!tokens) return EBAG_OK;
  if (int rc = row_matrix("dxs", dxs, lddxs, dim, dtype, &a.ld_in)) return rc;
  if (int rc = row_matrix("dx", dx, lddx, dim, dtype, &a.ld_out)) return rc;
  a.in = static_cast<const char*>(dxs);
  a.out = static_cast<char*>(dx);
  return launch_rows(pick_combine<true>(dtype), pick_combine<false>(dtype), a, true, "launch dispatch backward", stream);
}

int ebag_a2a_moe_combine(ebag_a2a_moe_t h, const void* ys, int64_t ldys, int64_t dim, int32_t dtype, int64_t tokens,
                         const int32_t* offsets, const int32_t* pos, const float* weights, void* out, int64_t ldo,
                         hipStream_t stream) {
  RowArgs a;
  if (int rc = row_args(h, dim, dtype, tokens, offsets, pos, &a)) return rc;
  if (!tokens) return EBAG_OK;
  if (!weights) return fail(EBAG_EINVAL, "null weights");
  if (int rc = row_matrix("ys", ys, ldys, dim, dtype, &a.ld_in)) return rc;
  if (int rc = row_matrix("out", out, ldo, dim, dtype, &a.ld_out)) return rc;
  a.in = static_cast<const char*>(ys);
  a.out = static_cast<char*>(out);
  a.weights = weights;
  return launch_rows(pick_combine<true>(dtype), pick_combine<false>(dtype), a, true, "launch combine", stream);
}

int ebag_a2a_moe_combine_backward(ebag_a2a_moe_t h, const void* dout, int64_t lddout, const void* ys, int64_t ldys,
                                  int64_t dim, int32_t dtype, int64_t tokens, const int32_t* offsets,
                                  const int32_t* pos, const float* weights, void* dys, int64_t lddys, float* dweights,
                                  hipStream_t stream) {
  RowArgs a;
  if (int rc = row_args(h, dim, dtype, tokens, offsets, pos, &a)) return rc;
  if (!tokens) return EBAG_OK;
  if (!weights || !dweights) return fail(EBAG_EINVAL, "null weights or dweights");
  if (int rc = row_matrix("dout", dout, lddout, dim, dtype, &a.ld_in)) return rc;
  if (int rc = row_matrix("ys", ys, ldys, dim, dtype, &a.ld_in2)) return rc;
  if (int rc = row_matrix("dys", dys, lddys, dim, dtype, &a.ld_out)) return rc;
  a.in = static_cast<const char*>(dout);
  a.in2 = static_cast<const char*>(ys);
  a.out = static_cast<char*>(dys);
  a.weights = weights;
  a.dweights = dweights;
  return launch_rows(pick_backward<true>(dtype), pick_backward<false>(dtype), a, false, "launch combine backward", stream);
}

void ebag_a2a_moe_destroy(ebag_a2a_moe_t h) { free_moe(h); }

}  // extern "C"
