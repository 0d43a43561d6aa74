// Tokens by expert (ebag_a2a_moe_* of include/ebag_a2a.h): the sort of the
// tokens' choices and the kernels that move and sum the tokens' rows.
#include <hip/hip_runtime.h>

#include <climits>
#include <new>

#include "common.h"
#include "ebag_a2a.h"
#include "in_flight.h"
#include "lanes.h"
#include "moe.h"
#include "vec16.h"

using namespace ebag;

namespace {

// ------------------------------------------------------------------- sort
//
// A stable counting sort: pos(i) = choices of smaller keys + earlier choices of
// the same key, the key being the expert, or `experts` for a dropped choice.  A
// workgroup of 16 waves takes chunks of 1024 to 4096 choices, a wave 64 of them
// in each of up to four batches, a lane each.  Inside a batch a lane's rank is
// the number of lower lanes with its key, found with a ballot per bit of the key;
// a counter per (wave, key) in LDS carries it from batch to batch, and sums over
// the waves and over the chunks before place the rest.  No atomic decides an order.
//
// Up to one chunk of 4096 one workgroup does it all (256 choices 3.4 us, 4096 7.3
// us, an empty launch 1.8 us); above, a first launch counts each workgroup's keys.
// Small chunks there: 131072 choices on 256 experts, 32 workgroups of 4096 17.6
// us, 128 of 1024 10.0 us; bound by the latency of its steps, not by bytes.

constexpr int kSortWaves = 16, kSortBatches = 4, kSortThreads = 64 * kSortWaves;
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
  int32_t batches;         // of a wave in a chunk
  int32_t experts;
  int32_t key_bits;        // bits of experts + 1
};

__device__ __forceinline__ uint32_t key_at(const SortArgs& a, uint32_t i) {
  if (i >= a.S) return a.experts + 1;  // no choice
  const uint32_t e = (uint32_t)a.experts_of[i];
  return e < (uint32_t)a.experts ? e : (uint32_t)a.experts;
}

__device__ __forceinline__ void wg_chunks(const SortArgs& a, uint32_t* first, uint32_t* last) {
  *first = blockIdx.x * a.chunks_per_wg;
  *last = *first + a.chunks_per_wg < a.chunks ? *first + a.chunks_per_wg : a.chunks;
}

// Choices of each key in a workgroup's chunks.
__global__ __launch_bounds__(kSortThreads) void moe_count_kernel(const SortArgs a) {
  __shared__ uint32_t total[kMaxExperts + 1];
  uint32_t first, last;
  wg_chunks(a, &first, &last);
  for (int e = threadIdx.x; e <= a.experts; e += kSortThreads) total[e] = 0;
  __syncthreads();
  for (uint32_t i = first * a.batches; i < last * a.batches; ++i) {
    const uint32_t key = key_at(a, i * kSortThreads + threadIdx.x);
    if (key <= (uint32_t)a.experts) atomicAdd(&total[key], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e <= a.experts; e += kSortThreads) a.counts[blockIdx.x * (a.experts + 1) + e] = total[e];
}

// ALONE: one workgroup has all choices, in one chunk.
template <bool ALONE>
__global__ __launch_bounds__(kSortThreads) void moe_place_kernel(const SortArgs a) {
  __shared__ uint32_t base[kMaxExperts + 1];    // where the next choice of each key goes
  __shared__ uint32_t before[kMaxExperts + 1];  // choices of each key in earlier workgroups
  __shared__ uint32_t wave_sum[kSortWaves];
  __shared__ uint16_t seen[kSortWaves][kMaxExperts + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int e = threadIdx.x;  // the key this thread sums (experts + 1 <= 1024 keys)
  const bool mine = e <= a.experts;

  // From a key's total, the first place of its choices over all workgroups; to be followed by a barrier.
  auto first_places = [&](uint32_t total, uint32_t earlier) {
    uint32_t upto = total;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t v = __shfl_up(upto, d);
      if (lane >= d) upto += v;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += wave_sum[w];
    if (mine) {
      base[e] = upto - total + earlier;
      if (blockIdx.x == 0) a.offsets[e] = (int32_t)(upto - total);
    }
  };

  uint32_t first, last;
  wg_chunks(a, &first, &last);
  if (!ALONE) {  // the workgroups' counts, a row of them to a wave
    if (mine) base[e] = before[e] = 0;
    __syncthreads();
    for (int k = lane; k <= a.experts; k += 64) {
      uint32_t total = 0, earlier = 0;
#pragma unroll 8
      for (uint32_t g = wave; g < gridDim.x; g += kSortWaves) {
        const uint32_t n = a.counts[g * (a.experts + 1) + k];
        total += n;
        if (g < blockIdx.x) earlier += n;
      }
      atomicAdd(&base[k], total);
      atomicAdd(&before[k], earlier);
    }
    __syncthreads();
    first_places(mine ? base[e] : 0, mine ? before[e] : 0);
  }
  for (uint32_t c = first; c < last || ALONE; ++c) {
    for (int k = lane; k <= a.experts; k += 64) seen[wave][k] = 0;
    __builtin_amdgcn_wave_barrier();
    uint32_t key[kSortBatches], rank[kSortBatches];
    const uint32_t i0 = (c * kSortThreads + wave * 64) * a.batches + lane;
#pragma unroll
    for (int b = 0; b < kSortBatches; ++b) key[b] = b < a.batches ? key_at(a, i0 + b * 64) : a.experts + 1;
#pragma unroll
    for (int b = 0; b < kSortBatches; ++b) {
      if (b >= a.batches) continue;
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
    if (mine) {
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t n = seen[w][e];
        seen[w][e] = (uint16_t)in_chunk;
        in_chunk += n;
      }
    }
    if (ALONE) first_places(in_chunk, 0);
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kSortBatches; ++b) {
      if (key[b] > (uint32_t)a.experts) continue;
      const uint32_t i = i0 + b * 64, p = base[key[b]] + seen[wave][key[b]] + rank[b];
      a.pos[i] = (int32_t)p;
      a.src[p] = (int32_t)i;
    }
    if (ALONE) return;
    __syncthreads();
    if (mine) base[e] += in_chunk;
  }
}

// ------------------------------------------------------------------- rows

constexpr int kRowThreads = 256;

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
  int32_t vecs;            // 16-byte vectors of a row; the last one ends where the row does
  int32_t last;            // its first byte
  int32_t twice;           // its elements that are the one's before, too
  int32_t tail;            // elements of a row of less than a vector
  int32_t lanes;           // lanes of a token: a power of two, 64 for rows of more than 32 vectors
  Divisor by_waves;        // waves of a token (rows of more than 32 vectors)
};

// Rows of more than 32 vectors have a wave to themselves, or one for every 128 of
// their vectors: neighbouring waves have neighbouring parts, so a row is read and
// written at one time (16384 tokens x 8 choices x 2048 bf16 dispatched: 172 us with
// the first part of every row first, 108 us like this).  The token and its places
// are the same for all lanes of a wave and sit in scalar registers.  Shorter rows
// share a wave.
//
// All of these move bytes only: 606 MB dispatched in 102 us (5.9 TB/s; a large copy
// reaches 5.1, a fill 6.9), combined in 115 us, and combine's gradients read and write
// 1.2 GB in 228 us.
template <bool WHOLE>
struct Place {
  int64_t token;
  int lane, lanes;
  int part;  // the wave's first, of a.parts, a.part_step apart
  bool any;
  __device__ __forceinline__ Place(const RowArgs& a) {
    if (WHOLE) {
      lanes = 64;
      lane = threadIdx.x & 63;
      const uint32_t g = blockIdx.x * (kRowThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      const uint32_t t = divide_by(a.by_waves, g);
      token = t;
      part = g - t * a.by_waves.d;
    } else {
      lanes = a.lanes;
      lane = threadIdx.x & (lanes - 1);
      token = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) / lanes;
      part = 0;
    }
    any = token < a.tokens;
  }
};

// Where vector v of a row begins.
__device__ __forceinline__ int64_t byte_of(const RowArgs& a, int v) { return v * 16 < a.last ? v * 16 : a.last; }

// Places below `kept` hold an expert's row, those up to S a dropped one.
__device__ __forceinline__ uint32_t kept_rows(const RowArgs& a) {
  const uint32_t n = (uint32_t)a.offsets[a.experts];
  return n < a.S ? n : a.S;
}

constexpr int kAtOnce = 8;

// Vectors of a row that a lane has at once, 64 apart.
template <bool WHOLE> constexpr int kVecs = WHOLE ? 2 : 1;

// How rows by place go past the caches, where all of them are more than these
// hold and nothing is won by keeping them.  Loads: 16384 tokens x 8 choices x 2048
// bf16 combined in 127 us through the caches, 115 us past them; 512 x 8 x 4096 (34
// MB) 9.0 and 10.1.  Stores, where rows are whole cache lines: the same two
// dispatched, 110 and 102 us; 2560 x 8 x 2048 15.5 and 17.4; rows of 1999, whose
// lines two rows share, 45 and 61 us.
enum Stream { CACHED = 0, LOADS = 1, BOTH = 2 };

template <bool STREAM>
__device__ __forceinline__ vec16 load_row(const char* p) {
  return STREAM ? __builtin_nontemporal_load(reinterpret_cast<const vec16_any*>(p)) : load16(p);
}

template <bool STREAM>
__device__ __forceinline__ void store_row(char* p, const vec16& v) {
  if (STREAM)
    __builtin_nontemporal_store(v, reinterpret_cast<vec16_any*>(p));
  else
    store16(p, v);
}

// xs[pos[n, j]] = x[n]: every row is read once and written `choices` times.
template <int DT, bool WHOLE, int STREAM>
__global__ __launch_bounds__(kRowThreads) void moe_dispatch_kernel(const RowArgs a) {
  typedef Type<DT> T;
  constexpr int U = kVecs<WHOLE>;
  const Place<WHOLE> at(a);
  if (!at.any) return;
  const uint32_t kept = kept_rows(a);
  const int32_t* pos = a.pos + at.token * a.choices;
  const char* row = a.in + at.token * a.ld_in;
  for (int v = at.lane + at.part * (U * at.lanes); v < a.vecs; v += U * at.lanes * (WHOLE ? a.by_waves.d : 1)) {
    vec16 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v + u * at.lanes < a.vecs) r[u] = load16(row + byte_of(a, v + u * at.lanes));
    for (int j = 0; j < a.choices; ++j) {
      const uint32_t p = (uint32_t)pos[j];
      if (p >= a.S) continue;
      char* to = a.out + p * a.ld_out;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v + u * at.lanes < a.vecs) store_row<STREAM == BOTH>(to + byte_of(a, v + u * at.lanes), p < kept ? r[u] : vec16{0, 0, 0, 0});
    }
  }
  if (at.part == 0) {
    for (int t = at.lane; t < a.tail; t += at.lanes) {
      const int64_t byte = t * (int)sizeof(typename T::elt);
      const typename T::elt r = *reinterpret_cast<const typename T::elt*>(row + byte);
      for (int j = 0; j < a.choices; ++j) {
        const uint32_t p = (uint32_t)pos[j];
        if (p < a.S) *reinterpret_cast<typename T::elt*>(a.out + p * a.ld_out + byte) = p < kept ? r : (typename T::elt)0;
      }
    }
  }
}

// out[n] = sum_j weights[n, j] * in[pos[n, j]].
template <int DT, bool WHOLE, int STREAM>
__global__ __launch_bounds__(kRowThreads) void moe_combine_kernel(const RowArgs a) {
  typedef Type<DT> T;
  constexpr int U = kVecs<WHOLE>;
  const Place<WHOLE> at(a);
  if (!at.any) return;
  const uint32_t kept = kept_rows(a);
  const int32_t* pos = a.pos + at.token * a.choices;
  const float* weights = a.weights ? a.weights + at.token * a.choices : nullptr;
  char* row = a.out + at.token * a.ld_out;
  for (int v = at.lane + at.part * (U * at.lanes); v < a.vecs; v += U * at.lanes * (WHOLE ? a.by_waves.d : 1)) {
    float sum[U][T::N] = {};
    for (int j0 = 0; j0 < a.choices; j0 += kAtOnce) {
      vec16 r[kAtOnce][U];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t p = j0 + i < a.choices ? (uint32_t)pos[j0 + i] : kept;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          r[i][u] = vec16{0, 0, 0, 0};
          if (p < kept && v + u * at.lanes < a.vecs) r[i][u] = load_row<STREAM >= LOADS>(a.in + p * a.ld_in + byte_of(a, v + u * at.lanes));
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (j0 + i >= a.choices || (uint32_t)pos[j0 + i] >= kept) continue;
        const float w = weights ? weights[j0 + i] : 1.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[T::N];
          T::widen(r[i][u], f);
#pragma unroll
          for (int n = 0; n < T::N; ++n) sum[u][n] = __builtin_fmaf(w, f[n], sum[u][n]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v + u * at.lanes < a.vecs) store16(row + byte_of(a, v + u * at.lanes), T::narrow(sum[u]));
  }
  if (at.part == 0) {
    for (int t = at.lane; t < a.tail; t += at.lanes) {
      const int64_t byte = t * (int)sizeof(typename T::elt);
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
// ys[pos[n, j]]>: one pass over dout and ys.  A token's waves, all of one workgroup,
// join their dot products in LDS.
template <int DT, bool WHOLE, int STREAM>
__global__ __launch_bounds__(kRowThreads) void moe_combine_backward_kernel(const RowArgs a) {
  typedef Type<DT> T;
  constexpr int U = kVecs<WHOLE>, WAVES = kRowThreads / 64;
  __shared__ float dots[WAVES][kAtOnce];
  const Place<WHOLE> at(a);
  const int wave = threadIdx.x >> 6, shared = WHOLE ? a.by_waves.d : 1;  // waves of the token
  const bool spread = shared > 1;
  if (!at.any) {
    if (spread)
      for (int j0 = 0; j0 < a.choices; j0 += kAtOnce) {  // the workgroup's other tokens meet at these
        __syncthreads();
        __syncthreads();
      }
    return;
  }
  const uint32_t kept = kept_rows(a);
  const int32_t* pos = a.pos + at.token * a.choices;
  const float* weights = a.weights + at.token * a.choices;
  const char* row = a.in + at.token * a.ld_in;
  const int step = U * at.lanes, first = at.lane + at.part * step, stride = shared * step;
  for (int j0 = 0; j0 < a.choices; j0 += kAtOnce) {
    float dot[kAtOnce] = {};
    for (int v = first; v < a.vecs; v += stride) {
      vec16 d[U], y[kAtOnce][U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        d[u] = vec16{0, 0, 0, 0};
        if (v + u * at.lanes < a.vecs) d[u] = load16(row + byte_of(a, v + u * at.lanes));
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t p = j0 + i < a.choices ? (uint32_t)pos[j0 + i] : kept;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          y[i][u] = vec16{0, 0, 0, 0};
          if (p < kept && v + u * at.lanes < a.vecs) y[i][u] = load_row<STREAM >= LOADS>(a.in2 + p * a.ld_in2 + byte_of(a, v + u * at.lanes));
        }
      }
      float f[U][T::N];
#pragma unroll
      for (int u = 0; u < U; ++u) T::widen(d[u], f[u]);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (j0 + i >= a.choices) continue;
        const uint32_t p = (uint32_t)pos[j0 + i];
        if (p >= a.S) continue;
        const float w = p < kept ? weights[j0 + i] : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float g[T::N], s[T::N];
          T::widen(y[i][u], g);
          // Elements that the last vector repeats count once, whatever they hold: both factors are 0, as 0 in place of one
          // would make an infinity in the other a NaN.
          float d[T::N];
#pragma unroll
          for (int n = 0; n < T::N; ++n) d[n] = f[u][n];
          if (a.twice && v + u * at.lanes == a.vecs - 1) {
#pragma unroll
            for (int n = 0; n < T::N; ++n) {
              d[n] = n < a.twice ? 0.f : d[n];
              g[n] = n < a.twice ? 0.f : g[n];
            }
          }
#pragma unroll
          for (int n = 0; n < T::N; ++n) {
            // Rounded to fp32 and then to the type, in every instance: the empty statement keeps the compiler from an
            // instruction that rounds a product to fp16 at once.
            s[n] = w * f[u][n];
            asm("" : "+v"(s[n]));
            s[n] = p < kept ? s[n] : 0.f;
            if (p < kept) dot[i] = __builtin_fmaf(d[n], g[n], dot[i]);
          }
          if (v + u * at.lanes < a.vecs) store_row<STREAM == BOTH>(a.out + p * a.ld_out + byte_of(a, v + u * at.lanes), T::narrow(s));
        }
      }
    }
    for (int t = at.lane; t < a.tail && at.part == 0; t += at.lanes) {
      const int64_t byte = t * (int)sizeof(typename T::elt);
      const float d = T::widen(*reinterpret_cast<const typename T::elt*>(row + byte));
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (j0 + i >= a.choices) continue;
        const uint32_t p = (uint32_t)pos[j0 + i];
        float s = 0.f;
        if (p < kept) {
          s = weights[j0 + i] * d;
          dot[i] = __builtin_fmaf(d, T::widen(*reinterpret_cast<const typename T::elt*>(a.in2 + p * a.ld_in2 + byte)), dot[i]);
        }
        if (p < a.S) *reinterpret_cast<typename T::elt*>(a.out + p * a.ld_out + byte) = T::narrow(s);
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (j0 + i >= a.choices) continue;
      dot[i] = sum_lanes(dot[i], at.lanes);
      if (spread) {
        if (at.lane == 0) dots[wave][i] = dot[i];
      } else if (at.lane == 0) {
        a.dweights[at.token * a.choices + j0 + i] = dot[i];
      }
    }
    if (spread) {
      __syncthreads();
      const int i = at.lane;
      if (at.part == 0 && i < kAtOnce && j0 + i < a.choices) {
        float sum = 0.f;
        for (int w = wave; w < wave + shared; ++w) sum += dots[w][i];
        a.dweights[at.token * a.choices + j0 + i] = sum;
      }
      __syncthreads();
    }
  }
}

typedef void (*row_fn)(const RowArgs);

template <int DT, bool WHOLE>
row_fn pick_dispatch(int stream) {
  return stream == BOTH ? moe_dispatch_kernel<DT, WHOLE, BOTH> : moe_dispatch_kernel<DT, WHOLE, CACHED>;
}
template <int DT, bool WHOLE>
row_fn pick_combine(int stream) {
  return stream ? moe_combine_kernel<DT, WHOLE, LOADS> : moe_combine_kernel<DT, WHOLE, CACHED>;
}
template <int DT, bool WHOLE>
row_fn pick_backward(int stream) {
  return stream == BOTH    ? moe_combine_backward_kernel<DT, WHOLE, BOTH>
         : stream == LOADS ? moe_combine_backward_kernel<DT, WHOLE, LOADS>
                           : moe_combine_backward_kernel<DT, WHOLE, CACHED>;
}

enum Which { DISPATCH, COMBINE, BACKWARD };

template <int DT>
row_fn pick(Which which, bool whole, int stream) {
  switch (which) {
    case DISPATCH: return whole ? pick_dispatch<DT, true>(stream) : pick_dispatch<DT, false>(stream);
    case COMBINE: return whole ? pick_combine<DT, true>(stream) : pick_combine<DT, false>(stream);
    default: return whole ? pick_backward<DT, true>(stream) : pick_backward<DT, false>(stream);
  }
}

int hipf(hipError_t e, const char* what) { return fail(EBAG_EHIP, "%s: %s", what, hipGetErrorString(e)); }

void free_moe(ebag_a2a_moe_plan* h) {
  if (!h) return;
  if (h->sort.done) (void)hipEventDestroy(h->sort.done);
  (void)hipFree(h->d_counts);
  delete h;
}

// Checks a row call's shape and fills what all of them share.
int row_args(ebag_a2a_moe_plan* h, int64_t dim, int32_t dtype, int64_t tokens, const int32_t* offsets,
             const int32_t* pos, RowArgs* a) {
  if (int rc = check_moe_plan(h, tokens)) return rc;
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
  const int64_t bytes = dim * elt;  // up to 2^31 - 4
  a->vecs = bytes < 16 ? 0 : (int32_t)((bytes + 15) / 16);
  a->last = (int32_t)(bytes - 16);
  a->twice = bytes < 16 ? 0 : (int32_t)((a->vecs * 16LL - bytes) / elt);
  a->tail = bytes < 16 ? (int32_t)dim : 0;
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

int launch_rows(Which which, int dtype, RowArgs& a, const char* what, hipStream_t stream) {
  // Waves of a token, a power of two; of one workgroup where they join sums.
  const int most = which == BACKWARD ? kRowThreads / 64 : 64;
  int waves = 1;
  if (a.lanes == 64)
    while (waves < most && waves * 64 * kVecs<true> < a.vecs && a.tokens * waves * 2 < INT_MAX) waves *= 2;
  a.by_waves = make_divisor(waves);
  const int64_t wgs = (a.tokens * waves + kRowThreads / a.lanes - 1) / (kRowThreads / a.lanes);
  if (wgs > INT_MAX) return fail(EBAG_EINVAL, "too many tokens for one launch");
  const int64_t row = (int64_t)a.last + 16;
  int past = CACHED;
  if (a.S * row > (int64_t)128 << 20) {
    const bool lines = row % 128 == 0 && a.ld_out % 128 == 0 && reinterpret_cast<uintptr_t>(a.out) % 128 == 0;
    past = lines && which != COMBINE ? BOTH : LOADS;
  }
  const bool whole = a.lanes == 64;
  const row_fn fn = dtype == EBAG_F32 ? pick<0>(which, whole, past) : dtype == EBAG_F16 ? pick<1>(which, whole, past) : pick<2>(which, whole, past);
  hipLaunchKernelGGL(fn, dim3((unsigned)wgs), dim3(kRowThreads), 0, stream, a);
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
  if (max_tokens < 0 || max_tokens > (INT_MAX - kSortThreads * kSortBatches) / choices)
    return fail(EBAG_EINVAL, "max_tokens=%lld: max_tokens * choices must be at most 2^31 - 4097", (long long)max_tokens);
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
  if (int rc = check_moe_plan(h, tokens)) return rc;
  if (!offsets || (tokens && (!experts_of || !pos || !src))) return fail(EBAG_EINVAL, "null experts_of, offsets, pos or src");
  SortArgs a{};
  a.experts_of = experts_of;
  a.offsets = offsets;
  a.pos = pos;
  a.src = src;
  a.counts = h->d_counts;
  a.S = (uint32_t)(tokens * h->choices);
  a.experts = h->experts;
  while (1 << a.key_bits < a.experts + 2) ++a.key_bits;
  const uint32_t batch = kSortThreads;
  if (a.S <= batch * kSortBatches) {
    a.chunks = a.chunks_per_wg = 1;
    a.batches = a.S <= batch ? 1 : (int32_t)((a.S + batch - 1) / batch);
    hipLaunchKernelGGL(moe_place_kernel<true>, dim3(1), dim3(kSortThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? EBAG_OK : hipf(e, "launch the sort");
  }
  if (int rc = check_busy(h->sort, stream, "sort")) return rc;
  a.batches = 1;
  while (a.batches < kSortBatches && a.S > batch * a.batches * kSortMaxWgs) a.batches *= 2;
  a.chunks = (a.S + batch * a.batches - 1) / (batch * a.batches);
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
  return launch_rows(DISPATCH, dtype, a, "launch dispatch", stream);
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
  return launch_rows(COMBINE, dtype, a, "launch dispatch backward", stream);
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
  return launch_rows(COMBINE, dtype, a, "launch combine", stream);
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
  return launch_rows(BACKWARD, dtype, a, "launch combine backward", stream);
}

void ebag_a2a_moe_destroy(ebag_a2a_moe_t h) { free_moe(h); }

}  // extern "C"
