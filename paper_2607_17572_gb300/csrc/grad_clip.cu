// The global norm of many gradient tensors and the clip by it (include/jagg.h).
//
//   norm = sqrt(sum_t sum_i g_ti^2),  coef = min(1, max_norm / (norm + eps)),  out = coef g
//
// Two launches for any number of tensors up to CLIP_TENSORS: one writes a partial sum per CTA, the
// next adds them in every CTA (the same order everywhere, so the same coefficient) and scales.  The
// tensors' addresses travel as kernel parameters: nothing has to be copied to the device first, and
// a captured graph keeps its own list.
#include <algorithm>
#include <vector>

#include "fp8.cuh"

namespace jagg {
namespace {

constexpr int CLIP_TENSORS = 1000;  // of a launch: the list fits the 32764 bytes of kernel parameters
constexpr int CLIP_FEW = 100;       // a shorter list for launches of few tensors (3 KB to pass instead of 28)
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_CHUNK = 32 * CLIP_THREADS;  // elements of a CTA's step: 8 or 4 16-byte loads per thread
constexpr int CLIP_KEEP = 80 << 20;  // bytes that the first pass leaves in the L2 (129 MB) for the second
constexpr int CLIP_CTAS_PER_SM = 4;
constexpr int CLIP_CTAS = 640;  // most CTAs of a launch (rows of partial sums)

template <int N>
struct ClipList {
  const void* in[N];
  void* out[N];
  int64_t numel[N];
  int32_t first[N + 1];  // first chunk of each tensor; first[count] is the total
  int count;
};
static_assert(sizeof(ClipList<CLIP_TENSORS>) + 64 <= 32764, "kernel parameters");

// The tensor of chunk c: the last t with first[t] <= c (empty tensors share their successor's start).
template <int N>
__device__ __forceinline__ int tensor_of(const ClipList<N>& l, int c) {
  int lo = 0, hi = l.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.first[mid] <= c)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <typename T> constexpr int kVec = 16 / sizeof(T);

template <typename T>
__device__ __forceinline__ void unpack(uint4 w, float (&v)[kVec<T>]) {
  if constexpr (sizeof(T) == 4) {
    v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y);
    v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
  } else {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&v)[kVec<T>]) {
  if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  } else {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<uint32_t*>(&t);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
}

// A thread's 32 elements of a chunk: whole vectors where tensor and chunk allow, single elements
// (in strides of the CTA) otherwise.
template <typename T>
struct Run {
  static constexpr int VECS = 32 / kVec<T>;
  uint4 w[VECS];
};

__device__ __forceinline__ double block_sum(double v, double* red) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < CLIP_THREADS / 32; ++i) s += red[i];
  return s;
}

template <typename T, int N>
__global__ void __launch_bounds__(CLIP_THREADS) square_sum_kernel(const __grid_constant__ ClipList<N> l, double* part) {
  constexpr int VEC = kVec<T>, VECS = Run<T>::VECS;
  __shared__ double red[CLIP_THREADS / 32];
  pdl_wait();
  double sum = 0.0;
  const int total = l.first[l.count];
  const int keep = total - CLIP_KEEP / (CLIP_CHUNK * (int)sizeof(T));  // from here on chunks are to stay in the L2
  for (int c = blockIdx.x; c < total; c += gridDim.x) {
    const int t = tensor_of(l, c);
    const T* g = static_cast<const T*>(l.in[t]);
    const int64_t at = (int64_t)(c - l.first[t]) * CLIP_CHUNK, left = l.numel[t] - at;
    float v[32];
    if (left >= CLIP_CHUNK && (reinterpret_cast<uintptr_t>(g) & 15) == 0) {
      uint4 w[VECS];
#pragma unroll
      for (int i = 0; i < VECS; ++i) {
        const uint4* from = reinterpret_cast<const uint4*>(g + at + (int64_t)(i * CLIP_THREADS + threadIdx.x) * VEC);
        w[i] = c < keep ? __ldcs(from) : *from;
      }
#pragma unroll
      for (int i = 0; i < VECS; ++i) unpack<T>(w[i], reinterpret_cast<float(&)[VEC]>(v[i * VEC]));
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int64_t k = threadIdx.x + (int64_t)i * CLIP_THREADS;
        v[i] = k < left ? ld(g + at + k) : 0.f;
      }
    }
    float p = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) p = fmaf(v[i], v[i], p);
    // a sum near the ends of f32's range may have lost terms to overflow or underflow
    if (p < 3e38f && p > 1e-25f) {
      sum += (double)p;
    } else {
      float any = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) any = fp8::amax(any, v[i]);
      if (any != 0.f) {
#pragma unroll 1
        for (int i = 0; i < 32; ++i) sum = fma((double)v[i], (double)v[i], sum);
      }
    }
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The sum of all partial sums, the same in every thread of every CTA.
__device__ __forceinline__ double total_of(const double* part, int parts, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += CLIP_THREADS) s += part[i];
  return block_sum(s, red);
}

__global__ void __launch_bounds__(CLIP_THREADS) norm_kernel(const double* part, int parts, float* out) {
  __shared__ double red[CLIP_THREADS / 32];
  pdl_wait();
  const double s = total_of(part, parts, red);
  if (threadIdx.x == 0) out[0] = (float)sqrt(s);
}

template <typename T, int N>
__global__ void __launch_bounds__(CLIP_THREADS)
    clip_kernel(const __grid_constant__ ClipList<N> l, const double* part, int parts, double max_norm, double eps,
                int write_norm, float* out2) {
  constexpr int VEC = kVec<T>, VECS = Run<T>::VECS;
  __shared__ double red[CLIP_THREADS / 32];
  pdl_wait();
  const double norm = sqrt(total_of(part, parts, red));
  const double below = norm + eps;
  // nothing to clip where all gradients are 0, or without a limit
  const double ratio = below == 0.0 || (isinf(max_norm) && !isnan(norm)) ? 1.0 : max_norm / below;
  const float coef = ratio >= 1.0 ? 1.f : (float)ratio;        // a NaN stays one
  if (write_norm && blockIdx.x == 0 && threadIdx.x == 0) {
    out2[0] = (float)norm;
    out2[1] = coef;
  }
  // last chunks first: the L2 still holds what the first pass read last
  const int total = l.first[l.count];
  for (int c = total - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const int t = tensor_of(l, c);
    const T* g = static_cast<const T*>(l.in[t]);
    T* o = static_cast<T*>(l.out[t]);
    if (coef == 1.f && g == o) continue;
    const int64_t at = (int64_t)(c - l.first[t]) * CLIP_CHUNK, left = l.numel[t] - at;
    if (left >= CLIP_CHUNK && ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(o)) & 15) == 0) {
      uint4 w[VECS];
#pragma unroll
      for (int i = 0; i < VECS; ++i)
        w[i] = __ldcs(reinterpret_cast<const uint4*>(g + at + (int64_t)(i * CLIP_THREADS + threadIdx.x) * VEC));
#pragma unroll
      for (int i = 0; i < VECS; ++i) {
        float v[VEC];
        unpack<T>(w[i], v);
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] *= coef;
        __stcs(reinterpret_cast<uint4*>(o + at + (int64_t)(i * CLIP_THREADS + threadIdx.x) * VEC), pack<T>(v));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int64_t k = threadIdx.x + (int64_t)i * CLIP_THREADS;
        if (k < left) st(o + at + k, ld(g + at + k) * coef);
      }
    }
  }
}

int launches_of(int count) { return count <= 0 ? 1 : (count + CLIP_TENSORS - 1) / CLIP_TENSORS; }

int ctas_of(int chunks) {
  const int most = CLIP_CTAS_PER_SM * sm_count();
  const int n = most < CLIP_CTAS ? most : CLIP_CTAS;
  return chunks < 1 ? 1 : chunks < n ? chunks : n;
}

// Tensors first .. first + n - 1 as a launch's list.
template <int N>
int fill(ClipList<N>& l, const void* const* grads, void* const* out, const int64_t* numel, int n, int* chunks) {
  int64_t c = 0;
  for (int i = 0; i < n; ++i) {
    l.in[i] = grads[i];
    l.out[i] = out ? out[i] : const_cast<void*>(grads[i]);
    l.numel[i] = numel[i];
    l.first[i] = (int32_t)c;
    c += (numel[i] + CLIP_CHUNK - 1) / CLIP_CHUNK;
  }
  if (c > INT32_MAX - CLIP_CTAS) {
    set_last_error("grad_clip: %lld elements in one launch", (long long)c * CLIP_CHUNK);
    return JAGG_ERR_UNSUPPORTED;
  }
  l.first[n] = (int32_t)c;
  l.count = n;
  *chunks = (int)c;
  return JAGG_OK;
}

struct ClipCall {
  const void* const* grads;
  void* const* out;
  const int64_t* numel;
  int count;
  double max_norm, eps;
  float* norm_out;
  double* part;
  bool clip;
  cudaStream_t stream;
};

template <typename T, int N>
int run_lists(const ClipCall& c) {
  const int lists = launches_of(c.count);
  std::vector<ClipList<N>> all;
  try {
    all.resize(lists);
  } catch (...) {
    set_last_error("grad_clip: out of host memory for the lists of %d tensors", c.count);
    return JAGG_ERR_ARG;
  }
  int parts = 0;
  for (int i = 0; i < lists; ++i) {
    const int at = i * CLIP_TENSORS, n = c.count - at < CLIP_TENSORS ? c.count - at : CLIP_TENSORS;
    int chunks = 0;
    JAGG_TRY(fill(all[i], c.grads + at, c.out ? c.out + at : nullptr, c.numel + at, n, &chunks));
  }
  for (int i = 0; i < lists; ++i) {
    const int ctas = ctas_of(all[i].first[all[i].count]);
    JAGG_CUDA_TRY(launch(square_sum_kernel<T, N>, ctas, CLIP_THREADS, 0, c.stream, all[i], c.part + parts));
    JAGG_LAUNCHED();
    parts += ctas;
  }
  if (!c.clip) {
    JAGG_CUDA_TRY(launch(norm_kernel, 1, CLIP_THREADS, 0, c.stream, (const double*)c.part, parts, c.norm_out));
    JAGG_LAUNCHED();
    return JAGG_OK;
  }
  for (int i = lists - 1; i >= 0; --i) {
    const int ctas = ctas_of(all[i].first[all[i].count]);
    JAGG_CUDA_TRY(launch(clip_kernel<T, N>, ctas, CLIP_THREADS, 0, c.stream, all[i], (const double*)c.part, parts,
                         c.max_norm, c.eps, i == 0 ? 1 : 0, c.norm_out));
    JAGG_LAUNCHED();
  }
  return JAGG_OK;
}

// What is written must not overlap anything else: two CTAs would scale an element twice, or read it scaled.
int check_overlap(const char* who, const ClipCall& c, int es) {
  struct Span {
    uintptr_t first, last;  // bytes first .. last - 1
    bool written;
  };
  std::vector<Span> v;
  try {
    v.reserve(c.out ? 2 * (size_t)c.count : c.count);
  } catch (...) {
    set_last_error("%s: out of host memory for %d tensors", who, c.count);
    return JAGG_ERR_ARG;
  }
  bool sorted = true;
  auto add = [&](const void* p, int64_t n, bool written) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    if (!v.empty() && a < v.back().first) sorted = false;
    v.push_back({a, a + (uintptr_t)n * es, written});
  };
  for (int i = 0; i < c.count; ++i) {
    if (c.numel[i] == 0) continue;
    const bool own = !c.out || c.out[i] == c.grads[i];
    add(c.grads[i], c.numel[i], own);
    if (!own) add(c.out[i], c.numel[i], true);
  }
  if (!sorted) std::sort(v.begin(), v.end(), [](const Span& a, const Span& b) { return a.first < b.first; });
  uintptr_t read = 0, written = 0;  // how far what came before reaches
  for (const Span& s : v) {
    JAGG_CHECK_ARG(s.first >= written && (!s.written || s.first >= read),
                   "%s: a tensor that is written overlaps another (at %p)", who, reinterpret_cast<void*>(s.first));
    (s.written ? written : read) = std::max(s.written ? written : read, s.last);
  }
  return JAGG_OK;
}

int run(const char* who, const ClipCall& c, int dtype, const void* ws, size_t ws_bytes) {
  JAGG_CHECK_ARG(fp8::is_dtype(dtype), "%s: bad dtype", who);
  JAGG_CHECK_ARG(c.count >= 0 && (c.count == 0 || (c.grads && c.numel)), "%s: %d tensors / null list", who, c.count);
  JAGG_CHECK_ARG(c.norm_out && fp8::aligned(c.norm_out, 4), "%s: null or misaligned norm_out", who);
  const int64_t need = jagg_grad_clip_workspace_bytes(c.count);
  if (!ws || (int64_t)ws_bytes < need) {
    set_last_error("%s: workspace %zu < %lld bytes", who, ws ? ws_bytes : (size_t)0, (long long)need);
    return JAGG_ERR_WORKSPACE;
  }
  JAGG_CHECK_ARG(fp8::aligned(ws, 8), "%s: workspace not 8-byte aligned", who);
  const int es = fp8::size_of(dtype);
  for (int i = 0; i < c.count; ++i) {
    JAGG_CHECK_ARG(c.numel[i] >= 0, "%s: tensor %d has %lld elements", who, i, (long long)c.numel[i]);
    if (c.numel[i] == 0) continue;
    JAGG_CHECK_ARG(c.grads[i] && (!c.out || c.out[i]), "%s: tensor %d is null", who, i);
    JAGG_CHECK_ARG(fp8::aligned(c.grads[i], es) && (!c.out || fp8::aligned(c.out[i], es)),
                   "%s: tensor %d is not aligned to its elements", who, i);
  }
  if (c.clip) JAGG_TRY(check_overlap(who, c, es));
  double total = 0.0;
  for (int i = 0; i < c.count; ++i) total += (double)c.numel[i];
  const int tok = prof_start(c.stream);
  if (dtype == JAGG_DTYPE_F32)
    JAGG_TRY((c.count <= CLIP_FEW ? run_lists<float, CLIP_FEW>(c) : run_lists<float, CLIP_TENSORS>(c)));
  else
    JAGG_TRY((c.count <= CLIP_FEW ? run_lists<bf16, CLIP_FEW>(c) : run_lists<bf16, CLIP_TENSORS>(c)));
  prof_stop(tok, c.stream, PROF_GRAD_CLIP, 0.0, total * es * (c.clip ? 2 : 1));
  return JAGG_OK;
}

}  // namespace
}  // namespace jagg

using namespace jagg;

extern "C" int64_t jagg_grad_clip_workspace_bytes(int count) { return (int64_t)launches_of(count) * CLIP_CTAS * 8; }

extern "C" int jagg_grad_norm(const void* const* grads, const int64_t* numel, int count, int dtype, float* norm_out,
                              void* ws, size_t ws_bytes, cudaStream_t stream) {
  const ClipCall c{grads, nullptr, numel, count, 0.0, 0.0, norm_out, static_cast<double*>(ws), false, stream};
  return run("jagg_grad_norm", c, dtype, ws, ws_bytes);
}

extern "C" int jagg_grad_clip(void* const* grads, void* const* out, const int64_t* numel, int count, int dtype,
                              double max_norm, double eps, float* norm_out, void* ws, size_t ws_bytes,
                              cudaStream_t stream) {
  JAGG_CHECK_ARG(max_norm >= 0.0 && eps >= 0.0, "jagg_grad_clip: max_norm=%g and eps=%g must not be negative", max_norm,
                 eps);
  const ClipCall c{grads, out, numel, count, max_norm, eps, norm_out, static_cast<double*>(ws), true, stream};
  return run("jagg_grad_clip", c, dtype, ws, ws_bytes);
}
