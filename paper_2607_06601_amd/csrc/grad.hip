// Global gradient norm over many tensors, and clipping:
//   norm = sqrt(sum of x^2) or max |x| over all elements of all tensors,
//   dst = src * c, c = min(1, max_norm / norm).
//
// The list of tensors lies on the device as one record for each piece of at
// most 16 KB (GRAD_PIECE) of a tensor, written once by the list's
// initialisation, so that one launch covers any number of tensors and a block
// finds its work by one load.  Bound by HBM: the norm reads every element,
// the scaling reads and writes it.  Squares are summed in fp64 (any finite
// fp32 element's square is a finite fp64 number; each of up to 2^19 threads adds
// its share one by one, so the sum over n elements is off by at most
// (n / 2^19 + 30) 2^-53 of it, 2^-42 for 10^9 elements), in an order that
// depends only on the list; the largest magnitude is taken on the bit
// patterns, whose order puts NaN above infinity.  Layer of 1.3B, 1.1 GB: norm
// 220 us, scaling 408 (5.0 and 5.4 TB/s, means); where a destination lies
// otherwise within 16 bytes than its source, an element a lane, the call takes
// 982 us for 632.
#include "kernels.hpp"

namespace tr {

constexpr int GRAD_PIECE = 16384;  // bytes
constexpr int GRAD_THREADS = 256;

static __host__ __device__ int elem_bytes(int dtype) { return dtype == TRIROUTE_BF16 ? 2 : 4; }

// Pieces of a tensor: all but the first start at 16-byte addresses of src.
int64_t grad_pieces(const triroute_grad_tensor &t) {
  const int64_t bytes = t.numel * elem_bytes(t.dtype);
  return t.numel <= 0 ? 0 : (bytes + int64_t(uintptr_t(t.src) & 15) + GRAD_PIECE - 1) / GRAD_PIECE;
}

// One thread per piece of up to GRAD_BATCH tensors, whose descriptors travel as kernel
// arguments (no copy from host memory).
__global__ __launch_bounds__(GRAD_THREADS) void grad_list_kernel(GradBatch b, GradRec *__restrict__ rec) {
  const GradDesc d = b.t[blockIdx.y];
  const int64_t pieces = b.first[blockIdx.y + 1] - b.first[blockIdx.y];
  const int es = elem_bytes(d.dtype);
  const int64_t lead = int64_t(uintptr_t(d.src) & 15);
  for (int64_t j = int64_t(blockIdx.x) * GRAD_THREADS + threadIdx.x; j < pieces;
       j += int64_t(gridDim.x) * GRAD_THREADS) {
    // bytes [from, to) of the tensor
    const int64_t from = j == 0 ? 0 : j * GRAD_PIECE - lead;
    const int64_t end = d.numel * es, to = min(end, (j + 1) * GRAD_PIECE - lead);
    GradRec r;
    r.src = (const uint8_t *)d.src + from;
    r.dst = d.dst ? (uint8_t *)d.dst + from : nullptr;
    r.n = int(to - from) / es;
    r.dtype = d.dtype;
    rec[b.first[blockIdx.y] + j] = r;
  }
}

hipError_t launch_grad_list(const GradBatch &b, int n, int64_t most, GradRec *rec, hipStream_t st) {
  const int64_t bx = std::min<int64_t>((most + GRAD_THREADS - 1) / GRAD_THREADS, 1024);
  if (n > 0 && bx > 0) grad_list_kernel<<<dim3(unsigned(bx), n), GRAD_THREADS, 0, st>>>(b, rec);
  return hipGetLastError();
}

// A piece in three parts: elements before the first 16-byte address of src, 16-byte
// words, elements after the last.
struct Split {
  int head, words, tail;
};
template <int ES>
__device__ __forceinline__ Split split_piece(const void *p, int n) {
  const int mis = int(uintptr_t(p) & 15);
  Split s;
  s.head = min(n, mis ? (16 - mis) / ES : 0);
  s.words = (n - s.head) / (16 / ES);
  s.tail = n - s.head - s.words * (16 / ES);
  return s;
}

// What a thread carries over the elements that it meets.
template <bool MAX> struct GradAcc;
template <> struct GradAcc<false> {
  double v = 0.0;
  __device__ void add(float x) { v = fma(double(x), double(x), v); }
  __device__ static double join(double a, double b) { return a + b; }
};
template <> struct GradAcc<true> {
  uint32_t v = 0;
  __device__ void add(float x) { v = max(v, __float_as_uint(x) & 0x7FFFFFFFu); }
  // of magnitudes: the larger bit pattern (NaN above all numbers)
  __device__ static double join(double a, double b) {
    return __double_as_longlong(a) >= __double_as_longlong(b) ? a : b;
  }
};

template <bool MAX>
__device__ __forceinline__ double block_join(double v, double *red) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = GradAcc<MAX>::join(v, __shfl_xor(v, m, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < GRAD_THREADS / 64; ++w) v = GradAcc<MAX>::join(v, red[w]);
  __syncthreads();
  return v;
}

template <typename T>
__device__ __forceinline__ void word_floats(const uint4 &w, float *v);
template <>
__device__ __forceinline__ void word_floats<float>(const uint4 &w, float *v) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(u[i]);
}
template <>
__device__ __forceinline__ void word_floats<bf16>(const uint4 &w, float *v) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
}

template <typename T, class A>
__device__ __forceinline__ void norm_piece(const GradRec &r, A &acc) {
  constexpr int EW = 16 / int(sizeof(T));
  const T *p = (const T *)r.src;
  const Split s = split_piece<int(sizeof(T))>(p, r.n);
  const uint4 *w = (const uint4 *)(p + s.head);
  constexpr int U = GRAD_PIECE / 16 / GRAD_THREADS;  // words a thread
  uint4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = threadIdx.x + u * GRAD_THREADS;
    v[u] = i < s.words ? w[i] : make_uint4(0u, 0u, 0u, 0u);
  }
  float e = 0.f;  // one of the odd elements
  if (int(threadIdx.x) < s.head)
    e = Act<T>::ld(p, threadIdx.x);
  else if (int(threadIdx.x) < s.head + s.tail)
    e = Act<T>::ld(p, s.words * EW + threadIdx.x);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x[EW];
    word_floats<T>(v[u], x);
#pragma unroll
    for (int i = 0; i < EW; ++i) acc.add(x[i]);
  }
  acc.add(e);
}

template <bool MAX>
__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(const GradRec *__restrict__ rec,
                                                                 int64_t pieces,
                                                                 double *__restrict__ part) {
  __shared__ double red[GRAD_THREADS / 64];
  GradAcc<MAX> acc;
  for (int64_t c = blockIdx.x; c < pieces; c += gridDim.x) {
    const GradRec r = rec[c];
    if (r.dtype == TRIROUTE_BF16)
      norm_piece<bf16>(r, acc);
    else
      norm_piece<float>(r, acc);
  }
  double v;
  if constexpr (MAX)
    v = double(__uint_as_float(acc.v));
  else
    v = acc.v;
  v = block_join<MAX>(v, red);
  if (threadIdx.x == 0) part[blockIdx.x] = v;
}

// The norm from the blocks' partial values, in one order everywhere.
template <bool MAX>
__device__ __forceinline__ double join_parts(const double *__restrict__ part, int nparts, double *red) {
  double v[GRAD_MAX_BLOCKS / GRAD_THREADS];
#pragma unroll
  for (int u = 0; u < GRAD_MAX_BLOCKS / GRAD_THREADS; ++u) {
    const int i = threadIdx.x + u * GRAD_THREADS;
    v[u] = i < nparts ? part[i] : 0.0;
  }
#pragma unroll
  for (int u = 1; u < GRAD_MAX_BLOCKS / GRAD_THREADS; ++u) v[0] = GradAcc<MAX>::join(v[0], v[u]);
  const double t = block_join<MAX>(v[0], red);
  return MAX ? t : sqrt(t);
}

template <bool MAX>
__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_finish_kernel(const double *__restrict__ part,
                                                                        int nparts,
                                                                        double *__restrict__ norm) {
  __shared__ double red[GRAD_THREADS / 64];
  const double v = join_parts<MAX>(part, nparts, red);
  if (threadIdx.x == 0) *norm = v;
}

// x c in fp32 (the rounding of an fp32 tensor's value), rounded to bf16 where the tensor is
template <typename T>
__device__ __forceinline__ uint4 scale_word(const uint4 &w, float c);
template <>
__device__ __forceinline__ uint4 scale_word<float>(const uint4 &w, float c) {
  float v[4];
  word_floats<float>(w, v);
  return make_uint4(__float_as_uint(v[0] * c), __float_as_uint(v[1] * c), __float_as_uint(v[2] * c),
                    __float_as_uint(v[3] * c));
}
template <>
__device__ __forceinline__ uint4 scale_word<bf16>(const uint4 &w, float c) {
  float v[8];
  word_floats<bf16>(w, v);
  return make_uint4(pk_bf16(v[0] * c, v[1] * c), pk_bf16(v[2] * c, v[3] * c),
                    pk_bf16(v[4] * c, v[5] * c), pk_bf16(v[6] * c, v[7] * c));
}
__device__ __forceinline__ void scale_elem(const float *s, float *d, int i, float c) { d[i] = s[i] * c; }
__device__ __forceinline__ void scale_elem(const bf16 *s, bf16 *d, int i, float c) {
  d[i] = bf16(pk_bf16(bf2f(s[i]) * c, 0.f));
}

template <typename T>
__device__ __forceinline__ void scale_piece(const GradRec &r, float c) {
  constexpr int EW = 16 / int(sizeof(T));
  const T *p = (const T *)r.src;
  T *d = (T *)r.dst;
  const Split s = split_piece<int(sizeof(T))>(p, r.n);
  if ((uintptr_t(d + s.head) & 15) == 0) {
    const uint4 *w = (const uint4 *)(p + s.head);
    uint4 *o = (uint4 *)(d + s.head);
    constexpr int U = GRAD_PIECE / 16 / GRAD_THREADS;
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = threadIdx.x + u * GRAD_THREADS;
      if (i < s.words) v[u] = w[i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = threadIdx.x + u * GRAD_THREADS;
      if (i < s.words) o[i] = scale_word<T>(v[u], c);
    }
    if (int(threadIdx.x) < s.head)
      scale_elem(p, d, threadIdx.x, c);
    else if (int(threadIdx.x) < s.head + s.tail)
      scale_elem(p, d, s.words * EW + threadIdx.x, c);
  } else {  // src and dst lie differently within 16 bytes
    for (int i = threadIdx.x; i < r.n; i += GRAD_THREADS) scale_elem(p, d, i, c);
  }
}

// PARTS: the norm comes as the partial values of grad_norm_kernel, which every
// block joins for itself (16 KB from the L2, against one more launch), and the
// first block stores it; otherwise as *norm.
template <bool PARTS, bool MAX>
__global__ __launch_bounds__(GRAD_THREADS) void grad_scale_kernel(const GradRec *__restrict__ rec,
                                                                  int64_t pieces,
                                                                  const double *__restrict__ part,
                                                                  int nparts, double max_norm,
                                                                  double *__restrict__ norm) {
  __shared__ double red[GRAD_THREADS / 64];
  double n;
  if constexpr (PARTS) {
    n = join_parts<MAX>(part, nparts, red);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
  } else {
    n = *norm;
  }
  // (a NaN norm gives NaN everywhere, an infinite one 0 and NaN: as the formula says)
  const float c = n <= max_norm ? 1.f : float(max_norm / n);
  for (int64_t i = blockIdx.x; i < pieces; i += gridDim.x) {
    const GradRec r = rec[i];
    if (c == 1.f && r.dst == r.src) continue;  // x * 1 is there already
    if (r.dtype == TRIROUTE_BF16)
      scale_piece<bf16>(r, c);
    else
      scale_piece<float>(r, c);
  }
}

static unsigned grad_blocks(int64_t pieces) {
  return unsigned(std::max<int64_t>(1, std::min<int64_t>(pieces, GRAD_MAX_BLOCKS)));
}

hipError_t launch_grad_norm(const GradRec *rec, int64_t pieces, bool mx, double *part, double *norm,
                            hipStream_t st) {
  const unsigned nb = grad_blocks(pieces);
  if (mx)
    grad_norm_kernel<true><<<nb, GRAD_THREADS, 0, st>>>(rec, pieces, part);
  else
    grad_norm_kernel<false><<<nb, GRAD_THREADS, 0, st>>>(rec, pieces, part);
  if (norm) {
    if (mx)
      grad_norm_finish_kernel<true><<<1, GRAD_THREADS, 0, st>>>(part, int(nb), norm);
    else
      grad_norm_finish_kernel<false><<<1, GRAD_THREADS, 0, st>>>(part, int(nb), norm);
  }
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradRec *rec, int64_t pieces, const double *norm, double max_norm,
                             hipStream_t st) {
  grad_scale_kernel<false, false><<<grad_blocks(pieces), GRAD_THREADS, 0, st>>>(
      rec, pieces, nullptr, 0, max_norm, const_cast<double *>(norm));
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradRec *rec, int64_t pieces, bool mx, double max_norm, double *part,
                            double *norm, hipStream_t st) {
  const hipError_t err = launch_grad_norm(rec, pieces, mx, part, nullptr, st);
  if (err != hipSuccess) return err;
  const unsigned nb = grad_blocks(pieces);
  if (mx)
    grad_scale_kernel<true, true><<<nb, GRAD_THREADS, 0, st>>>(rec, pieces, part, int(nb), max_norm, norm);
  else
    grad_scale_kernel<true, false><<<nb, GRAD_THREADS, 0, st>>>(rec, pieces, part, int(nb), max_norm, norm);
  return hipGetLastError();
}

}  // namespace tr
