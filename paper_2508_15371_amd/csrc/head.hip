// head.hip - the vocabulary projection ("head") around the logit pass: the product in 8-bit
// integers that makes logit rows, and the softmax cross entropy of hidden rows over the whole
// vocabulary with its gradients, which keeps no logits.  Entry points: include/cmsd.h.
//
// Every product is D[m][n] = sum_k A[m][k] B[n][k] on the matrix cores with 16x16 tiles, of
// which a lane holds four consecutive m of one n.  m is the axis that lies contiguous in the
// output (the vocabulary of a logit row, the width of a gradient row), so a lane stores
// vectors, and a softmax over the vocabulary is first a loop over a lane's registers.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "cmsd.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Bf16 {
  uint16_t bits;
};

constexpr int kWave = 64;
constexpr int kRowBytes = 128;  // of k that a tile holds per row: one cache line
constexpr int kChunks = kRowBytes / 16;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) {
  return x;
}
// To the nearest, ties to even; a NaN stays one.
template <>
__device__ __forceinline__ Bf16 from_float<Bf16>(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return Bf16{(uint16_t)((u >> 16) | 0x40u)};
  return Bf16{(uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16)};
}

// ----------------------------------------------------------------------------- matrix cores
// One step over 64 bytes of k: lane l holds bytes 16*(l/16) .. +15 of row l%16 of either side.
template <typename T>
struct Mma;
template <>
struct Mma<Bf16> {
  typedef f32x4 Acc;
  static __device__ __forceinline__ Acc mma(u32x4 a, u32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
  }
};
template <>
struct Mma<float> {
  typedef f32x4 Acc;
  // a lane's four values stand at k = 4g..4g+3 on both sides; instruction j takes the j-th
  static __device__ __forceinline__ Acc mma(u32x4 a, u32x4 b, Acc c) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
};
template <>
struct Mma<int8_t> {
  typedef i32x4 Acc;
  static __device__ __forceinline__ Acc mma(u32x4 a, u32x4 b, Acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// One side of a product: element (row, k) at p[row*stride + k], or p[k*stride + row] where
// the loader is a transposing one.
struct Side {
  const void* p;
  int64_t stride;
  int64_t rows;
};

// Where the tiles of a launch lie: tile (m, n) and part s of k.
struct Grid {
  int32_t tiles_m, tiles_n, parts;
  int64_t k, k_part;  // k in all, and of one part (a multiple of a tile's k)
};

enum class Load { Rows, Columns };  // k contiguous in memory, or the row index

// 16 bytes of k of one row, zeros past `left` elements.
template <typename T>
__device__ __forceinline__ u32x4 row_chunk(const T* p, int64_t left) {
  constexpr int E = 16 / sizeof(T);
  u32x4 v = {0u, 0u, 0u, 0u};
  if (left >= E) {
    __builtin_memcpy(&v, p, 16);
  } else {
    T x[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
      x[j] = T{};
      if (j < left) x[j] = p[j];
    }
    __builtin_memcpy(&v, x, 16);
  }
  return v;
}

// The chunks of one side's tile that a thread brings: into registers, then into LDS.
// Chunk c of row r lies at position c ^ (r & 7) of the row's eight: the sixteen lanes that
// read one chunk of sixteen rows then take every bank alike.
template <typename T, int ROWS, int THREADS, Load LOAD>
struct Bring {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int N = ROWS * kChunks / THREADS;
  static_assert(N * THREADS == ROWS * kChunks, "whole chunks per thread");
  u32x4 v[N];

  __device__ __forceinline__ void load(const Side& s, int64_t row0, int64_t k0, int64_t k_end, int t) {
    const T* p = static_cast<const T*>(s.p);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * THREADS + t;
      v[i] = u32x4{0u, 0u, 0u, 0u};
      if (LOAD == Load::Rows) {
        const int64_t row = row0 + at / kChunks, k = k0 + (at % kChunks) * E;
        if (row < s.rows && k < k_end) v[i] = row_chunk<T>(p + row * s.stride + k, k_end - k);
      } else {
        const int64_t row = row0 + at % ROWS, k = k0 + (at / ROWS) * E;
        if (row < s.rows) {
          T x[E];
#pragma unroll
          for (int j = 0; j < E; ++j) {
            x[j] = T{};
            if (k + j < k_end) x[j] = p[(k + j) * s.stride + row];
          }
          __builtin_memcpy(&v[i], x, 16);
        }
      }
    }
  }
  __device__ __forceinline__ void store(char* lds, int t) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = i * THREADS + t;
      const int row = LOAD == Load::Rows ? at / kChunks : at % ROWS;
      const int c = LOAD == Load::Rows ? at % kChunks : at / ROWS;
      *reinterpret_cast<u32x4*>(lds + row * kRowBytes + ((c ^ (row & 7)) << 4)) = v[i];
    }
  }
};

// ----------------------------------------------------------------------------- the product
// A workgroup's tile of BM x BN, in WM x WN waves.
template <int BM_, int BN_, int WM_, int WN_>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int THREADS = WM * WN * kWave;
  static constexpr int MI = BM / WM / 16, NI = BN / WN / 16;  // 16x16 tiles of a wave
  static constexpr int LDS = (BM + BN) * kRowBytes;
};

template <class TL>
struct Place {  // where a lane's values of its wave's tile lie in the output
  int64_t m0, n0;
  int wm, lane, tile_m, part;
  __device__ __forceinline__ int64_t m(int mi) const { return m0 + mi * 16 + (lane >> 4) * 4; }  // of four
  __device__ __forceinline__ int64_t n(int ni) const { return n0 + ni * 16 + (lane & 15); }
};

template <typename T, class TL, Load LA, Load LB, class Epilogue>
__global__ __launch_bounds__(TL::THREADS) void k_product(Side a, Side b, Grid g, Epilogue e) {
  constexpr int BK = kRowBytes / sizeof(T);
  __shared__ __attribute__((aligned(16))) char lds[TL::LDS];
  char* const la = lds;
  char* const lb = lds + TL::BM * kRowBytes;
  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave % TL::WM, wn = wave / TL::WM;

  const uint32_t tiles = (uint32_t)g.tiles_m * (uint32_t)g.tiles_n;
  const int part = blockIdx.x / tiles;
  const uint32_t at = blockIdx.x % tiles;
  const int tm = at / g.tiles_n, tn = at % g.tiles_n;
  const int64_t m0 = (int64_t)tm * TL::BM, n0 = (int64_t)tn * TL::BN;
  const int64_t k_begin = part * g.k_part;
  const int64_t k_end = k_begin + g.k_part < g.k ? k_begin + g.k_part : g.k;

  typename Mma<T>::Acc acc[TL::MI][TL::NI];
#pragma unroll
  for (int i = 0; i < TL::MI; ++i)
#pragma unroll
    for (int j = 0; j < TL::NI; ++j) acc[i][j] = typename Mma<T>::Acc{};

  Bring<T, TL::BM, TL::THREADS, LA> ra;
  Bring<T, TL::BN, TL::THREADS, LB> rb;
  ra.load(a, m0, k_begin, k_end, t);
  rb.load(b, n0, k_begin, k_end, t);
  for (int64_t k = k_begin; k < k_end; k += BK) {
    __syncthreads();  // the former tile has been read
    ra.store(la, t);
    rb.store(lb, t);
    __syncthreads();
    if (k + BK < k_end) {
      ra.load(a, m0, k + BK, k_end, t);
      rb.load(b, n0, k + BK, k_end, t);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      u32x4 fa[TL::MI], fb[TL::NI];
      const int pos = ((s * 4 + (lane >> 4)) ^ (lane & 7)) << 4;
#pragma unroll
      for (int i = 0; i < TL::MI; ++i)
        fa[i] = *reinterpret_cast<const u32x4*>(la + (wm * TL::MI * 16 + i * 16 + (lane & 15)) * kRowBytes + pos);
#pragma unroll
      for (int j = 0; j < TL::NI; ++j)
        fb[j] = *reinterpret_cast<const u32x4*>(lb + (wn * TL::NI * 16 + j * 16 + (lane & 15)) * kRowBytes + pos);
#pragma unroll
      for (int i = 0; i < TL::MI; ++i)
#pragma unroll
        for (int j = 0; j < TL::NI; ++j) acc[i][j] = Mma<T>::mma(fa[i], fb[j], acc[i][j]);
    }
  }
  Place<TL> w;
  w.m0 = m0 + wm * TL::MI * 16;
  w.n0 = n0 + wn * TL::NI * 16;
  w.wm = wm;
  w.lane = lane;
  w.tile_m = tm;
  w.part = part;
  __syncthreads();  // the epilogue may take the LDS
  e.template run<TL>(acc, w, a.rows, b.rows, lds, wn, t);
}

// Four consecutive values of a row, as one vector where that is aligned and inside.
template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&x)[4], int64_t left) {
  struct alignas(4 * sizeof(T)) V {
    T v[4];
  };
  if (left >= 4 && ((uintptr_t)p & (4 * sizeof(T) - 1)) == 0) {
    V v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v.v[i] = from_float<T>(x[i]);
    *reinterpret_cast<V*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = from_float<T>(x[i]);
  }
}

// Logit rows out of the integer sums: one scale per token and one per vocabulary entry.
template <typename T>
struct LogitRows {
  const float* hidden_scales;
  const float* weight_scales;
  float scale;
  T* out;
  int64_t stride;

  template <class TL, class Acc>
  __device__ __forceinline__ void run(Acc& acc, const Place<TL>& w, int64_t M, int64_t N, char*, int, int) const {
#pragma unroll
    for (int i = 0; i < TL::MI; ++i) {
      const int64_t m = w.m(i);
      float sw[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) sw[r] = m + r < M ? weight_scales[m + r] : 0.f;
#pragma unroll
      for (int j = 0; j < TL::NI; ++j) {
        const int64_t n = w.n(j);
        if (n >= N || m >= M) continue;
        const float sh = hidden_scales[n] * scale;
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = (float)acc[i][j][r] * sh * sw[r];
        store4(out + n * stride + m, x, M - m);
      }
    }
  }
};

// A tile's share of a row's softmax: the largest logit and the sum of exponentials over it.
struct Share {
  float top, sum;
};
__device__ __forceinline__ Share join(Share x, Share y) {
  // the order of a pair changes nothing; an empty share (top = -inf, sum = 0) adds nothing
  const float top = fmaxf(x.top, y.top);
  if (top == -INFINITY) return Share{top, x.sum + y.sum};
  return Share{top, x.sum * __builtin_amdgcn_exp2f((x.top - top) * kLog2e) +
                        y.sum * __builtin_amdgcn_exp2f((y.top - top) * kLog2e)};
}

// Shares of every row's softmax, and the label's logit.
struct SoftmaxShares {
  float scale;
  const int32_t* labels;
  Share* shares;  // [n][tiles_m]
  int32_t tiles_m;
  float* at_label;  // [n]

  template <class TL, class Acc>
  __device__ __forceinline__ void run(Acc& acc, const Place<TL>& w, int64_t M, int64_t N, char* lds, int wn,
                                      int t) const {
    Share* red = reinterpret_cast<Share*>(lds);  // [WM][BN]
    static_assert(TL::WM * TL::BN * (int)sizeof(Share) <= TL::LDS, "fits the tiles' space");
#pragma unroll
    for (int j = 0; j < TL::NI; ++j) {
      const int64_t n = w.n(j);
      const int64_t label = n < N ? labels[n] : -1;
      float top = -INFINITY;
      bool bad = false;
#pragma unroll
      for (int i = 0; i < TL::MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t m = w.m(i) + r;
          const float z = acc[i][j][r] * scale;
          if (m < M) {
            top = fmaxf(top, z);
            bad |= z != z;
            if (m == label) at_label[n] = z;
          }
        }
      float sum = 0.f;
      const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < TL::MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (w.m(i) + r < M) sum += __builtin_amdgcn_exp2f((acc[i][j][r] * scale - from) * kLog2e);
      Share s{top, bad ? NAN : sum};
#pragma unroll
      for (int d = 16; d < kWave; d *= 2) s = join(s, Share{__shfl_xor(s.top, d), __shfl_xor(s.sum, d)});
      if (w.lane < 16) red[w.wm * TL::BN + wn * TL::NI * 16 + j * 16 + w.lane] = s;
    }
    __syncthreads();
    for (int c = t; c < TL::BN; c += TL::THREADS) {
      const int64_t n = w.n0 - wn * TL::NI * 16 + c;
      if (n >= N) continue;
      Share s = red[c];
#pragma unroll
      for (int k = 1; k < TL::WM; ++k) s = join(s, red[k * TL::BN + c]);
      shares[n * tiles_m + w.tile_m] = s;
    }
  }
};

// The gradient by the logits, g * scale * (softmax - [v = label]), of a piece of the
// vocabulary, rounded to the type of the products that take it.
template <typename T>
struct LogitGradient {
  float scale;
  const int32_t* labels;
  const float* lse;
  const float* grad_loss;
  int64_t first, vocab;  // the piece's first entry; entries in all
  T* out;
  int64_t stride;

  template <class TL, class Acc>
  __device__ __forceinline__ void run(Acc& acc, const Place<TL>& w, int64_t M, int64_t N, char*, int, int) const {
#pragma unroll
    for (int j = 0; j < TL::NI; ++j) {
      const int64_t n = w.n(j);
      if (n >= N) continue;
      const int64_t label = labels[n];
      const bool counts = label >= 0 && label < vocab;
      const float g = grad_loss[n] * scale, less = -lse[n] * kLog2e, mul = scale * kLog2e;
#pragma unroll
      for (int i = 0; i < TL::MI; ++i) {
        const int64_t m = w.m(i);
        if (m >= M) continue;
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], mul, less));
          x[r] = counts ? (p - (first + m + r == label ? 1.f : 0.f)) * g : 0.f;
        }
        store4(out + n * stride + m, x, M - m);
      }
    }
  }
};

// A product as it is: rounded to T, or (T = float, slabs) each part of k into a slab of its
// own, added to what a former piece left there.
template <typename T>
struct Plain {
  T* out;
  int64_t stride, slab;
  bool add;

  template <class TL, class Acc>
  __device__ __forceinline__ void run(Acc& acc, const Place<TL>& w, int64_t M, int64_t N, char*, int, int) const {
    T* const o = out + w.part * slab;
#pragma unroll
    for (int j = 0; j < TL::NI; ++j) {
      const int64_t n = w.n(j);
#pragma unroll
      for (int i = 0; i < TL::MI; ++i) {
        const int64_t m = w.m(i);
        if (n >= N || m >= M) continue;
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = acc[i][j][r];
          if (add && m + r < M) x[r] += to_float(o[n * stride + m + r]);
        }
        store4(o + n * stride + m, x, M - m);
      }
    }
  }
};

// ----------------------------------------------------------------------------- small kernels
__device__ __forceinline__ Share wave_join(Share s) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) s = join(s, Share{__shfl_xor(s.top, d), __shfl_xor(s.sum, d)});
  return s;
}

// One wave per row: its shares joined, in an order that its count fixes.
__global__ __launch_bounds__(256) void k_loss(const Share* shares, int32_t tiles_m, const float* at_label,
                                              const int32_t* labels, int64_t n_rows, int64_t vocab, float* loss,
                                              float* lse) {
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (n >= n_rows) return;
  Share s{-INFINITY, 0.f};
  for (int i = lane; i < tiles_m; i += kWave) s = join(s, shares[n * tiles_m + i]);
  s = wave_join(s);
  if (lane == 0) {
    const float l = s.top + logf(s.sum);
    const int64_t label = labels[n];
    lse[n] = l;
    loss[n] = label < 0 ? 0.f : (label < vocab ? l - at_label[n] : NAN);
  }
}

// The slabs of a product summed, in their order, into rows of T.
template <typename T>
__global__ __launch_bounds__(256) void k_sum_slabs(const float* slabs, int32_t parts, int64_t slab, int64_t rows,
                                                   int64_t width, T* out, int64_t stride) {
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < rows * width; at += (int64_t)gridDim.x * 256) {
    float x = slabs[at];
    for (int p = 1; p < parts; ++p) x += slabs[p * slab + at];
    out[at / width * stride + at % width] = from_float<T>(x);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_zero_rows(T* out, int64_t rows, int64_t width, int64_t stride) {
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < rows * width; at += (int64_t)gridDim.x * 256)
    out[at / width * stride + at % width] = from_float<T>(0.f);
}

// One workgroup per row: its largest magnitude, then its codes.  A code is the whole number
// next to x / scale (ties to even), with both quotients in double precision: in single a
// quotient next to a border falls on either side of it.
template <typename T>
__global__ __launch_bounds__(256) void k_quantize(const T* x, int64_t stride, int64_t width, int8_t* codes,
                                                  int64_t code_stride, float* scales) {
  __shared__ float tops[4];
  const int t = threadIdx.x;
  const T* const row = x + blockIdx.x * stride;
  float top = 0.f;
  bool bad = false;
  for (int64_t i = t; i < width; i += 256) {
    const float v = fabsf(to_float(row[i]));
    top = fmaxf(top, v);
    bad |= !(v < INFINITY);
  }
  if (bad) top = INFINITY;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  if ((t & 63) == 0) tops[t >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const bool finite = top < INFINITY;
  const float scale = finite ? (float)((double)top / 127.0) : NAN;
  if (t == 0) scales[blockIdx.x] = scale;
  int8_t* const out = codes + blockIdx.x * code_stride;
  for (int64_t i = t; i < width; i += 256) {
    double q = 0.0;
    if (finite && scale > 0.f) q = fmin(fmax(rint((double)to_float(row[i]) / (double)scale), -127.0), 127.0);
    out[i] = (int8_t)(int)q;
  }
}

// ----------------------------------------------------------------------------- host
cmsd_status launched() { return hipGetLastError() == hipSuccess ? CMSD_OK : CMSD_ERR_LAUNCH; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
bool launch_fits(int64_t groups, int threads) { return groups < ((int64_t)1 << 32) / threads; }

typedef Tile<64, 64, 2, 2> SimpleTile;

constexpr int64_t kMostRows = (int64_t)1 << 24;   // of hidden
constexpr int64_t kMostWidth = (int64_t)1 << 17;  // an int32 sum of 2^17 - 1 products of codes holds
constexpr int64_t kMostStride = (int64_t)1 << 40;

template <class TL>
bool product_fits(int64_t rows_m, int64_t rows_n, int parts) {
  return launch_fits(ceil_div(rows_m, TL::BM) * ceil_div(rows_n, TL::BN) * parts, TL::THREADS);
}
template <typename T, class TL, Load LA, Load LB, class Epilogue>
void launch_product(const Side& a, const Side& b, int64_t k, int parts, const Epilogue& e, hipStream_t st) {
  constexpr int BK = kRowBytes / sizeof(T);
  Grid g;
  g.tiles_m = (int32_t)ceil_div(a.rows, TL::BM);
  g.tiles_n = (int32_t)ceil_div(b.rows, TL::BN);
  g.k = k;
  g.k_part = round_up(ceil_div(k, parts), BK);
  g.parts = parts;
  const int64_t groups = (int64_t)g.tiles_m * g.tiles_n * parts;
  hipLaunchKernelGGL((k_product<T, TL, LA, LB, Epilogue>), dim3((unsigned)groups), dim3(TL::THREADS), 0, st, a, b, g, e);
}

bool sizes_ok(int64_t n_rows, int64_t vocab, int64_t width) {
  return n_rows >= 0 && n_rows < kMostRows && vocab >= 2 && vocab <= INT32_MAX && width >= 1 && width < kMostWidth;
}
bool stride_ok(int64_t stride, int64_t width) { return stride >= width && stride < kMostStride; }
bool finite(float x) { return x - x == 0.f; }

// ------------------------------------------------------------------ the gradient's plan
// The vocabulary is taken in pieces: the gradient by a piece's logits is formed in the
// workspace (rounded to the inputs' type: products on the matrix cores take it so) and
// multiplied with the weight's rows (into the hidden rows' gradient) and with the hidden
// rows (into the weight's).
struct GradPlan {
  int64_t piece;                   // vocabulary entries of a piece
  int hidden_parts, weight_parts;  // parts of k of the two products
  size_t logits_at, hidden_at, weight_at, bytes;
};
constexpr int64_t kPieceBytes = (int64_t)1 << 28;  // of a piece's logit gradients
int parts_for(int64_t tiles, int64_t k, int64_t least_k) {
  int64_t parts = 1024 / (tiles < 1 ? 1 : tiles);
  const int64_t most = k / least_k;
  parts = parts < most ? parts : most;
  return (int)(parts < 1 ? 1 : (parts > 64 ? 64 : parts));
}
GradPlan grad_plan(int64_t n, int64_t vocab, int64_t width, int es) {
  GradPlan p;
  p.piece = kPieceBytes / (n * es) / 256 * 256;
  if (p.piece < 256) p.piece = 256;
  if (p.piece > vocab) p.piece = vocab;
  const int64_t stride = round_up(p.piece, 128);
  p.hidden_parts = parts_for(ceil_div(width, 64) * ceil_div(n, 64), p.piece, 512);
  p.weight_parts = parts_for(ceil_div(width, 64) * ceil_div(p.piece, 64), n, 512);
  size_t at = 0;
  p.logits_at = at;
  at += (size_t)round_up(n * stride * es, 256);
  p.hidden_at = at;
  if (p.hidden_parts > 1 || p.piece < vocab) at += (size_t)round_up(p.hidden_parts * n * width * 4, 256);
  p.weight_at = at;
  if (p.weight_parts > 1) at += (size_t)round_up(p.weight_parts * p.piece * width * 4, 256);
  p.bytes = at;
  return p;
}

struct LossArgs {
  const void* hidden;
  int64_t hidden_stride;
  const void* weight;
  int64_t weight_stride;
  const int32_t* labels;
  float scale;
  int64_t n, vocab, width;
};

size_t loss_bytes(int64_t n, int64_t vocab) {
  return (size_t)round_up(n * ceil_div(vocab, SimpleTile::BM) * (int64_t)sizeof(Share), 256) + (size_t)round_up(n * 4, 256);
}

template <typename T>
cmsd_status enqueue_loss(const LossArgs& a, float* loss, float* lse, void* workspace, hipStream_t st) {
  typedef SimpleTile TL;
  SoftmaxShares e;
  e.scale = a.scale;
  e.labels = a.labels;
  e.tiles_m = (int32_t)ceil_div(a.vocab, TL::BM);
  e.shares = static_cast<Share*>(workspace);
  e.at_label = reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                        round_up(a.n * (int64_t)e.tiles_m * (int64_t)sizeof(Share), 256));
  const Side w{a.weight, a.weight_stride, a.vocab}, h{a.hidden, a.hidden_stride, a.n};
  if (!product_fits<TL>(a.vocab, a.n, 1)) return CMSD_ERR_ARG;
  launch_product<T, TL, Load::Rows, Load::Rows>(w, h, a.width, 1, e, st);
  hipLaunchKernelGGL(k_loss, dim3((unsigned)ceil_div(a.n, 4)), dim3(256), 0, st, e.shares, e.tiles_m, e.at_label,
                     a.labels, a.n, a.vocab, loss, lse);
  return launched();
}

// Workgroups of 256 for so many elements (a thread takes further ones past the limit).
unsigned element_groups(int64_t elements) {
  const int64_t groups = ceil_div(elements, 256);
  return (unsigned)(groups < (1 << 20) ? groups : 1 << 20);
}

template <typename T>
void sum_slabs(const float* slabs, int parts, int64_t slab, int64_t rows, int64_t width, void* out, int64_t stride,
               hipStream_t st) {
  hipLaunchKernelGGL(k_sum_slabs<T>, dim3(element_groups(rows * width)), dim3(256), 0, st, slabs, parts, slab, rows,
                     width, static_cast<T*>(out), stride);
}

template <typename T>
cmsd_status enqueue_grad(const LossArgs& a, const float* lse, const float* grad_loss, void* grad_hidden,
                         int64_t gh_stride, void* grad_weight, int64_t gw_stride, void* workspace, hipStream_t st) {
  typedef SimpleTile TL;
  const GradPlan p = grad_plan(a.n, a.vocab, a.width, sizeof(T));
  char* const ws = static_cast<char*>(workspace);
  T* const dz = reinterpret_cast<T*>(ws + p.logits_at);
  const int64_t dz_stride = round_up(p.piece, 128);
  float* const hs = reinterpret_cast<float*>(ws + p.hidden_at);
  float* const wsl = reinterpret_cast<float*>(ws + p.weight_at);
  const bool slabs = p.hidden_parts > 1 || p.piece < a.vocab;
  const Side h{a.hidden, a.hidden_stride, a.n};
  if (!product_fits<TL>(p.piece, a.n, 1) || (grad_hidden && !product_fits<TL>(a.width, a.n, p.hidden_parts)) ||
      (grad_weight && !product_fits<TL>(a.width, p.piece, p.weight_parts)))
    return CMSD_ERR_ARG;
  for (int64_t v = 0; v < a.vocab; v += p.piece) {
    const int64_t m = a.vocab - v < p.piece ? a.vocab - v : p.piece;
    const Side w{static_cast<const T*>(a.weight) + v * a.weight_stride, a.weight_stride, m};
    LogitGradient<T> e{a.scale, a.labels, lse, grad_loss, v, a.vocab, dz, dz_stride};
    launch_product<T, TL, Load::Rows, Load::Rows>(w, h, a.width, 1, e, st);
    if (grad_hidden) {
      const Side wt{w.p, w.stride, a.width}, d{dz, dz_stride, a.n};
      if (slabs)
        launch_product<T, TL, Load::Columns, Load::Rows>(wt, d, m, p.hidden_parts,
                                                         Plain<float>{hs, a.width, a.n * a.width, v > 0}, st);
      else
        launch_product<T, TL, Load::Columns, Load::Rows>(
            wt, d, m, 1, Plain<T>{static_cast<T*>(grad_hidden), gh_stride, 0, false}, st);
    }
    if (grad_weight) {
      const Side ht{a.hidden, a.hidden_stride, a.width}, dt{dz, dz_stride, m};
      T* const out = static_cast<T*>(grad_weight) + v * gw_stride;
      if (p.weight_parts > 1) {
        launch_product<T, TL, Load::Columns, Load::Columns>(ht, dt, a.n, p.weight_parts,
                                                            Plain<float>{wsl, a.width, m * a.width, false}, st);
        sum_slabs<T>(wsl, p.weight_parts, m * a.width, m, a.width, out, gw_stride, st);
      } else {
        launch_product<T, TL, Load::Columns, Load::Columns>(ht, dt, a.n, 1, Plain<T>{out, gw_stride, 0, false}, st);
      }
    }
  }
  if (grad_hidden && slabs)
    sum_slabs<T>(hs, p.hidden_parts, a.n * a.width, a.n, a.width, grad_hidden, gh_stride, st);
  return launched();
}

template <typename T>
cmsd_status enqueue_zero(void* out, int64_t rows, int64_t width, int64_t stride, hipStream_t st) {
  hipLaunchKernelGGL(k_zero_rows<T>, dim3(element_groups(rows * width)), dim3(256), 0, st, static_cast<T*>(out), rows, width,
                     stride);
  return launched();
}

cmsd_status loss_args(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                      int32_t dtype, const int32_t* labels, float scale, int64_t n_rows, int64_t vocab, int64_t width,
                      LossArgs& a) {
  if (dtype != CMSD_F32 && dtype != CMSD_BF16) return CMSD_ERR_DTYPE;
  if (!sizes_ok(n_rows, vocab, width) || !stride_ok(hidden_stride, width) || !stride_ok(weight_stride, width) ||
      !finite(scale))
    return CMSD_ERR_ARG;
  const size_t es = dtype == CMSD_F32 ? 4 : 2;
  if (!aligned(hidden, es) || !aligned(weight, es) || !aligned(labels, 4)) return CMSD_ERR_ARG;
  if (n_rows > 0 && (!hidden || !weight || !labels)) return CMSD_ERR_ARG;
  a = LossArgs{hidden, hidden_stride, weight, weight_stride, labels, scale, n_rows, vocab, width};
  return CMSD_OK;
}

}  // namespace

extern "C" {

cmsd_status cmsd_quantize_rows(const void* rows, int32_t dtype, int64_t n_rows, int64_t width, int64_t row_stride,
                               int8_t* codes, int64_t code_stride, float* scales, void* stream) {
  if (dtype != CMSD_F32 && dtype != CMSD_BF16) return CMSD_ERR_DTYPE;
  if (n_rows < 0 || n_rows > INT32_MAX || width < 1 || width >= kMostWidth || !stride_ok(row_stride, width) ||
      !stride_ok(code_stride, width))
    return CMSD_ERR_ARG;
  if (n_rows == 0) return CMSD_OK;
  if (!rows || !codes || !scales || !aligned(rows, dtype == CMSD_F32 ? 4 : 2) || !aligned(scales, 4))
    return CMSD_ERR_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  constexpr int64_t kMost = (int64_t)1 << 22;  // rows of one launch
  for (int64_t r = 0; r < n_rows; r += kMost) {
    const unsigned n = (unsigned)(n_rows - r < kMost ? n_rows - r : kMost);
    if (dtype == CMSD_F32)
      hipLaunchKernelGGL(k_quantize<float>, dim3(n), dim3(256), 0, st, static_cast<const float*>(rows) + r * row_stride,
                         row_stride, width, codes + r * code_stride, code_stride, scales + r);
    else
      hipLaunchKernelGGL(k_quantize<Bf16>, dim3(n), dim3(256), 0, st, static_cast<const Bf16*>(rows) + r * row_stride,
                         row_stride, width, codes + r * code_stride, code_stride, scales + r);
  }
  return launched();
}

cmsd_status cmsd_head_logits(const int8_t* hidden, int64_t hidden_stride, const float* hidden_scales,
                             const int8_t* weight, int64_t weight_stride, const float* weight_scales, float scale,
                             int64_t n_rows, int64_t vocab, int64_t width, void* logits, int32_t dtype,
                             int64_t logit_stride, void* stream) {
  if (dtype != CMSD_F32 && dtype != CMSD_BF16) return CMSD_ERR_DTYPE;
  if (!sizes_ok(n_rows, vocab, width) || !stride_ok(hidden_stride, width) || !stride_ok(weight_stride, width) ||
      !stride_ok(logit_stride, vocab) || !finite(scale))
    return CMSD_ERR_ARG;
  if (n_rows == 0) return CMSD_OK;
  if (!hidden || !hidden_scales || !weight || !weight_scales || !logits) return CMSD_ERR_ARG;
  if (!aligned(hidden_scales, 4) || !aligned(weight_scales, 4) || !aligned(logits, dtype == CMSD_F32 ? 4 : 2))
    return CMSD_ERR_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const Side w{weight, weight_stride, vocab}, h{hidden, hidden_stride, n_rows};
  if (!product_fits<SimpleTile>(vocab, n_rows, 1)) return CMSD_ERR_ARG;
  if (dtype == CMSD_F32)
    launch_product<int8_t, SimpleTile, Load::Rows, Load::Rows>(
        w, h, width, 1, LogitRows<float>{hidden_scales, weight_scales, scale, static_cast<float*>(logits), logit_stride},
        st);
  else
    launch_product<int8_t, SimpleTile, Load::Rows, Load::Rows>(
        w, h, width, 1, LogitRows<Bf16>{hidden_scales, weight_scales, scale, static_cast<Bf16*>(logits), logit_stride},
        st);
  return launched();
}

size_t cmsd_head_loss_workspace_bytes(int64_t n_rows, int64_t vocab) {
  if (n_rows <= 0 || !sizes_ok(n_rows, vocab, 1)) return 0;
  return loss_bytes(n_rows, vocab);
}

cmsd_status cmsd_head_loss(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                           int32_t dtype, const int32_t* labels, float scale, int64_t n_rows, int64_t vocab,
                           int64_t width, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                           void* stream) {
  LossArgs a;
  const cmsd_status s =
      loss_args(hidden, hidden_stride, weight, weight_stride, dtype, labels, scale, n_rows, vocab, width, a);
  if (s != CMSD_OK) return s;
  if (n_rows == 0) return CMSD_OK;
  if (!loss || !lse || !aligned(loss, 4) || !aligned(lse, 4)) return CMSD_ERR_ARG;
  if (!workspace || !aligned(workspace, 8) || workspace_bytes < loss_bytes(n_rows, vocab)) return CMSD_ERR_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return dtype == CMSD_F32 ? enqueue_loss<float>(a, loss, lse, workspace, st)
                           : enqueue_loss<Bf16>(a, loss, lse, workspace, st);
}

size_t cmsd_head_loss_grad_workspace_bytes(int64_t n_rows, int64_t vocab, int64_t width, int32_t dtype) {
  if (n_rows <= 0 || !sizes_ok(n_rows, vocab, width) || (dtype != CMSD_F32 && dtype != CMSD_BF16)) return 0;
  return grad_plan(n_rows, vocab, width, dtype == CMSD_F32 ? 4 : 2).bytes;
}

cmsd_status cmsd_head_loss_grad(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                                int32_t dtype, const int32_t* labels, const float* lse, const float* grad_loss,
                                float scale, int64_t n_rows, int64_t vocab, int64_t width, void* grad_hidden,
                                int64_t grad_hidden_stride, void* grad_weight, int64_t grad_weight_stride,
                                void* workspace, size_t workspace_bytes, void* stream) {
  LossArgs a;
  const cmsd_status s =
      loss_args(hidden, hidden_stride, weight, weight_stride, dtype, labels, scale, n_rows, vocab, width, a);
  if (s != CMSD_OK) return s;
  const int es = dtype == CMSD_F32 ? 4 : 2;
  if (!grad_hidden && !grad_weight && n_rows > 0) return CMSD_ERR_ARG;
  if (grad_hidden && (!aligned(grad_hidden, es) || !stride_ok(grad_hidden_stride, width))) return CMSD_ERR_ARG;
  if (grad_weight && (!aligned(grad_weight, es) || !stride_ok(grad_weight_stride, width))) return CMSD_ERR_ARG;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (n_rows == 0) {  // a sum over no rows
    if (!grad_weight) return CMSD_OK;
    return dtype == CMSD_F32 ? enqueue_zero<float>(grad_weight, vocab, width, grad_weight_stride, st)
                             : enqueue_zero<Bf16>(grad_weight, vocab, width, grad_weight_stride, st);
  }
  if (!lse || !grad_loss || !aligned(lse, 4) || !aligned(grad_loss, 4)) return CMSD_ERR_ARG;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < grad_plan(n_rows, vocab, width, es).bytes)
    return CMSD_ERR_ARG;
  return dtype == CMSD_F32 ? enqueue_grad<float>(a, lse, grad_loss, grad_hidden, grad_hidden_stride, grad_weight,
                                                 grad_weight_stride, workspace, st)
                           : enqueue_grad<Bf16>(a, lse, grad_loss, grad_hidden, grad_hidden_stride, grad_weight,
                                                grad_weight_stride, workspace, st);
}

}  // extern "C"
