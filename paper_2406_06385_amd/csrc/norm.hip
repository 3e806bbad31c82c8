// Root-mean-square norm with the residual's addition, and its gradient.
//
// Forward, a token row of n values: h = x + r (the new residual stream, stored in the activation type),
// y = h g rho with rho = (mean(h^2) + eps)^(-1/2).  The norm is taken of the float32 sum, not of the stored
// one: each output is rounded once.  As int8 codes for the W4A8 projections, y = s c with s = max|y| / 127:
// rho cancels in c = rint(h g 127 / max|h g|), so one pass over the row finds the sum of squares and
// max|h g| together, and the row stays in registers between the two sides of that one reduction.
//
// Backward at the stored stream h: with a = mean(h^2), b = mean(g dy h), rho from a,
//     dx = rho g dy - h rho^3 b + dh,   dg = sum_t dy h rho.
// Both means come from one pass too, so nothing but h is kept from the forward.
//
// Both are bound by memory: a block (a wave where the row is short) owns a row and reads it once, eight
// values a thread and vector.  Rows need no alignment (gfx950 loads 16 bytes from any 2- or 4-byte boundary).
#include <algorithm>

#include "kernels.h"

namespace lrqat {

namespace {

// 16-byte vectors at the alignment of their elements
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

// Eight values from p; those at or past `valid` are 0.
__device__ __forceinline__ void load8(const uint16_t* p, int64_t valid, float* f) {
  if (valid >= 8) {
    const u32x4 v = *reinterpret_cast<const u32x4_a2*>(p);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f[2 * q] = bf16_lo(v[q]);
      f[2 * q + 1] = bf16_hi(v[q]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = e < valid ? bf16_to_f32(p[e]) : 0.f;
  }
}
__device__ __forceinline__ void load8(const float* p, int64_t valid, float* f) {
  if (valid >= 8) {
    const f32x4 a = *reinterpret_cast<const f32x4_a4*>(p), b = *reinterpret_cast<const f32x4_a4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[e] = a[e];
      f[4 + e] = b[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = e < valid ? p[e] : 0.f;
  }
}
__device__ __forceinline__ void store8(uint16_t* p, int64_t valid, const float* f) {
  if (valid >= 8) {
    *reinterpret_cast<u32x4_a2*>(p) =
        u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < valid) p[e] = __builtin_bit_cast(uint16_t, (__bf16)f[e]);
  }
}
__device__ __forceinline__ void store8(float* p, int64_t valid, const float* f) {
  if (valid >= 8) {
    *reinterpret_cast<f32x4_a4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<f32x4_a4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < valid) p[e] = f[e];
  }
}

// The larger of two magnitudes, or a NaN where either is one: as integers, NaN lies above infinity and that above numbers.
__device__ __forceinline__ float larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }

// Wave totals of a (and of b: a sum, or the largest of magnitudes), then of the row's waves, in a fixed order.
template <bool ONE, bool MAX>
__device__ __forceinline__ void row_reduce(float& a, float& b, float (*red)[2]) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    a += __shfl_xor(a, off);
    const float o = __shfl_xor(b, off);
    b = MAX ? larger(b, o) : b + o;
  }
  if constexpr (!ONE) {
    const int w = int(threadIdx.x >> 6), nw = int(blockDim.x >> 6);
    if ((threadIdx.x & 63) == 0) {
      red[w][0] = a;
      red[w][1] = b;
    }
    __syncthreads();
    a = red[0][0];
    b = red[0][1];
    for (int i = 1; i < nw; ++i) {
      a += red[i][0];
      b = MAX ? larger(b, red[i][1]) : b + red[i][1];
    }
  }
}

// ONE: a wave a row, four rows a block (blockDim 64 x 4); else a block a row.  8192 bfloat16 rows of 4096 values with
// a residual, to the stream and int8 codes: 49 us (4.8 TB/s, a large copy reaches 5.1); a single row 3.4 us.
template <class T, int NV, bool ONE>
__global__ __launch_bounds__(1024) void k_rmsnorm(NormArgs a) {
  __shared__ float red[16][2];
  __shared__ int redi[16];
  const int64_t row = ONE ? int64_t(blockIdx.x) * 4 + threadIdx.y : blockIdx.x;
  if (ONE && row >= a.T) return;
  const int64_t n = a.n;
  const int nt = ONE ? 64 : int(blockDim.x);
  const T* x = static_cast<const T*>(a.x) + row * n;
  const T* r = a.r ? static_cast<const T*>(a.r) + row * n : nullptr;
  float hg[NV][8];
  float ss = 0.f, mx = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t j = 8 * (int64_t(threadIdx.x) + int64_t(nt) * i), valid = n - j;
#pragma unroll
    for (int e = 0; e < 8; ++e) hg[i][e] = 0.f;
    if (valid > 0) {
      float h[8], g[8];
      load8(x + j, valid, h);
      load8(a.g + j, valid, g);
      if (r) {
        float v[8];
        load8(r + j, valid, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += v[e];
      }
      if (a.h) store8(static_cast<T*>(a.h) + row * n + j, valid, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss = __builtin_fmaf(h[e], h[e], ss);
        hg[i][e] = h[e] * g[e];
        mx = larger(mx, fabsf(hg[i][e]));
      }
    }
  }
  row_reduce<ONE, true>(ss, mx, red);
  const float rho = 1.f / __builtin_sqrtf(ss / float(n) + a.eps);
  if (a.y) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t j = 8 * (int64_t(threadIdx.x) + int64_t(nt) * i), valid = n - j;
      if (valid > 0) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = hg[i][e] * rho;
        store8(static_cast<T*>(a.y) + row * n + j, valid, y);
      }
    }
  }
  if (!a.codes) return;
  // 127 / mx would pass float32 from mx < 2^-121 on, and 0 times it be no 0: such rows are lifted by 2^64 first
  const float lift = mx < 0x1p-100f ? 0x1p64f : 1.f, inv = mx > 0.f ? 127.f / (mx * lift) : 0.f;
  int total = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t j = 8 * (int64_t(threadIdx.x) + int64_t(nt) * i);
    if (j < a.ldc) {  // the columns past n are 0
      u32x2 o;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = uint32_t(int(__builtin_rintf(__builtin_amdgcn_fmed3f(hg[i][4 * q + e] * lift * inv, -127.f, 127.f))));
        total += int(c[0]) + int(c[1]) + int(c[2]) + int(c[3]);
        o[q] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400u), __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u), 0x05040100u);
      }
      *reinterpret_cast<u32x2*>(a.codes + row * a.ldc + j) = o;
    }
  }
  if (a.nsum) {  // uniform
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off);
    if constexpr (!ONE) {
      if ((threadIdx.x & 63) == 0) redi[threadIdx.x >> 6] = total;
      __syncthreads();
      total = 0;
      for (int w = 0; w < int(blockDim.x >> 6); ++w) total += redi[w];
    }
    if (threadIdx.x == 0) a.nsum[row] = total;
  }
  // NaN where the row holds a NaN or an infinity, also one that a gain of 0 hides from mx: the row would read as zeros
  if (threadIdx.x == 0) a.sx[row] = larger(ss, mx) < __builtin_inff() ? rho * mx / 127.f : __builtin_nanf("");
}

// Eight values as they are loaded.
template <class T>
struct Raw;
template <>
struct Raw<uint16_t> {
  u32x4 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const u32x4_a2*>(p); }
  __device__ __forceinline__ float get(int e) const { return e & 1 ? bf16_hi(v[e >> 1]) : bf16_lo(v[e >> 1]); }
};
template <>
struct Raw<float> {
  f32x4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = *reinterpret_cast<const f32x4_a4*>(p);
    v[1] = *reinterpret_cast<const f32x4_a4*>(p + 4);
  }
  __device__ __forceinline__ float get(int e) const { return v[e >> 2][e & 3]; }
};

// Rows are dealt to the blocks (waves) in turn; a thread keeps its columns, so that its part of dg stays in
// registers and leaves once, as a row of the partial sums.  FULL, rows of whole vectors up to 16384 values (8192 in
// float32): the next row's loads are on their way while this one's sums meet, without a branch: threads past the row's
// end read its first vector and do not count it.  Otherwise the row is read again (from the caches) after its sums: of
// longer rows a thread's part does not fit beside dg.  8192 bfloat16 rows,
// the sums of dg included: of 5120 values 71 us (4.7 TB/s of h, dy, dh and dx), of 11008 141 us (read twice: 370).
template <class T, int NV, bool ONE, bool FULL>
__global__ __launch_bounds__(NV == 1 || (FULL && sizeof(T) == 4) ? 512 : 1024) void k_rmsnorm_bwd(NormBwdArgs a) {
  __shared__ float red[2][16][2];
  const int64_t n = a.n;
  const int nt = ONE ? 64 : int(blockDim.x);
  const int64_t owner = ONE ? blockIdx.x + int64_t(gridDim.x) * threadIdx.y : blockIdx.x;
  const int64_t owners = ONE ? int64_t(gridDim.x) * 4 : gridDim.x;
  const T* H = static_cast<const T*>(a.h);
  const T* DY = static_cast<const T*>(a.dy);
  const T* DH = static_cast<const T*>(a.dh);
  const auto column = [&](int i) { return 8 * (int64_t(threadIdx.x) + int64_t(nt) * i); };
  float dg[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[i][e] = 0.f;
  const auto factors = [&](float ss, float dot, float& rho, float& c) {
    rho = 1.f / __builtin_sqrtf(ss / float(n) + a.eps);
    c = rho * rho * (dot / float(n));
  };
  int turn = 0;
  if constexpr (FULL) {
    float g[NV][8];
    struct Row {
      Raw<T> h[NV], dy[NV], dh[NV];
    } cur, next;  // as they are loaded: values take twice the registers in bfloat16
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[i][e] = 0.f;
      if (column(i) < n) load8(a.g + column(i), 8, g[i]);
    }
    const auto fetch = [&](Row& to, int64_t row) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int64_t at = row * n + (column(i) < n ? column(i) : 0);
        to.h[i].load(H + at);
        to.dy[i].load(DY + at);
        if (DH) to.dh[i].load(DH + at);  // uniform over the launch
      }
    };
    if (owner < a.T) fetch(next, owner);
    for (int64_t row = owner; row < a.T; row += owners, turn ^= 1) {
      float ss = 0.f, dot = 0.f, rho, c;
      cur = next;
      fetch(next, min(row + owners, a.T - 1));
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (column(i) < n)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float h = cur.h[i].get(e);
            ss = __builtin_fmaf(h, h, ss);
            dot = __builtin_fmaf(g[i][e] * cur.dy[i].get(e), h, dot);
          }
      row_reduce<ONE, false>(ss, dot, red[turn]);  // two buffers: one barrier a row
      factors(ss, dot, rho, c);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (column(i) < n) {
          float d[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float h = cur.h[i].get(e), dy = cur.dy[i].get(e);
            d[e] = (DH ? cur.dh[i].get(e) : 0.f) + rho * (g[i][e] * dy - h * c);
            dg[i][e] = __builtin_fmaf(dy, h * rho, dg[i][e]);
          }
          store8(static_cast<T*>(a.dx) + row * n + column(i), 8, d);
        }
    }
  } else {
    const auto read = [&](int i, int64_t row, float* h, float* gdy, float* dy) {
      const int64_t j = column(i), valid = n - j;
      float g[8];
      load8(H + row * n + j, valid, h);
      load8(DY + row * n + j, valid, dy);
      load8(a.g + j, valid, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) gdy[e] = g[e] * dy[e];
    };
    for (int64_t row = owner; row < a.T; row += owners, turn ^= 1) {
      float ss = 0.f, dot = 0.f, rho, c;
      float h[8], gdy[8], dy[8], d[8];
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (column(i) < n) {
          read(i, row, h, gdy, dy);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ss = __builtin_fmaf(h[e], h[e], ss);
            dot = __builtin_fmaf(gdy[e], h[e], dot);
          }
        }
      row_reduce<ONE, false>(ss, dot, red[turn]);
      factors(ss, dot, rho, c);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (column(i) < n) {
          read(i, row, h, gdy, dy);
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = 0.f;
          if (DH) load8(DH + row * n + column(i), n - column(i), d);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            d[e] += rho * (gdy[e] - h[e] * c);
            dg[i][e] = __builtin_fmaf(dy[e], h[e] * rho, dg[i][e]);
          }
          store8(static_cast<T*>(a.dx) + row * n + column(i), n - column(i), d);
        }
    }
  }
  if (!a.part) return;
  if constexpr (ONE) {  // the block's four waves join theirs first
    __shared__ float join[3][64][8];
    if (threadIdx.y)
#pragma unroll
      for (int e = 0; e < 8; ++e) join[threadIdx.y - 1][threadIdx.x][e] = dg[0][e];
    __syncthreads();
    if (threadIdx.y) return;
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int e = 0; e < 8; ++e) dg[0][e] += join[w][threadIdx.x][e];
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int64_t j = column(i);
    if (j < n) store8(a.part + blockIdx.x * n + j, n - j, dg[i]);
  }
}

// dg = (accumulate ? dg : 0) + the partial rows, 16 slices of them added side by side and joined in order.
__global__ __launch_bounds__(1024) void k_rmsnorm_dgain(const float* __restrict__ part, int64_t nparts, int64_t n,
                                                         float* __restrict__ dg, int accumulate) {
  __shared__ float red[16][64];
  const int c = threadIdx.x & 63, sl = threadIdx.x >> 6;
  const int64_t j = int64_t(blockIdx.x) * 64 + c;
  float s = 0.f;
  if (j < n) {
#pragma unroll 8
    for (int64_t p = sl; p < nparts; p += 16) s += part[p * n + j];
  }
  red[sl][c] = s;
  __syncthreads();
  if (sl == 0 && j < n) {
    for (int i = 1; i < 16; ++i) s += red[i][c];
    dg[j] = (accumulate ? dg[j] : 0.f) + s;
  }
}

// Waves in flight.  Few leave the card idle while rows meet, many leave many partial rows to write and to add (those of
// a wave a row are joined four by four first).  us of both kernels, 8192 bfloat16 rows, at 1280 / 2048 / 4096 waves:
// 2048 values 43.0 / 32.2 / 34.6, 5120: 78.1 / 70.6 / 90.5, 11008: 140 / 141 / 173; at 2048: 128 values 10.0.
constexpr int kBwdWaves = 2048;

// Threads of a row and vectors of eight a thread: up to 512 threads with as few vectors as cover the row.
struct Shape {
  int nt, nv;
};
Shape shape_of(int64_t n, bool backward) {
  const int64_t vecs = (n + 7) / 8;
  Shape s{512, 1};
  while (s.nv < (backward ? 2 : 8) && int64_t(s.nt) * s.nv < vecs) s.nv *= 2;
  if (int64_t(s.nt) * s.nv < vecs) s.nt = 1024;  // (the gradient's rows stay in registers up to 16384 values)
  while (int64_t(s.nt) * s.nv < vecs) s.nv *= 2;
  s.nt = int((vecs + 64 * s.nv - 1) / (64 * s.nv)) * 64;
  return s;
}

// f(vectors a thread, wave a row) with both as compile-time constants
template <class F>
hipError_t by_shape(const Shape& s, F&& f) {
  using std::integral_constant;
  if (s.nt == 64 && s.nv == 1) return f(integral_constant<int, 1>{}, std::true_type{});
  switch (s.nv) {
    case 1: return f(integral_constant<int, 1>{}, std::false_type{});
    case 2: return f(integral_constant<int, 2>{}, std::false_type{});
    case 4: return f(integral_constant<int, 4>{}, std::false_type{});
    default: return f(integral_constant<int, 8>{}, std::false_type{});
  }
}

}  // namespace

hipError_t launch_rmsnorm(bool bf16, const NormArgs& a, hipStream_t st) {
  const Shape s = shape_of(a.n, false);
  return by_shape(s, [&](auto nv, auto one) {
    constexpr int NV = decltype(nv)::value;
    constexpr bool ONE = decltype(one)::value;
    const dim3 grid(unsigned(ONE ? (a.T + 3) / 4 : a.T)), block(unsigned(s.nt), ONE ? 4 : 1);
    if (bf16) k_rmsnorm<uint16_t, NV, ONE><<<grid, block, 0, st>>>(a);
    else k_rmsnorm<float, NV, ONE><<<grid, block, 0, st>>>(a);
    return hipGetLastError();
  });
}

// Rows of partial sums, one a block: a block for each of the 256 CUs, more where a block has few waves.
int64_t rmsnorm_bwd_parts(int64_t T, int64_t n) {
  const Shape s = shape_of(n, true);
  const bool one = s.nt == 64 && s.nv == 1;
  const int64_t most = std::max(256, kBwdWaves / (s.nt / 64));
  return std::min(T, one ? most / 4 : most);
}

hipError_t launch_rmsnorm_bwd(bool bf16, const NormBwdArgs& a, float* dgain, int accumulate, hipStream_t st) {
  const Shape s = shape_of(a.n, true);
  const int64_t parts = rmsnorm_bwd_parts(a.T, a.n);
  const hipError_t e = by_shape(s, [&](auto nv, auto one) {
    constexpr int NV = decltype(nv)::value;
    constexpr bool ONE = decltype(one)::value;
    const dim3 grid{unsigned(parts)}, block(unsigned(s.nt), ONE ? 4 : 1);
    const auto run = [&](auto type, auto full) { k_rmsnorm_bwd<decltype(type), NV, ONE, decltype(full)::value><<<grid, block, 0, st>>>(a); };
    const bool full = a.n % 8 == 0 && NV <= 2 && (bf16 || s.nt <= 512);
    if constexpr (NV <= 2) {
      if (full) bf16 ? run(uint16_t{}, std::true_type{}) : run(float{}, std::true_type{});
    }
    if (!full) bf16 ? run(uint16_t{}, std::false_type{}) : run(float{}, std::false_type{});
    return hipGetLastError();
  });
  if (e != hipSuccess || !a.part) return e;
  k_rmsnorm_dgain<<<unsigned((a.n + 63) / 64), 1024, 0, st>>>(a.part, parts, a.n, dgain, accumulate);
  return hipGetLastError();
}

}  // namespace lrqat
