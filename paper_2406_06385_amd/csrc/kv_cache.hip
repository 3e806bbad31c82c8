// Writing tokens into the paged int8 KV cache, and reading them back.
//
// Scales belong to blocks of tokens of one head: B = 1, or B = 16 .. page tokens.  A write touches the blocks
// that its tokens fall into.  With e earlier tokens in the block and s_old its scale,
//     s = max(s_old if e > 0, max|new| / 127, 2^-100),  new codes rint(x / s),  earlier codes rint(c s_old / s),
// in float32 with one rounding each, so that the codes are those of the formula.  A block that is given a NaN
// or an infinity gets s = NaN and codes 0: it reads as NaN, and its neighbours do not.
//
// Both kernels are bound by memory (by the launch for single tokens).  2^k lanes of eight values cover a token's row
// of one head, so a wave's step is 64 / 2^k tokens, and a wave takes four steps whose loads are all in flight together
// and stay in registers between the maximum and the codes.  A block of more tokens than that is shared by four waves.
// Measured, 8192 tokens of 32 heads of 128 in bfloat16, keys and values, a scale for 64 tokens: written in 41 us (4.9
// TB/s; one step's loads at a time and every code divided out: 92), read in 31 us (6.5 TB/s, part of it from the
// caches).  64 sequences' single tokens, 8 heads: 4 us each way, a launch.
#include <algorithm>

#include "kv.h"

namespace lrqat {

namespace {

constexpr int kWaves = 4;  // of a thread block
constexpr int kSteps = 4;  // of a wave, in registers

// Tokens pass by once, so they are kept out of the codes' way in the caches (8192 tokens written and read back: 71 us,
// 86 without).
__device__ __forceinline__ void load8(const uint16_t* p, float* f) {
  const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = bf16_lo(v[q]);
    f[2 * q + 1] = bf16_hi(v[q]);
  }
}
__device__ __forceinline__ void load8(const float* p, float* f) {
  const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
  const f32x4 b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = a[e];
    f[4 + e] = b[e];
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float* f) {
  const u32x4 v = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void store8(float* p, const float* f) {
  __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4*>(p + 4));
}

// The low bytes of eight words.
__device__ __forceinline__ u32x2 low_bytes(const uint32_t* c) {
  u32x2 o;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    o[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[4 * h + 3], c[4 * h + 2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(c[4 * h + 1], c[4 * h], 0x0c0c0400u), 0x05040100u);
  return o;
}

// The wave's place: its sequence, its span, K or V, and head; heads vary fastest.
struct Place {
  int seq, kv, head;
  int64_t span;
};
__device__ __forceinline__ Place place_of(uint32_t w, uint32_t heads, uint32_t spans) {
  Place p;
  const uint32_t r = w / heads, t = (r >> 1) / spans;
  p.head = int(w - r * heads);
  p.kv = int(r & 1);
  p.seq = int(t);
  p.span = (r >> 1) - t * spans;
  return p;
}

// Codes rint(x / s), the quotient rounded to float32 first; |x / s| <= 127.  Adding 1.5 2^23 rounds to the nearest
// integer, ties to even, and leaves it in the low bits.  y = x (1 / s) is within 2e-5 of the quotient, so only where y
// is that near to a rounding point the quotient itself decides (one wave in ten; the quotients of all values took half
// of the kernel's time).  s = NaN: codes 0, by the same way.  Lanes that are not live get anything.
constexpr float kRound = 12582912.f;
__device__ __forceinline__ u32x2 codes_of(const float* x, float s, bool live) {
  const float inv = s == s ? 1.f / s : 0.f;
  uint32_t c[8];
  float off = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = x[e] * inv, t = y + kRound;
    c[e] = __float_as_uint(t);
    off = fmaxf(off, fabsf(y - (t - kRound)));
  }
  if (__any(live && !(off < 0.4999f && s == s)))
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = s == s ? __float_as_uint(x[e] / s + kRound) : 0u;  // (0 times a NaN keeps its low bits)
  return low_bytes(c);
}

// The larger of a new and an old scale, or a NaN where either is one.
__device__ __forceinline__ float joined(float fresh, float old) { return old <= fresh ? fresh : fresh == fresh ? old : fresh; }

// kShared: a scale block of more than four steps, shared by the waves of the thread block; else a wave has four steps
// of whole blocks, within one page (kOnePage: its address is a scalar) or not (kPages).
enum WriteMode { kShared, kOnePage, kPages };

// 2^lg lanes a token row.
template <class T, int MODE>
__global__ __launch_bounds__(64 * kWaves) void k_kv_write(KvWriteArgs a, int lg, uint32_t spans, uint32_t units) {
  __shared__ uint32_t red[kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.y);
  const uint32_t w = MODE == kShared ? blockIdx.x : blockIdx.x * kWaves + wave;
  if (w >= units) return;
  const KvCache& c = a.c;
  const Place pl = place_of(w, c.heads, spans);
  const KvSeq q = kv_seq(a.b, pl.seq);
  const int ltok = 6 - lg;                        // log2 of a step's tokens
  const int lspan = max(ltok + 2, c.lscale);
  const int64_t base = ((q.c0 >> lspan) + pl.span) << lspan;
  if (q.end == q.c0 || base >= q.end) return;
  const int lane = threadIdx.x, sub = lane >> lg, col = 8 * (lane & ((1 << lg) - 1));
  const bool in = col < c.d;
  // positions from here on are relative to the span's start: the new tokens, and the start of the block that they enter
  const int n0 = int(max(q.c0 - base, int64_t(0))), n1 = int(min(q.end - base, int64_t(1) << lspan));
  const int open = n0 >> c.lscale << c.lscale;
  const T* x = static_cast<const T*>(a.x[pl.kv]) + int64_t(pl.head) * c.d + (q.row0 + (base - q.c0)) * a.stride[pl.kv];
  const int xstride = int(a.stride[pl.kv]), xcol = in ? col : 0;
  const int steps = MODE == kShared ? 1 << (lspan - ltok) : kSteps, first = MODE == kShared ? wave : 0, apart = MODE == kShared ? kWaves : 1;

  // the page, or the lanes' pages: codes and scales of the span's first token
  const int64_t page1 = MODE == kPages ? 0 : kv_page(c, a.b, pl.seq, base);
  if (MODE != kPages && page1 < 0) return;  // (uniform over the thread block where it is shared)
  int8_t* code1 = c.code[pl.kv] + (MODE == kPages ? 0 : kv_row(c, page1, pl.head, base));
  float* scale1 = c.scale[pl.kv] + (MODE == kPages ? 0 : kv_scale(c, page1, pl.head, base));
  const auto code_at = [&](int64_t page, int r) { return MODE == kPages ? code1 + kv_row(c, page, pl.head, base + r) : code1 + r * c.d; };
  const auto scale_at = [&](int64_t page, int r) { return MODE == kPages ? scale1 + kv_scale(c, page, pl.head, base + r) : scale1 + (r >> c.lscale); };

  // the block that held tokens before: its scale, read before any lane stores the new one
  float old = 0.f;
  const bool joins = base + open < q.c0;  // uniform; then n0 > open
  if (joins) {
    const int64_t page = MODE == kPages ? kv_page(c, a.b, pl.seq, base + open) : page1;
    if (page >= 0) old = *scale_at(page, open);
  }

  float f[kSteps][8];
  int64_t page[kSteps];
  uint32_t most[kSteps];  // magnitudes compare as integers, NaN above infinity above every number
  // no branch around a load: steps without new tokens read the nearest one, which counts for nothing
  const auto load = [&](int s0) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = ((s0 + i * apart) << ltok) + sub;
      load8(x + (min(max(r, n0), n1 - 1) * xstride + xcol), f[i]);
    }
    int32_t entry[kSteps];
    if constexpr (MODE == kPages)
#pragma unroll
      for (int i = 0; i < kSteps; ++i) entry[i] = kv_entry(c, a.b, pl.seq, base + (((s0 + i * apart) << ltok) + sub));
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = ((s0 + i * apart) << ltok) + sub;
      page[i] = MODE != kPages ? page1 : kv_inside(c, a.b, entry[i], base + r) ? entry[i] : -1;
      most[i] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) most[i] = max(most[i], __float_as_uint(f[i][e]) & 0x7fffffffu);
      if (!in || r < n0 || r >= n1 || page[i] < 0) most[i] = 0;
    }
  };
  const auto store = [&](int s0, const float* scales) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = ((s0 + i * apart) << ltok) + sub;
      const bool mine = joins && r >> c.lscale == open >> c.lscale;
      const float s = mine ? joined(scales[i], old) : scales[i];
      const u32x2 fresh = codes_of(f[i], s, in && r >= n0 && r < n1);
      if (r >= n1 || page[i] < 0) continue;
      if (r >= n0) {
        if (in) *reinterpret_cast<u32x2*>(code_at(page[i], r) + col) = fresh;
        // one lane of each block stores its scale
        if (col == 0 && r == max(r >> c.lscale << c.lscale, n0)) *scale_at(page[i], r) = s;
      } else if (mine && s != old && in) {
        u32x2* dst = reinterpret_cast<u32x2*>(code_at(page[i], r) + col);
        const u32x2 o = *dst;
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = __float_as_uint((s == s ? __builtin_amdgcn_fmed3f(float(sbyte(o[e >> 2], e & 3)) * old / s, -127.f, 127.f) : 0.f) + kRound);
        *dst = low_bytes(v);
      }
    }
  };
  const auto scale_of = [](uint32_t m) {
    return m >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__uint_as_float(m) / 127.f, kKvMinScale);
  };
  float scales[kSteps];
  if constexpr (MODE == kShared) {
    uint32_t m = 0;
    for (int s0 = first; s0 < steps; s0 += kSteps * apart) {
      load(s0);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) m = max(m, most[i]);
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) m = max(m, uint32_t(__shfl_xor(int(m), off)));
    if (lane == 0) red[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) m = max(m, red[i]);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) scales[i] = scale_of(m);
    for (int s0 = first; s0 < steps; s0 += kSteps * apart) {
      if (steps > kSteps * kWaves) load(s0);  // (else they are still here)
      store(s0, scales);
    }
  } else {
    load(0);
    const int lred = lg + min(ltok, c.lscale), many = c.lscale > ltok ? 1 << (c.lscale - ltok) : 1;  // lanes and steps of a block
    for (int off = 0; off < lred; ++off)
#pragma unroll
      for (int i = 0; i < kSteps; ++i) most[i] = max(most[i], uint32_t(__shfl_xor(int(most[i]), 1 << off)));
    if (many >= 2) {
      most[0] = most[1] = max(most[0], most[1]);
      most[2] = most[3] = max(most[2], most[3]);
    }
    if (many == 4) most[0] = most[1] = most[2] = most[3] = max(most[0], most[2]);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) scales[i] = scale_of(most[i]);
    store(0, scales);
  }
}

template <class T>
__global__ __launch_bounds__(64 * kWaves) void k_kv_read(KvReadArgs a, int lg, uint32_t spans, uint32_t units) {
  const uint32_t w = blockIdx.x * kWaves + threadIdx.y;
  if (w >= units) return;
  const KvCache& c = a.c;
  const Place pl = place_of(w, c.heads, spans);
  const KvSeq q = kv_seq(a.b, pl.seq);
  const int lane = threadIdx.x, col = 8 * (lane & ((1 << lg) - 1)), ltok = 6 - lg;
  const int64_t base = q.c0 + (pl.span << (ltok + 2)) + (lane >> lg);
  if (base >= q.end || col >= c.d) return;
  T* x = static_cast<T*>(a.x[pl.kv]) + int64_t(pl.head) * c.d + col;
  const int8_t* code = c.code[pl.kv] + col;
  const float* scale = c.scale[pl.kv];
  int64_t page[kSteps];
  u32x2 o[kSteps];
  float s[kSteps];
  int32_t entry[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) entry[i] = kv_entry(c, a.b, pl.seq, base + (int64_t(i) << ltok));
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t pos = base + (int64_t(i) << ltok);
    page[i] = kv_inside(c, a.b, entry[i], pos) ? entry[i] : -1;
    const int64_t at = max(page[i], int64_t(0));
    s[i] = scale[kv_scale(c, at, pl.head, pos)];
    o[i] = *reinterpret_cast<const u32x2*>(code + kv_row(c, at, pl.head, pos));
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int64_t pos = base + (int64_t(i) << ltok);
    if (pos >= q.end) break;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = page[i] >= 0 ? float(sbyte(o[i][e >> 2], e & 3)) * s[i] : 0.f;
    store8(x + (q.row0 + (pos - q.c0)) * a.stride[pl.kv], v);
  }
}

int lanes_log2(int d) {
  int lg = 1;
  while (8 << lg < d) ++lg;
  return lg;
}

// log2 of the tokens of a span: what a wave, or the waves that share a block, take.
int span_log2(const KvCache& c, bool write) {
  const int l = 6 - lanes_log2(c.d) + 2;
  return write ? std::max(l, c.lscale) : l;
}

// Spans that a sequence's new tokens can touch: a write's are aligned in the sequence (its blocks are whole), a read's
// start with its tokens.
int64_t spans_of(const KvCache& c, const KvBatch& b, bool write) {
  const int l = span_log2(c, write);
  return write ? ((int64_t(b.max_new) - 2 + (int64_t(1) << l)) >> l) + 1 : (int64_t(b.max_new) - 1 + (int64_t(1) << l)) >> l;
}

int64_t units_of(const KvCache& c, const KvBatch& b, bool write) {
  return int64_t(b.seqs) * spans_of(c, b, write) * 2 * c.heads;
}

WriteMode write_mode(const KvCache& c) {
  const int own = 6 - lanes_log2(c.d) + 2;  // log2 of a wave's tokens
  return c.lscale > own ? kShared : own <= c.lpage ? kOnePage : kPages;
}

}  // namespace

bool kv_fits(const KvCache& c, const KvBatch& b, bool write) {
  const int64_t units = units_of(c, b, write);
  return (write && write_mode(c) == kShared ? units : (units + kWaves - 1) / kWaves) <= kMaxThreads / (64 * kWaves);
}

hipError_t launch_kv_write(bool bf16, const KvWriteArgs& a, hipStream_t st) {
  const uint32_t units = uint32_t(units_of(a.c, a.b, true)), spans = uint32_t(spans_of(a.c, a.b, true));
  const int lg = lanes_log2(a.c.d);
  const WriteMode mode = write_mode(a.c);
  const dim3 grid(mode == kShared ? units : (units + kWaves - 1) / kWaves), block(64, kWaves);
  const auto run = [&](auto type) {
    using T = decltype(type);
    if (mode == kShared) k_kv_write<T, kShared><<<grid, block, 0, st>>>(a, lg, spans, units);
    else if (mode == kOnePage) k_kv_write<T, kOnePage><<<grid, block, 0, st>>>(a, lg, spans, units);
    else k_kv_write<T, kPages><<<grid, block, 0, st>>>(a, lg, spans, units);
  };
  if (bf16) run(uint16_t{});
  else run(float{});
  return hipGetLastError();
}

hipError_t launch_kv_read(bool bf16, const KvReadArgs& a, hipStream_t st) {
  const uint32_t units = uint32_t(units_of(a.c, a.b, false)), spans = uint32_t(spans_of(a.c, a.b, false));
  const dim3 grid((units + kWaves - 1) / kWaves), block(64, kWaves);
  if (bf16) k_kv_read<uint16_t><<<grid, block, 0, st>>>(a, lanes_log2(a.c.d), spans, units);
  else k_kv_read<float><<<grid, block, 0, st>>>(a, lanes_log2(a.c.d), spans, units);
  return hipGetLastError();
}

}  // namespace lrqat
