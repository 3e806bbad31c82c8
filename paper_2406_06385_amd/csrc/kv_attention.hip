// Attention over the paged int8 cache.
//
// Row i of a head has the query q, key j the codes k_j, v_j and the scales a_j, b_j.  With
//     t_j = scale log2(e) a_j (q . k_j) + log2(b_j),   m = max t_j - 14,   w_j = 2^(t_j - m)  in (0, 2^14]
// the output is  sum_j w_j v_j / sum_j (w_j / b_j): the values' scales ride in the exponent, so that one
// exponential a score serves both sums, and the matrix product of the numerator takes the codes as they are.
// Codes are exact in bfloat16 (keys, beside bfloat16 queries) and in half precision (values); the weights are
// rounded to the 11 bits of half precision there (its subnormals begin 2^28 below the largest weight), everything
// else is float32.
//
// The products are computed transposed, S^T = K Q^T and O^T = V^T W^T: a query row is a column of the result,
// so a lane's scores all belong to one row, its running maximum and sum need two exchanges a step, and the
// scores leave the first product in the lanes that the second one wants them in.  The order of the contracted
// index is free as long as both operands use the same one: keys are dealt to the rows of the first product so
// that each lane ends up with 16 consecutive keys, and their values are read a few bytes of 16 rows at a time,
// which makes the transposition part of the conversion.  With few rows nothing but the join of the waves goes through
// LDS; with many, the block's waves share what they read there.
//
// Rows of the query tokens and of the query heads that share a key/value head are one list: grouped heads read
// the cache once.  A long axis is split over blocks (whole chunks of keys, so that ragged batches stay even),
// and the splits are joined by a second kernel in their order.
#include <algorithm>

#include "kv.h"

namespace lrqat {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kRowTile = kKvRowTile, kStep = kKvStep;

__device__ __forceinline__ f32x4 mfma16_bf16(const u32x4& p, const u32x4& q, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16_f16(const u32x4& p, const u32x4& q, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  f16x2 v;
  v[0] = (_Float16)lo;
  v[1] = (_Float16)hi;
  return __builtin_bit_cast(uint32_t, v);
}
// two integers in [-2048, 2048]: exact whatever the rounding
__device__ __forceinline__ uint32_t pack_code_f16x2(int lo, int hi) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(float(lo), float(hi)));
}
// codes 0..7 of two words as bfloat16
__device__ __forceinline__ u32x4 codes_bf16(uint32_t a, uint32_t b) {
  return u32x4{pack_bf16x2(float(sbyte(a, 0)), float(sbyte(a, 1))), pack_bf16x2(float(sbyte(a, 2)), float(sbyte(a, 3))),
               pack_bf16x2(float(sbyte(b, 0)), float(sbyte(b, 1))), pack_bf16x2(float(sbyte(b, 2)), float(sbyte(b, 3)))};
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// A value's scale as the exponent takes it: never below the least one (a NaN stays).
__device__ __forceinline__ float sane(float s) { return s < kKvMinScale ? kKvMinScale : s; }

constexpr float kNone = -__builtin_inff();
constexpr float kBias = 14.f;  // the largest weight is 2^14
// What the exponents are taken from, given the largest one: kBias below it.  From 2^25 on float32 may put that 16 below,
// and half precision ends short of 2^16; so there, where an exponent is a multiple of 4 anyway, without the bias.
__device__ __forceinline__ float below(float mx) {
  const float m = mx - kBias;
  return mx - m <= kBias + 1.f ? m : mx;  // (mx where it is an infinity)
}

// Denominators are held in units of 2^16: a key of a block of zeros adds 2^14 / 2^-100 or twice that, of which float32
// would hold 2^13; as it is, 2^29, and what the largest scales of bfloat16 values add, 2^14 / 2^121, stays normal too.
// A lane's terms of a step are added up before they are taken to that unit.
constexpr float kDen = 0x1p-16f;
// 1 / l; 0 where no key was seen, NaN where a NaN was.
__device__ __forceinline__ float reciprocal(float l) { return l > 0.f ? kDen / l : l == l ? 0.f : l; }

// What a block works on.
struct Tile {
  int seq, head, split;
  int64_t row0, c0;  // first row of the sequence in the batch, its cached tokens
  int r0, rows;      // the tile's first row; rows (token, shared head) of the sequence
  int last;          // the last position that any row of the sequence sees
  bool split_up;               // the sequence has more than one split: partial results
};
// The splits of a row tile are neighbours, then come the heads (so that an XCD keeps to few of them), then the row
// tiles, where many rows are in play from the last one, which has the most keys of a causal prompt.
__device__ __forceinline__ bool tile_of(const KvAttnArgs& a, int rows_per_tile, bool last_first, Tile& t) {
  uint32_t w = blockIdx.x;
  t.split = int(w % uint32_t(a.nsplit));
  w /= uint32_t(a.nsplit);
  t.head = int(w % uint32_t(a.c.heads));
  w /= uint32_t(a.c.heads);
  const uint32_t i = w % a.tiles;
  t.r0 = int(last_first ? a.tiles - 1 - i : i) * rows_per_tile;
  t.seq = int(w / a.tiles);
  const KvSeq q = kv_seq(a.b, t.seq);
  t.row0 = q.row0;
  t.c0 = q.c0;
  t.rows = int(q.end - q.c0) * a.group;
  t.last = int(min(q.end, int64_t(a.b.width) << a.c.lpage) - 1);
  t.split_up = kv_split_up(t.last, a.chunk, a.nsplit);
  return t.r0 < t.rows;
}
// The last key that row r of the tile's sequence sees; -1 past its rows.
__device__ __forceinline__ int row_limit(const KvAttnArgs& a, const Tile& t, int r) {
  if (r >= t.rows) return -1;
  return a.causal ? int(min(t.c0 + int64_t(uint32_t(r) / uint32_t(a.group)), int64_t(t.last))) : t.last;
}
// A result as it is stored: values of scales below the least one are 0.
__device__ __forceinline__ float result(float x) { return fabsf(x) < 0x1p-92f ? 0.f : x; }

// ---------------------------------------------------------------- few rows
// A block owns 16 rows, and its NW waves take steps of 64 keys in turn, straight from memory.  Keys are loaded for
// the next step as soon as this step's scores are done with theirs, values when their product is, so that loads are
// in flight all the time without a second set of registers; table entries are read a step ahead of that.
// Bound by memory where there are units enough: 64 sequences of 4096 keys, 32 heads of 128, 226 us (5.1 TB/s); one
// token over 32768 keys, 8 heads, 16 us (4.2 TB/s) and 4 for the join.  The first version, a step at a time: 278, 36.
// DH: 64 DH >= d.  TOK: a scale a token, else a scale for 16 or more.
template <int DH, bool TOK, int NW>
__global__ __launch_bounds__(64 * NW, DH == 4 ? 1 : 2) void k_kv_attn_rows(KvAttnArgs a) {
  constexpr int VB = 4 * DH;  // bytes of a value row a lane reads
  constexpr int NS = TOK ? 16 : 1;
  __shared__ float red_ml[NW][16][2];
  __shared__ f32x4 red_o[NW / 2][VB][64];
  Tile tl;
  if (!tile_of(a, kRowTile, false, tl)) return;
  const KvCache& c = a.c;
  const int lane = threadIdx.x & 63, i16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6));
  const int d = c.d;

  // the lane's row: a query token and one of the heads that share the keys
  const int rr = tl.r0 + i16;
  const bool valid = rr < tl.rows;
  const uint32_t qi = uint32_t(rr) / uint32_t(a.group), head = tl.head * a.group + uint32_t(rr) % uint32_t(a.group);
  const int64_t token = tl.row0 + qi;
  const int limit = row_limit(a, tl, rr);
  const int k0 = tl.split * a.chunk, k1 = kv_split_end(tl.split, a.nsplit, a.chunk, row_limit(a, tl, min(tl.r0 + kRowTile, tl.rows) - 1) + 1);
  if (k0 >= k1 && tl.split > 0) return;  // (split 0 of a sequence without keys writes its zeros)

  u32x4 qf[DH][2];
#pragma unroll
  for (int h = 0; h < DH; ++h)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int col = 64 * h + 16 * g + 8 * u;
      qf[h][u] = valid && col < d ? *reinterpret_cast<const u32x4*>(a.q + token * a.q_stride + int64_t(head) * d + col) : u32x4{0u, 0u, 0u, 0u};
    }
  f32x4 o[VB];
#pragma unroll
  for (int e = 0; e < VB; ++e) o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNone, l = 0.f;

  // Row i of score product t is key 16 (i / 4) + 4 t + i % 4 of the step; a lane's scores are then keys 16 g .. + 15.
  // No branch stands around a load, so that waits for them can be counted: columns past d are those of column 0
  // (their queries are 0, their results not stored).
  const int pk = 16 * (i16 >> 2), pv = 16 * g;
  int koff[DH];
#pragma unroll
  for (int h = 0; h < DH; ++h) koff[h] = (i16 & 3) * d + (64 * h + 16 * g < d ? 64 * h + 16 * g : 0);
  const int voff = VB * i16 < d ? VB * i16 : 0;
  const int32_t* table = a.b.table + int64_t(tl.seq) * a.b.width;
  auto entry = [&](int pos) { return table[min(pos >> c.lpage, a.b.width - 1)]; };
  auto inside = [&](int page) { return page >= 0 && page < c.pages; };
  int page_k, page_v, next_k, next_v;  // table entries of the keys and values at hand, and of the next step's
  u32x4 kc[4][DH];
  uint32_t vc[16][DH];
  float sk[NS], sv[NS];
  auto load_k = [&](int kb) {
    const int8_t* p = c.code[0] + kv_row(c, inside(page_k) ? page_k : 0, tl.head, kb + pk);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int h = 0; h < DH; ++h) kc[t][h] = *reinterpret_cast<const u32x4*>(p + koff[h] + 4 * t * d);
  };
  auto load_v = [&](int kb) {
    const int page = inside(page_v) ? page_v : 0;
    const int64_t is = kv_scale(c, page, tl.head, kb + pv);
    if constexpr (TOK) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<f32x4*>(sk + 4 * i) = *reinterpret_cast<const f32x4*>(c.scale[0] + is + 4 * i);
        *reinterpret_cast<f32x4*>(sv + 4 * i) = *reinterpret_cast<const f32x4*>(c.scale[1] + is + 4 * i);
      }
    } else {
      sk[0] = c.scale[0][is];
      sv[0] = c.scale[1][is];
    }
    const int8_t* p = c.code[1] + kv_row(c, page, tl.head, kb + pv) + voff;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if constexpr (DH == 1) vc[j][0] = *reinterpret_cast<const uint32_t*>(p + j * d);
      if constexpr (DH == 2) *reinterpret_cast<u32x2*>(vc[j]) = *reinterpret_cast<const u32x2*>(p + j * d);
      if constexpr (DH == 4) *reinterpret_cast<u32x4*>(vc[j]) = *reinterpret_cast<const u32x4*>(p + j * d);
    }
  };
  // a step at kb; the next one's loads where there is one
  auto step = [&](int kb, auto more) {
    constexpr bool MORE = decltype(more)::value;
    const int kn = kb + kStep * NW;
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int h = 0; h < DH; ++h)
#pragma unroll
        for (int u = 0; u < 2; ++u) s[t] = mfma16_bf16(codes_bf16(kc[t][h][2 * u], kc[t][h][2 * u + 1]), qf[h][u], s[t]);
    }
    const bool held = inside(page_v);
    if constexpr (MORE) {
      page_k = next_k;
      load_k(kn);
    }
    float w[16], rb[NS], lb[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const float b = sane(sv[i]);
      lb[i] = __builtin_amdgcn_logf(b);
      rb[i] = __builtin_amdgcn_rcpf(fmaxf(b, kKvMinScale));  // finite for every b: what no row sees must not leave a NaN
    }
    const int seen = held ? limit - (kb + pv) : -1;
    float mx = kNone;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float x = __builtin_fmaf(s[j >> 2][j & 3], sk[TOK ? j : 0] * a.qk, lb[TOK ? j : 0]);
      w[j] = j <= seen ? x : kNone;
      mx = fmaxf(mx, w[j]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = below(fmaxf(mx, __shfl_xor(mx, 32)));
    const float m1 = fmaxf(m, mx), mf = m1 == kNone ? 0.f : m1;
    const float alpha = exp2_(m - mf);
    m = m1;
    l *= alpha;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < VB; ++e) o[e] *= alpha;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      w[j] = exp2_(w[j] - mf);
      sum = __builtin_fmaf(w[j], rb[TOK ? j : 0], sum);
    }
    l = __builtin_fmaf(sum, kDen, l);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      u32x4 p;
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = pack_f16x2(w[8 * u + 2 * i], w[8 * u + 2 * i + 1]);
#pragma unroll
      for (int e = 0; e < VB; ++e) {
        u32x4 vf;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vf[i] = pack_code_f16x2(sbyte(vc[8 * u + 2 * i][e >> 2], e & 3), sbyte(vc[8 * u + 2 * i + 1][e >> 2], e & 3));
        o[e] = mfma16_f16(vf, p, o[e]);
      }
    }
    if constexpr (MORE) {
      page_v = next_v;
      load_v(kn);
      next_k = entry(kn + kStep * NW + pk);
      next_v = entry(kn + kStep * NW + pv);
    }
  };
  int kb = k0 + kStep * wave;
  if (kb < k1) {
    page_k = entry(kb + pk);
    page_v = entry(kb + pv);
    next_k = entry(kb + kStep * NW + pk);
    next_v = entry(kb + kStep * NW + pv);
    load_k(kb);
    load_v(kb);
    for (; kb + kStep * NW < k1; kb += kStep * NW) step(kb, std::true_type{});
    step(kb, std::false_type{});
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // join the waves: to the common maximum, then in a fixed tree
  if (g == 0) {
    red_ml[wave][i16][0] = m;
    red_ml[wave][i16][1] = l;
  }
  __syncthreads();
  float mt = kNone;
#pragma unroll
  for (int i = 0; i < NW; ++i) mt = fmaxf(mt, red_ml[i][i16][0]);
  const float mtf = mt == kNone ? 0.f : mt;
  l = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) l += red_ml[i][i16][1] * exp2_(red_ml[i][i16][0] - mtf);
  const float f = exp2_(m - mtf);
#pragma unroll
  for (int e = 0; e < VB; ++e) o[e] *= f;
#pragma unroll
  for (int half = NW / 2; half > 0; half /= 2) {
    if (wave >= half && wave < 2 * half)
#pragma unroll
      for (int e = 0; e < VB; ++e) red_o[wave - half][e][lane] = o[e];
    __syncthreads();
    if (wave < half)
#pragma unroll
      for (int e = 0; e < VB; ++e) o[e] += red_o[wave][e][lane];
    __syncthreads();
  }
  if (wave > 0 || !valid) return;
  // element v of o[e]: column VB (4 g + v) + e
  if (!tl.split_up) {
    const float r = reciprocal(l);
    uint16_t* dst = a.o + token * a.o_stride + int64_t(head) * d + 4 * VB * g;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (VB * (4 * g + v) >= d) break;
      uint32_t x[VB / 2];
#pragma unroll
      for (int e = 0; e < VB; e += 2) x[e / 2] = pack_bf16x2(result(o[e][v] * r), result(o[e + 1][v] * r));
#pragma unroll
      for (int i = 0; i < VB / 4; ++i) *reinterpret_cast<u32x2*>(dst + VB * v + 4 * i) = u32x2{x[2 * i], x[2 * i + 1]};
    }
  } else {
    const int64_t at = (int64_t(tl.split) * a.b.tokens + token) * a.hq + head;
    float* dst = a.part_o + at * d + 4 * VB * g;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (VB * (4 * g + v) >= d) break;
#pragma unroll
      for (int e = 0; e < VB; e += 4) *reinterpret_cast<f32x4*>(dst + VB * v + e) = f32x4{o[e][v], o[e + 1][v], o[e + 2][v], o[e + 3][v]};
    }
    if (g == 0) {
      a.part_ml[2 * at] = mt;
      a.part_ml[2 * at + 1] = l;
    }
  }
}

// ---------------------------------------------------------------- many rows
// A block's waves own 32 rows each (the columns of their products) and share the keys and values of a step,
// converted once into LDS: keys as bfloat16 rows, values as half-precision columns.  The next step's codes are on
// their way while this one's products run, and its pages are known by then; one barrier a step.
// Keys and values lie in 16-byte pieces of eight elements, in rows of an odd number of pieces, so that the 16 lanes
// of a read phase fall on different banks and every read of a lane has one base address.
// A causal prompt of 8192 tokens, 32 query and 8 key/value heads of 128, a scale a token: 630 us (870 TFLOP/s).  A
// wave's step is 32 matrix instructions (1024 clocks), 270 others and 56 reads of 16 bytes a lane from LDS, and its
// two waves a SIMD overlap little: probes without the values' product, the scales, the conversion into LDS or the
// exponentials were 147, 91, 62 and 48 us faster (of 655), about what each takes alone, and 40 address instructions
// fewer gained 25.  Slower were the products of one half of a step beside the exponentials of the other (644 at 32 rows
// a wave, 780 at 64), scales broadcast across lanes (670 of 660) and every other wave half a step late.
__device__ __forceinline__ f32x16 mfma32_f16(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <int DP, bool TOK>  // DP: 64, 128 or 256 >= d; the columns past d are 0
struct ManyLds {
  static constexpr int NS = TOK ? kStep : kStep / 16;
  static constexpr int KP = DP / 8 + 1, VP = kStep / 8 + 1;  // pieces of a row, and one
  float fig[2][3][NS];    // score factor, log2 of the value's scale, its reciprocal
  u32x4 k[2][kStep][KP];  // row i of a half: the key whose number has bits 2 and 3 of i exchanged
  u32x4 v[2][DP][VP];     // row 32 e + i: column (DP / 32) i + e
};

template <int DP, bool TOK, int NW>
__global__ __launch_bounds__(64 * NW, DP == 256 ? 1 : 2) void k_kv_attn_many(KvAttnArgs a) {
  constexpr int NT = 64 * NW, NS = ManyLds<DP, TOK>::NS;
  // a thread's part of a step: KI pieces of 16 codes of a key, KT keys apart; VI blocks of four columns of VT
  // values, VS keys apart.  A wave's keys lie within 16, so that its page is one scalar.
  constexpr int KT = NT / (DP / 16), KI = kStep > KT ? kStep / KT : 1;
  constexpr int VT = DP / 4 * (kStep / 8) < NT ? 4 : 8, VS = VT * (NT / (DP / 4)), VI = kStep > VS ? kStep / VS : 1;
  static_assert(KT % 16 == 0 && (VI == 1 || VS % 16 == 0) && 64 / (DP / 16) <= 16 && VT * (DP / 4 < 64 ? 64 / (DP / 4) : 1) <= 16, "a wave's keys");
  extern __shared__ __attribute__((aligned(16))) uint8_t many_lds[];
  ManyLds<DP, TOK>& lds = *reinterpret_cast<ManyLds<DP, TOK>*>(many_lds);
  Tile tl;
  if (!tile_of(a, 32 * NW, true, tl)) return;
  const KvCache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, c32 = lane & 31, hh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d = c.d;

  const int w0 = tl.r0 + 32 * wave, rr = w0 + c32;
  const bool valid = rr < tl.rows;
  const uint32_t qi = uint32_t(rr) / uint32_t(a.group), head = tl.head * a.group + uint32_t(rr) % uint32_t(a.group);
  const int64_t token = tl.row0 + qi;
  const int limit = row_limit(a, tl, rr);
  const int wave_first = row_limit(a, tl, w0), wave_last = row_limit(a, tl, min(w0 + 31, max(tl.rows - 1, w0)));
  const int k0 = tl.split * a.chunk, k1 = kv_split_end(tl.split, a.nsplit, a.chunk, row_limit(a, tl, min(tl.r0 + 32 * NW, tl.rows) - 1) + 1);
  if (k0 >= k1 && tl.split > 0) return;

  u32x4 qf[DP / 16];
#pragma unroll
  for (int kk = 0; kk < DP / 16; ++kk) {
    const int col = 16 * kk + 8 * hh;
    qf[kk] = valid && col < d ? *reinterpret_cast<const u32x4*>(a.q + token * a.q_stride + int64_t(head) * d + col) : u32x4{0u, 0u, 0u, 0u};
  }
  f32x16 o[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) o[t] = f32x16{};
  float m = kNone, l = 0.f;

  // Loads have no branch around them, so that the waits for them can be counted: threads beyond a step's keys read
  // what others read too, and columns past d are those of column 0 (their queries are 0, their results not stored).
  const int kcol = 16 * (tid % (DP / 16)), krow = tid / (DP / 16) % kStep;
  const int vcol = 4 * (tid % (DP / 4)), vrow = VT * (tid / (DP / 4)) % kStep;
  const bool kin = KT <= kStep || tid < kStep * (DP / 16), vin = VS <= kStep || tid < kStep / VT * (DP / 4);  // uniform over a wave
  uint32_t koff = (krow & 15) * d + (kcol < d ? kcol : 0), voff = (vrow & 15) * d + (vcol < d ? vcol : 0);
  const int kgrp = __builtin_amdgcn_readfirstlane(krow & ~15), vgrp = __builtin_amdgcn_readfirstlane(vrow & ~15);
  const int side = tid / NS & 1, sn = (tid % NS) * (TOK ? 1 : 16);
  u32x4 kr[KI];
  uint32_t vr[VI][VT];
  float srow = 0.f;
  bool sheld = false;
  // Addresses are a scalar of the wave and 32 bits of the lane.  Table entries of the next loads, as they are: nothing
  // may wait for them where they are read (the codes' loads are ahead of them), so they are loaded as vectors though
  // every lane of a wave reads the same one of kpage[i] and of vpage[i].
  int kpage[KI], vpage[VI], spage = 0;
  uint32_t zero = 0;
  const auto lane_part = [](uint32_t& x) {  // kept apart from the scalar, for which a loop would otherwise widen it
    asm volatile("" : "+v"(x));
    return x;
  };
  const int32_t* table = a.b.table + int64_t(tl.seq) * a.b.width;
  const int lp = c.lpage, in_page = (1 << lp) - 1, ls = lp - c.lscale;
  auto entry = [&](int pos) { return *reinterpret_cast<const int32_t*>(reinterpret_cast<const char*>(table + min(pos >> lp, a.b.width - 1)) + lane_part(zero)); };
  auto pages = [&](int kb) {
#pragma unroll
    for (int i = 0; i < KI; ++i) kpage[i] = entry(kb + kgrp + KT * i);
#pragma unroll
    for (int i = 0; i < VI; ++i) vpage[i] = entry(kb + vgrp + VS * i);
    spage = table[uint32_t(min((kb + sn) >> lp, a.b.width - 1))];
  };
  const uint32_t npages = uint32_t(min(c.pages, int64_t(INT32_MAX)));
  auto inside = [&](int page) { return uint32_t(page) < npages; };
  const uint64_t page_codes = uint64_t(c.heads) * uint64_t(d) << lp;
  const int8_t* codes_k = c.code[0] + (int64_t(tl.head) << lp) * d;
  const int8_t* codes_v = c.code[1] + (int64_t(tl.head) << lp) * d;
  const float* scales = (side ? c.scale[1] : c.scale[0]) + (int64_t(tl.head) << ls);
  const uint32_t page_scales = uint32_t(c.heads) << ls;
  auto load = [&](int kb) {
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const int page = __builtin_amdgcn_readfirstlane(kpage[i]);
      const int8_t* p = codes_k + uint32_t(inside(page) ? page : 0) * page_codes + uint32_t(((kb + kgrp + KT * i) & in_page) * d);
      kr[i] = *reinterpret_cast<const u32x4*>(p + lane_part(koff));
    }
#pragma unroll
    for (int i = 0; i < VI; ++i) {
      const int page = __builtin_amdgcn_readfirstlane(vpage[i]);
      const int8_t* p = codes_v + uint32_t(inside(page) ? page : 0) * page_codes + uint32_t(((kb + vgrp + VS * i) & in_page) * d);
#pragma unroll
      for (int j = 0; j < VT; ++j) vr[i][j] = *reinterpret_cast<const uint32_t*>(p + j * d + lane_part(voff));
    }
    sheld = inside(spage) & (kb + sn <= tl.last);  // (the last position lies within the table)
    const uint32_t in_scales = (kb + sn) >> c.lscale & ((1 << ls) - 1);
    srow = scales[uint64_t(uint32_t(inside(spage) ? spage : 0)) * page_scales + in_scales];
  };
  auto stage = [&](int buf) {
    if (kin)
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int row = krow + KT * i, r = (row & ~12) | (row & 4) << 1 | (row & 8) >> 1;
#pragma unroll
        for (int u = 0; u < 2; ++u) lds.k[buf][r][kcol / 8 + u] = codes_bf16(kr[i][2 * u], kr[i][2 * u + 1]);
      }
    if (vin)
#pragma unroll
      for (int i = 0; i < VI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t x[VT / 2];
#pragma unroll
          for (int j = 0; j < VT / 2; ++j) x[j] = pack_code_f16x2(sbyte(vr[i][2 * j], e), sbyte(vr[i][2 * j + 1], e));
          const int col = vcol + e, row = vrow + VS * i;
          u32x4* dst = &lds.v[buf][32 * (col % (DP / 32)) + col / (DP / 32)][row / 8];
          if constexpr (VT == 8) *dst = u32x4{x[0], x[1], x[2], x[3]};
          else reinterpret_cast<u32x2*>(dst)[(row >> 2) & 1] = u32x2{x[0], x[1]};
        }
    // keys that no row sees (in no page, or past the sequence's end): weight 0 whatever the memory holds
    const float b = sane(srow);
    if (tid < NS) {
      lds.fig[buf][0][tid] = sheld ? srow * a.qk : 0.f;
    } else if (tid < 2 * NS) {
      lds.fig[buf][1][tid - NS] = sheld ? __builtin_amdgcn_logf(b) : kNone;
      lds.fig[buf][2][tid - NS] = sheld ? __builtin_amdgcn_rcpf(fmaxf(b, kKvMinScale)) : 0.f;
    }
  };

  const int steps = (k1 - k0 + kStep - 1) / kStep;                        // of the block
  const int mine = min(steps, (wave_last + 1 - k0 + kStep - 1) / kStep);  // of the wave (perhaps <= 0)
  f32x16 s[2];  // scores of a step's halves
  auto scores = [&](int buf) {
    s[0] = s[1] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < DP / 16; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t) s[t] = mfma32(lds.k[buf][32 * t + c32][2 * kk + hh], qf[kk], s[t]);
    // six reads ahead of the products (a prompt of 8192 tokens 671 -> 657 us)
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int i = 0; i < DP / 8 - 6; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);
  };
  // element 8 u + j of s[t]: key 32 t + 16 u + 8 hh + j of the step
  auto figures = [&](const float* from, int t, int u, float* x) {
    if constexpr (TOK) {
#pragma unroll
      for (int q = 0; q < 2; ++q) *reinterpret_cast<f32x4*>(x + 4 * q) = *reinterpret_cast<const f32x4*>(from + 32 * t + 16 * u + 8 * hh + 4 * q);
    } else {
      x[0] = from[2 * t + u];
    }
  };
  // weights of the step at kb, and their product with its values
  auto weigh = [&](int kb, int buf) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float f[TOK ? 8 : 1], b[TOK ? 8 : 1];
        figures(lds.fig[buf][0], t, u, f);
        figures(lds.fig[buf][1], t, u, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[t][8 * u + j] = __builtin_fmaf(s[t][8 * u + j], f[TOK ? j : 0], b[TOK ? j : 0]);
      }
    if (kb + kStep - 1 > wave_first) {  // some row sees less than all of the step's keys
      const int seen = limit - kb - 8 * hh;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 16; ++j) s[t][j] = 32 * t + 16 * (j >> 3) + (j & 7) <= seen ? s[t][j] : kNone;
    }
    float mx = kNone;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, s[t][j]);
    // The maximum follows only from twice the weight on (weights stay within 2^15; the difference is exact where it is
    // near that, a sum would be rounded): few steps pay for it, or for the exchange between the two lanes of a row.
    if (__any(mx - m > kBias + 1.f)) {
      const float m1 = fmaxf(m, below(fmaxf(mx, __shfl_xor(mx, 32)))), alpha = exp2_(m - (m1 == kNone ? 0.f : m1));
      m = m1;
      l *= alpha;
#pragma unroll
      for (int e = 0; e < DP / 32; ++e) o[e] *= alpha;
    }
    const float mf = m == kNone ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float r[TOK ? 8 : 1], w[8];
        figures(lds.fig[buf][2], t, u, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          w[j] = exp2_(s[t][8 * u + j] - mf);
          sum = __builtin_fmaf(w[j], r[TOK ? j : 0], sum);
        }
        u32x4 p;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = pack_f16x2(w[2 * i], w[2 * i + 1]);
#pragma unroll
        for (int e = 0; e < DP / 32; ++e) o[e] = mfma32_f16(lds.v[buf][32 * e + c32][4 * t + 2 * u + hh], p, o[e]);
      }
    l = __builtin_fmaf(sum, kDen, l);
  };

  if (steps > 0) {
    pages(k0);
    load(k0);
    pages(k0 + kStep);
    stage(0);
  }
  __syncthreads();
  for (int n = 0; n < steps; ++n) {
    const int kb = k0 + kStep * n;
    load(kb + kStep);  // (past the last step: keys that are not used)
    pages(kb + 2 * kStep);
    if (n < mine) {
      scores(n & 1);
      weigh(kb, n & 1);
    }
    stage((n + 1) & 1);
    __syncthreads();
  }
  l += __shfl_xor(l, 32);
  if (!valid) return;
  // element 4 v + i of o[e]: column (DP / 32) (8 v + 4 hh + i) + e
  constexpr int CE = DP / 32;
  const float r = reciprocal(l);
  const int64_t at = (int64_t(tl.split) * a.b.tokens + token) * a.hq + head;
  uint16_t* out = a.o + token * a.o_stride + int64_t(head) * d;
#pragma unroll
  for (int i = 0; i < 16 * CE; i += 4) {  // the lane's columns in fours: element x of the four
    const auto value = [&](int x) { return o[(i + x) % CE][(i + x) / CE]; };
    const int col = CE * (8 * (i / CE / 4) + 4 * hh) + i % (4 * CE);
    if (col >= d) continue;
    const f32x4 x = {value(0), value(1), value(2), value(3)};
    if (tl.split_up) *reinterpret_cast<f32x4*>(a.part_o + at * d + col) = x;
    else
      *reinterpret_cast<u32x2*>(out + col) =
          u32x2{pack_bf16x2(result(x[0] * r), result(x[1] * r)), pack_bf16x2(result(x[2] * r), result(x[3] * r))};
  }
  if (tl.split_up && hh == 0) {
    a.part_ml[2 * at] = m;
    a.part_ml[2 * at + 1] = l;
  }
}

// The splits of a row joined.  G threads' groups share the row's splits, every G-th one each, and their sums meet in
// a fixed tree; each group has four columns a thread.  G = 32 with blocks of 32 columns of one row where rows are few
// (a decoding step: the row's splits all at once); G = 1 with as many whole rows as fit a block otherwise.  Bound by
// its launch and one trip to memory: 32 heads of one token, 64 splits, 4 us; G = 1, 1000 rows of 32 heads of 64 in
// three splits, 6 us.
template <int G>
__global__ __launch_bounds__(256) void k_kv_attn_join(KvAttnArgs a, uint32_t tasks) {
  __shared__ float red[4];
  __shared__ f32x4 red_o[4][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = a.c.d;
  // task: a row's place in its sequence, its head and (G > 1) its part of the columns
  uint32_t w;
  int col, first;
  if constexpr (G > 1) {
    const uint32_t parts = uint32_t(d + 31) / 32;
    w = blockIdx.x / parts;
    col = int(blockIdx.x % parts) * 32 + 4 * (threadIdx.x & 7);
    first = threadIdx.x >> 3;
  } else {
    const uint32_t lanes = uint32_t(d) / 4, per = 256 / lanes;
    w = blockIdx.x * per + threadIdx.x / lanes;
    if (threadIdx.x / lanes >= per || w >= tasks) return;
    col = int(threadIdx.x % lanes) * 4;
    first = 0;
  }
  const int head = int(w % uint32_t(a.hq));
  w /= uint32_t(a.hq);
  const int qi = int(w % uint32_t(a.b.max_new)), seq = int(w / uint32_t(a.b.max_new));
  const KvSeq q = kv_seq(a.b, seq);
  if (qi >= q.end - q.c0) return;
  const int64_t last = min(q.end, int64_t(a.b.width) << a.c.lpage) - 1;
  if (!kv_split_up(last, a.chunk, a.nsplit)) return;  // written already
  const int64_t token = q.row0 + qi;
  const int64_t limit = a.causal ? min(q.c0 + qi, last) : last;
  const int ns = kv_splits(limit, a.chunk, a.nsplit);
  const int64_t step = a.b.tokens * a.hq, at0 = token * a.hq + head;
  const bool in = col < d;
  // the common maximum (every wave or thread for itself); then the splits' outputs in that scale
  float mt = kNone;
  for (int s = G > 1 ? lane : 0; s < ns; s += G > 1 ? 64 : 1) mt = fmaxf(mt, a.part_ml[2 * (s * step + at0)]);
  if constexpr (G > 1)
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) mt = fmaxf(mt, __shfl_xor(mt, off));
  const float mtf = mt == kNone ? 0.f : mt;
  float l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = first; s < ns; s += G) {
    const float f = exp2_(a.part_ml[2 * (s * step + at0)] - mtf);
    l += f * a.part_ml[2 * (s * step + at0) + 1];
    if (in) acc += f * *reinterpret_cast<const f32x4*>(a.part_o + (s * step + at0) * d + col);
  }
  if constexpr (G > 1) {
#pragma unroll
    for (int off = 8; off < 64; off <<= 1) {
      l += __shfl_xor(l, off);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], off);
    }
    if (lane < 8) red_o[wave][lane] = acc;
    if (lane == 0) red[wave] = l;
    __syncthreads();
    if (threadIdx.x >= 8 || !in) return;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      l += red[i];
      acc += red_o[i][lane];
    }
  }
  const float r = reciprocal(l);
  *reinterpret_cast<u32x2*>(a.o + token * a.o_stride + int64_t(head) * d + col) =
      u32x2{pack_bf16x2(result(acc[0] * r), result(acc[1] * r)), pack_bf16x2(result(acc[2] * r), result(acc[3] * r))};
}

template <int DH, int NW>
void launch_rows(const KvAttnArgs& a, unsigned blocks, hipStream_t st) {
  if (a.c.lscale == 0) k_kv_attn_rows<DH, true, NW><<<blocks, 64 * NW, 0, st>>>(a);
  else k_kv_attn_rows<DH, false, NW><<<blocks, 64 * NW, 0, st>>>(a);
}

template <int DP, int NW>
void launch_many(const KvAttnArgs& a, unsigned blocks, hipStream_t st) {
  if (a.c.lscale == 0) k_kv_attn_many<DP, true, NW><<<blocks, 64 * NW, sizeof(ManyLds<DP, true>), st>>>(a);
  else k_kv_attn_many<DP, false, NW><<<blocks, 64 * NW, sizeof(ManyLds<DP, false>), st>>>(a);
}

bool wide_join(int64_t tasks, int nsplit) { return nsplit > 4 && tasks < 2048; }
int64_t join_blocks(int64_t tasks, int d, int nsplit) {
  return wide_join(tasks, nsplit) ? tasks * ((d + 31) / 32) : (tasks + 256 / (d / 4) - 1) / (256 / (d / 4));
}

}  // namespace

bool kv_attention_fits(const KvCache& c, const KvBatch& b, int hq, const KvAttnPlan& p) {
  const int64_t tasks = int64_t(b.seqs) * b.max_new * hq;  // (rows of tiles and of the join are counted in 32 bits)
  return tasks < INT32_MAX / 8 && p.blocks <= kMaxThreads / (64 * p.waves) &&
         (p.nsplit == 1 || join_blocks(tasks, c.d, p.nsplit) <= kMaxThreads / 256);
}

hipError_t launch_kv_attention(const KvAttnArgs& a, const KvAttnPlan& p, hipStream_t st) {
  const unsigned blocks = unsigned(p.blocks);
  const int d = a.c.d;
  if (p.rows == kRowTile) {
    if (p.waves == 8) d <= 64 ? launch_rows<1, 8>(a, blocks, st) : launch_rows<2, 8>(a, blocks, st);
    else d <= 64 ? launch_rows<1, 4>(a, blocks, st) : d <= 128 ? launch_rows<2, 4>(a, blocks, st) : launch_rows<4, 4>(a, blocks, st);
  } else if (p.rows == 128) {
    d <= 64 ? launch_many<64, 4>(a, blocks, st) : d <= 128 ? launch_many<128, 4>(a, blocks, st) : launch_many<256, 4>(a, blocks, st);
  } else {
    d <= 64 ? launch_many<64, 8>(a, blocks, st) : launch_many<128, 8>(a, blocks, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const int64_t tasks = int64_t(a.b.seqs) * a.b.max_new * a.hq;
  const unsigned joins = unsigned(join_blocks(tasks, d, p.nsplit));
  if (wide_join(tasks, p.nsplit)) k_kv_attn_join<32><<<joins, 256, 0, st>>>(a, uint32_t(tasks));
  else k_kv_attn_join<1><<<joins, 256, 0, st>>>(a, uint32_t(tasks));
  return hipGetLastError();
}

}  // namespace lrqat
