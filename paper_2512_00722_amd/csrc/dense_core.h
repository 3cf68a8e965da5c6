// Device code shared by the kernels over caches that are read in full: one pass of
// decode attention over contiguous tokens, and the joining of partial results.
#pragma once

#include <float.h>

#include <type_traits>

#include "device_common.h"
#include "internal.h"

namespace spec {

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The running maximum before the first logit: finite, so that logits of -inf
// weigh nothing from the first tile on.
constexpr float kNoMax = -FLT_MAX;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Transposing LDS read: within each 16-lane group, lane i receives element
// (i & 3) of the 8-byte pieces read by lanes (i >> 2) + 4j, j = 0..3.
__device__ __forceinline__ bf16x4 lds_read_tr(const uint16_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
      (__attribute__((address_space(3))) bf16x4*)(p));
}

__device__ __forceinline__ bf16x8 to_bf16x8(const float* p) {  // round to nearest even
  bf16x8 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bf16x2 h = __builtin_convertvector(floatx2{p[2 * j], p[2 * j + 1]}, bf16x2);
    r[2 * j] = h[0];
    r[2 * j + 1] = h[1];
  }
  return r;
}
// Takes what to_bf16x8 gave off eight values (exactly) and rounds the rest.
__device__ __forceinline__ bf16x8 next_bf16x8(float* p, bf16x8 high) {
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] -= (float)high[e];
  return to_bf16x8(p);
}

// LDS tiles of whole 256-byte rows: the 16-byte pieces of a row stand at piece ^
// swizzle(row), so that the 16 rows which a quarter of a K read touches lie in
// different banks, and so do the four rows of a transposing V read.
__device__ __forceinline__ int swizzle(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

// Between a wavefront's own LDS writes and reads.
__device__ __forceinline__ void wave_sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// max / sum over the four lanes {l, l^16, l^32, l^48} (one head's lanes).
__device__ __forceinline__ float quad_max(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Decode attention of up to 16 query heads of one KV head over a contiguous cache,
// by some wavefronts: chunk c of 32 tokens belongs to wavefront c mod n_parts,
// whatever the length, so that it divides evenly and nothing but the length has to
// arrive before the first rows are requested.
constexpr int kDecodeChunk = 32;

struct DecodeUnit {
  const uint16_t* q;    // the unit's first query head; heads are d apart
  const uint16_t* k;    // the sequence's rows of the KV head
  const uint16_t* v;
  int64_t rs;           // elements between tokens
  int heads;            // query heads, at most 16
  int count;            // visible tokens: 0 .. n_sink - 1, the others `shift` further on
  int n_sink, shift;
  int part, n_parts;    // this wavefront among those of the unit
  float scale_log2;
};

// bf16 elements of a wavefront's V tile: a whole chunk, or (HALF) its 16-token halves
// in turn.
constexpr int kTileElems = kDecodeChunk * kHeadDim;
constexpr int tile_elems(bool half) { return half ? kTileElems / 2 : kTileElems; }

// A wavefront's share token by token, without the matrix cores, for the rare sums that
// hold an infinity or a NaN: an infinity times a weight's parts is not that times the
// weight, and a token whose logit is -inf counts for nothing, whatever its row of V holds
// (in a part of nothing but such tokens as well, which joins leave out).  As decode_unit
// leaves them, l_run not yet added up over a head's lanes.
__device__ __forceinline__ void unit_by_token(const DecodeUnit& u, float& m_run, float& l_run,
                                              floatx4 (&acc)[8]) {
  const int lane = threadIdx.x & 63, r16 = lane & 15, kg = lane >> 4;
  const uint16_t* q = u.q + (r16 < u.heads ? r16 : 0) * kHeadDim + 4 * kg;
  auto four = [](const uint16_t* p) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    return floatx4{bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y)};
  };
  m_run = kNoMax;
  l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 8; ++db) acc[db] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int c = kDecodeChunk * u.part; c < u.count; c += kDecodeChunk * u.n_parts) {
#pragma unroll 1
    for (int j = c; j < min(c + kDecodeChunk, u.count); ++j) {
      const int64_t off = (int64_t)(j + (j < u.n_sink ? 0 : u.shift)) * u.rs + 4 * kg;
      float s = 0.f;
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const floatx4 x = four(q + 16 * db), y = four(u.k + off + 16 * db);
#pragma unroll
        for (int i = 0; i < 4; ++i) s = fmaf(x[i], y[i], s);
      }
      s = quad_sum(s) * u.scale_log2;
      const float mn = fmaxf(m_run, s);
      const float alpha = exp2_fast(m_run - mn), p = exp2_fast(s - mn);
      m_run = mn;
      l_run = l_run * alpha + (kg == 0 ? p : 0.f);
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const floatx4 y = four(u.v + off + 16 * db);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[db][i] = fmaf(acc[db][i], alpha, s == -INFINITY ? 0.f : p * y[i]);
      }
    }
  }
}

// A wavefront's share: maximum and sum of head r16 (l_run complete) and O^T[16 db + 4 kg
// + i][head r16]; keep(head, token, logits of four tokens) is called for every four
// logits (log2 units) of its chunks.  V: its V tile.
template <bool HALF, class Keep>
__device__ __forceinline__ void decode_unit(const DecodeUnit& u, uint16_t* V, float& m_run,
                                            float& l_run, floatx4 (&acc)[8], Keep&& keep) {
  const int lane = threadIdx.x & 63;
  const int r16 = lane & 15;  // head of this lane; token of a K tile row
  const int kg = lane >> 4;
  bf16x8 qf[4];  // Q^T: column r16, dimensions 32 s + 8 kg ..
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const uint4 w = r16 < u.heads ? ldg16(u.q + r16 * kHeadDim + 8 * kg + 32 * s)
                                  : make_uint4(0, 0, 0, 0);
    qf[s] = __builtin_bit_cast(bf16x8, w);
  }
  const int step = kDecodeChunk * u.n_parts;  // tokens between a wavefront's chunks
  const int first = kDecodeChunk * u.part;
  // Rows behind the last token read the last: they are never used with a weight.
  auto row = [&](const uint16_t* base, int j) {
    j = min(j, u.count - 1);
    return base + (int64_t)(j + (j < u.n_sink ? 0 : u.shift)) * u.rs;
  };
  uint4 kr[2][4], vr[8];
  auto load_k = [&](int c) {  // MFMA A operand: token 16 t + r16, dimensions 32 s + 8 kg ..
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint16_t* p = row(u.k, c + 16 * t + r16) + 8 * kg;
#pragma unroll
      for (int s = 0; s < 4; ++s) kr[t][s] = ldg16_stream(p + 32 * s);
    }
  };
  constexpr int VH = HALF ? 4 : 8;  // loads of a V tile
  auto load_v = [&](int c, int r0) {  // whole rows: token 4 r + kg, dimensions 8 r16 ..
#pragma unroll
    for (int r = r0; r < r0 + VH; ++r)
      vr[r] = ldg16_stream(row(u.v, c + 4 * r + kg) + 8 * r16);
  };
  auto put_v = [&](int r0) {
#pragma unroll
    for (int r = 0; r < VH; ++r) {
      const int t = 4 * r + kg;
      *reinterpret_cast<uint4*>(V + t * kHeadDim + ((r16 ^ swizzle(t)) << 3)) = vr[r0 + r];
    }
  };
  // transposed V: tokens 16 h + 4 kg .. + 3, dimensions 16 db + r16
  auto get_v = [&](int h, int db) {
    const int t = 16 * h + 4 * kg + (r16 >> 2);
    const int piece = 2 * db + ((r16 >> 1) & 1);
    return lds_read_tr(V + t * kHeadDim + ((piece ^ swizzle(t)) << 3) + 4 * (r16 & 1));
  };

  m_run = kNoMax;
  l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 8; ++db) acc[db] = floatx4{0.f, 0.f, 0.f, 0.f};
  if (first < u.count) {
    load_v(first, 0);
    __builtin_amdgcn_sched_barrier(0);
    load_k(first);
    __builtin_amdgcn_sched_barrier(0);
    if (HALF) load_v(first, 4);
    __builtin_amdgcn_sched_barrier(0);
  }
  // Each register buffer is refilled as soon as it is consumed; loads retire in
  // issue order, so that every wait is a partial one.
  for (int c = first; c < u.count; c += step) {
    put_v(0);
    load_v(c + step, 0);
    __builtin_amdgcn_sched_barrier(0);
    floatx4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[t][i]), qf[i],
                                                       s[t], 0, 0, 0);
    }
    load_k(c + step);
    __builtin_amdgcn_sched_barrier(0);

    // S[head r16][token 16 t + 4 kg + i]
    float p[8];
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = s[t][i] * u.scale_log2;
        p[4 * t + i] = c + 16 * t + 4 * kg + i < u.count ? x : -INFINITY;
        mx = fmaxf(mx, p[4 * t + i]);
      }
      keep(r16, c + 16 * t + 4 * kg, p + 4 * t);
    }
    mx = quad_max(mx);
    const float mn = fmaxf(m_run, mx);
    const float alpha = exp2_fast(m_run - mn);
    m_run = mn;
    l_run *= alpha;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = exp2_fast(p[i] - mn);
      l_run += p[i];
    }
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] *= alpha;
    // Weights enter as three bf16 numbers, 2^-26 relative at most: a pair's 2^-17 would be
    // most of the result's error over some thousand tokens, and the third is free in a kernel
    // bound by memory (321 us with either; 32 layers x 8 sequences x 2048 tokens).
    const bf16x8 ph = to_bf16x8(p), pl = next_bf16x8(p, ph), pt = next_bf16x8(p, pl);
    wave_sync_lds();
    if constexpr (HALF) {
      typedef short shortx4 __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h == 1) {
          wave_sync_lds();
          put_v(4);
          load_v(c + step, 4);
          __builtin_amdgcn_sched_barrier(0);
          wave_sync_lds();
        }
        const bf16x4 hi = h ? __builtin_shufflevector(ph, ph, 4, 5, 6, 7)
                            : __builtin_shufflevector(ph, ph, 0, 1, 2, 3);
        const bf16x4 lo = h ? __builtin_shufflevector(pl, pl, 4, 5, 6, 7)
                            : __builtin_shufflevector(pl, pl, 0, 1, 2, 3);
        const bf16x4 th = h ? __builtin_shufflevector(pt, pt, 4, 5, 6, 7)
                            : __builtin_shufflevector(pt, pt, 0, 1, 2, 3);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
          const shortx4 vf = __builtin_bit_cast(shortx4, get_v(0, db));
          acc[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
              vf, __builtin_bit_cast(shortx4, hi), acc[db], 0, 0, 0);
          acc[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
              vf, __builtin_bit_cast(shortx4, lo), acc[db], 0, 0, 0);
          acc[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
              vf, __builtin_bit_cast(shortx4, th), acc[db], 0, 0, 0);
        }
      }
    } else {
      // slots 8 kg .. + 7 of a multiplication: tokens 4 kg .. + 3 and 16 + 4 kg .. + 3
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const bf16x8 vf =
            __builtin_shufflevector(get_v(0, db), get_v(1, db), 0, 1, 2, 3, 4, 5, 6, 7);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, ph, acc[db], 0, 0, 0);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl, acc[db], 0, 0, 0);
        acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pt, acc[db], 0, 0, 0);
      }
    }
    wave_sync_lds();  // the tile is rewritten by the next chunk
  }
  float odd = 0.f;
#pragma unroll
  for (int db = 0; db < 8; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) odd = fmaf(acc[db][i], 0.f, odd);
  if (__any(odd != odd)) unit_by_token(u, m_run, l_run, acc);
  l_run = quad_sum(l_run);
}

// Where several wavefronts share a unit, a wavefront's accumulators stand in its V tile
// (which it no longer needs): 16 heads of 128 floats.  Four floats of head h, dimensions
// 4 d4 ..: pieces are swizzled so that the 16 heads of a store lie in different banks.
static_assert(kTileElems * 2 == 16 * kHeadDim * 4, "results fill the V tile");
__device__ __forceinline__ int result_at(int h, int d4) {
  return h * kHeadDim + ((d4 ^ ((h & 7) << 2)) << 2);
}
__device__ __forceinline__ void leave_results(uint16_t* V, float2* ml, float m_run, float l_run,
                                              const floatx4 (&acc)[8]) {
  const int r16 = threadIdx.x & 15, kg = (threadIdx.x >> 4) & 3;
  float* res = reinterpret_cast<float*>(V);
#pragma unroll
  for (int db = 0; db < 8; ++db)
    *reinterpret_cast<float4*>(res + result_at(r16, 4 * db + kg)) =
        make_float4(acc[db][0], acc[db][1], acc[db][2], acc[db][3]);
  if (kg == 0) ml[r16] = make_float2(m_run, l_run);
}

// The joined partial results of one output row, as one thread sees it: its four
// dimensions, weights 2^(m - M).
struct Join {
  float M = kNoMax, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void rescale(float m) {
    const float f = exp2f(M - m);
    M = m;
    L *= f;
    o.x *= f;
    o.y *= f;
    o.z *= f;
    o.w *= f;
  }
  __device__ __forceinline__ void add(const float2 ml, const float4 x) {  // ml.x <= M
    const float f = exp2f(ml.x - M);
    L += ml.y * f;
    o.x += x.x * f;
    o.y += x.y * f;
    o.z += x.z * f;
    o.w += x.w * f;
  }
  __device__ __forceinline__ float inv() const { return L == 0.f ? 0.f : 1.f / L; }
  __device__ __forceinline__ float lse() const { return (M + log2f(L)) * kLn2; }
};

// The results of wavefronts w0, w0 + HB, .. < W, head h, dimensions 4 d4 .. (after
// decode_unit).
template <int W, int HB>
__device__ __forceinline__ Join join_waves(const uint16_t (*tiles)[kTileElems],
                                           const float2 (*ml)[16], int w0, int h, int d4) {
  Join j;
#pragma unroll
  for (int w = w0; w < W; w += HB) j.M = fmaxf(j.M, ml[w][h].x);
#pragma unroll
  for (int w = w0; w < W; w += HB)
    j.add(ml[w][h], *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(tiles[w]) +
                                                     result_at(h, d4)));
  return j;
}

// A decode launch: units (layer, sequence, KV head, column group of at most 16 query
// heads), each split over n_split workgroups.
struct DecodeArgs {
  const uint16_t* q;       // [n_layers][B][H_q][d]
  const uint16_t* k;       // caches
  const uint16_t* v;
  const int32_t* lens;     // [B] cached tokens
  float* out;              // [n_layers*B][H_q][d]; null: partial results are left
  float* lse;              // [n_layers*B][H_q] or null
  float* part_acc;         // [n_layers*B][n_split][H_q][d]
  float* part_ml;          // [n_layers*B][n_split][H_q][2]
  float* logits;           // [n_layers*B][H_q][logit_stride], log2 units, or null
  float* weights;          // added to, [units][L_cap]; or, overwritten, [units][logit_stride]
  int64_t stride_layer, stride_b, logit_stride;
  int B, H_q, H_kv, heads, R, L_cap, k_max, n_sink, n_split;  // heads: of a column group
  int add_weights;
  float scale_log2;
};

// What becomes of the logits.
enum Keep { kKeepNone = 0, kKeepLogits = 1, kKeepWeights = 2 };

// LDS pitch of a head's logits: heads in different banks.
__host__ __device__ inline int logit_pitch(int k_max) { return (k_max + 31) / 32 * 32 + 16; }

// One workgroup of such a launch: HB consecutive column groups, W / HB wavefronts each
// (the KV heads' pieces of a token's row are then read at the same time).
// KEEP = kKeepWeights (n_split = 1): the logits stay in LDS until their sums are known,
// and the heads' weights are added up there; memory sees one value per token
// instead of one per token and head, which matters as any steady writing takes a
// kernel that streams from 6.5 to 5 TB/s.
template <int W, int HB, int KEEP, bool HALF = false>
__device__ __forceinline__ void decode_block(const DecodeArgs& a, int block,
                                             uint16_t (*tiles)[tile_elems(HALF)],
                                             float2 (*ml)[16], float* lds_logits) {
  static_assert(!HALF || W == HB, "half tiles do not hold a wavefront's results");
  const int groups = a.H_kv * a.R / HB;
  const int wave = threadIdx.x >> 6;
  const int split = block % a.n_split, rest = block / a.n_split;
  const int gv0 = rest % groups * HB, gv = gv0 + wave % HB;
  const int lb = rest / groups, b = lb % a.B;
  const int len = clampi(a.lens[b], 0, a.L_cap);
  const size_t row0 = (size_t)lb * a.H_q + (size_t)gv0 * a.heads;  // first query head
  const size_t part0 = ((size_t)lb * a.n_split + split) * a.H_q + (size_t)gv0 * a.heads;
  const int64_t base = (int64_t)(lb / a.B) * a.stride_layer + (int64_t)b * a.stride_b +
                       (int64_t)(gv / a.R) * kHeadDim;
  DecodeUnit u;
  u.q = a.q + (row0 + wave % HB * a.heads) * kHeadDim;
  u.k = a.k + base;
  u.v = a.v + base;
  u.rs = (int64_t)a.H_kv * kHeadDim;
  u.heads = a.heads;
  u.count = min(len, a.k_max);
  u.n_sink = min(a.n_sink, u.count);
  u.shift = len - u.count;
  u.part = split * (W / HB) + wave / HB;
  u.n_parts = a.n_split * (W / HB);
  u.scale_log2 = a.scale_log2;
  const int pitch = logit_pitch(a.k_max), own = wave % HB * a.heads;
  float m_run, l_run;
  floatx4 acc[8];
  decode_unit<HALF>(u, tiles[wave], m_run, l_run, acc, [&](int h, int tok, const float* x) {
    if (KEEP == kKeepNone || h >= a.heads) return;
    float* p = KEEP == kKeepWeights ? lds_logits + (own + h) * pitch + tok
                                    : a.logits + (row0 + own + h) * a.logit_stride + tok;
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  });

  // a head all of whose logits are -inf has no weights: 2^(-inf - inf) = 0
  __shared__ float lse2[KEEP == kKeepWeights ? 16 * HB : 1];
  if constexpr (W == HB) {  // a wavefront's results are the unit's
    const int r16 = threadIdx.x & 15, kg = (threadIdx.x >> 4) & 3;
    if (r16 < a.heads) {
      const int h = own + r16;
      const float f = !a.out ? 1.f : l_run == 0.f ? 0.f : 1.f / l_run;
      float* dst = (a.out ? a.out + (row0 + h) * kHeadDim : a.part_acc + (part0 + h) * kHeadDim) +
                   4 * kg;
#pragma unroll
      for (int db = 0; db < 8; ++db)
        *reinterpret_cast<float4*>(dst + 16 * db) =
            make_float4(acc[db][0] * f, acc[db][1] * f, acc[db][2] * f, acc[db][3] * f);
      if (kg == 0) {
        if (!a.out) reinterpret_cast<float2*>(a.part_ml)[part0 + h] = make_float2(m_run, l_run);
        else if (a.lse) a.lse[row0 + h] = (m_run + log2f(l_run)) * kLn2;
        if (KEEP == kKeepWeights) lse2[h] = l_run == 0.f ? INFINITY : m_run + log2f(l_run);
      }
    }
  } else {
    leave_results(tiles[wave], ml[wave], m_run, l_run, acc);
    __syncthreads();
    for (int e = threadIdx.x; e < HB * a.heads * 32; e += W * 64) {
      const int h = e >> 5, d4 = e & 31;  // query head among the workgroup's
      const int w0 = HB == 1 ? 0 : h / a.heads;
      const Join j = join_waves<W, HB>(tiles, ml, w0, h - w0 * a.heads, d4);
      if (a.out) {
        const float inv = j.inv();
        reinterpret_cast<float4*>(a.out + (row0 + h) * kHeadDim)[d4] =
            make_float4(j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv);
        if (a.lse && d4 == 0) a.lse[row0 + h] = j.lse();
      } else {
        reinterpret_cast<float4*>(a.part_acc + (part0 + h) * kHeadDim)[d4] = j.o;
        if (d4 == 0) reinterpret_cast<float2*>(a.part_ml)[part0 + h] = make_float2(j.M, j.L);
      }
      if (KEEP == kKeepWeights && d4 == 0) lse2[h] = j.L == 0.f ? INFINITY : j.M + log2f(j.L);
    }
  }
  if constexpr (KEEP == kKeepWeights) {
    __syncthreads();
    const int64_t pitch_w = a.add_weights ? a.L_cap : a.logit_stride;
    float* w = a.weights + ((int64_t)lb * a.H_kv * a.R + gv0) * pitch_w;
    for (int hb = 0; hb < HB; ++hb, w += pitch_w) {
      for (int t = threadIdx.x; t < u.count; t += W * 64) {
        float sum = 0.f;
        for (int h = hb * a.heads; h < (hb + 1) * a.heads; ++h)
          sum += exp2_fast(lds_logits[h * pitch + t] - lse2[h]);
        w[t] = a.add_weights ? w[t] + sum : sum;
      }
    }
  }
}

// Joins parts 0 .. n-1 of a row (at(s): pointers to a part's (max, sum) and
// accumulators) by S groups of 32 threads, of which group 0 has the result.
// Eight parts of a group are requested together: one round trip for up to 8 S
// parts.  Parts whose sum is 0 are left out: their accumulators may never have
// been written.  All threads of the workgroup call.
template <int S, class At>
__device__ __forceinline__ Join join_parts(int n, At&& at) {
  constexpr int kBatch = 8;
  __shared__ float2 ml_lds[8];
  __shared__ float4 acc_lds[8][32];
  const int slot = threadIdx.x >> 5, d4 = threadIdx.x & 31, part = slot % S;
  Join j;
  for (int s0 = part; s0 < n; s0 += kBatch * S) {
    float2 ml[kBatch];
    float4 x[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {  // clamped: every load is issued
      const float* acc;
      const float2* pair;
      at(min(s0 + u * S, n - 1), pair, acc);
      ml[u] = *pair;
      x[u] = reinterpret_cast<const float4*>(acc)[d4];
    }
    float m = j.M;
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (s0 + u * S < n && ml[u].y != 0.f) m = fmaxf(m, ml[u].x);
    j.rescale(m);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (s0 + u * S < n && ml[u].y != 0.f) j.add(ml[u], x[u]);
  }
  if constexpr (S > 1) {
    if (d4 == 0) ml_lds[slot] = make_float2(j.M, j.L);
    acc_lds[slot][d4] = j.o;
    __syncthreads();
    if (part == 0) {
      float m = j.M;
      for (int p = 1; p < S; ++p) m = fmaxf(m, ml_lds[slot + p].x);
      j.rescale(m);
      for (int p = 1; p < S; ++p) j.add(ml_lds[slot + p], acc_lds[slot + p][d4]);
    }
  }
  return j;
}

// Groups of 32 threads that join a row of n partial results: one per eight, whose
// loads are a single round trip.  Calls launch(integral constant).
template <class F>
void with_parts(int n, F&& launch) {
  if (n <= 8) launch(std::integral_constant<int, 1>{});
  else if (n <= 16) launch(std::integral_constant<int, 2>{});
  else if (n <= 32) launch(std::integral_constant<int, 4>{});
  else launch(std::integral_constant<int, 8>{});
}
inline dim3 merge_grid(int64_t rows, int s) { return dim3((unsigned)((rows * s + 7) / 8)); }

}  // namespace spec
