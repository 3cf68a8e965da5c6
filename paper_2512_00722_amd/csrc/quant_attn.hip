// Decode attention over caches held in 4 or 8 bits: all rows or a sliding window with
// sinks, and selected rows.
//
// One pass with a running maximum and sum (log2 units), as over bf16 caches
// (dense_core.h), but for the operands:
//  * S^T = K Q^T: the matrix cores' sum over the dimensions may take them in any order,
//    so that a lane has the 32 of one group of one token, in one or two 16-byte loads
//    that stay whole, and one scale; Q is read in the same order;
//  * O^T += V^T P^T: the same lanes' parts of V go to LDS as bf16 rows and are read back
//    transposed.
// A part becomes bf16 by half an instruction per element; every value is exact, so that
// the result is that of the bf16 attention over what spec_quant_read gives, to the
// rounding of the sums.
#include "dense_core.h"
#include "quant_core.h"

namespace spec {
namespace {

constexpr int kW = 8;  // wavefronts of a workgroup

struct QuantArgs {
  const uint16_t* q;       // [n_layers][B][H_q][d]
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* scales;
  const int32_t* lens;     // [B] tokens, or selected ones
  const int32_t* idx;      // [B][n_sets][k_max]
  float* out;              // [n_layers*B][H_q][d]; null: partial results are left
  float* lse;              // [n_layers*B][H_q] or null
  float* part_acc;         // [n_layers*B][n_split][H_q][d]
  float* part_ml;          // [n_layers*B][n_split][H_q][2]
  int64_t kv_stride_layer, kv_stride_b, scale_stride_layer, scale_stride_b;
  int B, H_q, H_kv, heads, R, L_cap, k_max, n_sets, n_sink, n_split;  // heads: of a column group
  float scale_log2;
};

struct QuantUnit {
  const uint16_t* q;       // the unit's first query head; heads are d apart
  const uint8_t* k;        // the sequence's rows of the KV head
  const uint8_t* v;
  const uint8_t* scales;
  const int32_t* idx;      // INDEXED: the rows' tokens, within 0 .. last
  int64_t rs;              // bytes between tokens; of scales: ss
  int ss;
  int last;
  int heads, count;        // query heads, at most 16; visible tokens
  int n_sink, shift;       // else: 0 .. n_sink - 1, the others `shift` further on
  int part, n_parts;       // this wavefront among those of the unit
  float scale_log2;
};

template <bool INDEXED>
__device__ __forceinline__ int token_of(const QuantUnit& u, int j) {
  if (INDEXED) return clampi(u.idx[j], 0, u.last);
  return j + (j < u.n_sink ? 0 : u.shift);
}

// A wavefront's share token by token, without the matrix cores, for the rare sums that
// hold an infinity or a NaN, as unit_by_token() has it for bf16 caches.
template <int BITS, bool INDEXED>
__device__ __forceinline__ void quant_unit_by_token(const QuantUnit& u, float& m_run,
                                                    float& l_run, floatx4 (&acc)[8]) {
  const int lane = threadIdx.x & 63, r16 = lane & 15, kg = lane >> 4;
  const uint16_t* q = u.q + (r16 < u.heads ? r16 : 0) * kHeadDim + 4 * kg;
  m_run = kNoMax;
  l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 8; ++db) acc[db] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int c = kDecodeChunk * u.part; c < u.count; c += kDecodeChunk * u.n_parts) {
#pragma unroll 1
    for (int j = c; j < min(c + kDecodeChunk, u.count); ++j) {
      const int64_t t = token_of<INDEXED>(u, j);
      const uint2 sc = *reinterpret_cast<const uint2*>(u.scales + t * u.ss);
      float s = 0.f;
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const uint2 x = *reinterpret_cast<const uint2*>(q + 16 * db);
        const floatx4 y = elements4<BITS>(u.k + t * u.rs, 16 * db + 4 * kg,
                                          scale_of(sc.x, db / 2));
        s = fmaf(bf16lo(x.x), y[0], s);
        s = fmaf(bf16hi(x.x), y[1], s);
        s = fmaf(bf16lo(x.y), y[2], s);
        s = fmaf(bf16hi(x.y), y[3], s);
      }
      s = quad_sum(s) * u.scale_log2;
      const float mn = fmaxf(m_run, s);
      const float alpha = exp2_fast(m_run - mn), p = exp2_fast(s - mn);
      m_run = mn;
      l_run = l_run * alpha + (kg == 0 ? p : 0.f);
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const floatx4 y = elements4<BITS>(u.v + t * u.rs, 16 * db + 4 * kg,
                                          scale_of(sc.y, db / 2));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[db][i] = fmaf(acc[db][i], alpha, s == -INFINITY ? 0.f : p * y[i]);
      }
    }
  }
}

template <int BITS>
__device__ __forceinline__ RowPart<BITS> load_part(const uint8_t* p) {
  RowPart<BITS> r;
#pragma unroll
  for (int i = 0; i < BITS / 4; ++i)
    r.w[i] = ldg16_stream(reinterpret_cast<const uint16_t*>(p) + 8 * i);
  return r;
}

// A wavefront's share: chunks of 32 tokens, of which lane (r16, kg) has dimensions 32 kg ..
// of tokens r16 and 16 + r16.  Results as decode_unit's.  V: its V tile.
template <int BITS, bool INDEXED>
__device__ __forceinline__ void quant_unit(const QuantUnit& u, uint16_t* V, float& m_run,
                                           float& l_run, floatx4 (&acc)[8]) {
  const int lane = threadIdx.x & 63;
  const int r16 = lane & 15;  // head of this lane; token of a K tile row
  const int kg = lane >> 4;
  bf16x8 qf[4];  // Q^T: column r16, dimensions 32 kg + 8 s ..
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const uint4 w = r16 < u.heads ? ldg16(u.q + r16 * kHeadDim + kGroup * kg + 8 * s)
                                  : make_uint4(0, 0, 0, 0);
    qf[s] = __builtin_bit_cast(bf16x8, w);
  }
  const int step = kDecodeChunk * u.n_parts;  // tokens between a wavefront's chunks
  const int first = kDecodeChunk * u.part;
  RowPart<BITS> kr[2], vr[2];
  uint2 sc[2];
  int64_t tok[2];
  // Rows behind the last token read the last: they are never used with a weight.
  auto next_tokens = [&](int c) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      tok[t] = token_of<INDEXED>(u, min(c + 16 * t + r16, u.count - 1));
  };
  auto load_v = [&]() {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t] = *reinterpret_cast<const uint2*>(u.scales + tok[t] * u.ss);
      vr[t] = load_part<BITS>(u.v + tok[t] * u.rs + part_bytes(BITS) * kg);
    }
  };
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      kr[t] = load_part<BITS>(u.k + tok[t] * u.rs + part_bytes(BITS) * kg);
  };
  auto put_v = [&]() {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = 16 * t + r16;
      const float scale = scale_of(sc[t].y, kg);
#pragma unroll
      for (int s = 0; s < 4; ++s)
        *reinterpret_cast<bf16x8*>(V + row * kHeadDim + (((4 * kg + s) ^ swizzle(row)) << 3)) =
            elements8<BITS>(vr[t], s, scale);
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
    next_tokens(first);
    load_v();
    load_k();
    next_tokens(first + step);
    __builtin_amdgcn_sched_barrier(0);
  }
  // Each register buffer is refilled as soon as it is consumed.
  for (int c = first; c < u.count; c += step) {
    const float ks[2] = {scale_of(sc[0].x, kg), scale_of(sc[1].x, kg)};
    put_v();
    load_v();
    __builtin_amdgcn_sched_barrier(0);
    floatx4 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(elements8<BITS>(kr[t], i, ks[t]), qf[i],
                                                       s[t], 0, 0, 0);
    }
    load_k();
    next_tokens(c + 2 * step);
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
    // Weights enter as three bf16 numbers, 2^-26 relative at most, as over bf16 caches.
    const bf16x8 ph = to_bf16x8(p), pl = next_bf16x8(p, ph), pt = next_bf16x8(p, pl);
    wave_sync_lds();
    // slots 8 kg .. + 7 of a multiplication: tokens 4 kg .. + 3 and 16 + 4 kg .. + 3
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const bf16x8 vf =
          __builtin_shufflevector(get_v(0, db), get_v(1, db), 0, 1, 2, 3, 4, 5, 6, 7);
      acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, ph, acc[db], 0, 0, 0);
      acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl, acc[db], 0, 0, 0);
      acc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pt, acc[db], 0, 0, 0);
    }
    wave_sync_lds();  // the tile is rewritten by the next chunk
  }
  float odd = 0.f;
#pragma unroll
  for (int db = 0; db < 8; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) odd = fmaf(acc[db][i], 0.f, odd);
  if (__any(odd != odd)) quant_unit_by_token<BITS, INDEXED>(u, m_run, l_run, acc);
  l_run = quad_sum(l_run);
}

// HB consecutive column groups (KV heads of the same tokens, whose pieces of a row are
// then read at the same time), kW / HB wavefronts each.
template <int BITS, bool INDEXED, int HB>
__global__ __launch_bounds__(kW * 64) __attribute__((amdgpu_waves_per_eu(4)))
void quant_decode_kernel(QuantArgs a) {
  __shared__ __align__(16) uint16_t tiles[kW][kTileElems];
  __shared__ float2 ml[kW][16];
  const int groups = a.H_kv * a.R / HB;
  const int wave = threadIdx.x >> 6;
  const int split = blockIdx.x % a.n_split, rest = blockIdx.x / a.n_split;
  const int gv0 = rest % groups * HB, gv = gv0 + wave % HB, g = gv / a.R;
  const int lb = rest / groups, layer = lb / a.B, b = lb % a.B;
  const size_t row0 = (size_t)lb * a.H_q + (size_t)gv0 * a.heads;  // first query head
  const size_t part0 = ((size_t)lb * a.n_split + split) * a.H_q + (size_t)gv0 * a.heads;
  const int64_t base = layer * a.kv_stride_layer + b * a.kv_stride_b + g * row_bytes(BITS);
  const int len = clampi(a.lens[b], 0, INDEXED ? a.k_max : a.L_cap);
  QuantUnit u;
  u.q = a.q + (row0 + wave % HB * a.heads) * kHeadDim;
  u.k = a.k + base;
  u.v = a.v + base;
  u.scales = a.scales + layer * a.scale_stride_layer + b * a.scale_stride_b + g * kScaleBytes;
  u.idx = INDEXED ? a.idx + ((int64_t)b * a.n_sets + (a.n_sets == 1 ? 0 : g)) * a.k_max : nullptr;
  u.rs = (int64_t)a.H_kv * row_bytes(BITS);
  u.ss = a.H_kv * kScaleBytes;
  u.last = a.L_cap - 1;
  u.heads = a.heads;
  u.count = min(len, a.k_max);
  u.n_sink = min(a.n_sink, u.count);
  u.shift = len - u.count;
  u.part = split * (kW / HB) + wave / HB;
  u.n_parts = a.n_split * (kW / HB);
  u.scale_log2 = a.scale_log2;
  float m_run, l_run;
  floatx4 acc[8];
  quant_unit<BITS, INDEXED>(u, tiles[wave], m_run, l_run, acc);

  leave_results(tiles[wave], ml[wave], m_run, l_run, acc);
  __syncthreads();
  for (int e = threadIdx.x; e < HB * a.heads * 32; e += kW * 64) {
    const int h = e >> 5, d4 = e & 31;  // query head among the workgroup's
    const int w0 = HB == 1 ? 0 : h / a.heads;
    const Join j = join_waves<kW, HB>(tiles, ml, w0, h - w0 * a.heads, d4);
    if (a.out) {
      const float inv = j.inv();
      reinterpret_cast<float4*>(a.out + (row0 + h) * kHeadDim)[d4] =
          make_float4(j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv);
      if (a.lse && d4 == 0) a.lse[row0 + h] = j.lse();
    } else {
      reinterpret_cast<float4*>(a.part_acc + (part0 + h) * kHeadDim)[d4] = j.o;
      if (d4 == 0) reinterpret_cast<float2*>(a.part_ml)[part0 + h] = make_float2(j.M, j.L);
    }
  }
}

template <int S>
__global__ __launch_bounds__(256) void quant_merge_kernel(DecodeArgs a, float* out, float* lse,
                                                          int64_t n_out) {
  decode_merge<S>(a, blockIdx.x, out, lse, n_out);
}

// How a launch is divided: hb column groups per workgroup, each over n_split of them.
struct QuantPlan {
  int hb, n_split;
};

QuantPlan quant_plan(const QuantDims& d, int k_max) {
  const int64_t groups = (int64_t)d.H_kv * (d.G / group_heads(d.G));
  int hb = kW;
  while (groups % hb) hb /= 2;
  const int64_t wgs = (int64_t)d.n_layers * d.B * groups / hb;
  const int64_t chunks = (k_max + kDecodeChunk - 1) / kDecodeChunk;
  const int64_t most = (chunks + kW / hb - 1) / (kW / hb);
  int64_t n = 2 * kCUs / wgs;
  if (n > most) n = most;
  return {hb, n < 1 ? 1 : (int)n};
}
int decode_tokens(const QuantDims& d) {
  const int64_t n = (int64_t)d.window + d.n_sink;
  return (int)(n < d.L_cap ? n : d.L_cap);
}
size_t quant_part_acc_bytes(const QuantDims& d, int n_split) {
  return n_split > 1 ? align_up(sizeof(float) * kHeadDim * (size_t)d.n_layers * d.B * n_split *
                                d.H_q)
                     : 0;
}
size_t quant_part_bytes(const QuantDims& d, int n_split) {
  return quant_part_acc_bytes(d, n_split) +
         (n_split > 1 ? align_up(sizeof(float) * 2 * (size_t)d.n_layers * d.B * n_split * d.H_q)
                      : 0);
}

template <int BITS, bool INDEXED>
void launch_kernel(const QuantArgs& a, int hb, unsigned blocks, hipStream_t s) {
  if (hb == 8) quant_decode_kernel<BITS, INDEXED, 8><<<blocks, kW * 64, 0, s>>>(a);
  else if (hb == 4) quant_decode_kernel<BITS, INDEXED, 4><<<blocks, kW * 64, 0, s>>>(a);
  else if (hb == 2) quant_decode_kernel<BITS, INDEXED, 2><<<blocks, kW * 64, 0, s>>>(a);
  else quant_decode_kernel<BITS, INDEXED, 1><<<blocks, kW * 64, 0, s>>>(a);
}

hipError_t launch_quant(const QuantDims& d, int k_max, int n_sink, const uint16_t* q,
                        const QuantCache& c, const int32_t* idx, const int32_t* lens, float* out,
                        float* lse, void* ws, hipStream_t s) {
  const QuantPlan p = quant_plan(d, k_max);
  const int heads = group_heads(d.G);
  QuantArgs a{};
  a.q = q;
  a.k = c.k;
  a.v = c.v;
  a.scales = c.scales;
  a.lens = lens;
  a.idx = idx;
  a.out = out;
  a.lse = lse;
  a.kv_stride_layer = d.kv_stride_layer;
  a.kv_stride_b = d.kv_stride_b;
  a.scale_stride_layer = d.scale_stride_layer;
  a.scale_stride_b = d.scale_stride_b;
  a.B = d.B;
  a.H_q = d.H_q;
  a.H_kv = d.H_kv;
  a.heads = heads;
  a.R = d.G / heads;
  a.L_cap = d.L_cap;
  a.k_max = k_max;
  a.n_sets = d.n_sets;
  a.n_sink = n_sink;
  a.n_split = p.n_split;
  a.scale_log2 = d.scale * kLog2e;
  if (p.n_split > 1) {
    a.out = nullptr;
    a.part_acc = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) +
                                         quant_part_acc_bytes(d, p.n_split));
  }
  const int64_t blocks = (int64_t)d.n_layers * d.B * d.H_kv * a.R / p.hb * p.n_split;
  if (blocks > INT32_MAX / (kW * 64)) return hipErrorInvalidValue;
  if (d.bits == 4) {
    if (idx) launch_kernel<4, true>(a, p.hb, (unsigned)blocks, s);
    else launch_kernel<4, false>(a, p.hb, (unsigned)blocks, s);
  } else {
    if (idx) launch_kernel<8, true>(a, p.hb, (unsigned)blocks, s);
    else launch_kernel<8, false>(a, p.hb, (unsigned)blocks, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  DecodeArgs m{};
  m.part_acc = a.part_acc;
  m.part_ml = a.part_ml;
  m.n_split = p.n_split;
  m.H_q = d.H_q;
  const int64_t n_out = (int64_t)d.n_layers * d.B * d.H_q;
  with_parts(p.n_split, [&](auto S) {
    quant_merge_kernel<S.value><<<merge_grid(n_out, S.value), 256, 0, s>>>(m, out, lse, n_out);
  });
  return hipGetLastError();
}

}  // namespace

size_t quant_decode_ws_bytes(const QuantDims& d) {
  return quant_part_bytes(d, quant_plan(d, decode_tokens(d)).n_split);
}
size_t quant_sparse_ws_bytes(const QuantDims& d) {
  return quant_part_bytes(d, quant_plan(d, d.k_max).n_split);
}

hipError_t launch_quant_decode(const QuantDims& d, const uint16_t* q, const QuantCache& c,
                               const int32_t* lens, float* out, float* lse, void* ws,
                               hipStream_t s) {
  return launch_quant(d, decode_tokens(d), d.n_sink, q, c, nullptr, lens, out, lse, ws, s);
}
hipError_t launch_quant_sparse_decode(const QuantDims& d, const uint16_t* q, const QuantCache& c,
                                      const int32_t* idx, const int32_t* counts, float* out,
                                      float* lse, void* ws, hipStream_t s) {
  return launch_quant(d, d.k_max, d.k_max, q, c, idx, counts, out, lse, ws, s);
}

}  // namespace spec
