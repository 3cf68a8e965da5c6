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
#include "quant_plan.h"

namespace spec {
namespace {

struct QuantArgs {
  const uint16_t* q;       // [n_layers][B][H_q][d]
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* scales;
  const int32_t* lens;     // [B] tokens, or selected ones
  const int32_t* idx;      // [B][n_sets][k_max]
  float* out;              // [n_layers*B][H_q][d]; null: partial results are left
  float* lse;              // [n_layers*B][H_q] or null
  float* part_acc;         // [n_layers][B n_split][H_q][d]: a layer's parts, by sequence
  float* part_ml;          // [n_layers][B n_split][H_q][2]
  int64_t kv_stride_layer, kv_stride_b, scale_stride_layer, scale_stride_b;
  int B, H_q, H_kv, heads, R, L_cap, k_max, n_sets, n_sink;  // heads: of a column group
  int ub_log2, n_split;    // see QuantPlan
  int32_t* parts;          // [B + 1], or null: where each sequence's parts begin (see Parts)
  float scale_log2;
};

struct QuantUnit {
  const uint16_t* q;       // the unit's first query head; heads are d apart, those of the
  int q_stride;            // next KV head q_stride
  const uint8_t* k;        // the sequence's rows of the first KV head
  const uint8_t* v;
  const uint8_t* scales;
  const int32_t* idx;      // INDEXED: the rows' tokens, clamped into 0 .. last; those of the
  int64_t idx_stride;      // next KV head idx_stride on
  int64_t rs;              // bytes between tokens; of scales: ss
  int ss;
  int last, k_max;         // INDEXED: k_max: indices of a set
  int heads, count;        // query heads of a KV head, at most 16; visible tokens
  int n_sink, shift;       // else: tokens 0 .. n_sink - 1, the others `shift` further on
  int part, n_parts;       // this wavefront among those of the unit
  float scale_log2;

  // Chunks of up to 32 tokens that stand together: of the sinks, then of the others.
  __device__ __forceinline__ int chunks() const {
    return (n_sink + kDecodeChunk - 1) / kDecodeChunk +
           (count - n_sink + kDecodeChunk - 1) / kDecodeChunk;
  }
  __device__ __forceinline__ int valid(int c) const {
    const int sinks = (n_sink + kDecodeChunk - 1) / kDecodeChunk;
    return min(kDecodeChunk, c < sinks ? n_sink - kDecodeChunk * c
                                       : count - n_sink - kDecodeChunk * (c - sinks));
  }
  __device__ __forceinline__ void chunk(int c, int& start, int& n) const {
    const int sinks = (n_sink + kDecodeChunk - 1) / kDecodeChunk;
    start = c < sinks ? kDecodeChunk * c : n_sink + shift + kDecodeChunk * (c - sinks);
    n = valid(c);
  }
};

template <bool INDEXED>
__device__ __forceinline__ int64_t token_of(const QuantUnit& u, int h, int j) {
  if (INDEXED) return clampi(u.idx[h * u.idx_stride + j], 0, u.last);
  return j + (j < u.n_sink ? 0 : u.shift);
}

// A wavefront's share token by token, without the matrix cores, for the rare sums that
// hold an infinity or a NaN, as unit_by_token() has it for bf16 caches, and for logits beyond
// kFusedMost: there the logits are rounded before the maximum is taken off, so that the
// greatest token weighs 1.  Below, weights are those of quant_unit(): equal logits weigh the
// same in every wavefront, whichever way it went.
template <int BITS, bool INDEXED>
__device__ __forceinline__ void quant_unit_by_token(const QuantUnit& u, int h, float& m_run,
                                                    float& l_run, floatx4 (&acc)[8]) {
#pragma clang fp contract(off)  // a logit's product and difference stay two roundings
  const int lane = threadIdx.x & 63, r16 = lane & 15, kg = lane >> 4;
  const uint16_t* q = u.q + h * u.q_stride + (r16 < u.heads ? r16 : 0) * kHeadDim + 4 * kg;
  const uint8_t* k = u.k + h * row_bytes(BITS);
  const uint8_t* v = u.v + h * row_bytes(BITS);
  m_run = kNoMax;
  l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 8; ++db) acc[db] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int sinks = (u.n_sink + kDecodeChunk - 1) / kDecodeChunk;
#pragma unroll 1
  for (int c = u.part; c < u.chunks(); c += u.n_parts) {
    const int j0 = c < sinks ? kDecodeChunk * c : u.n_sink + kDecodeChunk * (c - sinks);
#pragma unroll 1
    for (int j = j0; j < j0 + u.valid(c); ++j) {
      const int64_t t = token_of<INDEXED>(u, h, j);
      const uint2 sc = *reinterpret_cast<const uint2*>(u.scales + t * u.ss + h * kScaleBytes);
      float s = 0.f;
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const uint2 x = *reinterpret_cast<const uint2*>(q + 16 * db);
        const floatx4 y = elements4<BITS>(k + t * u.rs, 16 * db + 4 * kg, scale_of(sc.x, db / 2));
        s = fmaf(bf16lo(x.x), y[0], s);
        s = fmaf(bf16hi(x.x), y[1], s);
        s = fmaf(bf16lo(x.y), y[2], s);
        s = fmaf(bf16hi(x.y), y[3], s);
      }
      const float sum = quad_sum(s);
      s = sum * u.scale_log2;
      const float mn = fmaxf(m_run, s);
      const float alpha = exp2_fast(m_run - mn);
      const float p =
          exp2_fast(fabsf(mn) < kFusedMost ? fmaf(sum, u.scale_log2, -mn) : s - mn);
      m_run = mn;
      l_run = l_run * alpha + (kg == 0 ? p : 0.f);
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const floatx4 y = elements4<BITS>(v + t * u.rs, 16 * db + 4 * kg, scale_of(sc.y, db / 2));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[db][i] = fmaf(acc[db][i], alpha, s == -INFINITY ? 0.f : p * y[i]);
      }
    }
  }
  l_run = quad_sum(l_run);
}

// The matrix cores' 16 columns are 16 / GW copies of the GW query heads of a KV head.
// S^T is worked out in the first (the others' queries are zeros, which cost less power: 1372
// us for 1385 at the sizes below); of a lane's eight tokens copy L takes numbers
// 8 GW / 16 L .., so that the softmax of a token is worked out once.  In the second
// product a copy's column then has the tokens of its own as its lanes made them, and in
// the places of the others', which it would leave empty, their weights' lower parts: the
// copies' sums together are that of all tokens by weights of three bf16 numbers
// (2^-26 relative at most), for GW = 4 in one multiplication instead of three, for GW = 8
// in two (32 layers x 8 sequences x 32768 tokens, 4 heads of each of 8 KV heads, 4 bits: 1391
// us, with three multiplications of everything 1583).
template <int GW>
struct Columns {
  static constexpr int COPIES = 16 / GW, OWN = 8 / COPIES;  // tokens of a copy
  static constexpr int MULS = GW == 4 ? 1 : GW == 8 ? 2 : 3;

  // v of the copies in MASK (bits: lanes 4 b .. 4 b + 3 of 16), rotated by ROT lanes; else old
  template <int ROT, int MASK>
  static __device__ __forceinline__ uint32_t put(uint32_t old, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)v, ROT == 0 ? 0xE4 : 0x120 + ROT,
                                                 0xf, MASK, false);
  }
  template <int ROT, int MASK>
  static __device__ __forceinline__ float choose(float old, float v) {
    return __uint_as_float(put<ROT, MASK>(__float_as_uint(old), __float_as_uint(v)));
  }
  // The first copy's v.
  static __device__ __forceinline__ float first(float v) {
    if constexpr (GW == 4) v = choose<12, 8>(choose<8, 4>(choose<4, 2>(v, v), v), v);
    else if constexpr (GW == 8) v = choose<8, 12>(v, v);
    return v;
  }
  // A lane's own values of the first copy's eight.
  static __device__ __forceinline__ void own(const float (&p)[8], float (&q)[OWN]) {
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
      q[i] = p[i];
      if constexpr (GW == 4) {
        q[i] = choose<4, 2>(q[i], p[2 + i]);
        q[i] = choose<8, 4>(q[i], p[4 + i]);
        q[i] = choose<12, 8>(q[i], p[6 + i]);
      } else if constexpr (GW == 8) {
        q[i] = choose<8, 12>(q[i], p[4 + i]);
      }
    }
  }
  // The operands of the second product, of a lane's own weights (which are used up).
  static __device__ __forceinline__ void weights(float (&q)[OWN], bf16x8 (&w)[MULS]) {
    uint32_t part[3][OWN / 2];
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int j = 0; j < OWN / 2; ++j) {
        const bf16x2 x = __builtin_convertvector(floatx2{q[2 * j], q[2 * j + 1]}, bf16x2);
        part[k][j] = __builtin_bit_cast(uint32_t, x);
        q[2 * j] -= (float)x[0];
        q[2 * j + 1] -= (float)x[1];
      }
    uint32_t r[MULS][4];
    if constexpr (GW == 4) {
      r[0][0] = put<8, 4>(put<4, 2>(put<0, 1>(0, part[0][0]), part[1][0]), part[2][0]);
      r[0][1] = put<8, 8>(put<4, 4>(put<0, 2>(0, part[0][0]), part[1][0]), part[2][0]);
      r[0][2] = put<8, 1>(put<4, 8>(put<0, 4>(0, part[0][0]), part[1][0]), part[2][0]);
      r[0][3] = put<8, 2>(put<4, 1>(put<0, 8>(0, part[0][0]), part[1][0]), part[2][0]);
    } else if constexpr (GW == 8) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        r[0][j] = put<8, 12>(part[0][j], part[1][j]);
        r[0][2 + j] = put<8, 3>(part[0][j], part[1][j]);
        r[1][j] = put<0, 3>(0, part[2][j]);
        r[1][2 + j] = put<0, 12>(0, part[2][j]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) r[k][j] = part[k][j];
    }
#pragma unroll
    for (int k = 0; k < MULS; ++k)
      w[k] = __builtin_bit_cast(bf16x8, make_uint4(r[k][0], r[k][1], r[k][2], r[k][3]));
  }
  // The sum of the copies.
  static __device__ __forceinline__ float sum(float v) {
    if constexpr (GW == 4) v += dpp_f<0x124>(v);
    if constexpr (GW <= 8) v += dpp_f<0x128>(v);
    return v;
  }
};

// Where a 16-byte piece of a row of V in bf16 stands among the row's 16.  A transposing
// read takes pieces 2 db and 2 db + 1 of eight rows 4 a .. 4 a + 3, 4 a + 4 .. at a time, over
// all banks; a write takes 8 pieces 4 kg + s, kg = 0 .. 3, of a row of two heads (8 bits: of
// one head 2 p + s, p = 0 .. 7), over half of them, so that those have to differ modulo 8.
__device__ __forceinline__ int v_place(int h, int row, int piece) {
  return piece ^ ((row & 3) << 2 | (row >> 2 & 1) << 1 | (row >> 3 & 1)) ^ (piece >> 3) ^ 2 * h;
}

// LDS of a wavefront: V in bf16, [NH][32 tokens][256 bytes], and before it the chunk's K as
// it is held; scales [32 tokens][NH][8].
template <int NH>
struct WaveTile {
  uint16_t v[NH][kTileElems];
  uint8_t scales[kDecodeChunk * NH * kScaleBytes];
};

// A wavefront's share of NH neighbouring KV heads: chunks of 32 tokens.  Lines of 128 bytes
// are what a card moves fastest (K and V of 8 heads x 32768 tokens x 256 in 4 bits, loads
// alone: 7.3 TB/s by lines in the order of the lanes, 5.7 by 64-byte rows of a head, the
// matrix cores' order): two heads in 4 bits, one in 8.  A lane loads 16-byte pieces, K goes
// through LDS as it is held, V as bf16 (from where it is read transposed); both by the
// wavefront itself, so that none waits for another.  Lane (r16, kg) then has dimensions
// 32 kg .. of K of tokens r16 and 16 + r16.  Results as decode_unit's, for each head; returns
// the heads (bits) whose sums hold an infinity or a NaN or whose logits go beyond kFusedMost,
// which quant_unit_by_token() has yet to work out.
template <int BITS, int NH, int GW, bool INDEXED>
__device__ __forceinline__ uint32_t quant_unit(const QuantUnit& u, WaveTile<NH>& T,
                                               float (&m_run)[NH], float (&l_run)[NH],
                                               floatx4 (&acc)[NH][8]) {
  using C = Columns<GW>;
  constexpr int P = NH * BITS;         // pieces of a token's row
  constexpr int RI = 64 / P;           // rows of a load
  constexpr int NI = kDecodeChunk / RI;
  constexpr int SP = 16 * 8 / BITS / 8;  // bf16 pieces of 8 elements of a piece
  const int lane = threadIdx.x & 63;
  const int r16 = lane & 15;  // column of this lane; token of a K tile row
  const int kg = lane >> 4;
  const int lrow = lane / P, lpiece = lane % P;   // of a load
  const int lhead = lpiece / BITS, lpart = lpiece % BITS;
  bf16x8 qf[NH][4];  // Q^T: column r16, dimensions 32 kg + 8 s ..
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint4 w = r16 < u.heads ? ldg16(u.q + h * u.q_stride + r16 * kHeadDim + kGroup * kg +
                                            8 * s)
                                    : make_uint4(0, 0, 0, 0);
      qf[h][s] = __builtin_bit_cast(bf16x8, w);
    }
  uint4 kr[NI], vr[NI];
  uint2 sc;
  int tok[NI], tok_s;
  const uint8_t *kb, *vb, *sb;
  int64_t off[NI];
  // Where chunk c stands: the rows behind its last are read as that one.
  auto locate = [&](int c) {
    if (!INDEXED) {
      int start, valid;
      u.chunk(c, start, valid);
      kb = u.k + (int64_t)start * u.rs;
      vb = u.v + (int64_t)start * u.rs;
      sb = u.scales + (int64_t)start * u.ss;
#pragma unroll
      for (int i = 0; i < NI; ++i) tok[i] = min(RI * i + lrow, valid - 1);
      tok_s = min(lane / NH % kDecodeChunk, valid - 1);
    } else {
      kb = u.k;
      vb = u.v;
      sb = u.scales;
    }
  };
  auto indices = [&](int c) {  // INDEXED: of chunk c
#pragma unroll
    for (int i = 0; i < NI; ++i)
      tok[i] = u.idx[lhead * u.idx_stride + min(kDecodeChunk * c + RI * i + lrow, u.count - 1)];
    tok_s = u.idx[lane % NH * u.idx_stride +
                  min(kDecodeChunk * c + lane / NH % kDecodeChunk, u.count - 1)];
  };
  // K and scales of the chunk that has been located; before them, as loads arrive in order,
  // the indices of chunk `then`.
  auto load_k = [&](int then) {
    if (INDEXED) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
        off[i] = (int64_t)clampi(tok[i], 0, u.last) * u.rs + 16 * lpiece;
      const uint8_t* s = sb + (int64_t)clampi(tok_s, 0, u.last) * u.ss + lane % NH * kScaleBytes;
      indices(then);
      __builtin_amdgcn_sched_barrier(0);
      sc = *reinterpret_cast<const uint2*>(s);
    } else {
#pragma unroll
      for (int i = 0; i < NI; ++i) off[i] = (uint32_t)(tok[i] * (int)u.rs + 16 * lpiece);
      sc = *reinterpret_cast<const uint2*>(sb + (uint32_t)(tok_s * u.ss + lane % NH * kScaleBytes));
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
      kr[i] = ldg16_stream(reinterpret_cast<const uint16_t*>(kb + off[i]));
  };
  auto load_v = [&]() {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      vr[i] = ldg16_stream(reinterpret_cast<const uint16_t*>(vb + off[i]));
  };
  // K's pieces, the 16 rows of a read in different banks
  uint8_t* const K = reinterpret_cast<uint8_t*>(T.v);
  auto k_at = [&](int row, int piece) {
    return K + row * 16 * P + 16 * (piece ^ (P == 8 ? row >> 1 & 7 : row >> 2 & 3));
  };
  auto v_at = [&](int h, int row, int piece) {
    return T.v[h] + row * kHeadDim + (v_place(h, row, piece) << 3);
  };
  // transposed V: tokens 16 t + 4 kg .. + 3, dimensions 16 db + r16
  auto get_v = [&](int h, int t, int db) {
    return lds_read_tr(v_at(h, 16 * t + 4 * kg + (r16 >> 2), 2 * db + ((r16 >> 1) & 1)) +
                       4 * (r16 & 1));
  };

#pragma unroll
  for (int h = 0; h < NH; ++h) {
    m_run[h] = kNoMax;
    l_run[h] = 0.f;
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[h][db] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  int first[NI], first_s;
  if (INDEXED) {
    // The first chunk's indices do not wait for the number of rows: those behind the last
    // row, whatever they are, give way to that of the chunk's first row.
    const int j0 = min(kDecodeChunk * u.part, u.k_max - 1);
#pragma unroll
    for (int i = 0; i < NI; ++i)
      first[i] = u.idx[lhead * u.idx_stride + min(j0 + RI * i + lrow, u.k_max - 1)];
    first_s = u.idx[lane % NH * u.idx_stride +
                    min(j0 + lane / NH % kDecodeChunk, u.k_max - 1)];
#pragma unroll
    for (int i = 0; i < NI; ++i) asm volatile("" : "+v"(first[i]));
    asm volatile("" : "+v"(first_s));
  }
  const int chunks = u.chunks();
  if (u.part < chunks) {
    if (INDEXED) {
      const int row0 = __builtin_amdgcn_readfirstlane(first[0]);
      const int row1 = NH == 1 ? row0 : __builtin_amdgcn_readlane(first[0], BITS);
#pragma unroll
      for (int i = 0; i < NI; ++i)
        tok[i] = kDecodeChunk * u.part + RI * i + lrow < u.count ? first[i]
                 : lhead == 0 ? row0 : row1;
      tok_s = kDecodeChunk * u.part + lane / NH % kDecodeChunk < u.count ? first_s
              : lane % NH == 0 ? row0 : row1;
    }
    locate(u.part);
    load_k(min(u.part + u.n_parts, chunks - 1));
    load_v();
    __builtin_amdgcn_sched_barrier(0);
  }
  for (int c = u.part; c < chunks; c += u.n_parts) {
    // Behind a wavefront's last chunk the sequence's last is requested, which nobody uses: the
    // loads stay without a branch, and a wavefront waits for them at its end.
    const int next = min(c + u.n_parts, chunks - 1);
    *reinterpret_cast<uint2*>(T.scales + lane % (kDecodeChunk * NH) * kScaleBytes) = sc;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      *reinterpret_cast<uint4*>(k_at(RI * i + lrow, lpiece)) = kr[i];
    locate(next);
    load_k(min(next + u.n_parts, chunks - 1));
    __builtin_amdgcn_sched_barrier(0);
    wave_sync_lds();
    RowPart<BITS> kf[NH][2];
    float ks[NH][2], vs[NI];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int row = 16 * t + r16;
#pragma unroll
        for (int w = 0; w < BITS / 4; ++w)
          kf[h][t].w[w] = *reinterpret_cast<const uint4*>(
              k_at(row, h * BITS + kg * (BITS / 4) + w));
        ks[h][t] = scale_of(T.scales[(row * NH + h) * kScaleBytes + kg], 0);
      }
#pragma unroll
    for (int i = 0; i < NI; ++i)
      vs[i] = scale_of(T.scales[((RI * i + lrow) * NH + lhead) * kScaleBytes + 4 +
                                lpart / (BITS / 4)], 0);
    wave_sync_lds();
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      RowPart<BITS> x{};
      x.w[0] = vr[i];
#pragma unroll
      for (int s = 0; s < SP; ++s)
        *reinterpret_cast<bf16x8*>(v_at(lhead, RI * i + lrow, SP * lpart + s)) =
            elements8<BITS>(x, s, vs[i]);
    }
    load_v();
    __builtin_amdgcn_sched_barrier(0);
    wave_sync_lds();

    // S[head r16][token 16 t + 4 kg + i], of all heads step by step: their chains of
    // instructions fill each other's gaps.
    float p[NH][8], mx[NH];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        floatx4 s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(elements8<BITS>(kf[h][t], i, ks[h][t]),
                                                      qf[h][i], s, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[h][4 * t + i] = s[i];
      }
    const int valid = u.valid(c);
    if (valid < kDecodeChunk) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (16 * (i / 4) + 4 * kg + i % 4 >= valid)
#pragma unroll
          for (int h = 0; h < NH; ++h) p[h][i] = -INFINITY;
    }
    bool more = false;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      mx[h] = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) mx[h] = fmaxf(mx[h], p[h][i]);
      mx[h] = C::first(quad_max(mx[h])) * u.scale_log2;
      more |= mx[h] > m_run[h];
    }
    if (__any(more)) {  // seldom but in the first chunks
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const float mn = fmaxf(m_run[h], mx[h]);
        const float alpha = exp2_fast(m_run[h] - mn);
        m_run[h] = mn;
        l_run[h] *= alpha;
#pragma unroll
        for (int db = 0; db < 8; ++db) acc[h][db] *= alpha;
      }
    }
    bf16x8 w[NH][C::MULS];
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      float q[C::OWN];
      C::own(p[h], q);
#pragma unroll
      for (int i = 0; i < C::OWN; ++i) {
        q[i] = exp2_fast(fmaf(q[i], u.scale_log2, -m_run[h]));
        l_run[h] += q[i];
      }
      C::weights(q, w[h]);
    }
    // slots 8 kg .. + 7 of a multiplication: tokens 4 kg .. + 3 and 16 + 4 kg .. + 3
#pragma unroll
    for (int db = 0; db < 8; ++db)
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const bf16x8 vf =
            __builtin_shufflevector(get_v(h, 0, db), get_v(h, 1, db), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int k = 0; k < C::MULS; ++k)
          acc[h][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, w[h][k], acc[h][db], 0, 0, 0);
      }
    wave_sync_lds();  // the tile is rewritten by the next chunk
  }
  uint32_t odd_heads = 0;
#pragma unroll
  for (int h = 0; h < NH; ++h) {
    float odd[4] = {0.f, 0.f, 0.f, 0.f};  // short chains
    l_run[h] = quad_sum(C::sum(l_run[h]));
#pragma unroll
    for (int db = 0; db < 8; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[h][db][i] = C::sum(acc[h][db][i]);
        odd[i] = fmaf(acc[h][db][i], 0.f, odd[i]);
      }
    const float any = (odd[0] + odd[1]) + (odd[2] + odd[3]);
    // Maxima only rise: smaller ones than -kFusedMost before the last have weights of 0, or
    // sums that the last one makes a NaN of.
    const bool far = u.part < chunks && fabsf(m_run[h]) >= kFusedMost;
    if (__any(any != any || far)) odd_heads |= 1u << h;
  }
  return odd_heads;
}

// Visible tokens of a sequence and how they lie.
struct Visible {
  int count, shift, n_sink;
  __device__ __forceinline__ Visible(const QuantArgs& a, int b, int most) {
    const int len = clampi(a.lens[b], 0, most);
    count = min(len, a.k_max);
    shift = len - count;
    n_sink = shift == 0 ? 0 : min(a.n_sink, count);
  }
  __device__ __forceinline__ int chunks() const {
    return (n_sink + kDecodeChunk - 1) / kDecodeChunk +
           (count - n_sink + kDecodeChunk - 1) / kDecodeChunk;
  }
};

// A layer's B n_split parts dealt to its sequences by their lengths, at least one each:
// the least of 64 numbers q of chunks, from the mean up, with which parts of q chunks are
// no more than there are.  Sequences of as many chunks have n_split each.  Every workgroup
// works it out for itself (about 15 instructions a sequence): a ragged batch then takes as
// long as its tokens, not as its longest sequence (us, 8 KV heads, at most: 8 layers x 16 of
// 16384 tokens in 4 bits 209, with n_split each 232; 2 x 32 of 8192 67 and 85; 4 x 7 of 30000
// in 8 bits 147 and 183).
struct Parts {
  int b, first, n;  // the sequence of part j, its first part and their number; b < 0: none
  __device__ __forceinline__ Parts(const QuantArgs& a, int j, int most, int waves_log2) {
    const int lane = threadIdx.x & 63;
    const int P = a.B * a.n_split;
    const int own =
        lane < a.B ? (Visible(a, lane, most).chunks() + (1 << waves_log2) - 1) >> waves_log2 : 0;
    int start, end;  // of the lane's sequence; of all
    if (__all(lane >= a.B || own == __builtin_amdgcn_readfirstlane(own))) {
      b = j / a.n_split;
      first = b * a.n_split;
      n = a.n_split;
      start = lane * a.n_split;
      end = P;
    } else {
      int64_t total = 0;
      for (int s = 0; s < a.B; ++s) total += __builtin_amdgcn_readlane(own, s);
      const int64_t mean = total < P ? 1 : total / P;
      const float rq = 1.f / (float)(mean + mean * lane / 32 + lane);
      auto parts = [](int chunks, float r) { return max(1, (int)ceilf((float)chunks * r)); };
      int sum = 0;
      for (int s = 0; s < a.B; ++s) sum += parts(__builtin_amdgcn_readlane(own, s), rq);
      const uint64_t fits = __ballot(sum <= P);
      const float r = __uint_as_float(
          __builtin_amdgcn_readlane(__float_as_uint(rq), fits ? __builtin_ctzll(fits) : 63));
      const int mine = parts(own, r);
      b = -1;
      first = n = start = 0;
      int next = 0;
      for (int s = 0; s < a.B; ++s) {
        const int m = __builtin_amdgcn_readlane(mine, s);
        if (lane == s) start = next;
        if (j >= next && j < next + m) {
          b = s;
          first = next;
          n = m;
        }
        next += m;
      }
      end = min(next, P);
    }
    if (blockIdx.x == 0 && threadIdx.x < 64) {
      if (lane < a.B) a.parts[lane] = min(start, P);
      if (lane == 0) a.parts[a.B] = end;
    }
  }
};

// The results of a unit's wavefronts, w0 and every 2^ub_log2-th from it on, of head h of KV
// head hu, dimensions 4 d4 ..: all of them are under way before the first is used.  With
// heads counted by powers of two beside it, which need no division, the end of a workgroup
// takes 0.4 to 1.6 us less than with loops and divisions by their numbers (1 x 4096 tokens, 4
// heads of each of 8 KV heads: 5.5 us of 5.9 before the joining launch; 4 layers x 5 of 10016, 7
// of each of 4: 29.3 of 30.9).
template <int W, int NH, int N = W>
__device__ __forceinline__ Join join_unit(const WaveTile<NH> (&tiles)[W],
                                          const float2 (&ml)[W][NH][16], int ub_log2, int w0,
                                          int hu, int h, int d4) {
  if constexpr (N > 1)
    if (W >> ub_log2 < N) return join_unit<W, NH, N / 2>(tiles, ml, ub_log2, w0, hu, h, d4);
  float2 x[N];
  float4 v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int w = w0 + i * (W / N);
    x[i] = ml[w][hu][h];
    v[i] = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(tiles[w].v[hu]) +
                                            result_at(h, d4));
  }
  Join j;
#pragma unroll
  for (int i = 0; i < N; ++i) j.M = fmaxf(j.M, x[i].x);
#pragma unroll
  for (int i = 0; i < N; ++i) j.add(x[i], v[i]);
  return j;
}

// 2^ub_log2 units (NH KV heads and a column group each) of the same tokens side by side, an
// equal number of the W wavefronts each.
template <int W, int BITS, int NH, int GW, bool INDEXED>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(2)))
void quant_decode_kernel(QuantArgs a) {
  __shared__ __align__(16) WaveTile<NH> tiles[W];
  __shared__ float2 ml[W][NH][16];
  __shared__ int first_head[W];  // of a wavefront's unit
  const int units = (a.H_kv / NH * a.R) >> a.ub_log2;  // workgroups of a (layer, sequence, part)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int most = INDEXED ? a.k_max : a.L_cap;
  int layer, b, split, n_parts, group;
  int64_t part;  // of all, where its results are left
  if (a.parts) {  // parts by length: [layer][group of units][part]
    const int per_layer = a.B * a.n_split, rest = blockIdx.x / per_layer;
    const int j = blockIdx.x % per_layer;
    group = rest % units;
    layer = rest / units;
    const Parts p(a, j, most, (W == 8 ? 3 : 2) - a.ub_log2);
    if (p.b < 0) return;  // uniform over the workgroup
    b = p.b;
    split = j - p.first;
    n_parts = p.n;
    part = (int64_t)layer * per_layer + j;
  } else {        // [layer][sequence][group of units][part]
    const int rest = blockIdx.x / a.n_split, lb = rest / units;
    split = blockIdx.x % a.n_split;
    n_parts = a.n_split;
    group = rest % units;
    layer = lb / a.B;
    b = lb % a.B;
    part = (int64_t)lb * a.n_split + split;
  }
  const int lb = layer * a.B + b;
  // unit: column group r of KV heads g .. g + NH - 1
  const int unit = (group << a.ub_log2) + (wave & ((1 << a.ub_log2) - 1));
  const int g = unit / a.R * NH, r = unit % a.R, G = a.heads * a.R;
  const int64_t base = layer * a.kv_stride_layer + b * a.kv_stride_b + g * row_bytes(BITS);
  const Visible vis(a, b, most);
  QuantUnit u;
  const int head0 = g * G + r * a.heads;
  u.q = a.q + ((int64_t)lb * a.H_q + head0) * kHeadDim;
  u.q_stride = G * kHeadDim;
  u.k = a.k + base;
  u.v = a.v + base;
  u.scales = a.scales + layer * a.scale_stride_layer + b * a.scale_stride_b + g * kScaleBytes;
  u.idx = INDEXED ? a.idx + ((int64_t)b * a.n_sets + (a.n_sets == 1 ? 0 : g)) * a.k_max : nullptr;
  u.idx_stride = a.n_sets == 1 ? 0 : a.k_max;
  u.rs = (int64_t)a.H_kv * row_bytes(BITS);
  u.ss = a.H_kv * kScaleBytes;
  u.last = a.L_cap - 1;
  u.k_max = a.k_max;
  u.heads = a.heads;
  u.count = vis.count;
  u.shift = vis.shift;
  u.n_sink = vis.n_sink;
  u.part = split * (W >> a.ub_log2) + (wave >> a.ub_log2);
  u.n_parts = n_parts * (W >> a.ub_log2);
  u.scale_log2 = a.scale_log2;
  float m_run[NH], l_run[NH];
  floatx4 acc[NH][8];
  const uint32_t odd = quant_unit<BITS, NH, GW, INDEXED>(u, tiles[wave], m_run, l_run, acc);

#pragma unroll
  for (int h = 0; h < NH; ++h)
    leave_results(tiles[wave].v[h], ml[wave][h], m_run[h], l_run[h], acc[h]);
  if ((threadIdx.x & 63) == 0) first_head[wave] = head0;
  if (odd) {  // uniform
#pragma unroll 1
    for (int h = 0; h < NH; ++h) {
      if (!(odd >> h & 1)) continue;
      quant_unit_by_token<BITS, INDEXED>(u, h, m_run[0], l_run[0], acc[0]);
      leave_results(tiles[wave].v[h], ml[wave][h], m_run[0], l_run[0], acc[0]);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < GW * NH * 32 << a.ub_log2; e += W * 64) {
    const int d4 = e & 31, h = (e >> 5) % GW, hu = (e >> 5) / GW % NH;
    const int w0 = (e >> 5) / (GW * NH);
    if (h >= a.heads) continue;
    const int head = first_head[w0] + hu * G + h;
    const Join j = join_unit<W, NH>(tiles, ml, a.ub_log2, w0, hu, h, d4);
    if (a.out) {
      const int64_t row = (int64_t)lb * a.H_q + head;
      const float inv = j.inv();
      reinterpret_cast<float4*>(a.out + row * kHeadDim)[d4] =
          make_float4(j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv);
      if (a.lse && d4 == 0) a.lse[row] = j.lse();
    } else {
      const int64_t row = part * a.H_q + head;
      reinterpret_cast<float4*>(a.part_acc + row * kHeadDim)[d4] = j.o;
      if (d4 == 0) reinterpret_cast<float2*>(a.part_ml)[row] = make_float2(j.M, j.L);
    }
  }
}

struct MergeArgs {
  const float* part_acc;
  const float* part_ml;
  const int32_t* parts;
  float* out;
  float* lse;
  uint32_t n_out, B, H_q;  // n_out: 2^26 at most
  int n_split;
};

// 8 / S output rows per workgroup, 32 threads (4 dimensions each) and S of them.
template <int S>
__global__ __launch_bounds__(256) void quant_merge_kernel(MergeArgs a) {
  const uint32_t want = blockIdx.x * (8 / S) + (threadIdx.x >> 5) / S;
  const uint32_t orow = want < a.n_out ? want : a.n_out - 1;
  const int d4 = threadIdx.x & 31;
  const uint32_t lb = orow / a.H_q, h = orow - lb * a.H_q;
  int64_t first = (int64_t)lb * a.n_split;
  int n = a.n_split;
  if (a.parts) {
    const uint32_t layer = lb / a.B, b = lb - layer * a.B;
    first = (int64_t)layer * a.B * a.n_split + a.parts[b];
    n = a.parts[b + 1] - a.parts[b];
  }
  const Join j = join_parts<S>(n, [&](int s, const float2*& ml, const float*& acc) {
    const int64_t row = (first + s) * a.H_q + h;
    ml = reinterpret_cast<const float2*>(a.part_ml) + row;
    acc = a.part_acc + row * kHeadDim;
  });
  if (want >= a.n_out || (threadIdx.x >> 5) % S != 0) return;
  const float inv = j.inv();
  reinterpret_cast<float4*>(a.out + (int64_t)orow * kHeadDim)[d4] =
      make_float4(j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv);
  if (a.lse && d4 == 0) a.lse[orow] = j.lse();
}

size_t quant_part_acc_bytes(const QuantDims& d, int n_split) {
  return n_split > 1 ? align_up(sizeof(float) * kHeadDim * (size_t)d.n_layers * d.B * n_split *
                                d.H_q)
                     : 0;
}
constexpr size_t kDealtBytes = align_up(sizeof(int32_t) * (kMostDealt + 1));
size_t quant_part_bytes(const QuantDims& d, int n_split) {
  return quant_part_acc_bytes(d, n_split) +
         (n_split > 1 ? align_up(sizeof(float) * 2 * (size_t)d.n_layers * d.B * n_split * d.H_q) +
                            kDealtBytes
                      : 0);
}

template <int BITS, int NH, int GW, bool INDEXED>
void launch_columns(const QuantArgs& a, int w, unsigned blocks, hipStream_t s) {
  if (w == 8) quant_decode_kernel<8, BITS, NH, GW, INDEXED><<<blocks, 512, 0, s>>>(a);
  else quant_decode_kernel<4, BITS, NH, GW, INDEXED><<<blocks, 256, 0, s>>>(a);
}

template <int BITS, int NH, bool INDEXED>
void launch_rows(const QuantArgs& a, int w, unsigned blocks, hipStream_t s) {
  if (a.heads <= 4) launch_columns<BITS, NH, 4, INDEXED>(a, w, blocks, s);
  else if (a.heads <= 8) launch_columns<BITS, NH, 8, INDEXED>(a, w, blocks, s);
  else launch_columns<BITS, NH, 16, INDEXED>(a, w, blocks, s);
}

template <bool INDEXED>
void launch_kernel(const QuantArgs& a, int bits, const QuantPlan& p, unsigned blocks,
                   hipStream_t s) {
  if (bits == 8) launch_rows<8, 1, INDEXED>(a, p.w, blocks, s);
  else if (p.nh == 2) launch_rows<4, 2, INDEXED>(a, p.w, blocks, s);
  else launch_rows<4, 1, INDEXED>(a, p.w, blocks, s);
}

hipError_t launch_quant(const QuantDims& d, int k_max, int n_sink, const uint16_t* q,
                        const QuantCache& c, const int32_t* idx, const int32_t* lens, float* out,
                        float* lse, void* ws, hipStream_t s) {
  const QuantPlan p = d.plan;
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
  a.ub_log2 = p.ub_log2;
  a.n_split = p.n_split;
  a.scale_log2 = d.scale * kLog2e;
  if (p.n_split > 1) {
    a.out = nullptr;
    a.part_acc = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) +
                                         quant_part_acc_bytes(d, p.n_split));
    if (p.deal)
      a.parts = reinterpret_cast<int32_t*>(static_cast<char*>(ws) +
                                           quant_part_bytes(d, p.n_split) - kDealtBytes);
  }
  const int64_t blocks =
      ((int64_t)d.n_layers * d.B * (d.H_kv / p.nh) * a.R >> p.ub_log2) * p.n_split;
  if (blocks > INT32_MAX / (p.w * 64)) return hipErrorInvalidValue;
  if (idx) launch_kernel<true>(a, d.bits, p, (unsigned)blocks, s);
  else launch_kernel<false>(a, d.bits, p, (unsigned)blocks, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_split == 1) return e;
  const uint32_t n_out = (uint32_t)(d.n_layers * d.B) * d.H_q;
  const MergeArgs m{a.part_acc, a.part_ml, a.parts, out, lse, n_out, (uint32_t)d.B,
                    (uint32_t)d.H_q, p.n_split};
  with_parts(p.n_split, [&](auto S) {
    quant_merge_kernel<S.value><<<merge_grid(n_out, S.value), 256, 0, s>>>(m);
  });
  return hipGetLastError();
}

}  // namespace

QuantPlan quant_plan(const QuantDims& d, bool selected) { return plan_of(d, selected); }
size_t quant_attn_ws_bytes(const QuantDims& d) { return quant_part_bytes(d, d.plan.n_split); }

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
