// Attention of many query rows over one range of cached tokens, on gfx950: the
// chunks of window attention (Sec. 4.3's GQA layout; the rows are the query
// tokens of a sequence times the query heads of a KV head), and the shared part
// of prefix attention (the rows are the sequences of the batch times the heads).
//
// One pass over the tokens with a running maximum and sum per row:
//     m' = max(m, max_t s_t),  l' = l 2^(m-m') + sum_t 2^(s_t-m'),
//     O' = O 2^(m-m') + sum_t 2^(s_t-m') v_t,     s_t = scale log2(e) q.k_t
// Tiles of TOK tokens go through two or three stages in LDS: later tiles' loads go
// there directly, issued between this one's products.  (By way of registers, their
// issue and the LDS writes took 1200 of a tile's 3200 cycles with 64 rows, as a
// wavefront waits where the path is full: 2 x 4096 tokens 294 us against 271, 512
// tokens 17 against 15.)  The largest chunks reach 1.0 PFLOP/s of the 1.2 of a library
// product of bf16 (its limit is power: with zeros it reaches 1.7, and the chunks lose
// 10 % of their time).  More stages, products of the next tile beside this one's
// exponentials, and wavefronts half a tile apart changed that by 2 % at most.
// A wavefront owns 32 rows:
//  * S^T = K Q^T with v_mfma_f32_32x32x16_bf16 leaves a row's logits in one lane
//    (and its partner 32 lanes on), so that the softmax needs one lane swap;
//  * O^T += V^T P^T takes P from those registers as they are: the token order
//    inside a multiplication is free, and V is read transposed from LDS
//    (ds_read_b64_tr_b16) in the same order.
#include "dense_core.h"

namespace spec {
namespace {

constexpr int kD = kHeadDim;
typedef float floatx16 __attribute__((ext_vector_type(16)));
// The maximum is moved, and what has been added up rescaled, only once a logit
// is 2^8 above it: until then weights are up to 2^8, which neither the fp32 sums
// nor the bf16 weights (whose precision is relative) notice.
constexpr float kSlack = 8.f;

struct TileArgs {
  const uint16_t* q;      // [units / H_kv][T][H_q][d]
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* lens;    // window: cached tokens [B]; prefix: [1] or null (L_cap)
  const int32_t* q_lens;  // window: [B] or null (T)
  uint16_t* out;          // window, one split: [units / H_kv][T][H_q][d] bf16
  float* lse;             // [units / H_kv][T][H_q] or null
  float* part_acc;        // [units][n_rt][n_split][ROWS][d]
  float* part_ml;         // [units][n_rt][n_split][ROWS][2]
  int64_t stride_layer, stride_b;  // elements between layers / sequences of K and V
  int B, T, H_q, H_kv, G, L_cap, window, n_sink;
  int n_units, n_rt, n_split, split_tok;
  float scale_log2;
  DecodeArgs own;         // prefix: the sequences' own tokens, by
  int own_blocks;         // the first workgroups of the launch,
  int own_hb;             // one or four column groups each
};

// The value of the lane 32 on (each row lives in two lanes).
__device__ __forceinline__ float pair_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Visible tokens of the query items i0..i1 of one sequence (len cached tokens, n
// query tokens, item i at position len - n + i), numbered 0 .. count-1: the first
// n_sink are themselves, the others stand `shift` further on.
struct Range {
  int count, n_sink, shift;
};
__device__ __forceinline__ Range window_range(const TileArgs& a, int p0, int i0, int i1) {
  const int hi = p0 + i1 + 1;  // behind the last visible token
  if (hi <= 0) return {0, 0, 0};
  const int s = min(a.n_sink, hi);
  const int lo = max(p0 + i0 - a.window + 1, s);
  return {s + hi - lo, s, lo - s};
}

// The same token by token, for the rare sums that hold infinities or NaNs: of rows that
// a query does not see, or whose logit is -inf, they are selected away; and for logits
// beyond kFusedMost, which are rounded before the maximum is taken off (below, weights are
// those of the matrix cores' path).  The wavefront's tokens are j0 .. j0 + run - 1 and those
// `step` further on, up to j1.  A lane has the dimensions 32 db + 8 e + 4 kg .. + 3 of its
// row, as the accumulators do.
template <bool WINDOW, class TokenOf>
__device__ __forceinline__ void attend_by_token(const TileArgs& a, const uint16_t* q,
                                                const uint16_t* k, const uint16_t* v, int64_t rs,
                                                int kg, int j0, int j1, int run, int step, int pos,
                                                TokenOf&& token_of, float& m_run, float& l_run,
                                                floatx16 (&acc)[4]) {
#pragma clang fp contract(off)  // a logit's product and difference stay two roundings
  auto four = [](const uint16_t* p, float (&f)[4]) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    f[0] = bf16lo(x.x);
    f[1] = bf16hi(x.x);
    f[2] = bf16lo(x.y);
    f[3] = bf16hi(x.y);
  };
  m_run = kNoMax;
  l_run = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db) acc[db] = 0.f;
#pragma unroll 1
  for (int j = j0, left = run; j < j1; left = left == 1 ? run : left - 1,
           j += left == run ? step - run + 1 : 1) {
    const int t = token_of(j);
    const int64_t off = (int64_t)t * rs + 4 * kg;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float x[4], y[4];
      four(q + 4 * kg + 8 * e, x);
      four(k + off + 8 * e, y);
      for (int i = 0; i < 4; ++i) s = fmaf(x[i], y[i], s);
    }
    const bool see = !WINDOW || (t <= pos && (t < a.n_sink || t > pos - a.window));
    const float all = pair_sum(s), sum = see ? all : -INFINITY;
    s = see ? all * a.scale_log2 : -INFINITY;
    const float mn = fmaxf(m_run, s);
    const float alpha = exp2_fast(m_run - mn);
    const float p = exp2_fast(fabsf(mn) < kFusedMost ? fmaf(sum, a.scale_log2, -mn) : s - mn);
    m_run = mn;
    l_run = l_run * alpha + (kg == 0 ? p : 0.f);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float y[4];
      four(v + off + 8 * e, y);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        acc[e >> 2][4 * (e & 3) + i] =
            acc[e >> 2][4 * (e & 3) + i] * alpha + (s == -INFINITY ? 0.f : p * y[i]);
    }
  }
}

// s_waitcnt immediate (gfx9 encoding: vmcnt[3:0], expcnt[6:4], lgkmcnt[11:8], vmcnt[5:4]
// in bits [15:14]) that waits for the vector-memory count only.
constexpr int waitcnt_vm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }

// Global-to-LDS copy of 16 bytes per lane: lane l's bytes land at lds + 16 l (M0 holds
// the wave-uniform base).  From inline assembly, as the compiler, which cannot tell the
// stage being read from the one being filled, would wait for all pending loads
// before every LDS read.  It has no output registers; the kernel does the waiting.
// Nothing else in this file uses M0 (tests/test_isa_dense_cpu.py).
// A load that reads M0 needs a wait state after the write, which the compiler puts in
// for its own: .long is s_nop 0, as a word since those checks want the two listed side
// by side (tests/test_isa_m0_cpu.py has what is encoded).
__device__ __forceinline__ void load_to_lds(const void* g, const void* lds) {
  const uint32_t base = (uint32_t)(uintptr_t)lds;
  asm volatile("s_mov_b32 m0, %0\n\t.long 0xbf800000\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(base)), "v"(g)
               : "memory", "m0");
}

// RW x TW wavefronts: RW groups of 32 rows, TW parts of each tile's tokens.
// WINDOW: masked rows of a sequence; else every row sees all tokens.  SPLITP:
// weights as a bf16 pair (2^-17 relative) for fp32 results, or with few rows, which
// leave the matrix cores idle, as three bf16 numbers (2 % of the time of 32 rows, but 9 %
// of that of 64 and 13 % of that of 256); else rounded to bf16 once (2^-8), as the result
// is, for that takes the matrix cores: 2 x 4096 tokens 277 us, with a pair 373; 8192, window
// 1024, 157 and 205; 5 x 257 at most 24.1 and 27.3.  It makes the error of the whole output
// 2.3e-3 (root of mean squares) instead of the 1.7e-3 of rounding the exact one.
template <int RW, int TW, int TOK, bool WINDOW, bool SPLITP>
__global__ __launch_bounds__(RW* TW * 64) __attribute__((amdgpu_waves_per_eu(TOK == 64 ? 2 : 1)))
void tile_attn_kernel(TileArgs a) {
  constexpr int ROWS = 32 * RW;
  constexpr int NB = TOK / (32 * TW);      // 32-token blocks of a wavefront
  constexpr int LD = TOK / 4 / (RW * TW);  // loads of a wavefront for K, and for V: 4 rows each
  // Tiles in LDS: a workgroup of eight wavefronts is alone on its CU, with room for a third
  // (2 x 4096 tokens not in the caches: 302 us, with two 307), and 64 rows on a long prefix,
  // which wait for memory, are faster so than two workgroups of two stages (us, 16
  // sequences: 8 layers of 32768 tokens 266, with two stages 291; one of 65536 70 and 76; 2
  // of 20011 63.8 and 66.7; one of 1000 14.6 and 14.6; slower where the own tokens are many
  // beside it, 4 of 16384 and 1024 own ones 116 and 110, one of 4096 and 777 28.4 and 25.4).
  constexpr int STAGES = RW * TW == 8 || (!WINDOW && RW == 2) ? 3 : 2;
  __shared__ __align__(16) uint16_t lds[STAGES][2][TOK * kD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rw = wave % RW, tw = wave / RW;
  const int c32 = lane & 31, kg = lane >> 5;
  int block = blockIdx.x;
  if (!WINDOW) {  // own tokens: memory-bound work beside that of the matrix cores
    if (block < a.own_blocks) {
      constexpr int W = RW * TW;
      static_assert(W * kTileElems <= STAGES * 2 * TOK * kD, "room for the wavefronts' V tiles");
      __shared__ float2 ml[W][16];
      auto tiles = reinterpret_cast<uint16_t(*)[kTileElems]>(&lds[0][0][0]);
      if (a.own_hb == 4) decode_block<W, 4, kKeepNone>(a.own, block, tiles, ml, nullptr);
      else decode_block<W, 1, kKeepNone>(a.own, block, tiles, ml, nullptr);
      return;
    }
    block -= a.own_blocks;
  }

  // Units run fastest over the workgroups: those of one KV head keep to one XCD
  // where the units are a multiple of 8, and share its L2.  The last rows, which
  // see the most tokens, go first.
  const int u = block % a.n_units;
  const int rest = block / a.n_units;
  const int split = rest % a.n_split;
  const int rt = a.n_rt - 1 - rest / a.n_split;
  const int lb = u / a.H_kv, g = u % a.H_kv;
  const int b = lb % a.B;

  int n_items = a.T, p0 = 0;
  Range rg;
  const int r0 = rt * ROWS;
  if (WINDOW) {
    const int len = clampi(a.lens[b], 0, a.L_cap);
    if (a.q_lens) n_items = clampi(a.q_lens[b], 0, a.T);
    p0 = len - n_items;
  }
  const int n_rows = n_items * a.G;
  if (r0 >= n_rows) return;  // uniform
  const int i0 = r0 / a.G, i1 = (min(r0 + ROWS, n_rows) - 1) / a.G;
  if (WINDOW) rg = window_range(a, p0, i0, i1);
  else rg = {a.lens ? clampi(a.lens[0], 0, a.L_cap) : a.L_cap, 0, 0};
  const int v0 = split * a.split_tok;
  const int v1 = min(v0 + a.split_tok, rg.count);
  const int n_tiles = v1 > v0 ? (v1 - v0 + TOK - 1) / TOK : 0;

  // this lane's row
  const int row = r0 + rw * 32 + c32;
  const bool row_ok = row < n_rows;
  const int rc = min(row, n_rows - 1);
  const int item = rc / a.G;
  const int pos = p0 + item;
  const size_t orow = ((size_t)lb * a.T + item) * a.H_q + (size_t)g * a.G + (rc - item * a.G);

  bf16x8 qf[8];
  {
    const uint16_t* qp = a.q + orow * kD + 8 * kg;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = __builtin_bit_cast(bf16x8, ldg16(qp + 16 * s));
    // Waited for here: in the loop the wait would cover the tiles' loads as well.
#pragma unroll
    for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(qf[s]));
  }

  const int64_t rs = (int64_t)a.H_kv * kD;
  const int64_t base = (int64_t)(lb / a.B) * a.stride_layer + (int64_t)b * a.stride_b + g * kD;
  auto token_of = [&](int j) { return j + (j < rg.n_sink ? 0 : rg.shift); };
  // A load brings four rows, 16 bytes per lane, to where they are read from (swizzle);
  // rows behind the range are its last one.  Tiles behind the last are loaded, and not
  // read, so that no branch stands between the multiplications.
  auto issue = [&](int it, int stage, int e) {
    const int r0 = (wave * LD + e / 2) * 4, r = r0 + (lane >> 4);
    const int j = min(v0 + it * TOK + r, v1 - 1);
    const int64_t off = base + (int64_t)token_of(j) * rs + (((lane & 15) ^ swizzle(r)) * 8);
    load_to_lds((e % 2 ? a.v : a.k) + off, &lds[stage][e % 2][r0 * kD]);
  };

  // Tiles that every row sees whole need no mask: those before `clear`, but for the ones
  // on the window's edge, edge0 .. edge1 - 1.
  int clear, edge0 = 0, edge1 = 0;
  {
    int last = v1 - 1;  // the last token that the first query sees
    if (WINDOW) {
      const int p = p0 + i0;
      last = min(last, p - rg.shift >= rg.n_sink ? p - rg.shift : min(p, rg.n_sink - 1));
      const int out = p0 + i1 - a.window - rg.shift;  // the last one the last does not see
      if (rg.n_sink <= out) {
        edge0 = max(rg.n_sink - v0, 0) / TOK;
        edge1 = out >= v0 ? (out - v0) / TOK + 1 : 0;
      }
    }
    clear = max(last + 1 - v0, 0) / TOK;
  }
  // This row sees tokens 0 .. sinks - 1 and lo .. lo + n - 1 of the range.
  int sinks = 0, lo = 0, n = v1;
  if (WINDOW) {
    sinks = min(min(rg.n_sink, pos + 1), v1);
    lo = max(rg.n_sink, pos - a.window + 1 - rg.shift);
    n = max(min(pos + 1 - rg.shift, v1) - lo, 0);
  }

  float m_run = kNoMax, l_run = 0.f;
  floatx16 acc[4];  // O^T[32 db + 8 (i / 4) + 4 kg + i % 4][row]
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[db][i] = 0.f;

  // LDS offsets of this lane: K rows c32 of a block, V rows of a transposing read
  const int ksw = kg ^ swizzle(c32);
  const int a16 = lane & 15, half16 = (lane >> 4) & 1;

  // Each wavefront waits for its own loads of a tile, those of later ones being in flight,
  // before the barrier in front of its use.
  constexpr int kWait = waitcnt_vm((STAGES - 2) * 2 * LD);
  if (n_tiles > 0) {
#pragma unroll
    for (int t = 0; t < STAGES - 1; ++t)
#pragma unroll
      for (int e = 0; e < 2 * LD; ++e) issue(t, t, e);
    __builtin_amdgcn_s_waitcnt(kWait);
    __syncthreads();
  }

  int now = 0, then = STAGES - 1;  // stages of this tile, and of the one that is requested
  for (int it = 0; it < n_tiles; ++it) {
    const uint16_t* Kt = lds[now][0];
    const uint16_t* Vt = lds[now][1];

    // S^T of this wavefront's blocks: token 32 blk + 8 (i / 4) + 4 kg + i % 4.  Between
    // the products a later tile's loads, into the stage that was last read before the
    // previous barrier; as no LDS read moves across those, K is read kAhead products
    // before it is needed (8192 tokens, window 1024: 158 us, read beside them 164).
    floatx16 s[NB];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) s[blk] = 0.f;
    constexpr int kOps = 8 * NB, kAhead = 5;
    auto k_operand = [&](int c) {
      const uint16_t* kp = Kt + ((tw * NB + c / 8) * 32 + c32) * kD;
      return *reinterpret_cast<const bf16x8*>(kp + (((2 * (c % 8)) ^ ksw) * 8));
    };
    bf16x8 kf[kOps];
#pragma unroll
    for (int c = 0; c < kAhead; ++c) kf[c] = k_operand(c);
#pragma unroll
    for (int c = 0; c < kOps; ++c) {
      if (c + kAhead < kOps) kf[c + kAhead] = k_operand(c + kAhead);
      s[c / 8] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], qf[c % 8], s[c / 8], 0, 0, 0);
#pragma unroll
      for (int e = c * LD / (4 * NB); e < (c + 1) * LD / (4 * NB); ++e)
        issue(it + STAGES - 1, then, e);
    }

    if (it >= clear || (WINDOW && it >= edge0 && it < edge1)) {
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = v0 + it * TOK + (tw * NB + blk) * 32 + 8 * (i >> 2) + 4 * kg + (i & 3);
          bool see = (uint32_t)(j - lo) < (uint32_t)n;
          if (WINDOW) see = see | (j < sinks);
          s[blk][i] = see ? s[blk][i] : -INFINITY;
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // few conditions at a time
        }
    }

    float mx = -INFINITY;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[blk][i]);
    mx = pair_max(mx) * a.scale_log2;
    if (__any(mx > m_run + kSlack)) {
      const float mn = fmaxf(m_run, mx);
      const float alpha = exp2_fast(m_run - mn);
      m_run = mn;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < 4; ++db) acc[db] *= alpha;
    }

    constexpr bool kThird = SPLITP && RW == 1;
    bf16x8 ph[2 * NB], pl[SPLITP ? 2 * NB : 1], pt[kThird ? 2 * NB : 1];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      float p[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = exp2_fast(fmaf(s[blk][i], a.scale_log2, -m_run));
        l_run += p[i];
      }
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        ph[2 * blk + m] = to_bf16x8(p + 8 * m);
        if constexpr (SPLITP) pl[2 * blk + m] = next_bf16x8(p + 8 * m, ph[2 * blk + m]);
        if constexpr (kThird) pt[2 * blk + m] = next_bf16x8(p + 8 * m, pl[2 * blk + m]);
      }
    }

    // O^T += V^T P^T: slots 8 kg .. 8 kg + 7 of a multiplication are tokens
    // 16 m + 4 kg + 0..3 and 16 m + 8 + 4 kg + 0..3, as this lane holds P.
#pragma unroll
    for (int m = 0; m < 2 * NB; ++m) {
      const uint16_t* vp = Vt + (tw * NB * 32 + 16 * m + 4 * kg + (a16 >> 2)) * kD + 4 * (a16 & 1);
      const int lo0 = (2 * half16 + ((a16 >> 1) & 1)) ^ kg;
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const int hi4 = 4 * (db ^ (a16 >> 2));
        const bf16x4 x = lds_read_tr(vp + (hi4 + lo0) * 8);
        const bf16x4 y = lds_read_tr(vp + 8 * kD + (hi4 + (lo0 ^ 2)) * 8);
        const bf16x8 vf = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, ph[m], acc[db], 0, 0, 0);
        if constexpr (SPLITP)
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pl[m], acc[db], 0, 0, 0);
        if constexpr (kThird)
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pt[m], acc[db], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(kWait);
    __syncthreads();
    now = now == STAGES - 1 ? 0 : now + 1;
    then = then == STAGES - 1 ? 0 : then + 1;
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // loads past the last tile, before LDS is
  __syncthreads();                            // used anew or given back
  // Where an infinity or a NaN got into the sums, they are taken again without the matrix
  // cores: a weight of 0 does not keep one of a row that this query does not see, or whose
  // logit is -inf, out of them (0 x NaN), nor is an infinity of one that it sees the
  // product with a weight's parts.  So they are where a row's logits go beyond kFusedMost
  // (maxima only rise: those of before weigh 0, or leave a NaN).
  {
    float odd = 0.f;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd = fmaf(acc[db][i], 0.f, odd);
    if (__any(odd != odd || (fabsf(m_run) >= kFusedMost && m_run != kNoMax)))
      attend_by_token<WINDOW>(a, a.q + orow * kD, a.k + base, a.v + base, rs, kg,
                              v0 + tw * NB * 32, v1, NB * 32, TOK, pos, token_of, m_run, l_run,
                              acc);
  }
  l_run = pair_sum(l_run);

  // The parts of a row group, joined by its first wavefront: accumulators stand
  // in the same lanes of each.
  if constexpr (TW > 1) {
    static_assert((TW - 1) * RW * 64 * (64 + 2) * 4 <= sizeof(lds), "merge area");
    float* mem = reinterpret_cast<float*>(lds);
    constexpr int kPer = 64 * 66;  // floats of a wavefront: 16 x 64 float4, 64 x (m, l)
    if (tw > 0) {
      float* w = mem + ((tw - 1) * RW + rw) * kPer;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<float4*>(w + ((db * 4 + e) * 64 + lane) * 4) = make_float4(
              acc[db][4 * e], acc[db][4 * e + 1], acc[db][4 * e + 2], acc[db][4 * e + 3]);
      *reinterpret_cast<float2*>(w + 64 * 64 + lane * 2) = make_float2(m_run, l_run);
    }
    __syncthreads();
    if (tw > 0) return;
#pragma unroll
    for (int o = 1; o < TW; ++o) {
      const float* w = mem + ((o - 1) * RW + rw) * kPer;
      const float2 ml = *reinterpret_cast<const float2*>(w + 64 * 64 + lane * 2);
      const float mn = fmaxf(m_run, ml.x);
      const float f0 = exp2_fast(m_run - mn), f1 = exp2_fast(ml.x - mn);
      m_run = mn;
      l_run = l_run * f0 + ml.y * f1;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 x = *reinterpret_cast<const float4*>(w + ((db * 4 + e) * 64 + lane) * 4);
          acc[db][4 * e] = acc[db][4 * e] * f0 + x.x * f1;
          acc[db][4 * e + 1] = acc[db][4 * e + 1] * f0 + x.y * f1;
          acc[db][4 * e + 2] = acc[db][4 * e + 2] * f0 + x.z * f1;
          acc[db][4 * e + 3] = acc[db][4 * e + 3] * f0 + x.w * f1;
        }
    }
  }

  if (!row_ok) return;
  if (WINDOW && a.n_split == 1) {
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    uint16_t* dst = a.out + orow * kD + 4 * kg;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x4 h = __builtin_convertvector(
            floatx4{acc[db][4 * e] * inv, acc[db][4 * e + 1] * inv, acc[db][4 * e + 2] * inv,
                     acc[db][4 * e + 3] * inv}, bf16x4);
        *reinterpret_cast<uint2*>(dst + 32 * db + 8 * e) = __builtin_bit_cast(uint2, h);
      }
    if (a.lse && kg == 0) a.lse[orow] = (m_run + log2f(l_run)) * kLn2;
    return;
  }
  // a part without tokens leaves a sum of 0, and no accumulators
  const size_t prow = (((size_t)u * a.n_rt + rt) * a.n_split + split) * ROWS + rw * 32 + c32;
  if (kg == 0) reinterpret_cast<float2*>(a.part_ml)[prow] = make_float2(m_run, l_run);
  if (n_tiles == 0) return;
  float* dst = a.part_acc + prow * kD + 4 * kg;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<float4*>(dst + 32 * db + 8 * e) = make_float4(
          acc[db][4 * e], acc[db][4 * e + 1], acc[db][4 * e + 2], acc[db][4 * e + 3]);
}

// 8 / S output rows per workgroup, 32 threads (4 dimensions each) and S of them.
template <int S>
__global__ __launch_bounds__(256) void window_merge_kernel(TileArgs a, int rows_per_tile,
                                                           int64_t n_out) {
  const int64_t want = (int64_t)blockIdx.x * (8 / S) + (threadIdx.x >> 5) / S;
  const int64_t orow = want < n_out ? want : n_out - 1;
  const int d4 = threadIdx.x & 31;
  const int h = (int)(orow % a.H_q);
  const int64_t rest = orow / a.H_q;
  const int i = (int)(rest % a.T), lb = (int)(rest / a.T);
  const bool live = want < n_out && !(a.q_lens && i >= clampi(a.q_lens[lb % a.B], 0, a.T));
  const int g = h / a.G;
  const int r = i * a.G + (h - g * a.G);
  const size_t part = ((size_t)lb * a.H_kv + g) * a.n_rt + r / rows_per_tile;
  const Join j = join_parts<S>(live ? a.n_split : 0, [&](int s, const float2*& ml,
                                                         const float*& acc) {
    const size_t prow = (part * a.n_split + s) * rows_per_tile + r % rows_per_tile;
    ml = reinterpret_cast<const float2*>(a.part_ml) + prow;
    acc = a.part_acc + prow * kD;
  });
  if (!live || (threadIdx.x >> 5) % S != 0) return;
  const float inv = j.inv();
  const bf16x4 o = __builtin_convertvector(
      floatx4{j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv}, bf16x4);
  reinterpret_cast<uint2*>(a.out + orow * kD)[d4] = __builtin_bit_cast(uint2, o);
  if (a.lse && d4 == 0) a.lse[orow] = j.lse();
}

// The prefix's partial results and those of the sequence's own tokens.
template <int S>
__global__ __launch_bounds__(256) void prefix_merge_kernel(TileArgs a, int rows_per_tile,
                                                           float* out, float* lse,
                                                           int64_t n_out) {
  const int64_t want = (int64_t)blockIdx.x * (8 / S) + (threadIdx.x >> 5) / S;
  const int64_t orow = want < n_out ? want : n_out - 1;
  const int d4 = threadIdx.x & 31;
  const int h = (int)(orow % a.H_q);
  const int64_t lb = orow / a.H_q;                         // layer * batch + sequence
  const int b = (int)(lb % a.T), layer = (int)(lb / a.T);  // T: the batch
  const int g = h / a.G;
  const int r = b * a.G + (h - g * a.G);
  const size_t part = ((size_t)layer * a.H_kv + g) * a.n_rt + r / rows_per_tile;
  const Join j = join_parts<S>(a.n_split + a.own.n_split, [&](int s, const float2*& ml,
                                                              const float*& acc) {
    const bool pre = s < a.n_split;
    const size_t prow = pre ? (part * a.n_split + s) * rows_per_tile + r % rows_per_tile
                            : ((size_t)lb * a.own.n_split + (s - a.n_split)) * a.H_q + h;
    ml = reinterpret_cast<const float2*>(pre ? a.part_ml : a.own.part_ml) + prow;
    acc = (pre ? a.part_acc : a.own.part_acc) + prow * kD;
  });
  if (want >= n_out || (threadIdx.x >> 5) % S != 0) return;
  const float inv = j.inv();
  reinterpret_cast<float4*>(out + orow * kD)[d4] =
      make_float4(j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv);
  if (lse && d4 == 0) lse[orow] = j.lse();
}

// Rows of a workgroup, tokens of a tile, and how the tokens are split.
struct TilePlan {
  int rows, tok, n_rt, n_split, split_tok;
};

// Tokens of a part at least.  us with 128 / 256 / 512: 4 sequences on a prefix of 500
// tokens 11.7 / 12.9 / 15.5, 1000 13.8 / 14.0 / 16.8, 2000 14.9 / 16.3 / 18.7, 4000 20.7 /
// 17.0 / 20.4; 16 sequences on 4000 23.0 / 18.7 / 20.8; 16 queries over 4096 tokens 17.4 /
// 17.3 / 19.6.
constexpr int kMinSplit = 256;

// Splits a row tile's `most` tokens into about n parts.
void split_tokens(TilePlan& p, int64_t most, int64_t n) {
  const int64_t per = ((most + n - 1) / n + p.tok - 1) / p.tok * p.tok;
  p.split_tok = (int)(per < p.tok ? p.tok : per);
  p.n_split = (int)((most + p.split_tok - 1) / p.split_tok);
  if (p.n_split < 1) p.n_split = 1;
}

size_t tile_acc_bytes(int64_t units, const TilePlan& p) {
  return align_up(sizeof(float) * kD * (size_t)units * p.n_rt * p.n_split * p.rows);
}
size_t tile_ml_bytes(int64_t units, const TilePlan& p) {
  return align_up(sizeof(float) * 2 * (size_t)units * p.n_rt * p.n_split * p.rows);
}

template <bool WINDOW, bool SPLITP>
hipError_t launch_tiles(const TilePlan& p, const TileArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.n_units * a.n_rt * a.n_split + a.own_blocks;
  if (n > UINT32_MAX / 512) return hipErrorInvalidValue;  // threads of a launch
  const dim3 grid((unsigned)n);
  if (p.rows == 256) tile_attn_kernel<8, 1, 64, WINDOW, SPLITP><<<grid, 512, 0, s>>>(a);
  else if (p.rows == 128) tile_attn_kernel<4, 1, 64, WINDOW, SPLITP><<<grid, 256, 0, s>>>(a);
  else if (p.rows == 64) tile_attn_kernel<2, 2, 64, WINDOW, SPLITP><<<grid, 256, 0, s>>>(a);
  else tile_attn_kernel<1, 4, 128, WINDOW, SPLITP><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

// Rows and splits of window chunks by estimated time, in microseconds.  A CU needs
// `full` for a tile of each kind where it has enough workgroups, and a workgroup
// alone `alone`; `ends` tiles' time goes into its beginning and end, and `edge`
// more into the masked tiles of a window's far edge (256 rows: no other workgroup
// shares the CU and covers them).  A further split costs a launch and the rows'
// partial results, written and read once each.
// Measured (us, rows / splits; 32 query and 8 KV heads):
//   8192 tokens                256/1 531  128/1 556   64/1 664
//   8192 tokens, window 1024   128/1 164  256/1 179   64/1 194
//   2048 tokens                128/1  56   64/1  58  256/1  61  128/2  86
//   1024 tokens                 64/1  23  128/1  27  256/1  34   64/2  44
//   512 of 8192 tokens         256/4  83  128/4  89   64/2  99   64/1 112
//   128 of 32768 tokens       256/16  84 128/16  89   64/8  99   64/1 414
//   32 of 16384 tokens         64/16  28 128/32  28   32/8  34   64/8  39
//   8 x 16 of 4096 tokens       64/4  33   32/2  35   64/2  40
TilePlan window_plan(const DenseDims& d) {
  struct Kind {
    int rows, tok;
    double full, alone, ends, edge;
  };
  constexpr Kind kKinds[4] = {{256, 64, 1.94, 1.44, 3.2, 2.},
                              {128, 64, 1.02, 1.25, 3., 0.},
                              {64, 64, 0.62, 0.81, 3., 0.},
                              {32, 128, 1.2, 1.2, 2., 0.}};
  constexpr double kMergeLaunch = 5., kMergeBytes = 4e6;  // us, bytes / us
  const int64_t units = (int64_t)d.n_layers * d.B * d.H_kv, rows = (int64_t)d.T * d.G;
  const int64_t cap = d.L_cap;
  // mean over the query tokens i of min(window, L_cap - T + i + 1)
  const double before = cap > d.T ? (double)(cap - d.T) : 0.;
  const double w = d.window < cap ? (double)d.window : (double)cap;
  const double mean = w <= before ? w
                      : w >= cap  ? before + 0.5 * d.T
                                  : w - 0.5 * (w - before) * (w - before) / d.T;
  TilePlan best{};
  double least = 0.;
  for (const Kind& k : kKinds) {
    TilePlan p{k.rows, k.tok, (int)((rows + k.rows - 1) / k.rows), 1, 0};
    // a row tile covers at most (rows - 2) / G + 2 query tokens
    const int64_t span = (k.rows - 2) / d.G + 1;
    int64_t most = (int64_t)d.window + d.n_sink + span;
    if (most > cap) most = cap;
    double avg = mean + 0.5 * span + d.n_sink;
    if (avg > most) avg = (double)most;
    for (int64_t n = 1; n == 1 || n <= (most + kMinSplit - 1) / kMinSplit; n *= 2) {
      split_tokens(p, most, n);
      const int64_t wgs = units * p.n_rt * p.n_split;
      if (n > 1 && wgs > 4 * kCUs) break;
      const double ends = k.ends + (w < cap ? k.edge : 0.);
      const double longest = p.split_tok / p.tok + ends;
      const double work = avg / p.n_split / p.tok + ends;
      double t = (double)((wgs + kCUs - 1) / kCUs) * work * k.full;
      if (t < longest * k.alone) t = longest * k.alone;
      if (p.n_split > 1)
        t += kMergeLaunch +
             (double)units * (double)rows * p.n_split * (2 * 4 * (kD + 2)) / kMergeBytes;
      if (best.rows == 0 || t < least) {
        best = p;
        least = t;
      }
    }
  }
  return best;
}

// Prefix: units are (layer, KV head), rows the batch's query rows of a unit.  Few
// rows fill the chip by splits of the prefix alone: into a workgroup per CU, or two of 128
// rows, which share one.  us, 2 layers of 20011 tokens, rows of a workgroup / workgroups
// per CU:
//    64 query rows   64/1  49   64/2  59  128/1  58  128/2  55  256/1  70
//    96              64/1  68   64/2  81  128/1  71  128/2  62  256/1  74
//   136              64/2 110             128/1 106  128/2  80  256/1  81  256/2  95
//   256              64/1 111  64/2 120   128/1  99  128/2  93  256/1  91  256/2 115
//   264              64/2 160             128/1 136  128/2 122  256/1 126  256/2 139
TilePlan prefix_plan(const DenseDims& d) {
  const int64_t units = (int64_t)d.n_layers * d.H_kv, rows = (int64_t)d.B * d.G;
  TilePlan p{};
  p.rows = rows > 128 ? 256 : rows > 64 ? 128 : rows > 32 ? 64 : 32;
  p.tok = p.rows == 32 ? 128 : 64;
  p.n_rt = (int)((rows + p.rows - 1) / p.rows);
  const int64_t wgs = units * p.n_rt;
  const int64_t target = p.rows == 128 ? 2 * kCUs : kCUs;
  int64_t ns = (target + wgs - 1) / wgs;
  const int64_t cap = ((int64_t)d.P_cap + kMinSplit - 1) / kMinSplit;
  if (ns > cap) ns = cap;
  split_tokens(p, d.P_cap, ns < 1 ? 1 : ns);
  return p;
}

}  // namespace

size_t window_ws_bytes(const DenseDims& d) {
  const TilePlan p = window_plan(d);
  const int64_t units = (int64_t)d.n_layers * d.B * d.H_kv;
  return p.n_split > 1 ? tile_acc_bytes(units, p) + tile_ml_bytes(units, p) : 0;
}

hipError_t launch_window(const DenseDims& d, const uint16_t* q, const uint16_t* k,
                         const uint16_t* v, const int32_t* lens, const int32_t* q_lens,
                         uint16_t* out, float* lse, void* ws, hipStream_t s) {
  const TilePlan p = window_plan(d);
  const int64_t units = (int64_t)d.n_layers * d.B * d.H_kv;
  TileArgs a{q, k, v, lens, q_lens, out, lse, nullptr, nullptr, d.kv_stride_layer, d.kv_stride_b,
             d.B, d.T, d.H_q, d.H_kv, d.G, d.L_cap, d.window, d.n_sink, (int)units, p.n_rt,
             p.n_split, p.split_tok, d.scale * kLog2e, DecodeArgs{}, 0, 1};
  if (p.n_split > 1) {
    a.part_acc = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + tile_acc_bytes(units, p));
  }
  hipError_t e = launch_tiles<true, false>(p, a, s);
  if (e != hipSuccess || p.n_split == 1) return e;
  const int64_t n_out = (int64_t)d.n_layers * d.B * d.T * d.H_q;
  with_parts(p.n_split, [&](auto S) {
    window_merge_kernel<S.value><<<merge_grid(n_out, S.value), 256, 0, s>>>(a, p.rows, n_out);
  });
  return hipGetLastError();
}

namespace {

// The own tokens' workgroups, of as many wavefronts as the tiles': hb column groups each,
// over n_split of them.  Four groups side by side where that leaves a workgroup per CU,
// and a few chunks to a wavefront (us with four groups, and one: 2 layers of 20011 tokens
// and 16 sequences of 777 64.8 and 67.2, 4 of 16384 and 32 of 512 127 and 138, 4 of 32768
// and 64 of 1024 398 and 409, one of 4096 and 16 of 777 29.0 and 28.4).
struct OwnPlan {
  int hb, n_split;
};
OwnPlan own_plan(const DenseDims& d, const TilePlan& p) {
  const int64_t groups = (int64_t)d.H_kv * (d.G / group_heads(d.G));
  OwnPlan best{1, 1};
  for (int hb = groups % 4 == 0 ? 4 : 1; hb >= 1; hb /= 4) {
    const int64_t wgs = (int64_t)d.n_layers * d.B * groups / hb;
    const int64_t tokens = 4 * kDecodeChunk * (p.rows == 256 ? 8 : 4) / hb;
    const int64_t most = (d.L_cap + tokens - 1) / tokens, n = (kCUs + wgs - 1) / wgs;
    best = {hb, (int)(n < most ? n : most)};
    if (n <= most) break;
  }
  return best;
}
size_t own_acc_bytes(const DenseDims& d, int n_split) {
  return align_up(sizeof(float) * kD * (size_t)d.n_layers * d.B * n_split * d.H_q);
}
size_t own_ml_bytes(const DenseDims& d, int n_split) {
  return align_up(sizeof(float) * 2 * (size_t)d.n_layers * d.B * n_split * d.H_q);
}

}  // namespace

size_t prefix_decode_ws_bytes(const DenseDims& d) {
  const TilePlan p = prefix_plan(d);
  const int64_t units = (int64_t)d.n_layers * d.H_kv;
  const int ns = own_plan(d, p).n_split;
  return tile_acc_bytes(units, p) + tile_ml_bytes(units, p) + own_acc_bytes(d, ns) +
         own_ml_bytes(d, ns);
}

hipError_t launch_prefix_decode(const DenseDims& d, const uint16_t* q, const uint16_t* k_prefix,
                                const uint16_t* v_prefix, const int32_t* prefix_len,
                                const uint16_t* k, const uint16_t* v, const int32_t* lens,
                                float* out, float* lse, void* ws, hipStream_t s) {
  const TilePlan p = prefix_plan(d);
  const int64_t units = (int64_t)d.n_layers * d.H_kv;
  const OwnPlan own = own_plan(d, p);
  const int heads = group_heads(d.G), R = d.G / heads, ns = own.n_split;
  char* w = static_cast<char*>(ws);
  TileArgs a{q, k_prefix, v_prefix, prefix_len, nullptr, nullptr, nullptr,
             reinterpret_cast<float*>(w), reinterpret_cast<float*>(w + tile_acc_bytes(units, p)),
             d.prefix_stride_layer, 0, 1, d.B, d.H_q, d.H_kv, d.G, d.P_cap, 0, 0, (int)units,
             p.n_rt, p.n_split, p.split_tok, d.scale * kLog2e, DecodeArgs{}, 0, 1};
  w += tile_acc_bytes(units, p) + tile_ml_bytes(units, p);
  a.own = DecodeArgs{q, k, v, lens, nullptr, nullptr, reinterpret_cast<float*>(w),
                     reinterpret_cast<float*>(w + own_acc_bytes(d, ns)), nullptr, nullptr,
                     d.kv_stride_layer, d.kv_stride_b, 0, d.B, d.H_q, d.H_kv, heads, R, d.L_cap,
                     d.L_cap, d.L_cap, ns, 0, d.scale * kLog2e};
  a.own_blocks = (int)((int64_t)d.n_layers * d.B * d.H_kv * R / own.hb * ns);
  a.own_hb = own.hb;
  const hipError_t e = launch_tiles<false, true>(p, a, s);
  if (e != hipSuccess) return e;
  const int64_t n_out = (int64_t)d.n_layers * d.B * d.H_q;
  with_parts(p.n_split + ns, [&](auto S) {
    prefix_merge_kernel<S.value><<<merge_grid(n_out, S.value), 256, 0, s>>>(a, p.rows, out, lse,
                                                                           n_out);
  });
  return hipGetLastError();
}

}  // namespace spec
