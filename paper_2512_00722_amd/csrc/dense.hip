// Decode attention over caches that are read in full: a sliding window with sinks,
// and with the weights added up per token.
//
// Workgroups of four wavefronts take one, two or four column groups (layer,
// sequence, KV head, at most 16 query heads) or one of n_split parts of them
// (dense_core.h).  The kernel is bound by memory; what a launch reaches of it depends
// on two things (DecodePlan): one workgroup per CU, and wavefronts side by side on
// the KV heads of the same tokens, whose rows share DRAM pages.
#include "dense_core.h"

namespace spec {
namespace {

constexpr int kW = 4;

template <int HB, int KEEP, bool HALF>
__global__ __launch_bounds__(kW * 64) __attribute__((amdgpu_waves_per_eu(2)))
void decode_kernel(DecodeArgs a) {
  extern __shared__ __align__(16) float lds_logits[];
  __shared__ __align__(16) uint16_t tiles[kW][tile_elems(HALF)];
  __shared__ float2 ml[kW][16];
  decode_block<kW, HB, KEEP, HALF>(a, blockIdx.x, tiles, ml, lds_logits);
}

// 8 / S output rows per workgroup, 32 threads (4 dimensions each) and S of them.
template <int S>
__device__ __forceinline__ void decode_merge(const DecodeArgs& a, int block, float* out,
                                             float* lse, int64_t n_out) {
  const int64_t want = (int64_t)block * (8 / S) + (threadIdx.x >> 5) / S;
  const int64_t orow = want < n_out ? want : n_out - 1;
  const int d4 = threadIdx.x & 31;
  const int h = (int)(orow % a.H_q);
  const int64_t lb = orow / a.H_q;
  const Join j = join_parts<S>(a.n_split, [&](int s, const float2*& ml, const float*& acc) {
    const size_t prow = ((size_t)lb * a.n_split + s) * a.H_q + h;
    ml = reinterpret_cast<const float2*>(a.part_ml) + prow;
    acc = a.part_acc + prow * kHeadDim;
  });
  if (want >= n_out || (threadIdx.x >> 5) % S != 0) return;
  const float inv = j.inv();
  reinterpret_cast<float4*>(out + orow * kHeadDim)[d4] =
      make_float4(j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv);
  if (lse && d4 == 0) lse[orow] = j.lse();
}
template <int S>
__global__ __launch_bounds__(256) void decode_merge_kernel(DecodeArgs a, float* out, float* lse,
                                                           int64_t n_out) {
  decode_merge<S>(a, blockIdx.x, out, lse, n_out);
}

// A workgroup's threads are PARTS parts of a set's rows by 256 / PARTS groups of
// four tokens.
constexpr int accum_tokens(int parts) { return 4 * 256 / parts; }
constexpr int kAccumMerge = 4;  // parts of decode_merge in the same launch

struct AccumArgs {
  const float* rows;    // [lb][n_rows][stride]: logits (log2 units), or weights (lse null)
  const float* lse;     // [lb][n_rows]
  const int32_t* counts;
  float* weights;       // [lb][n_sets][L_cap]
  int64_t stride;
  int B, n_rows, n_sets, L_cap, tiles;  // tiles: workgroups of a weights row
  // Logits of a pass in parts: the first workgroups join its results, and the others
  // its sums for themselves, which saves a launch (24 units of 1500 tokens: 10.0 us, 12.3
  // with it).
  int merge_blocks;     // 0: one part
  DecodeArgs of;
  float* out;
  float* out_lse;
  int64_t n_out;
};

// weights[lb][set][t] += sum over the set's rows of the weight, 2^(logit - lse log2(e)),
// in a fixed order.  A thread has four tokens of every PARTS-th row, four of them
// requested together; the parts are added in LDS.
template <int PARTS>
__global__ __launch_bounds__(256) void accum_kernel(AccumArgs a) {
  constexpr int TOK = accum_tokens(PARTS);
  constexpr int ROWS = 4 * PARTS;       // rows at a time
  constexpr int LANES = 256 / ROWS;     // that join a row's sums
  __shared__ float4 sums[PARTS][TOK / 4];
  __shared__ float z_lds[ROWS];
  if ((int)blockIdx.x < a.merge_blocks) {
    decode_merge<kAccumMerge>(a.of, blockIdx.x, a.out, a.out_lse, a.n_out);
    return;
  }
  const int block = blockIdx.x - a.merge_blocks;
  const int tile = block % a.tiles, rest = block / a.tiles;
  const int set = rest % a.n_sets, lb = rest / a.n_sets;
  const int count = clampi(a.counts[lb % a.B], 0, a.L_cap);
  if (tile * TOK >= count) return;  // uniform
  const int t4 = threadIdx.x % (TOK / 4), part = threadIdx.x / (TOK / 4);
  const int t0 = tile * TOK + t4 * 4;
  const int rows = a.n_rows / a.n_sets;
  const size_t r0 = (size_t)lb * a.n_rows + (size_t)set * rows;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int h0 = 0; h0 < rows; h0 += ROWS) {
    float4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const size_t r = r0 + min(h0 + part + PARTS * u, rows - 1);
      x[u] = *reinterpret_cast<const float4*>(a.rows + r * a.stride + min(t0, count - 1) / 4 * 4);
    }
    if (a.lse) {  // the rows' sums, in log2 units; +inf where there are no weights
      const int h = set * rows + min(h0 + (int)threadIdx.x / LANES, rows - 1);
      float m = kNoMax, l = 0.f;
      if (a.merge_blocks > 0) {
        const float2* ml = reinterpret_cast<const float2*>(a.of.part_ml) +
                           (size_t)lb * a.of.n_split * a.n_rows + h;
        for (int s = threadIdx.x % LANES; s < a.of.n_split; s += LANES) {
          const float2 x = ml[(size_t)s * a.n_rows];
          const float mn = fmaxf(m, x.x);
          l = l * exp2f(m - mn) + x.y * exp2f(x.x - mn);
          m = mn;
        }
#pragma unroll
        for (int o = 1; o < LANES; o *= 2) {
          const float m1 = __shfl_xor(m, o), l1 = __shfl_xor(l, o), mn = fmaxf(m, m1);
          l = l * exp2f(m - mn) + l1 * exp2f(m1 - mn);
          m = mn;
        }
        m += log2f(l);
      } else {
        m = a.lse[(size_t)lb * a.n_rows + h] * kLog2e;
      }
      __syncthreads();
      if (threadIdx.x % LANES == 0) z_lds[threadIdx.x / LANES] = m == -INFINITY ? INFINITY : m;
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (h0 + part + PARTS * u >= rows) continue;
      const float z = z_lds[part + PARTS * u];
      sum.x += a.lse ? exp2f(x[u].x - z) : x[u].x;
      sum.y += a.lse ? exp2f(x[u].y - z) : x[u].y;
      sum.z += a.lse ? exp2f(x[u].z - z) : x[u].z;
      sum.w += a.lse ? exp2f(x[u].w - z) : x[u].w;
    }
  }
  sums[part][t4] = sum;
  __syncthreads();
  float* row = a.weights + ((size_t)lb * a.n_sets + set) * a.L_cap;
  for (int t = threadIdx.x; t < TOK && tile * TOK + t < count; t += 256) {
    float add = 0.f;
    for (int p = 0; p < PARTS; ++p) add += reinterpret_cast<const float*>(sums[p])[t];
    row[tile * TOK + t] += add;
  }
}

hipError_t launch_accum(AccumArgs a, int64_t lb, hipStream_t s) {
  const int rows = a.n_rows / a.n_sets;
  const int parts = rows >= 16 ? 16 : rows >= 4 ? 4 : 1;
  a.tiles = (a.L_cap + accum_tokens(parts) - 1) / accum_tokens(parts);
  const int64_t blocks = (int64_t)a.tiles * a.n_sets * lb + a.merge_blocks;
  if (blocks > UINT32_MAX / 256) return hipErrorInvalidValue;  // threads of a launch
  const dim3 grid((unsigned)blocks);
  if (parts == 16) accum_kernel<16><<<grid, 256, 0, s>>>(a);
  else if (parts == 4) accum_kernel<4><<<grid, 256, 0, s>>>(a);
  else accum_kernel<1><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

// How a launch is divided: hb column groups per workgroup, each over n_split of them.
struct DecodePlan {
  int hb, n_split;
};

int64_t decode_units(const DenseDims& d) {
  return (int64_t)d.n_layers * d.B * d.H_kv * (d.G / group_heads(d.G));
}

// The largest of 4, 2, 1 that divides the column groups and is at most `most`.
int groups_per_block(const DenseDims& d, int64_t most) {
  const int64_t n = (int64_t)d.H_kv * (d.G / group_heads(d.G));
  return n % 4 == 0 && most >= 4 ? 4 : n % 2 == 0 && most >= 2 ? 2 : 1;
}

// One workgroup per CU is the best number throughout (us, 8 KV heads, bf16; 8 to 1024
// units of 256 to 16384 tokens were measured with 1, 2, 4 groups per workgroup and 1
// to 8 workgroups per CU): 64 units x 4096 tokens 26.0, with two per CU 28.4; 1024 x
// 2048 155.8, two 165.7, four 181.1.  Four groups beside each other are faster where a
// CU has some 400 tokens or more, as a wavefront then has several chunks: 128 x 1024
// 16.3 against 18.3 with one, 1024 x 2048 155.8 against 194.7; but 64 x 1024 12.1
// against 11.5.  Parts cost a merge of about 3.5 us, so that launches which fill the
// CUs with fewer groups per workgroup and no parts take those up to some 40 us (512
// x 256: 13.9 against 16.2), and short selections are not divided (8 x 256: 7.3
// against 8.0).
DecodePlan decode_plan(const DenseDims& d, int k_max) {
  const int64_t units = decode_units(d);
  const double per_cu = (double)units * k_max / kCUs;  // tokens
  const int64_t chunks = (k_max + kDecodeChunk - 1) / kDecodeChunk;
  if (per_cu < 400) {
    const int64_t most = (chunks + kW - 1) / kW;  // a chunk per wavefront at least
    int64_t n = kCUs / units;
    if (n > most) n = most;
    return {1, n < 2 || k_max <= 320 ? 1 : (int)n};
  }
  const int hb0 = groups_per_block(d, units / kCUs);
  if (per_cu < 1500 && units >= kCUs) return {hb0, 1};
  // Rounds of workgroups per CU: a last one that is not full, and more than one.
  const int hb = groups_per_block(d, 4);
  const int64_t most = (chunks + kW / hb - 1) / (kW / hb);
  const double time = (double)units * k_max / 12890;  // us at 6.6 TB/s
  double best = 1e30;
  DecodePlan p{hb, 1};
  for (int64_t n = 1; n <= most && units / hb * n <= 16 * kCUs + units / hb; ++n) {
    const int64_t wgs = units / hb * n, rounds = (wgs + kCUs - 1) / kCUs;
    const double cost = time * rounds * kCUs / wgs * (1 + 0.05 * (rounds < 4 ? rounds - 1 : 3)) +
                        (n > 1 ? 3.5 : 0);
    if (cost < best) {
      best = cost;
      p.n_split = (int)n;
    }
  }
  return p;
}
size_t part_acc_bytes(const DenseDims& d, int n_split) {
  return n_split > 1 ? align_up(sizeof(float) * kHeadDim * (size_t)d.n_layers * d.B * n_split *
                                d.H_q)
                     : 0;
}
size_t part_ml_bytes(const DenseDims& d, int n_split) {
  return n_split > 1 ? align_up(sizeof(float) * 2 * (size_t)d.n_layers * d.B * n_split * d.H_q)
                     : 0;
}

DecodeArgs decode_args(const DenseDims& d, int k_max, int n_sink, int n_split, const uint16_t* q,
                       const uint16_t* k, const uint16_t* v, const int32_t* lens, float* out,
                       float* lse, char* ws) {
  const int heads = group_heads(d.G);
  DecodeArgs a{q, k, v, lens, out, lse, nullptr, nullptr, nullptr, nullptr, d.kv_stride_layer,
               d.kv_stride_b, 0, d.B, d.H_q, d.H_kv, heads, d.G / heads, d.L_cap, k_max, n_sink,
               n_split, 0, d.scale * kLog2e};
  if (n_split > 1) {
    a.out = nullptr;
    a.part_acc = reinterpret_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(ws + part_acc_bytes(d, n_split));
  }
  return a;
}

// lds: bytes of a column group's logits (kKeepWeights: with four groups the V tiles
// are of 16 tokens, which leaves the LDS to the logits).
template <int KEEP>
hipError_t launch_decode(const DenseDims& d, const DecodeArgs& a, int hb, size_t lds,
                         hipStream_t s) {
  const int64_t blocks = decode_units(d) / hb * a.n_split;
  if (blocks > INT32_MAX / (kW * 64)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks), block(kW * 64);
  if (hb == 1) decode_kernel<1, KEEP, false><<<grid, block, lds, s>>>(a);
  else if (hb == 2) decode_kernel<2, KEEP, false><<<grid, block, 2 * lds, s>>>(a);
  else if constexpr (KEEP == kKeepWeights)
    decode_kernel<4, KEEP, true><<<grid, block, 4 * lds, s>>>(a);
  else decode_kernel<4, KEEP, false><<<grid, block, 4 * lds, s>>>(a);
  return hipGetLastError();
}

int window_tokens(const DenseDims& d) {
  const int64_t n = (int64_t)d.window + d.n_sink;
  return (int)(n < d.L_cap ? n : d.L_cap);
}

// Where the logits stay until their sums are known: in the LDS of the workgroup that
// has them all (no parts), or in memory.  us, 8 KV heads: 128 sequences and layers of
// 2048 tokens, 4 query heads each: four groups per workgroup 166, two 186, one 208,
// memory 229; of 4000 tokens 356 (two), 420, memory 450; 16 query heads each, 512 tokens:
// 52, 60, 61, memory 76.  Rates of a CU (GB/s) from those; fewer workgroups than CUs
// leave it idle, so that small launches go through memory in parts.
struct AccumPlan {
  DecodePlan plan;
  bool in_lds;    // else the logits go through memory
  bool in_place;  // in_lds: a set is one unit, which adds to the weights itself
};
size_t logit_lds(const DenseDims& d) {
  return sizeof(float) * group_heads(d.G) * logit_pitch(d.L_cap);
}
AccumPlan accum_plan(const DenseDims& d) {
  constexpr size_t kLds = 160 * 1024, kRest = 2 * 1024;  // of a CU; beside tiles and logits
  AccumPlan p{decode_plan(d, d.L_cap), false, false};
  const int64_t units = decode_units(d);
  const double bytes = 512.0 * d.L_cap;  // of a unit
  double best = units * bytes / 4.7e6 + 8;  // us, through memory
  for (int hb = groups_per_block(d, 4); hb >= 1; hb /= 2) {
    const size_t lds = hb * logit_lds(d) +
                       kW * sizeof(uint16_t) * tile_elems(hb == 4) + kRest;
    if (lds > kLds) continue;
    const int64_t wgs = units / hb, per_cu = hb == 4 ? 1 : lds <= kLds / 2 ? 2 : 1;
    const int64_t rounds = (wgs + kCUs * per_cu - 1) / (kCUs * per_cu);
    const double cu = hb == 4 ? 26e3 : hb == 2 ? 23e3 : 20.5e3;  // bytes per us
    const double time = rounds * per_cu * hb * bytes / cu + 5;
    if (time < best) {
      best = time;
      p.plan = {hb, 1};
      p.in_lds = true;
    }
  }
  p.in_place = p.in_lds && d.n_sets == d.H_kv && d.G == group_heads(d.G);
  return p;
}
int64_t accum_stride(const DenseDims& d) { return ((int64_t)d.L_cap + 31) / 32 * 32; }
// Logits [lb][H_q], or the units' weights [lb][H_kv R].
size_t accum_row_bytes(const DenseDims& d, const AccumPlan& p) {
  if (p.in_place) return 0;
  const int64_t rows = p.in_lds ? (int64_t)d.H_kv * (d.G / group_heads(d.G)) : d.H_q;
  return align_up(sizeof(float) * (size_t)d.n_layers * d.B * rows * accum_stride(d));
}
size_t accum_lse_bytes(const DenseDims& d) {
  return align_up(sizeof(float) * (size_t)d.n_layers * d.B * d.H_q);
}

}  // namespace

size_t window_decode_ws_bytes(const DenseDims& d) {
  const int n = decode_plan(d, window_tokens(d)).n_split;
  return part_acc_bytes(d, n) + part_ml_bytes(d, n);
}

hipError_t launch_window_decode(const DenseDims& d, const uint16_t* q, const uint16_t* k,
                                const uint16_t* v, const int32_t* lens, float* out, float* lse,
                                void* ws, hipStream_t s) {
  const int k_max = window_tokens(d);
  const DecodePlan p = decode_plan(d, k_max);
  const DecodeArgs a = decode_args(d, k_max, d.n_sink, p.n_split, q, k, v, lens, out, lse,
                                   static_cast<char*>(ws));
  const hipError_t e = launch_decode<kKeepNone>(d, a, p.hb, 0, s);
  if (e != hipSuccess || p.n_split == 1) return e;
  const int64_t n_out = (int64_t)d.n_layers * d.B * d.H_q;
  with_parts(p.n_split, [&](auto S) {
    decode_merge_kernel<S.value><<<merge_grid(n_out, S.value), 256, 0, s>>>(a, out, lse, n_out);
  });
  return hipGetLastError();
}

size_t accum_decode_ws_bytes(const DenseDims& d) {
  const AccumPlan p = accum_plan(d);
  return accum_row_bytes(d, p) + accum_lse_bytes(d) + part_acc_bytes(d, p.plan.n_split) +
         part_ml_bytes(d, p.plan.n_split);
}

hipError_t launch_accum_decode(const DenseDims& d, const uint16_t* q, const uint16_t* k,
                               const uint16_t* v, const int32_t* counts, float* weights,
                               float* out, float* lse, void* ws, hipStream_t s) {
  const AccumPlan p = accum_plan(d);
  char* w = static_cast<char*>(ws);
  float* rows = reinterpret_cast<float*>(w);
  w += accum_row_bytes(d, p);
  float* z = lse ? lse : reinterpret_cast<float*>(w);
  w += accum_lse_bytes(d);
  DecodeArgs a = decode_args(d, d.L_cap, d.L_cap, p.plan.n_split, q, k, v, counts, out, z, w);
  a.logit_stride = accum_stride(d);
  const int64_t lb = (int64_t)d.n_layers * d.B;
  if (p.in_lds) {
    a.add_weights = p.in_place;
    a.weights = p.in_place ? weights : rows;
    const hipError_t e = launch_decode<kKeepWeights>(d, a, p.plan.hb, logit_lds(d), s);
    if (e != hipSuccess || p.in_place) return e;
    return launch_accum({rows, nullptr, counts, weights, a.logit_stride, d.B, d.H_kv * a.R,
                         d.n_sets, d.L_cap, 0, 0, a, nullptr, nullptr, 0}, lb, s);
  }
  a.logits = rows;
  const hipError_t e = launch_decode<kKeepLogits>(d, a, p.plan.hb, 0, s);
  if (e != hipSuccess) return e;
  const int64_t n_out = lb * d.H_q;
  const int merge = p.plan.n_split > 1 ? (int)merge_grid(n_out, kAccumMerge).x : 0;
  return launch_accum({rows, z, counts, weights, a.logit_stride, d.B, d.H_q, d.n_sets, d.L_cap, 0,
                       merge, a, out, lse, n_out}, lb, s);
}

}  // namespace spec
