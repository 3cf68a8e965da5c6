// New rows into caches held in 4 or 8 bits, and rows back to bf16.
//
// Both are bound by memory: 5.6 to 6.6 TB/s of what they read and write in calls of 680 to 990
// MB, one after another on two sets of buffers in turn (as all times here; calls on one set
// find some of it in the caches).  A thread has eight elements of K and the same eight of V
// (one 16-byte bf16 load or store each), four threads a group, sixteen a row of a head.
#include "quant_core.h"

namespace spec {
namespace {

constexpr int kRowThreads = 16;               // of a row of a head
constexpr int kThreads = 256;
constexpr int kBlockRows = kThreads / kRowThreads;  // rows at a time
// Rows of a thread, whose loads are all in flight: two when writing the caches (8 layers x 2
// x 8192 tokens x 8 KV heads in 4 bits 114 us, one 111, four 115; in 8 bits 141, 136, 143;
// with the rows read back 205, 203, 206 and 265, 265, 264), one when reading them (8 x 8 x 2048
// selected rows in 4 bits 121, two 125, four 123; in 8 bits 142, 145, 146; 4 x 2 x 20011 rows in
// order 126, 135, 140 and 158, 161, 161).
constexpr int kAppendRows = 2;
constexpr int kReadRows = 1;

struct QuantIoArgs {
  uint8_t* k;
  uint8_t* v;
  uint8_t* scales;
  const uint16_t* k_in;   // append: new rows
  const uint16_t* v_in;
  uint16_t* k_out;        // read
  uint16_t* v_out;
  const int32_t* idx;     // read: [B][n_sets][rows] or null
  const int32_t* n;       // [B] rows of a sequence; null: all
  const int32_t* pos;     // append: [B]
  int64_t kv_stride_layer, kv_stride_b, scale_stride_layer, scale_stride_b;
  int B, n_lb, L_cap, H_kv, rows, n_sets;  // n_lb: layers x sequences; rows: T or k_max
};

template <int BITS>
__device__ __forceinline__ uint2 quantise8(const uint4& x, float scale) {
  uint2 r = make_uint2(0, 0);
  if constexpr (BITS == 4) {
    r.x = elements2<4, 0>(r.x, x.x, scale);
    r.x = elements2<4, 1>(r.x, x.y, scale);
    r.x = elements2<4, 2>(r.x, x.z, scale);
    r.x = elements2<4, 3>(r.x, x.w, scale);
  } else {
    r.x = elements2<8, 0>(r.x, x.x, scale);
    r.x = elements2<8, 1>(r.x, x.y, scale);
    r.y = elements2<8, 0>(r.y, x.z, scale);
    r.y = elements2<8, 1>(r.y, x.w, scale);
  }
  return r;
}

// Largest magnitude (bf16 bits) of the eight elements of each of a quad's threads.
__device__ __forceinline__ uint32_t quad_top(const uint4& x) {
  typedef uint16_t ushortx2 __attribute__((ext_vector_type(2)));
  auto mag = [](uint32_t w) { return __builtin_bit_cast(ushortx2, w & 0x7fff7fffu); };
  ushortx2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(x.x), mag(x.y)),
                                         __builtin_elementwise_max(mag(x.z), mag(x.w)));
  uint32_t t = m[0] > m[1] ? m[0] : m[1];
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xf, 0xf, false);
  t = t > o ? t : o;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xf, 0xf, false);
  return t > o ? t : o;
}

template <int BITS>
__device__ __forceinline__ void store8(uint8_t* row, int piece, const uint2& e) {
  if constexpr (BITS == 4) reinterpret_cast<uint32_t*>(row)[piece] = e.x;
  else reinterpret_cast<uint2*>(row)[piece] = e;
}

// Rows (token, head) of a sequence's new tokens stand in the caches as they come, from
// token pos on: those inside the caches are one range of rows.  STREAM: new rows that the
// caches do not hold are loaded past them (537 MB of them in 4 bits: 114 us, through the caches
// 121, and with the rows read back 205 and 226; in 8 bits 141 and 141, 265 and 280);
// others, which the program has just made, through them.  The rows are stored through the
// caches: past them the call takes 3% less (in 8 bits 10%), and reading the rows afterwards 15%
// more (10%).
template <int BITS, bool STREAM>
__global__ __launch_bounds__(kThreads) void append_kernel(QuantIoArgs a) {
  const int lb = blockIdx.z * gridDim.y + blockIdx.y;
  if (lb >= a.n_lb) return;
  const int layer = lb / a.B, b = lb % a.B;
  const int64_t pos = a.pos[b];
  const int n = a.n ? clampi(a.n[b], 0, a.rows) : a.rows;
  const int64_t lo = (pos < 0 ? -pos : 0) * a.H_kv;
  const int64_t hi = (pos + n < a.L_cap ? n : a.L_cap - pos) * a.H_kv;
  const int piece = threadIdx.x % kRowThreads;
  const int64_t r0 = (int64_t)blockIdx.x * (kBlockRows * kAppendRows) + threadIdx.x / kRowThreads;
  const int64_t in0 = (int64_t)lb * a.rows * a.H_kv * kHeadDim + 8 * piece;
  uint4 k[kAppendRows], v[kAppendRows];
#pragma unroll
  for (int u = 0; u < kAppendRows; ++u) {
    const int64_t r = r0 + u * kBlockRows;
    if (r < lo || r >= hi) continue;
    const uint16_t *kp = a.k_in + in0 + r * kHeadDim, *vp = a.v_in + in0 + r * kHeadDim;
    k[u] = STREAM ? ldg16_stream(kp) : ldg16(kp);
    v[u] = STREAM ? ldg16_stream(vp) : ldg16(vp);
  }
#pragma unroll
  for (int u = 0; u < kAppendRows; ++u) {
    const int64_t r = r0 + u * kBlockRows;
    if (r < lo || r >= hi) continue;  // uniform over a row's threads
    const int64_t to = pos * a.H_kv + r;  // row of the sequence's caches
    const int64_t at = layer * a.kv_stride_layer + b * a.kv_stride_b + to * row_bytes(BITS);
    const int ks = scale_byte<BITS>(quad_top(k[u])), vs = scale_byte<BITS>(quad_top(v[u]));
    store8<BITS>(a.k + at, piece, quantise8<BITS>(k[u], scale_of(ks, 0)));
    store8<BITS>(a.v + at, piece, quantise8<BITS>(v[u], scale_of(vs, 0)));
    if ((piece & 3) < 2)  // the first thread of a group has K's scale, the second V's
      a.scales[layer * a.scale_stride_layer + b * a.scale_stride_b + to * kScaleBytes +
               4 * (piece & 3) + piece / 4] = (uint8_t)((piece & 3) == 0 ? ks : vs);
  }
}

template <int BITS>
__device__ __forceinline__ uint2 load8(const uint8_t* row, int piece) {
  if constexpr (BITS == 4) return make_uint2(reinterpret_cast<const uint32_t*>(row)[piece], 0);
  else return reinterpret_cast<const uint2*>(row)[piece];
}

template <int BITS>
__device__ __forceinline__ uint4 values8(const uint2& e, float scale) {
  RowPart<BITS> p{};
  p.w[0].x = e.x;
  p.w[0].y = e.y;
  return __builtin_bit_cast(uint4, elements8<BITS>(p, 0, scale));
}

// A 16-byte store past the caches: in 4 bits 8 layers x 8 x 2048 selected rows take 121 us,
// with ordinary stores 130, one layer of them 14.3 and 16.2, one layer and the attention that
// reads the outputs next 32.6 and 37.0; in 8 bits 142 and 159, 16.9 and 18.6, 35.1 and 37.5.
__device__ __forceinline__ void store_stream(uint16_t* p, const uint4& x) {
  typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(uintx4{x.x, x.y, x.z, x.w}, reinterpret_cast<uintx4*>(p));
}

template <int BITS, bool INDEXED>
__global__ __launch_bounds__(kThreads) void read_kernel(QuantIoArgs a) {
  const int lb = blockIdx.z * gridDim.y + blockIdx.y;
  if (lb >= a.n_lb) return;
  const int layer = lb / a.B, b = lb % a.B;
  const int64_t hi = (int64_t)clampi(a.n[b], 0, a.rows) * a.H_kv;
  const int piece = threadIdx.x % kRowThreads;
  const int64_t b0 = (int64_t)blockIdx.x * (kBlockRows * kReadRows);
  const int64_t r0 = b0 + threadIdx.x / kRowThreads;
  if (b0 >= hi) return;  // uniform
  const int64_t kv0 = layer * a.kv_stride_layer + b * a.kv_stride_b;
  const int64_t s0 = layer * a.scale_stride_layer + b * a.scale_stride_b;
  int64_t from[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int64_t r = r0 + u * kBlockRows;
    from[u] = r < hi ? r : hi - 1;
    if (INDEXED) {
      const int64_t j = from[u] / a.H_kv;
      const int g = (int)(from[u] - j * a.H_kv), s = a.n_sets == 1 ? 0 : g;
      from[u] = (int64_t)clampi(a.idx[((int64_t)b * a.n_sets + s) * a.rows + j], 0, a.L_cap - 1) *
                    a.H_kv + g;
    }
  }
  uint2 k[kReadRows], v[kReadRows];
  uint8_t ks[kReadRows], vs[kReadRows];
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    k[u] = load8<BITS>(a.k + kv0 + from[u] * row_bytes(BITS), piece);
    v[u] = load8<BITS>(a.v + kv0 + from[u] * row_bytes(BITS), piece);
    ks[u] = a.scales[s0 + from[u] * kScaleBytes + piece / 4];
    vs[u] = a.scales[s0 + from[u] * kScaleBytes + 4 + piece / 4];
  }
  const int64_t out0 = (int64_t)lb * a.rows * a.H_kv * kHeadDim + 8 * piece;
#pragma unroll
  for (int u = 0; u < kReadRows; ++u) {
    const int64_t r = r0 + u * kBlockRows;
    if (r >= hi) continue;
    store_stream(a.k_out + out0 + r * kHeadDim, values8<BITS>(k[u], scale_of(ks[u], 0)));
    store_stream(a.v_out + out0 + r * kHeadDim, values8<BITS>(v[u], scale_of(vs[u], 0)));
  }
}

QuantIoArgs io_args(const QuantDims& d, const QuantCache& c, int rows) {
  QuantIoArgs a{};
  a.k = c.k;
  a.v = c.v;
  a.scales = c.scales;
  a.kv_stride_layer = d.kv_stride_layer;
  a.kv_stride_b = d.kv_stride_b;
  a.scale_stride_layer = d.scale_stride_layer;
  a.scale_stride_b = d.scale_stride_b;
  a.B = d.B;
  a.L_cap = d.L_cap;
  a.H_kv = d.H_kv;
  a.n_lb = d.n_layers * d.B;
  a.rows = rows;
  a.n_sets = d.n_sets;
  return a;
}

dim3 io_grid(const QuantDims& d, int rows, int thread_rows) {
  const int64_t per_block = kBlockRows * thread_rows, lb = (int64_t)d.n_layers * d.B;
  const int64_t y = lb < 32768 ? lb : 32768;
  return dim3((unsigned)(((int64_t)rows * d.H_kv + per_block - 1) / per_block), (unsigned)y,
              (unsigned)((lb + y - 1) / y));
}

}  // namespace

int64_t quant_io_blocks(const QuantDims& d, int rows) {
  return ((int64_t)rows * d.H_kv + kBlockRows - 1) / kBlockRows;
}

hipError_t launch_quant_append(const QuantDims& d, const QuantCache& c, const uint16_t* k_new,
                               const uint16_t* v_new, const int32_t* pos, const int32_t* n_new,
                               hipStream_t s) {
  QuantIoArgs a = io_args(d, c, d.T);
  a.k_in = k_new;
  a.v_in = v_new;
  a.n = n_new;
  a.pos = pos;
  const bool stream = (int64_t)d.n_layers * d.B * d.T * d.H_kv * kHeadDim * 4 > 64 << 20;
  const dim3 grid = io_grid(d, d.T, kAppendRows);
  if (d.bits == 4) {
    if (stream) append_kernel<4, true><<<grid, kThreads, 0, s>>>(a);
    else append_kernel<4, false><<<grid, kThreads, 0, s>>>(a);
  } else {
    if (stream) append_kernel<8, true><<<grid, kThreads, 0, s>>>(a);
    else append_kernel<8, false><<<grid, kThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_quant_read(const QuantDims& d, const QuantCache& c, const int32_t* idx,
                             const int32_t* counts, uint16_t* k_out, uint16_t* v_out,
                             hipStream_t s) {
  QuantIoArgs a = io_args(d, c, d.k_max);
  a.k_out = k_out;
  a.v_out = v_out;
  a.idx = idx;
  a.n = counts;
  const dim3 grid = io_grid(d, d.k_max, kReadRows);
  if (d.bits == 4) {
    if (idx) read_kernel<4, true><<<grid, kThreads, 0, s>>>(a);
    else read_kernel<4, false><<<grid, kThreads, 0, s>>>(a);
  } else {
    if (idx) read_kernel<8, true><<<grid, kThreads, 0, s>>>(a);
    else read_kernel<8, false><<<grid, kThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace spec
