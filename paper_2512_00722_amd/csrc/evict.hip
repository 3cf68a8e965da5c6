// Insertion into a bounded cache, evicting by accumulated attention weight.
//
// Per token set (layer, sequence, KV head or all heads) with c rows held, n new
// rows and a budget of k: C' = min(k, c + n) rows remain, the n' = min(n, C') last
// of the new ones among them, so E = C' - n' of the rows held: those that are
// protected (recent tokens and sinks), then the largest weights, ties to the lower
// slot.  Rows that stay keep their slot.  The slots below C' that hold none of
// them are filled, ascending: first by kept rows that stand at C' or above
// (ascending), then by the new rows in order.  Sources lie at C' or above or in the
// new rows, destinations below C', so the moves are independent of each other,
// and a full cache that takes n new rows writes n rows.
//
// The plan reads 8 bytes per slot (weight and token) and selects in LDS: a radix
// search for the E-th largest key.  One workgroup does a set, as the sets of a
// model's layers, sequences and heads are many.
#include "device_common.h"
#include "internal.h"
#include "select_common.h"

namespace spec {
namespace {

constexpr int kLdsKeys = 16384;  // slots whose keys fit the workgroup's LDS (64 KiB)

struct PlanArgs {
  const float* weights;    // [sets][L_cap]
  const int32_t* tokens;   // [sets][L_cap]
  const int32_t* counts;   // [B]
  const int32_t* keep;     // [B]
  const int32_t* pos;      // [B]
  const int32_t* n_new;    // [B] or null (T)
  int4* head;              // [sets]: slots filled, of them from the cache, first new row, C'
  int32_t* dst;            // [sets][L_cap] slots filled, ascending
  int32_t* src;            // [sets][L_cap] kept slots at C' or above, ascending
  int B, n_sets, L_cap, T, n_recent, n_sink;
};

// Protected rows count as +inf; NaN ranks with -inf, -0 with +0.
__device__ __forceinline__ uint32_t rank_key(float w, int32_t tok, int64_t recent_from,
                                             int n_sink) {
  if (tok >= recent_from || tok < n_sink) w = INFINITY;
  return order_key(w != w ? -INFINITY : w + 0.f);
}

template <int NT>
__global__ __launch_bounds__(NT) void evict_plan_kernel(PlanArgs a) {
  extern __shared__ uint32_t keys[];  // of all held slots, where they fit
  __shared__ int hist[256];
  __shared__ int sh[2 * NT / 64];
  __shared__ int sel[3];
  const int set = blockIdx.x;
  const int b = (set / a.n_sets) % a.B;
  const int tid = threadIdx.x;
  const int c = clampi(a.counts[b], 0, a.L_cap);
  const int n = a.n_new ? clampi(a.n_new[b], 0, a.T) : a.T;
  const int k = clampi(a.keep[b], 0, a.L_cap);
  const int after = (int)min((int64_t)k, (int64_t)c + n);
  const int taken = min(n, after);
  const int E = after - taken;  // rows held that stay, E <= c
  const float* w = a.weights + (size_t)set * a.L_cap;
  const int32_t* tok = a.tokens + (size_t)set * a.L_cap;
  int32_t* dst = a.dst + (size_t)set * a.L_cap;
  int32_t* src = a.src + (size_t)set * a.L_cap;
  const int64_t recent_from = (int64_t)a.pos[b] + n - a.n_recent;

  if (E == c || E == 0) {  // all stay, or none: no selection
    for (int i = tid; i < taken; i += NT) dst[i] = E + i;
    if (tid == 0) a.head[set] = make_int4(taken, 0, n - taken, after);
    return;
  }

  const bool in_lds = c <= kLdsKeys;
  if (in_lds) {
    for (int j = tid; j < c; j += NT) keys[j] = rank_key(w[j], tok[j], recent_from, a.n_sink);
  }
  auto key_at = [&](int j) -> uint32_t {
    return in_lds ? keys[j] : rank_key(w[j], tok[j], recent_from, a.n_sink);
  };

  // The E-th largest key: eight bits at a time.  Kept are the keys whose leading
  // bits are above `prefix`, and of those equal to it the first `need`.
  uint32_t prefix = 0, mask = 0;
  int need = E;
  bool all_equal = false;  // every key that matches the prefix is kept
  for (int shift = 24; shift >= 0 && !all_equal; shift -= 8) {
    for (int i = tid; i < 256; i += NT) hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < c; j += NT) {
      const uint32_t key = key_at(j);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1);
    }
    __syncthreads();
    find_bin<NT>(hist, 256, need, sh, sel);
    prefix |= (uint32_t)sel[0] << shift;
    mask |= 255u << shift;
    need -= sel[1];
    all_equal = sel[2] == need;
    __syncthreads();  // sel and hist are rewritten
  }

  // Every thread takes a run of consecutive slots, so that one scan orders them.
  const int most = max(c, after);
  const int per = (most + NT - 1) / NT;
  const int s0 = min(tid * per, most), s1 = min(s0 + per, most);
  int before = 0, unused, t0, t1;
  if (!all_equal) {
    int eq = 0;
    for (int j = s0; j < min(s1, c); ++j) eq += (key_at(j) & mask) == prefix;
    block_scan2<NT>(eq, 0, before, unused, t0, t1, sh);
  }
  auto walk = [&](auto&& f) {  // f(slot, kept) for this thread's slots
    int rank = before;
    for (int j = s0; j < s1; ++j) {
      bool kept = false;
      if (j < c) {
        const uint32_t key = key_at(j) & mask;
        kept = key > prefix || (key == prefix && (all_equal || rank < need));
        rank += key == prefix;
      }
      f(j, kept);
    }
  };
  int n_free = 0, n_src = 0;
  walk([&](int j, bool kept) {
    n_free += j < after && !kept;
    n_src += j >= after && kept;
  });
  int ef, es;
  block_scan2<NT>(n_free, n_src, ef, es, t0, t1, sh);
  walk([&](int j, bool kept) {
    if (j < after && !kept) dst[ef++] = j;
    if (j >= after && kept) src[es++] = j;
  });
  if (tid == 0) a.head[set] = make_int4(t0, t1, n - taken, after);
}

struct MoveArgs {
  uint16_t* k;             // [n_layers][B][L_cap][H_kv][d]
  uint16_t* v;
  const uint16_t* k_new;   // [n_layers][B][T][H_kv][d]
  const uint16_t* v_new;
  float* weights;
  int32_t* tokens;
  int32_t* counts;
  const int32_t* pos;
  const int4* head;
  const int32_t* dst;
  const int32_t* src;
  int64_t stride_layer, stride_b;
  int B, n_sets, L_cap, T, H_kv, blocks;  // workgroups of a set
};

// The planned rows of one set, 16 bytes a lane, K and V in turn; their weights
// and tokens; and, once per sequence, its count.
__global__ __launch_bounds__(256) void evict_move_kernel(MoveArgs a) {
  const int set = blockIdx.x / a.blocks, part = blockIdx.x % a.blocks;
  const int s = set % a.n_sets, lb = set / a.n_sets, b = lb % a.B, layer = lb / a.B;
  const int4 h = a.head[set];  // filled, from the cache, first new row, C'
  if (lb < a.B && s == 0 && part == 0 && threadIdx.x == 0) a.counts[b] = h.w;
  const size_t list = (size_t)set * a.L_cap;
  const int heads = a.H_kv / a.n_sets;      // of the set
  const int pieces = heads * (kHeadDim / 8);  // 16-byte pieces of a row
  const int64_t rs = (int64_t)a.H_kv * kHeadDim;
  const int64_t col = (int64_t)s * heads * kHeadDim;
  uint16_t* kc = a.k + (int64_t)layer * a.stride_layer + (int64_t)b * a.stride_b + col;
  uint16_t* vc = a.v + (int64_t)layer * a.stride_layer + (int64_t)b * a.stride_b + col;
  const int64_t new_off = (int64_t)lb * a.T * rs + col;
  const int64_t n = (int64_t)h.x * pieces;
  for (int64_t e = (int64_t)part * 256 + threadIdx.x; e < n; e += (int64_t)a.blocks * 256) {
    const int i = (int)(e / pieces);
    const int piece = (int)(e - (int64_t)i * pieces);
    const int d = a.dst[list + i];
    const int x = i < h.y ? a.src[list + i] : h.z + i - h.y;
    const uint16_t* ks = i < h.y ? kc + x * rs : a.k_new + new_off + x * rs;
    const uint16_t* vs = i < h.y ? vc + x * rs : a.v_new + new_off + x * rs;
    const uint4 kv = ldg16(ks + 8 * piece), vv = ldg16(vs + 8 * piece);
    *reinterpret_cast<uint4*>(kc + d * rs + 8 * piece) = kv;
    *reinterpret_cast<uint4*>(vc + d * rs + 8 * piece) = vv;
    if (piece == 0) {
      a.weights[list + d] = i < h.y ? a.weights[list + x] : 0.f;
      a.tokens[list + d] = i < h.y ? a.tokens[list + x] : a.pos[b] + x;
    }
  }
}

size_t head_bytes(int64_t sets) { return align_up(sizeof(int4) * (size_t)sets); }
size_t list_bytes(const DenseDims& d, int64_t sets) {
  return align_up(sizeof(int32_t) * (size_t)sets * d.L_cap);
}

}  // namespace

size_t evict_ws_bytes(const DenseDims& d) {
  const int64_t sets = (int64_t)d.n_layers * d.B * d.n_sets;
  return head_bytes(sets) + 2 * list_bytes(d, sets);
}

hipError_t launch_evict(const DenseDims& d, const EvictArgs& x, void* ws, hipStream_t s) {
  const int64_t sets = (int64_t)d.n_layers * d.B * d.n_sets;
  char* w = static_cast<char*>(ws);
  int4* head = reinterpret_cast<int4*>(w);
  int32_t* dst = reinterpret_cast<int32_t*>(w + head_bytes(sets));
  int32_t* src = reinterpret_cast<int32_t*>(w + head_bytes(sets) + list_bytes(d, sets));
  const PlanArgs p{x.weights, x.tokens, x.counts, x.keep, x.pos, x.n_new, head, dst, src,
                   d.B, d.n_sets, d.L_cap, d.T, d.n_recent, d.n_sink};
  const size_t lds = sizeof(uint32_t) * (size_t)(d.L_cap < kLdsKeys ? d.L_cap : kLdsKeys);
  const dim3 grid((unsigned)sets);
  if (d.L_cap <= 4096) evict_plan_kernel<256><<<grid, 256, lds, s>>>(p);
  else evict_plan_kernel<1024><<<grid, 1024, lds, s>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = (int)(sets >= 2048 ? 1 : 2048 / sets);
  const MoveArgs m{x.k, x.v, x.k_new, x.v_new, x.weights, x.tokens, x.counts, x.pos, head, dst,
                   src, d.kv_stride_layer, d.kv_stride_b, d.B, d.n_sets, d.L_cap, d.T, d.H_kv,
                   blocks};
  evict_move_kernel<<<dim3((unsigned)(sets * blocks)), 256, 0, s>>>(m);
  return hipGetLastError();
}

}  // namespace spec
