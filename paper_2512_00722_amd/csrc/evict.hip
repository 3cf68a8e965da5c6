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
// A set's selection reads 8 bytes per slot (weight and token) and is one
// workgroup's, as the sets of a model's layers, sequences and heads are many: a
// thread keeps the keys of a run of consecutive slots in registers, and the E-th
// largest key is found from counts in LDS of its digits of 11, 11 and 10 bits, done
// early once the keys that share the digits found all stay (32 sets of 8192 slots:
// the plan takes 11.5 us).  Where only a few rows go, as in a decode step, they are
// searched for one after another instead (2048 sets of 2048 slots, one row: 15.8 us a
// call, 27.8 by digits; the launch alone 13.1).  Many new rows are moved by a launch of
// its own at the rate of a copy (32 sets x 512 rows of 4 KB: 27.5 us, 4.9 TB/s).
#include <type_traits>

#include "device_common.h"
#include "internal.h"
#include "select_common.h"

namespace spec {
namespace {

struct EvictKernelArgs {
  EvictArgs x;
  int4* head;            // [B] head_of each sequence
  int32_t* pos;          // [B] x.pos, which may be the counts' memory
  int2* filled;          // [sets]: slots filled, of them from the cache
  int32_t* dst;          // [sets][L_cap] slots filled, ascending
  int32_t* src;          // [sets][L_cap] kept slots at C' or above, ascending
  int64_t stride_layer, stride_b;
  int B, n_sets, H_kv, L_cap, T, n_recent, n_sink;
  int blocks;            // workgroups of a set in the move
};

// Of a sequence: rows held before, E, C', first new row taken.
__device__ __forceinline__ int4 head_of(const EvictKernelArgs& a, int b) {
  const int c = clampi(a.x.counts[b], 0, a.L_cap);
  const int n = a.x.n_new ? clampi(a.x.n_new[b], 0, a.T) : a.T;
  const int k = clampi(a.x.keep[b], 0, a.L_cap);
  const int after = (int)min((int64_t)k, (int64_t)c + n);
  const int taken = min(n, after);
  return make_int4(c, after - taken, after, n - taken);
}
// Every workgroup of a plan reads the counts, so that they are rewritten in another
// launch: before a plan that moves the rows itself, else by the move.
__global__ __launch_bounds__(256) void evict_counts_kernel(EvictKernelArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= a.B) return;
  const int4 hd = head_of(a, b);
  a.head[b] = hd;
  a.pos[b] = a.x.pos[b];
  a.x.counts[b] = hd.z;
}
__device__ __forceinline__ int4 plan_head(const EvictKernelArgs& a, int set, bool move) {
  const int b = (set / a.n_sets) % a.B;
  if (move) return a.head[b];
  const int4 hd = head_of(a, b);
  if (set == b * a.n_sets && threadIdx.x == 0) {
    a.head[b] = hd;
    a.pos[b] = a.x.pos[b];
  }
  return hd;
}

// Protected rows count as +inf; NaN ranks with -inf, -0 with +0.
__device__ __forceinline__ uint32_t rank_key(float w, int32_t tok, int64_t recent_from,
                                             int n_sink) {
  if (tok >= recent_from || tok < n_sink) w = INFINITY;
  return order_key(w != w ? -INFINITY : w + 0.f);
}

// Slots j .. j + 3 of a row of `cap` values; what stands behind the row's end is
// any value of it.  No branch that differs between threads: all loads of a thread
// are in flight together.
template <class T>
__device__ __forceinline__ void four(const T* row, int j, int cap, T (&v)[4]) {
  typedef T vec __attribute__((ext_vector_type(4), aligned(4)));
  if (cap % 4 == 0) {  // whole pieces
    const vec x = *reinterpret_cast<const vec*>(row + min(j, cap - 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = row[min(j + i, cap - 1)];
  }
}

// Values of a thread that satisfy f, in four sums that do not wait for each other.
template <int PER, class F>
__device__ __forceinline__ int count_if(const uint32_t (&key)[PER], F&& f) {
  int n[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < PER; ++i) n[i & 3] += f(key[i]);
  return (n[0] + n[1]) + (n[2] + n[3]);
}

// The planned rows of one set by `step` threads from `first` on: 16 bytes a lane,
// K and V in turn, with their weights and tokens.
__device__ __forceinline__ void move_rows(const EvictKernelArgs& a, int set, int first_new,
                                          int2 filled, const int32_t* dst, const int32_t* src,
                                          int64_t first, int64_t step) {
  const int s = set % a.n_sets, lb = set / a.n_sets, b = lb % a.B, layer = lb / a.B;
  const int heads = a.H_kv / a.n_sets;        // of the set
  const int pieces = heads * (kHeadDim / 8);  // 16-byte pieces of a row
  const int64_t rs = (int64_t)a.H_kv * kHeadDim;
  const int64_t col = (int64_t)s * heads * kHeadDim;
  uint16_t* kc = a.x.k + (int64_t)layer * a.stride_layer + (int64_t)b * a.stride_b + col;
  uint16_t* vc = a.x.v + (int64_t)layer * a.stride_layer + (int64_t)b * a.stride_b + col;
  const int64_t new_off = (int64_t)lb * a.T * rs + col;
  float* w = a.x.weights + (size_t)set * a.L_cap;
  int32_t* tok = a.x.tokens + (size_t)set * a.L_cap;
  const int64_t n = (int64_t)filled.x * pieces;
  for (int64_t e = first; e < n; e += step) {
    const int i = (int)(e / pieces);
    const int piece = (int)(e - (int64_t)i * pieces);
    const bool held = i < filled.y;
    const int d = dst[i];
    const int x = held ? src[i] : first_new + i - filled.y;
    const uint16_t* ks = held ? kc + x * rs : a.x.k_new + new_off + x * rs;
    const uint16_t* vs = held ? vc + x * rs : a.x.v_new + new_off + x * rs;
    const uint4 kv = ldg16(ks + 8 * piece), vv = ldg16(vs + 8 * piece);
    *reinterpret_cast<uint4*>(kc + d * rs + 8 * piece) = kv;
    *reinterpret_cast<uint4*>(vc + d * rs + 8 * piece) = vv;
    if (piece == 0) {
      w[d] = held ? w[x] : 0.f;
      tok[d] = held ? tok[x] : a.pos[b] + x;
    }
  }
}

// f over a wavefront's values, in every lane.
template <class T, class F>
__device__ __forceinline__ T wave_reduce(T v, F&& f) {
  auto step = [&](auto ctrl) {
    v = f(v, (T)__builtin_amdgcn_update_dpp((int)v, (int)v, ctrl.value, 0xf, 0xf, false));
  };
  step(std::integral_constant<int, 0xB1>{});  // quads, then rows of 16
  step(std::integral_constant<int, 0x4E>{});
  step(std::integral_constant<int, 0x141>{});
  step(std::integral_constant<int, 0x140>{});
  auto a = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = f((T)a[0], (T)a[1]);
  auto b = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return f((T)b[0], (T)b[1]);
}

// The sum of NW values in LDS, the same in every lane.
template <int NW>
__device__ __forceinline__ int sum_of(const int* v) {
  int n = 0;
  if constexpr (NW <= 4) {
#pragma unroll
    for (int i = 0; i < NW; ++i) n += v[i];
  } else {
    n = (threadIdx.x & 63) < NW ? v[threadIdx.x & 63] : 0;
    n = wave_reduce(n, [](int x, int y) { return x + y; });
  }
  return __builtin_amdgcn_readfirstlane(n);
}

// Rows that go which are searched for one by one: eight take as long as the digits do
// (us a call, 2048 sets of 2048 slots: 1 row 15.8, 4 20.5, 6 24, 8 27.5 against 27 to 30; 512
// sets of 8192: 17, 21, 23, 25.4 against 24).
constexpr int kFewEvicted = 6;

constexpr int kDigitBins = 2048;

// MOVE: the workgroup moves the rows itself (few new rows); else it leaves the
// lists for evict_move_kernel.  A thread has slots PER tid .. + PER - 1.
template <int NT, int PER, bool MOVE>
__global__ __launch_bounds__(NT) void evict_plan_kernel(EvictKernelArgs a) {
  constexpr int NW = NT / 64;
  constexpr int kLds = 64;  // list entries kept in LDS (more go through memory)
  __shared__ int cnt[2][NW];
  __shared__ int eqs[2][NW];
  __shared__ int sh[2 * NW];
  __shared__ int hist[kDigitBins];
  __shared__ int sel[3];
  __shared__ int dst_l[MOVE ? kLds : 1], src_l[MOVE ? kLds : 1];
  const int set = blockIdx.x;
  const int b = (set / a.n_sets) % a.B;
  const int tid = threadIdx.x, wave = tid >> 6;
  const int4 hd = plan_head(a, set, MOVE);
  const int c = hd.x, E = hd.y, after = hd.z, taken = after - E;
  // hd.w + taken: the new rows (x.n_new may be the counts, which are rewritten by now)
  const int64_t recent_from =
      (int64_t)(MOVE ? a.pos : a.x.pos)[b] + hd.w + taken - a.n_recent;
  int32_t* dst = a.dst + (size_t)set * a.L_cap;
  int32_t* src = a.src + (size_t)set * a.L_cap;

  if (E == c || E == 0) {  // all stay, or none: no selection; uniform
    for (int i = tid; i < taken; i += NT) {
      dst[i] = E + i;
      if (MOVE && i < kLds) dst_l[i] = E + i;
    }
    const int2 filled = make_int2(taken, 0);
    if (!MOVE) {
      if (tid == 0) a.filled[set] = filled;
      return;
    }
    __syncthreads();
    move_rows(a, set, hd.w, filled, taken <= kLds ? dst_l : dst, src, tid, NT);
    return;
  }

  uint32_t key[PER];
  {
    const float* w = a.x.weights + (size_t)set * a.L_cap;
    const int32_t* tok = a.x.tokens + (size_t)set * a.L_cap;
    float wv[PER / 4][4];
    int32_t tv[PER / 4][4];
#pragma unroll
    for (int i = 0; i < PER / 4; ++i) {
      four(w, PER * tid + 4 * i, a.L_cap, wv[i]);
      four(tok, PER * tid + 4 * i, a.L_cap, tv[i]);
    }
    // slots that hold nothing rank below every key (the least is that of -inf)
#pragma unroll
    for (int i = 0; i < PER; ++i)
      key[i] = PER * tid + i < c
                   ? rank_key(wv[i / 4][i % 4], tv[i / 4][i % 4], recent_from, a.n_sink)
                   : 0u;
  }

  uint32_t cut = 0;   // kept: the keys above it, and
  int need = c;       // the first `need` of those equal to it
  int before = 0, unused, t0, t1;
  if (c - E <= kFewEvicted) {
    // Few go: the least keys one after another, until as many rows hold them.
    int gone = c - E;
    uint32_t above = 0;  // keys up to here are gone
    for (int it = 0;; ++it) {  // at most kFewEvicted times: each takes a key of some row
      uint32_t m = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < PER; ++i) m = key[i] > above && key[i] < m ? key[i] : m;
      m = wave_reduce(m, [](uint32_t x, uint32_t y) { return min(x, y); });
      if ((tid & 63) == 0) cnt[it & 1][wave] = (int)m;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NW; ++i) m = min(m, (uint32_t)cnt[it & 1][i]);
      m = __builtin_amdgcn_readfirstlane(m);
      int n = wave_reduce(count_if(key, [&](uint32_t x) { return x == m; }),
                          [](int x, int y) { return x + y; });
      if ((tid & 63) == 0) eqs[it & 1][wave] = n;
      __syncthreads();
      n = sum_of<NW>(eqs[it & 1]);
      cut = m;
      need = n - gone;
      if (n >= gone) break;
      gone -= n;
      above = m;
    }
    if (need > 0) {  // uniform: the last of several equal keys go
      const int eq = count_if(key, [&](uint32_t x) { return x == cut; });
      block_scan2<NT>(eq, 0, before, unused, t0, t1, sh);
    }
  } else {
    // Digits of 11, 11 and 10 bits from the top, counted in LDS, until the keys
    // that share the digits found all stay.
    constexpr uint32_t kTop = 0xff800000u;  // the key of +inf
    // protected rows are many, and one value: a wavefront's are added at once
    const int top = wave_reduce(count_if(key, [&](uint32_t x) { return x == kTop; }),
                                [](int x, int y) { return x + y; });
    uint32_t mask = 0;
    bool all = false;
    need = E;
#pragma unroll 1
    for (int shift = 21; shift >= 0 && !all; shift -= shift > 10 ? 11 : 10) {
      const int bins = shift > 0 ? kDigitBins : kDigitBins / 2;
      for (int i = tid; i < bins; i += NT) hist[i] = 0;
      __syncthreads();
      if (top && (tid & 63) == 0 && (kTop & mask) == cut)
        atomicAdd(&hist[(kTop >> shift) & (bins - 1)], top);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (key[i] - 1u < kTop - 1u && (key[i] & mask) == cut)
          atomicAdd(&hist[(key[i] >> shift) & (bins - 1)], 1);
      __syncthreads();
      find_bin<NT>(hist, bins, need, sh, sel);
      cut |= (uint32_t)sel[0] << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      need -= sel[1];
      all = sel[2] == need;
      __syncthreads();  // sel and hist are rewritten
    }
    if (all) {
      need = c;
    } else {  // uniform: only the first of several equal keys stay
      const int eq = count_if(key, [&](uint32_t x) { return x == cut; });
      block_scan2<NT>(eq, 0, before, unused, t0, t1, sh);
    }
  }
  uint32_t kept = 0;  // this thread's slots that stay
  {
    int rank = before;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      kept |= (uint32_t)(key[i] > cut || (key[i] == cut && rank < need)) << i;
      rank += key[i] == cut;
    }
  }
  uint32_t below = 0;  // those below C'
#pragma unroll
  for (int i = 0; i < PER; ++i) below |= (uint32_t)(PER * tid + i < after) << i;
  uint32_t fill = below & ~kept, held = kept & ~below;
  int ef, es;
  block_scan2<NT>(__popc(fill), __popc(held), ef, es, t0, t1, sh);
  const bool in_lds = MOVE && t0 <= kLds;  // uniform; t1 <= t0
  int32_t* dl = in_lds ? dst_l : dst;
  int32_t* sl = in_lds ? src_l : src;
  for (; fill; fill &= fill - 1) dl[ef++] = PER * tid + __ffs(fill) - 1;
  for (; held; held &= held - 1) sl[es++] = PER * tid + __ffs(held) - 1;
  const int2 filled = make_int2(t0, t1);
  if (!MOVE) {
    if (tid == 0) a.filled[set] = filled;
    return;
  }
  __syncthreads();
  move_rows(a, set, hd.w, filled, dl, sl, tid, NT);
}

// Longer caches: the keys are read anew in each of four passes of a radix search.
constexpr int kRadixThreads = 1024;
__global__ __launch_bounds__(kRadixThreads) void evict_plan_long_kernel(EvictKernelArgs a) {
  constexpr int NT = kRadixThreads;
  __shared__ int hist[256];
  __shared__ int sh[2 * NT / 64];
  __shared__ int sel[3];
  const int set = blockIdx.x;
  const int b = (set / a.n_sets) % a.B;
  const int tid = threadIdx.x;
  const int4 hd = plan_head(a, set, false);
  const int c = hd.x, E = hd.y, after = hd.z, taken = after - E;
  const float* w = a.x.weights + (size_t)set * a.L_cap;
  const int32_t* tok = a.x.tokens + (size_t)set * a.L_cap;
  int32_t* dst = a.dst + (size_t)set * a.L_cap;
  int32_t* src = a.src + (size_t)set * a.L_cap;
  const int64_t recent_from = (int64_t)a.x.pos[b] + hd.w + taken - a.n_recent;

  if (E == c || E == 0) {  // all stay, or none: no selection
    for (int i = tid; i < taken; i += NT) dst[i] = E + i;
    if (tid == 0) a.filled[set] = make_int2(taken, 0);
    return;
  }
  auto key_at = [&](int j) { return rank_key(w[j], tok[j], recent_from, a.n_sink); };

  // Kept are the keys whose leading bits are above `prefix`, and of those equal to
  // it the first `need`.
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
  if (tid == 0) a.filled[set] = make_int2(t0, t1);
}

// The planned rows, `blocks` workgroups to a set.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictKernelArgs a) {
  const int set = blockIdx.x / a.blocks, part = blockIdx.x % a.blocks;
  const int b = (set / a.n_sets) % a.B;
  const size_t list = (size_t)set * a.L_cap;
  if (blockIdx.x == b * a.n_sets * a.blocks && threadIdx.x == 0) a.x.counts[b] = a.head[b].z;
  move_rows(a, set, a.head[b].w, a.filled[set], a.dst + list, a.src + list,
            (int64_t)part * 256 + threadIdx.x, (int64_t)a.blocks * 256);
}

size_t head_bytes(const DenseDims& d) { return align_up(sizeof(int4) * (size_t)d.B); }
size_t pos_bytes(const DenseDims& d) { return align_up(sizeof(int32_t) * (size_t)d.B); }
size_t filled_bytes(int64_t sets) { return align_up(sizeof(int2) * (size_t)sets); }
size_t list_bytes(const DenseDims& d, int64_t sets) {
  return align_up(sizeof(int32_t) * (size_t)sets * d.L_cap);
}

// New rows that a set's own workgroup moves: it streams a few tens of GB/s, and
// a launch of its own costs about 4 us.
constexpr int kMoveInPlan = 32;

// Slots of a thread: few enough that its loads are in flight together, and as many
// threads as leave other workgroups their places (us a call, one new row: 2048 sets of 2048
// slots by 128 threads 16.9, 256 15.8, 512 19.9; 512 sets of 8192 by 256 threads 23.9, 512
// 17.2, 1024 18.7; 32 sets of 8192 12.7, 9.9, 9.5).
template <bool MOVE>
void launch_plan(int64_t sets, const EvictKernelArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)sets);
  if (a.L_cap <= 2048) evict_plan_kernel<256, 8, MOVE><<<grid, 256, 0, s>>>(a);
  else if (a.L_cap <= 4096) evict_plan_kernel<512, 8, MOVE><<<grid, 512, 0, s>>>(a);
  else if (a.L_cap <= 8192) evict_plan_kernel<512, 16, MOVE><<<grid, 512, 0, s>>>(a);
  else if (a.L_cap <= 16384) evict_plan_kernel<1024, 16, MOVE><<<grid, 1024, 0, s>>>(a);
  else evict_plan_kernel<1024, 32, MOVE><<<grid, 1024, 0, s>>>(a);
}
constexpr int kPlanSlots = 32768;  // what the widest of them holds

}  // namespace

size_t evict_ws_bytes(const DenseDims& d) {
  const int64_t sets = (int64_t)d.n_layers * d.B * d.n_sets;
  return head_bytes(d) + pos_bytes(d) + filled_bytes(sets) + 2 * list_bytes(d, sets);
}

hipError_t launch_evict(const DenseDims& d, const EvictArgs& x, void* ws, hipStream_t s) {
  const int64_t sets = (int64_t)d.n_layers * d.B * d.n_sets;
  char* w = static_cast<char*>(ws);
  int4* head = reinterpret_cast<int4*>(w);
  w += head_bytes(d);
  int32_t* pos = reinterpret_cast<int32_t*>(w);
  w += pos_bytes(d);
  int2* filled = reinterpret_cast<int2*>(w);
  w += filled_bytes(sets);
  int32_t* dst = reinterpret_cast<int32_t*>(w);
  int32_t* src = reinterpret_cast<int32_t*>(w + list_bytes(d, sets));
  const int blocks = (int)(sets >= 2048 ? 1 : 2048 / sets);
  const EvictKernelArgs a{x, head, pos, filled, dst, src, d.kv_stride_layer, d.kv_stride_b, d.B,
                          d.n_sets, d.H_kv, d.L_cap, d.T, d.n_recent, d.n_sink, blocks};
  const bool in_plan = d.T > 0 && d.T <= kMoveInPlan && d.L_cap <= kPlanSlots;
  if (in_plan) {
    evict_counts_kernel<<<dim3((unsigned)((d.B + 255) / 256)), 256, 0, s>>>(a);
    launch_plan<true>(sets, a, s);
    return hipGetLastError();
  }
  if (d.L_cap <= kPlanSlots) launch_plan<false>(sets, a, s);
  else evict_plan_long_kernel<<<dim3((unsigned)sets), kRadixThreads, 0, s>>>(a);
  evict_move_kernel<<<dim3((unsigned)(sets * blocks)), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace spec
