// The tokens' slots in the order of their experts, the tokens' rows in that order, and the
// experts' rows back to the tokens.
//
//   k_sort_few                     up to kFewSlots slots: one block
//   k_sort_count, _scan, _place    beyond: kBlockSlots slots per block
//   k_gather, k_combine            one wave per token and 64 vectors of its row
//   k_combine_bwd                  one wave per slot
//
// The sort is a counting sort that keeps the slots' order.  A wave takes a run of consecutive
// slots, 64 at a time; lanes with the same expert find each other by one ballot per bit of the
// id, so a slot's rank in its expert is the wave's count before it plus the lanes below.  The
// wave's counts start from those of the waves and blocks before it: no atomic decides an order.
// Latency bounds it: the ids are 4 bytes per slot, the order 8 (1600 slots 4.8 us, 8192 8.4 us
// in one block, 524288 in three launches of 4.6, 4.6 and 10 us).
//
// Rows move as 16 bytes per lane where size and alignment allow it, else element by element;
// HBM bounds them.  The gather goes by tokens, not by sorted rows: a token's row is read once
// and written to its k places, where going by sorted rows reads it k times, far apart in time.
// 65536 tokens (41000 with experts), k = 8, 1536 bf16 (1 GB of rows): gather 220 us,
// combine 285 (228 without gates and residual), combine_bwd 400; the whole case 4.8 TB/s, a copy 5.1.
#include <algorithm>

#include "abi_common.h"

namespace rft {
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxExperts = 1024, kMaxTopK = 16;
constexpr int64_t kFewSlots = 16384;
constexpr int64_t kBlockSlots = 8192;  // both: at most 64 kRun for a wave

struct Order {
  const int32_t* ids;  // expert_ids (sort) or nullptr
  int64_t n;           // T k
  int E, bits;         // ids fit `bits` bits
  int32_t *offsets, *slots, *places;
};

// Exclusive prefix sum over the block's threads, and the total.
__device__ __forceinline__ int block_scan(int v, int* sh, int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (lane == 63) sh[w] = s;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kSortWaves; ++i) {
    const int c = sh[i];
    before += i < w ? c : 0;
    all += c;
  }
  *total = all;
  __syncthreads();
  return before + s - v;
}

// The ids of the wave's slots [a, b), 64 kRun at most: all loads go out before the first is used.
constexpr int kRun = 16;
static_assert(kFewSlots <= kSortWaves * 64 * kRun && kBlockSlots <= kFewSlots, "a wave's run");
__device__ __forceinline__ void load_ids(const Order& o, int64_t a, int64_t b, int (&id)[kRun]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < kRun; ++i) id[i] = a + i * 64 + lane < b ? o.ids[a + i * 64 + lane] : -1;
}

// Counts per expert into h[E] (this wave's, in LDS).
__device__ __forceinline__ void count_slots(const Order& o, const int (&id)[kRun], int* h) {
#pragma unroll
  for (int i = 0; i < kRun; ++i)
    if ((unsigned)id[i] < (unsigned)o.E) atomicAdd(h + id[i], 1);
}

// The wave's slots [a, b) to their places; h[e]: the next place of expert e for this wave.
__device__ __forceinline__ void place_slots(const Order& o, int64_t a, int64_t b, const int (&id)[kRun],
                                            int* h) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    const int64_t s = a + i * 64 + lane;
    if (a + i * 64 >= b) break;
    const int e = id[i];
    const bool has = (unsigned)e < (unsigned)o.E;
    uint64_t peers = __builtin_amdgcn_ballot_w64(has);
    for (int q = 0; q < o.bits; ++q) {
      const uint64_t m = __builtin_amdgcn_ballot_w64((e >> q) & 1);
      peers &= (e >> q) & 1 ? m : ~m;
    }
    const int below = __builtin_popcountll(peers & ((1ull << lane) - 1));
    const int at = has ? h[e] + below : -1;
    __builtin_amdgcn_wave_barrier();
    if (has && below == 0) h[e] += __builtin_popcountll(peers);
    __builtin_amdgcn_wave_barrier();
    if (has) o.slots[at] = (int32_t)s;
    if (s < b) o.places[s] = at;
  }
}

// Counts h[wave][E] of a block to the waves' first places; base[e]: slots of earlier blocks.
// Returns in *n the slots with an expert, where whole (totals of the whole batch) is nullptr.
__device__ __forceinline__ void first_places(const Order& o, int* h, const int* whole,
                                             const int* before, int64_t step, bool write, int* sh,
                                             int* n) {
  const int e = threadIdx.x;
  int c = 0;
  if (e < o.E) {
    if (whole) {
      c = whole[e];
    } else {
#pragma unroll 4
      for (int w = 0; w < kSortWaves; ++w) c += h[w * o.E + e];
    }
  }
  int base = block_scan(c, sh, n);
  if (e < o.E) {
    if (write) o.offsets[e] = base;
    if (before) base += before[e * step];
    for (int w = 0; w < kSortWaves; ++w) {
      const int u = h[w * o.E + e];
      h[w * o.E + e] = base;
      base += u;
    }
  }
  if (write && e == 0) o.offsets[o.E] = *n;
  __syncthreads();
}

__device__ __forceinline__ void wave_run(int64_t from, int64_t to, int64_t& a, int64_t& b) {
  const int w = threadIdx.x >> 6;
  const int64_t per = ((to - from + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  a = min(to, from + w * per);
  b = min(to, a + per);
}

__global__ void __launch_bounds__(kSortThreads) k_sort_few(const Order o) {
  __shared__ int h[kSortWaves * kMaxExperts], sh[kSortWaves];  // h [wave][E]
  for (int i = threadIdx.x; i < kSortWaves * o.E; i += kSortThreads) h[i] = 0;
  __syncthreads();
  int64_t a, b;
  wave_run(0, o.n, a, b);
  int* const mine = h + (threadIdx.x >> 6) * o.E;
  int id[kRun];
  load_ids(o, a, b, id);
  count_slots(o, id, mine);
  __syncthreads();
  int n;
  first_places(o, h, nullptr, nullptr, 0, true, sh, &n);
  place_slots(o, a, b, id, mine);
  for (int64_t i = n + threadIdx.x; i < o.n; i += kSortThreads) o.slots[i] = -1;
}

// part [E][blocks]: counts of a block, then (scan) of the blocks before it; total [E].
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const Order o, int32_t* part, int64_t blocks) {
  __shared__ int h[kMaxExperts];
  for (int i = threadIdx.x; i < o.E; i += kSortThreads) h[i] = 0;
  __syncthreads();
  int64_t a, b;
  wave_run(blockIdx.x * kBlockSlots, min(o.n, (blockIdx.x + 1) * kBlockSlots), a, b);
  int id[kRun];
  load_ids(o, a, b, id);
  count_slots(o, id, h);
  __syncthreads();
  for (int i = threadIdx.x; i < o.E; i += kSortThreads) part[i * blocks + blockIdx.x] = h[i];
}

__global__ void __launch_bounds__(256) k_sort_scan(int E, int32_t* part, int64_t blocks, int32_t* total) {
  const int e = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (e >= E) return;
  int32_t* const p = part + e * blocks;
  int before = 0;
  for (int64_t i = lane; i - lane < blocks; i += 64) {
    const int v = i < blocks ? p[i] : 0;
    int s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(s, o, 64);
      if (lane >= o) s += u;
    }
    if (i < blocks) p[i] = before + s - v;
    before += __builtin_amdgcn_readlane(s, 63);
  }
  if (lane == 0) total[e] = before;
}

__global__ void __launch_bounds__(kSortThreads) k_sort_place(const Order o, const int32_t* part,
                                                             int64_t blocks, const int32_t* total) {
  __shared__ int h[kSortWaves * kMaxExperts], sh[kSortWaves];
  for (int i = threadIdx.x; i < kSortWaves * o.E; i += kSortThreads) h[i] = 0;
  __syncthreads();
  int64_t a, b;
  wave_run(blockIdx.x * kBlockSlots, min(o.n, (blockIdx.x + 1) * kBlockSlots), a, b);
  int* const mine = h + (threadIdx.x >> 6) * o.E;
  int id[kRun];
  load_ids(o, a, b, id);
  count_slots(o, id, mine);
  __syncthreads();
  int n;
  first_places(o, h, total, part + blockIdx.x, blocks, blockIdx.x == 0, sh, &n);
  place_slots(o, a, b, id, mine);
  const int64_t end = min(o.n, (blockIdx.x + 1) * kBlockSlots);
  for (int64_t i = max((int64_t)n, blockIdx.x * kBlockSlots) + threadIdx.x; i < end; i += kSortThreads)
    o.slots[i] = -1;
}

// ------------------------------------------------------------------- rows --
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// V elements of a row as fp32: 16 bytes (V = 8 of bf16, 4 of fp32), or one.
template <bool BF16, int V>
struct Vec {
  float v[V];
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    if constexpr (V == 1) {
      v[0] = BF16 ? bf16_to_f32(((const uint16_t*)p)[at]) : ((const float*)p)[at];
    } else if constexpr (BF16) {
      const u32x4 w = *(const u32x4*)((const uint16_t*)p + at);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[2 * q] = __uint_as_float(w[q] << 16);
        v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
      }
    } else {
      const floatx4 w = *(const floatx4*)((const float*)p + at);
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = w[q];
    }
  }
  __device__ __forceinline__ void store(void* p, int64_t at) const {
    if constexpr (V == 1) {
      if (BF16)
        ((uint16_t*)p)[at] = f32_to_bf16(v[0]);
      else
        ((float*)p)[at] = v[0];
    } else if constexpr (BF16) {
      u32x4 w;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        w[q] = (uint32_t)f32_to_bf16(v[2 * q]) | (uint32_t)f32_to_bf16(v[2 * q + 1]) << 16;
      *(u32x4*)((uint16_t*)p + at) = w;
    } else {
      *(floatx4*)((float*)p + at) = (floatx4){v[0], v[1], v[2], v[3]};
    }
  }
};

struct Rows {
  int64_t T, d, n;  // n = T k rows
  int k;
  int64_t units;    // waves per token (64 V elements each)
  const int32_t* places;
  const float* gates;  // or nullptr
};

// Wave (block of four) to token t and elements [c, c + V) of its row; false: none.
template <int V>
__device__ __forceinline__ bool unit_of(const Rows& r, int64_t& t, int64_t& c) {
  const int64_t u = block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  t = u / r.units;
  c = ((u - t * r.units) * 64 + (threadIdx.x & 63)) * V;
  return t < r.T;
}

// The sorted row of slot s; -1: none.
__device__ __forceinline__ int64_t place_of(const Rows& r, int64_t s) {
  const int p = __builtin_amdgcn_readfirstlane(r.places[s]);
  return (uint64_t)(int64_t)p < (uint64_t)r.n ? p : -1;
}

template <bool BF16, int V>
__global__ void __launch_bounds__(256) k_gather(const Rows r, const void* __restrict__ x, void* rows) {
  int64_t t, c;
  if (!unit_of<V>(r, t, c) || c >= r.d) return;
  Vec<BF16, V> a;
  a.load(x, t * r.d + c);
  for (int j = 0; j < r.k; ++j) {
    const int64_t s = t * r.k + j, p = place_of(r, s);
    if (p < 0) continue;
    Vec<BF16, V> b = a;
    if (r.gates) {
      const float g = r.gates[s];
#pragma unroll
      for (int q = 0; q < V; ++q) b.v[q] *= g;
    }
    b.store(rows, p * r.d + c);
  }
}

template <bool BF16, int V>
__global__ void __launch_bounds__(256) k_combine(const Rows r, const void* __restrict__ rows,
                                                 const void* residual, void* out) {
  constexpr int J = 4;  // rows in flight
  int64_t t, c;
  if (!unit_of<V>(r, t, c) || c >= r.d) return;
  Vec<BF16, V> sum;
  if (residual) {
    sum.load(residual, t * r.d + c);
  } else {
#pragma unroll
    for (int q = 0; q < V; ++q) sum.v[q] = 0.f;
  }
  for (int j0 = 0; j0 < r.k; j0 += J) {
    Vec<BF16, V> b[J];
    int64_t p[J];
#pragma unroll
    for (int i = 0; i < J; ++i) {
      p[i] = j0 + i < r.k ? place_of(r, t * r.k + j0 + i) : -1;
      if (p[i] >= 0) b[i].load(rows, p[i] * r.d + c);
    }
#pragma unroll
    for (int i = 0; i < J; ++i) {
      if (p[i] < 0) continue;
      const float g = r.gates ? r.gates[t * r.k + j0 + i] : 1.f;
#pragma unroll
      for (int q = 0; q < V; ++q) sum.v[q] = fmaf(g, b[i].v[q], sum.v[q]);
    }
  }
  sum.store(out, t * r.d + c);
}

template <bool BF16, int V>
__global__ void __launch_bounds__(256) k_combine_bwd(const Rows r, const void* __restrict__ d_out,
                                                     const void* rows, void* d_rows, float* d_gates) {
  const int64_t s = block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (s >= r.n) return;
  const int64_t t = s / r.k, p = place_of(r, s);
  const int lane = threadIdx.x & 63;
  float dot = 0.f;
  if (p >= 0) {
    const float g = r.gates ? r.gates[s] : 1.f;
    for (int64_t c = lane * V; c < r.d; c += 64 * V) {
      Vec<BF16, V> a, b;
      a.load(d_out, t * r.d + c);
      if (d_gates) {
        b.load(rows, p * r.d + c);
#pragma unroll
        for (int q = 0; q < V; ++q) dot = fmaf(a.v[q], b.v[q], dot);
      }
      if (d_rows) {
#pragma unroll
        for (int q = 0; q < V; ++q) a.v[q] *= g;
        a.store(d_rows, p * r.d + c);
      }
    }
  }
  if (d_gates) {
    dot = wave_sum_f(dot);
    if (lane == 0) d_gates[s] = dot;
  }
}

// ------------------------------------------------------------------- host --
rft_status check_order(const char* fn, const rft_expert_order* o) {
  if (!o) return fail(RFT_E_NULL, "%s: order is NULL", fn);
  if (o->n_experts < 1 || o->n_experts > kMaxExperts)
    return fail(RFT_E_SHAPE, "%s: n_experts=%d must be in [1, %d]", fn, o->n_experts, kMaxExperts);
  if (o->top_k < 1 || o->top_k > kMaxTopK)
    return fail(RFT_E_SHAPE, "%s: top_k=%d must be in [1, %d]", fn, o->top_k, kMaxTopK);
  if (o->T < 0 || o->T > 0x7fffffff / o->top_k)
    return fail(RFT_E_SHAPE, "%s: T=%lld rows of %d slots must be in [0, 2^31)", fn, (long long)o->T,
                o->top_k);
  return RFT_OK;
}

rft_status check_rows(const char* fn, const rft_expert_order* o, int dtype, int64_t d) {
  rft_status st = check_order(fn, o);
  if (st) return st;
  if (dtype != RFT_F32 && dtype != RFT_BF16) return fail(RFT_E_DTYPE, "%s: dtype %d unknown", fn, dtype);
  if (d < 1 || d > ((int64_t)1 << 24))
    return fail(RFT_E_SHAPE, "%s: d=%lld must be in [1, 2^24]", fn, (long long)d);
  if (o->T > 0 && !o->places) return fail(RFT_E_NULL, "%s: order.places is NULL", fn);
  return RFT_OK;
}

// Calls f(bf16, V) for the widest access that the row size and every array allow.
template <class F>
void by_access(int dtype, int64_t d, std::initializer_list<const void*> arrays, F f) {
  using std::integral_constant;
  const int64_t esz = dtype == RFT_BF16 ? 2 : 4;
  bool wide = d * esz % 16 == 0;
  for (const void* p : arrays) wide = wide && aligned16(p);
  if (dtype == RFT_BF16)
    wide ? f(std::true_type{}, integral_constant<int, 8>{}) : f(std::true_type{}, integral_constant<int, 1>{});
  else
    wide ? f(std::false_type{}, integral_constant<int, 4>{}) : f(std::false_type{}, integral_constant<int, 1>{});
}

Rows rows_of(const rft_expert_order& o, int64_t d, int V, const float* gates) {
  return {o.T, d, o.T * o.top_k, o.top_k, (d + 64 * V - 1) / (64 * V), o.places, gates};
}

int64_t sort_blocks(int64_t n) { return (n + kBlockSlots - 1) / kBlockSlots; }

}  // namespace
}  // namespace rft

using namespace rft;

extern "C" {

size_t rft_expert_sort_workspace_bytes(int64_t T, int32_t top_k, int32_t n_experts) {
  rft_expert_order o = {T, top_k, n_experts, nullptr, nullptr, nullptr};
  if (check_order("rft_expert_sort_workspace_bytes", &o)) return 0;
  const int64_t n = T * top_k;
  if (n <= kFewSlots) return 0;
  Carver c(nullptr);
  c.take<int32_t>((size_t)n_experts * sort_blocks(n));
  c.take<int32_t>(n_experts);
  return c.bytes();
}

rft_status rft_expert_sort(const int32_t* expert_ids, const rft_expert_order* order, void* ws,
                           size_t ws_bytes, void* stream) {
  const char* fn = "rft_expert_sort";
  rft_status st = check_order(fn, order);
  if (st) return st;
  if (!order->offsets || (order->T > 0 && (!expert_ids || !order->slots || !order->places)))
    return fail(RFT_E_NULL, "%s: expert_ids / offsets / slots / places is NULL", fn);
  const int64_t n = order->T * order->top_k;
  const int E = order->n_experts;
  if ((st = check_ws(fn, ws, ws_bytes, rft_expert_sort_workspace_bytes(order->T, order->top_k, E))))
    return st;
  Order o = {expert_ids, n, E, 0, order->offsets, order->slots, order->places};
  while (((E - 1) >> o.bits) > 0) ++o.bits;
  hipStream_t s = (hipStream_t)stream;
  if (n <= kFewSlots) {
    k_sort_few<<<1, kSortThreads, 0, s>>>(o);
  } else {
    Carver c(ws);
    const int64_t blocks = sort_blocks(n);
    int32_t* part = c.take<int32_t>((size_t)E * blocks);
    int32_t* total = c.take<int32_t>(E);
    k_sort_count<<<(unsigned)blocks, kSortThreads, 0, s>>>(o, part, blocks);
    k_sort_scan<<<(unsigned)((E + 3) / 4), 256, 0, s>>>(E, part, blocks, total);
    k_sort_place<<<(unsigned)blocks, kSortThreads, 0, s>>>(o, part, blocks, total);
  }
  RFT_HIP(hipGetLastError(), fn);
  return RFT_OK;
}

rft_status rft_expert_gather(const rft_expert_order* order, const void* x, int dtype, int64_t d,
                             const float* gates, void* rows, void* stream) {
  const char* fn = "rft_expert_gather";
  rft_status st = check_rows(fn, order, dtype, d);
  if (st) return st;
  if (order->T == 0) return RFT_OK;
  if (!x || !rows) return fail(RFT_E_NULL, "%s: x / rows is NULL", fn);
  by_access(dtype, d, {x, rows}, [&](auto bf, auto v) {
    const Rows r = rows_of(*order, d, decltype(v)::value, gates);
    k_gather<decltype(bf)::value, decltype(v)::value>
        <<<grid_xy((r.T * r.units + 3) / 4), 256, 0, (hipStream_t)stream>>>(r, x, rows);
  });
  RFT_HIP(hipGetLastError(), fn);
  return RFT_OK;
}

rft_status rft_expert_combine(const rft_expert_order* order, const void* rows, int dtype, int64_t d,
                              const float* gates, const void* residual, void* out, void* stream) {
  const char* fn = "rft_expert_combine";
  rft_status st = check_rows(fn, order, dtype, d);
  if (st) return st;
  if (order->T == 0) return RFT_OK;
  if (!rows || !out) return fail(RFT_E_NULL, "%s: rows / out is NULL", fn);
  by_access(dtype, d, {rows, out, residual}, [&](auto bf, auto v) {
    const Rows r = rows_of(*order, d, decltype(v)::value, gates);
    k_combine<decltype(bf)::value, decltype(v)::value>
        <<<grid_xy((r.T * r.units + 3) / 4), 256, 0, (hipStream_t)stream>>>(r, rows, residual, out);
  });
  RFT_HIP(hipGetLastError(), fn);
  return RFT_OK;
}

rft_status rft_expert_combine_bwd(const rft_expert_order* order, const void* d_out, const void* rows,
                                  int dtype, int64_t d, const float* gates, void* d_rows,
                                  float* d_gates, void* stream) {
  const char* fn = "rft_expert_combine_bwd";
  rft_status st = check_rows(fn, order, dtype, d);
  if (st) return st;
  if (order->T == 0 || (!d_rows && !d_gates)) return RFT_OK;
  if (!d_out || (d_gates && !rows)) return fail(RFT_E_NULL, "%s: d_out / rows is NULL", fn);
  by_access(dtype, d, {d_out, rows, d_rows}, [&](auto bf, auto v) {
    const Rows r = rows_of(*order, d, decltype(v)::value, gates);
    k_combine_bwd<decltype(bf)::value, decltype(v)::value>
        <<<grid_xy((r.n + 3) / 4), 256, 0, (hipStream_t)stream>>>(r, d_out, rows, d_rows, d_gates);
  });
  RFT_HIP(hipGetLastError(), fn);
  return RFT_OK;
}

}  // extern "C"
