// The 8-bit KV cache: pages and slots for new tokens, and the quantising write of their
// keys and values (spec_map_slots, spec_append_kv_fp8).
#include <cuda_bf16.h>

#include <algorithm>
#include <climits>

#include "kv_fp8.cuh"

namespace specv {
namespace {

// ---------------------------------------------------------------------------------
// Pages and slots
// ---------------------------------------------------------------------------------
// Every block scans the whole batch (its request sizes and page needs) into shared memory
// and then maps its share of the rows, so that one launch does what would otherwise take a
// scan and a dependent expansion. No block waits: the state that may be updated in place
// (kv_len, free_count) is read by that scan alone and written by the block that takes the last
// ticket; tickets are taken right behind the scan, when a block has no writes that the fence
// before its ticket would wait for. New pages are read from the free list, never from the table entries
// that other blocks are writing. Up to some 100,000 rows a call is a launch and a chain of three
// dependent reads (64 requests of 16 tokens: 4.7 us); above, the writes count (512 requests of 1
// to 4,096 tokens, 1.05 M rows: 8.7 us, 1.5 TB/s; half or twice the rows per block: 10.3 us both).
constexpr int kSlotThreads = 512;
constexpr int kSlotRowsPerBlock = 8 * kSlotThreads;  // rows the grid is sized for, per block

struct SlotParams {
  spec_slot_args_t a;
  uint32_t* ticket;
};

struct SeqSlots {
  int32_t len;     // tokens held; -1: not served
  int32_t first;   // table entry of its first new page; not served: kv_len
  int32_t before;  // pages that earlier sequences need (at most INT32_MAX)
};

struct Two {  // rows and pages, summed together
  int64_t rows, pages;
};

__device__ __forceinline__ Two warp_incl_scan(Two v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t r = __shfl_up_sync(0xffffffffu, v.rows, o), g = __shfl_up_sync(0xffffffffu, v.pages, o);
    if (lane >= o) {
      v.rows += r;
      v.pages += g;
    }
  }
  return v;
}

// Sums over the earlier threads of the block; *total over all.
__device__ __forceinline__ Two block_excl_scan(Two x, Two* sh, Two* total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  constexpr int kWarps = kSlotThreads / 32;
  const Two in = warp_incl_scan(x, lane);
  if (lane == 31) sh[w] = in;
  __syncthreads();
  // every warp sums the warps' totals for itself
  const Two all = warp_incl_scan(lane < kWarps ? sh[lane] : Two{0, 0}, lane);
  *total = {__shfl_sync(0xffffffffu, all.rows, kWarps - 1), __shfl_sync(0xffffffffu, all.pages, kWarps - 1)};
  const int64_t r = __shfl_sync(0xffffffffu, all.rows, w > 0 ? w - 1 : 0);
  const int64_t g = __shfl_sync(0xffffffffu, all.pages, w > 0 ? w - 1 : 0);
  __syncthreads();
  return {(w > 0 ? r : 0) + in.rows - x.rows, (w > 0 ? g : 0) + in.pages - x.pages};
}

__global__ void __launch_bounds__(kSlotThreads) map_slots_kernel(SlotParams p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  const spec_slot_args_t& a = p.a;
  int32_t* start = reinterpret_cast<int32_t*>(smem_raw);                // [batch + 1]
  SeqSlots* seq = reinterpret_cast<SeqSlots*>(start + a.batch + 1);      // [batch + 1]
  __shared__ Two sh[kSlotThreads / 32];
  __shared__ int s_last, s_taken;
  const int tid = threadIdx.x;
  const int P = a.page_size, MP = a.max_pages_per_seq;
  const int psh = (P & (P - 1)) == 0 ? __ffs(P) - 1 : -1;  // log2 of a power of two
  const int64_t cap = static_cast<int64_t>(MP) * P;
  pdl_wait_prior();
  const int count0 = min(max(*a.free_count, 0), a.free_capacity);
  if (tid == 0) s_taken = 0;
  Two carry = {0, 0};
  for (int b0 = 0; b0 < a.batch; b0 += kSlotThreads) {
    const int b = b0 + tid;
    int held_len = 0, len = -1, n = 0, need = 0, first = 0;
    if (b < a.batch) {
      n = a.num_new[b];
      len = held_len = a.kv_len[b];
      const bool fits = len >= 0 && n >= 0 && static_cast<int64_t>(len) + n <= cap;
      if (fits) {
        const int64_t held = static_cast<int64_t>(len) + a.reserved + P - 1;
        first = static_cast<int>(psh >= 0 ? held >> psh : held / P);
        const int end = len + n + P - 1;
        need = max(0, (psh >= 0 ? end >> psh : end / P) - first);
      } else {
        len = -1;
      }
      n = max(n, 0);
    }
    Two all;
    const Two before = block_excl_scan({n, need}, sh, &all);
    if (b < a.batch) {
      const int64_t pages = carry.pages + before.pages;
      start[b] = static_cast<int32_t>(min(carry.rows + before.rows, static_cast<int64_t>(INT32_MAX)));
      const bool served = len >= 0 && (need == 0 || pages + need <= count0);
      if (served && need > 0) atomicMax(&s_taken, static_cast<int>(pages) + need);
      seq[b] = {served ? len : -1, served ? first : held_len, static_cast<int32_t>(min(pages, static_cast<int64_t>(INT32_MAX)))};
    }
    carry.rows += all.rows;
    carry.pages += all.pages;
  }
  if (tid == 0) {
    start[a.batch] = static_cast<int32_t>(min(carry.rows, static_cast<int64_t>(INT32_MAX)));
    seq[a.batch].before = static_cast<int32_t>(min(carry.pages, static_cast<int64_t>(INT32_MAX)));
  }
  __syncthreads();
  uint32_t ticket = 0;
  if (gridDim.x > 1 && tid == 0) {
    asm volatile("fence.acq_rel.gpu;" ::: "memory");  // the block's reads of the state are before its ticket
    ticket = atomicAdd(p.ticket, 1u);
  }
  const int total = start[a.batch];

  // Four rows a thread, one search for their sequence; a page's first token puts it into the table.
  const int64_t step = static_cast<int64_t>(gridDim.x) * kSlotThreads * 4;
  const bool wide = ((reinterpret_cast<uintptr_t>(a.slots) | reinterpret_cast<uintptr_t>(a.positions) |
                      reinterpret_cast<uintptr_t>(a.row_seq)) & 15u) == 0;
  for (int64_t r0 = (static_cast<int64_t>(blockIdx.x) * kSlotThreads + tid) * 4; r0 < a.max_rows; r0 += step) {
    int lo = 0;
    if (r0 < total) {
      int hi = a.batch;  // largest b with start[b] <= r0
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= r0) lo = mid; else hi = mid;
      }
    }
    int slot[4], pos[4], sq[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      slot[e] = pos[e] = sq[e] = -1;
      const int64_t r = r0 + e;
      if (r >= total) continue;
      while (start[lo + 1] <= r) ++lo;
      sq[e] = lo;
      const SeqSlots s = seq[lo];
      const int i = static_cast<int>(r) - start[lo];
      if (s.len < 0) {
        pos[e] = s.first + i;
        continue;
      }
      pos[e] = s.len + i;
      const int idx = psh >= 0 ? pos[e] >> psh : pos[e] / P, place = pos[e] - idx * P;
      int32_t* entry = a.page_table + static_cast<int64_t>(lo) * MP + idx;
      int page;
      if (idx >= s.first) {
        page = __ldg(a.free_pages + (count0 - 1 - s.before - (idx - s.first)));
        if (place == 0) *entry = page;  // the page's first token is new: first * P >= len
      } else {
        page = *entry;
      }
      if (page >= 0 && page < a.num_pages) slot[e] = page * P + place;
    }
    if (wide && r0 + 4 <= a.max_rows) {
      *reinterpret_cast<int4*>(a.slots + r0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      if (a.positions) *reinterpret_cast<int4*>(a.positions + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      if (a.row_seq) *reinterpret_cast<int4*>(a.row_seq + r0) = make_int4(sq[0], sq[1], sq[2], sq[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (r0 + e >= a.max_rows) break;
        a.slots[r0 + e] = slot[e];
        if (a.positions) a.positions[r0 + e] = pos[e];
        if (a.row_seq) a.row_seq[r0 + e] = sq[e];
      }
    }
  }

  // Pages whose first token is a row past max_rows, page by page: there may be many more such rows
  // than pages, and behind a request of a wrong size their numbers end at INT32_MAX. Page i from
  // the free list's top is that of the last sequence with before <= i, if it is served.
  if (total > a.max_rows) {
    const int pages_end = min(seq[a.batch].before, s_taken);
    for (int64_t i = blockIdx.x * kSlotThreads + tid; i < pages_end; i += static_cast<int64_t>(gridDim.x) * kSlotThreads) {
      int lo = 0, hi = a.batch;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (seq[mid].before <= i) lo = mid; else hi = mid;
      }
      const SeqSlots s = seq[lo];
      const int64_t idx = s.first + (i - s.before);
      if (s.len >= 0 && start[lo] + (idx * P - s.len) >= a.max_rows)
        a.page_table[static_cast<int64_t>(lo) * MP + idx] = __ldg(a.free_pages + (count0 - 1 - i));
    }
  }

  // The block with the last ticket updates the state, which all have read.
  if (gridDim.x > 1) {
    if (tid == 0) {
      s_last = ticket == gridDim.x - 1;
      if (s_last) {
        *p.ticket = 0;
        asm volatile("fence.acq_rel.gpu;" ::: "memory");
      }
    }
    __syncthreads();
    if (!s_last) return;
  }
  for (int b = tid; b < a.batch; b += kSlotThreads) {
    const bool served = seq[b].len >= 0;
    const int len = served ? seq[b].len : seq[b].first, n = a.num_new[b];
    const bool fits = len >= 0 && n >= 0 && static_cast<int64_t>(len) + n <= cap;
    a.new_len[b] = served ? len + n : len;
    if (a.flags) a.flags[b] = served ? 0 : (fits ? 2 : 1);
  }
  for (int b = tid; b <= a.batch; b += kSlotThreads) a.row_start[b] = start[b];
  if (tid == 0) *a.new_free_count = count0 - s_taken;
}

// ---------------------------------------------------------------------------------
// Quantising write
// ---------------------------------------------------------------------------------
// A block takes kAppendRows rows of some KV heads. A row that is the first of its page in the
// window before it leads that page's rows; the block notes which row goes to each place of a
// led page once, for all heads, K and V. A group of one warp per 16 places then holds a
// page's new keys or values of one head in registers: one pass finds their largest
// magnitude, from it the page's scale, and the same registers are rounded and stored. Groups
// run free of each other. HBM traffic is the new rows once and their 8-bit form once (a page
// whose scale grows is read and written once more); memory bounds it: 8 prompts of 4,093 tokens,
// 8 heads of 128, take 35.3 us, 5.7 TB/s (0.84 of the measured copy rate; 44 us when the
// magnitudes were compared one by one). 64 blocks of 16 tokens: 4.5 us, the launch and two
// dependent reads. 16 or 64 rows a block: 38 us both.
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 32;
constexpr int kWin = SPEC_APPEND_WINDOW;

struct AppendParams {
  int rows, hkv, heads, num_pages;  // heads: per block
  int64_t k_stride, v_stride;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  const int32_t* slots;
  uint8_t* cache;
  float* scale;
  uint32_t* status;
};

// The largest finite magnitude of two packed bf16 values, as its bits.
__device__ __forceinline__ uint32_t finite_max2(uint32_t w, uint32_t m) {
  const uint32_t a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
  m = max(m, a < 0x7f80u ? a : 0u);
  return max(m, b < 0x7f80u ? b : 0u);
}

template <int D, int P>
__global__ void __launch_bounds__(kAppendThreads) append_fp8_kernel(AppendParams p) {
  constexpr int GW = P / 16;                        // warps per group
  constexpr int GROUPS = kAppendThreads / 32 / GW;  // groups per block
  constexpr int LPR = D / 8;                        // lanes per row of 8-element pieces
  constexpr int RPI = 32 / LPR;                     // rows per warp and step
  constexpr int STEPS = 16 / RPI;
  __shared__ int32_t win[kAppendRows + 2 * kWin];   // slots of the rows around the block's
  __shared__ int32_t leaders[kAppendRows];
  __shared__ int nlead;
  __shared__ int32_t row_of[kAppendRows][P];        // row written to each place of a led page, or -1
  __shared__ uint32_t amax[GROUPS][2][GW];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r0 = blockIdx.x * kAppendRows, head0 = blockIdx.y * p.heads;
  const int nheads = min(p.heads, p.hkv - head0);
  const int64_t max_slot = static_cast<int64_t>(p.num_pages) * P;
  if (tid == 0) nlead = 0;
  pdl_wait_prior();
  for (int i = tid; i < kAppendRows + 2 * kWin; i += kAppendThreads) {
    const int64_t r = static_cast<int64_t>(r0) - kWin + i;
    int s = r >= 0 && r < p.rows ? p.slots[r] : -1;
    if (s >= max_slot) {
      if (p.status && head0 == 0 && i >= kWin && i < kWin + kAppendRows)
        set_status(p.status, SPEC_FLAG_BAD_PAGE);
      s = -1;
    }
    win[i] = s;
  }
  __syncthreads();
  for (int i = warp; i < kAppendRows; i += kAppendThreads / 32) {
    const int s = win[kWin + i];
    if (s < 0) continue;  // warp-uniform
    bool earlier = false;
    for (int q = lane; q < kWin - 1; q += 32) {
      const int t = win[i + 1 + q];
      earlier |= t >= 0 && t / P == s / P;
    }
    if (__any_sync(0xffffffffu, earlier)) continue;
    int at = 0;
    if (lane == 0) {
      at = atomicAdd(&nlead, 1);
      leaders[at] = s / P;
    }
    at = __shfl_sync(0xffffffffu, at, 0);
    for (int q = lane; q < P; q += 32) row_of[at][q] = -1;
    __syncwarp();
    for (int q = lane; q < kWin; q += 32) {
      const int t = win[kWin + i + q];
      if (t >= 0 && t / P == s / P) row_of[at][t % P] = r0 + i + q;
    }
  }
  __syncthreads();
  const int items = nlead * nheads * 2;  // (leader, head, K or V)
  const int group = warp / GW, gwarp = warp % GW;
  const int sub = lane / LPR, piece = lane % LPR;
  int turn = 0;
  for (int it = group; it < items; it += GROUPS, turn ^= 1) {
    const int kind = it & 1, lead = (it >> 1) / nheads, head = head0 + (it >> 1) - lead * nheads;
    const int page = leaders[lead];
    const int32_t* rows = row_of[lead];
    const __nv_bfloat16* src = (kind ? p.v : p.k) + head * D + piece * 8;
    const int64_t stride = kind ? p.v_stride : p.k_stride;
    float* sp = p.scale + (static_cast<int64_t>(page) * p.hkv + head) * 2 + kind;
    const bool anew = rows[0] >= 0;
    const float old = anew ? kScaleMin : clamp_scale(*sp);
    uint4 x[STEPS];
    uint32_t written = 0, m = 0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int row = rows[gwarp * 16 + i * RPI + sub];
      x[i] = make_uint4(0, 0, 0, 0);
      if (row >= 0) {
        written |= 1u << i;
        x[i] = __ldg(reinterpret_cast<const uint4*>(src + row * stride));
      }
    }
    // Magnitudes of bf16 values compare like their bits, two in a word; Infs and NaNs, which
    // do not count, are above all others and are sorted out only where there are any.
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      m = __vmaxu2(m, __vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu));
      m = __vmaxu2(m, __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu));
    }
    m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
    if (m >= 0x7f80u) {
      m = 0;
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
        m = finite_max2(x[i].w, finite_max2(x[i].z, finite_max2(x[i].y, finite_max2(x[i].x, m))));
      m = __reduce_max_sync(0xffffffffu, m);
    }
    if (GW > 1) {  // over the group's warps; the two halves of amax take turns
      if (lane == 0) amax[group][turn][gwarp] = m;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(GW * 32) : "memory");
#pragma unroll
      for (int w = 0; w < GW; ++w) m = max(m, amax[group][turn][w]);
    }
    const float need = fp8_scale_of(m), sc = fmaxf(need, old);
    const float inv = 1.f / sc, grow = old / sc;
    uint8_t* dst = p.cache + ((static_cast<int64_t>(page) * p.hkv + head) * 2 + kind) * (P * D) + piece * 8;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      uint2* d = reinterpret_cast<uint2*>(dst + (gwarp * 16 + i * RPI + sub) * D);
      if (written >> i & 1) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[e] = to_e4m3x2(__uint_as_float(w[e] << 16) * inv, __uint_as_float(w[e] & 0xffff0000u) * inv);
        *d = make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
      } else if (!anew && grow != 1.f) {  // the page goes on at a larger scale
        const uint2 held = *d;
        const uint32_t w[4] = {held.x & 0xffffu, held.x >> 16, held.y & 0xffffu, held.y >> 16};
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = from_e4m3x2(w[e]);
          o[e] = to_e4m3x2(f.x * grow, f.y * grow);
        }
        *d = make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
      }
    }
    if (gwarp == 0 && lane == 0) *sp = sc;  // the group's warps read the old one before the barrier
    __syncwarp();
  }
}

template <int D>
cudaError_t launch_append_d(const AppendParams& p, int page_size, cudaStream_t stream) {
  const dim3 grid((p.rows - 1) / kAppendRows + 1, (p.hkv - 1) / p.heads + 1);
  auto kernel = page_size == 16   ? append_fp8_kernel<D, 16>
                : page_size == 32 ? append_fp8_kernel<D, 32>
                                  : append_fp8_kernel<D, 64>;
  return launch_overlapped(kernel, grid, kAppendThreads, 0, stream, p);
}

}  // namespace

size_t slot_smem(int batch) { return (batch + 1) * (4 + sizeof(SeqSlots)); }

cudaError_t launch_map_slots(const spec_slot_args_t& a, char* ws, cudaStream_t stream) {
  SlotParams p{a, reinterpret_cast<uint32_t*>(ws + kWsHeader)};
  const size_t smem = slot_smem(a.batch);
  (void)cudaGetLastError();
  if (smem > 48 * 1024) {  // the limit is one for all host threads, so every call sets the same
    const cudaError_t e = cudaFuncSetAttribute(map_slots_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(slot_smem(SPEC_SLOTS_MAX_BATCH)));
    if (e != cudaSuccess) return e;
  }
  const int grid = (a.max_rows - 1) / kSlotRowsPerBlock + 1;
  return launch_overlapped(map_slots_kernel, dim3(grid), kSlotThreads, smem, stream, p);
}

cudaError_t launch_append_fp8(const spec_append_fp8_args_t& a, int sms, cudaStream_t stream) {
  AppendParams p;
  const int64_t dense = static_cast<int64_t>(a.num_kv_heads) * a.head_dim;
  p.rows = a.rows;
  p.hkv = a.num_kv_heads;
  p.num_pages = a.num_pages;
  p.k_stride = a.k_row_stride ? a.k_row_stride : dense;
  p.v_stride = a.v_row_stride ? a.v_row_stride : dense;
  p.k = static_cast<const __nv_bfloat16*>(a.k);
  p.v = static_cast<const __nv_bfloat16*>(a.v);
  p.slots = a.slots;
  p.cache = static_cast<uint8_t*>(a.kv_cache);
  p.scale = a.kv_scale;
  p.status = a.status;
  // several heads per block where the rows alone fill the GPU: the search for led pages is
  // done once for all of them
  p.heads = 1;
  while (p.heads < 8 && p.heads < p.hkv &&
         static_cast<int64_t>((p.rows - 1) / kAppendRows + 1) * ((p.hkv - 1) / (2 * p.heads) + 1) >= 4 * sms)
    p.heads *= 2;
  (void)cudaGetLastError();
  return a.head_dim == 128 ? launch_append_d<128>(p, a.page_size, stream)
                           : launch_append_d<64>(p, a.page_size, stream);
}

}  // namespace specv
