// Sequences that go on from others or end (spec_fork_sequences), and copies of pages in the
// caches of all layers (spec_copy_pages).
#include "chunk.cuh"
#include "kv_fp8.cuh"

namespace specv {
namespace {

// ---------------------------------------------------------------------------------
// Forks
// ---------------------------------------------------------------------------------
constexpr int kForkThreads = 1024;
constexpr int kForkBlocks = 8;     // one cluster
constexpr int kNobody = INT32_MAX;
constexpr int kClaim = 1 << 30;    // claims of freed pages are stored as -kClaim - place

struct ForkParams {
  spec_fork_args_t a;
  int32_t* freed;  // [batch]: pages that each ended sequence frees
  int32_t* stage;  // [batch][max_pages_per_seq], or NULL: new_table is another array
};

// Every block of the cluster passes here; global writes before it are seen after it.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The block's exclusive prefix sum of v in thread order, and the total.
__device__ __forceinline__ int scan_block(int v, int* sh, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh[warp] = x;
  __syncthreads();
  int w = sh[lane];  // kForkThreads / 32 == 32 warps
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  const int before = warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0;
  *total = __shfl_sync(0xffffffffu, w, 31);
  __syncthreads();
  return before + x - v;
}

// One cluster. Each block works out for itself who goes on from whom and which pages the forks
// get (the same in all of them); rows of the table and pages are shared out by warps. Freed
// pages keep one order whatever the order of the blocks: a page goes to the last place that
// held it, by a minimum over the places, and places are counted in order.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const __grid_constant__ ForkParams p) {
  extern __shared__ int32_t smem[];
  const spec_fork_args_t& a = p.a;
  const int B = a.batch, P = a.page_size, MP = a.max_pages_per_seq;
  int32_t* keeper = smem;        // [B]: who goes on with a sequence's pages
  int32_t* fresh = smem + B;     // [B]: new pages before a fork's, -1: not a fork, -2: refused
  int32_t* length = smem + 2 * B;  // [B]: new lengths
  __shared__ int sh[32];
  __shared__ int s_taken;
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = blockIdx.x, blocks = gridDim.x;
  const int gwarp = (tid >> 5) * blocks + rank, warps = blocks * (kForkThreads / 32);
  pdl_wait_prior();
  const int count0 = min(max(*a.free_count, 0), a.free_capacity);

  auto len_ok = [&](int b) {
    const int n = a.kv_len[b];
    return n >= 0 && static_cast<int64_t>(n) + a.reserved <= static_cast<int64_t>(MP) * P;
  };
  // whom b goes on from (-1: nobody), b itself where the request or a length is out of range
  auto source = [&](int b, bool* bad) {
    const int q = a.parent[b];
    const bool ok = q >= -1 && q < B && len_ok(b) && (q < 0 || len_ok(q));
    *bad = !ok;
    return ok ? q : b;
  };
  auto held = [&](int n) { return static_cast<int>((static_cast<int64_t>(n) + a.reserved + P - 1) / P); };

  if (a.new_shares != a.shares)
    for (int i = rank * kForkThreads + tid; i < a.num_pages; i += blocks * kForkThreads) a.new_shares[i] = a.shares[i];
  if (a.new_free_pages != a.free_pages)
    for (int i = rank * kForkThreads + tid; i < a.free_capacity; i += blocks * kForkThreads)
      a.new_free_pages[i] = a.free_pages[i];
  for (int b = tid; b < B; b += kForkThreads) keeper[b] = kNobody;
  if (tid == 0) s_taken = 0;
  __syncthreads();
  for (int b = tid; b < B; b += kForkThreads) {
    bool bad;
    const int q = source(b, &bad);
    if (q >= 0) atomicMin(&keeper[q], q == b ? -1 : b);
  }
  __syncthreads();
  int64_t carry = 0;
  for (int b0 = 0; b0 < B; b0 += kForkThreads) {
    const int b = b0 + tid;
    int need = 0, n = 0, q = -1;
    bool bad = false, fork = false;
    if (b < B) {
      q = source(b, &bad);
      if (q >= 0) {
        n = a.kv_len[q];
        fork = q != b && keeper[q] != b;
        if (fork) need = held(n) - n / P;
      }
    }
    int all;
    const int64_t before = carry + scan_block(need, sh, &all);
    if (b < B) {
      const bool refused = fork && need > 0 && before + need > count0;
      if (fork && need > 0 && !refused) atomicMax(&s_taken, static_cast<int>(before) + need);
      fresh[b] = !fork ? -1 : (refused ? -2 : static_cast<int>(min(before, static_cast<int64_t>(kNobody))));
      length[b] = q < 0 || refused ? 0 : n;
      if (rank == 0 && a.flags) a.flags[b] = bad ? 1 : (refused ? 2 : 0);
    }
    carry += all;
  }
  __syncthreads();
  const int taken = s_taken;
  cluster_sync();  // holders are copied, lengths and the free count read by all

  // ---- tables, copies, holders ----
  auto ended = [&](int b) {  // nobody goes on with b's pages
    return keeper[b] == kNobody && len_ok(b);
  };
  int32_t* rows_out = p.stage ? p.stage : a.new_table;
  for (int b = gwarp; b < B; b += warps) {
    bool bad;
    const int q = source(b, &bad);
    const int32_t* own = a.page_table + static_cast<int64_t>(b) * MP;
    int32_t* out = rows_out + static_cast<int64_t>(b) * MP;
    if (q == b) {
      if (!p.stage)
        for (int i = lane; i < MP; i += 32) out[i] = own[i];
      if (lane == 0) a.copies[2 * b] = a.copies[2 * b + 1] = -1;
      continue;
    }
    const int32_t* from = a.page_table + static_cast<int64_t>(q < 0 ? 0 : q) * MP;
    const bool none = q < 0 || fresh[b] == -2;
    const int n = none ? 0 : a.kv_len[q], hold = none ? 0 : held(n);
    const int whole = fresh[b] >= 0 ? n / P : hold;  // pages held together with others, or taken over
    for (int i = lane; i < MP; i += 32) {
      int page = -1;
      if (i < whole) {
        page = from[i];
        if (fresh[b] >= 0 && page >= 0 && page < a.num_pages) atomicAdd(&a.new_shares[page], 1);
      } else if (i < hold) {
        page = a.free_pages[count0 - 1 - fresh[b] - (i - whole)];
      }
      out[i] = page;
    }
    if (lane == 0) {
      const bool copy = !none && fresh[b] >= 0 && n % P != 0;
      a.copies[2 * b] = copy ? from[whole] : -1;
      a.copies[2 * b + 1] = copy ? a.free_pages[count0 - 1 - fresh[b]] : -1;
    }
  }
  for (int b = gwarp; b < B; b += warps) {
    if (!ended(b)) continue;
    const int hold = held(a.kv_len[b]);
    const int32_t* own = a.page_table + static_cast<int64_t>(b) * MP;
    for (int i = lane; i < hold; i += 32)
      if (own[i] >= 0 && own[i] < a.num_pages) atomicSub(&a.new_shares[own[i]], 1);
  }
  cluster_sync();
  // ---- pages that nobody holds any more: the last place claims each ----
  for (int b = gwarp; b < B; b += warps) {
    if (!ended(b)) continue;
    const int hold = held(a.kv_len[b]);
    const int32_t* own = a.page_table + static_cast<int64_t>(b) * MP;
    for (int i = lane; i < hold; i += 32) {
      const int page = own[i];
      if (page >= 0 && page < a.num_pages && a.new_shares[page] < 0)
        atomicMin(&a.new_shares[page], -kClaim - (b * MP + i));
    }
  }
  cluster_sync();
  auto claimed = [&](const int32_t* own, int b, int i, int hold) {
    if (i >= hold) return false;
    const int page = own[i];
    return page >= 0 && page < a.num_pages && __ldcg(&a.new_shares[page]) == -kClaim - (b * MP + i);
  };
  for (int b = gwarp; b < B; b += warps) {
    int n = 0;
    if (ended(b)) {
      const int hold = held(a.kv_len[b]);
      const int32_t* own = a.page_table + static_cast<int64_t>(b) * MP;
      for (int i0 = 0; i0 < hold; i0 += 32) n += __popc(__ballot_sync(0xffffffffu, claimed(own, b, i0 + lane, hold)));
    }
    if (lane == 0) p.freed[b] = n;
  }
  cluster_sync();
  // ---- the free list, in the order of the places ----
  int base = count0 - taken;
  for (int b0 = 0; b0 < B; b0 += kForkThreads) {
    const int b = b0 + tid;
    int all;
    const int before = scan_block(b < B ? __ldcg(&p.freed[b]) : 0, sh, &all);
    if (b < B) fresh[b] = base + before;
    base += all;
  }
  __syncthreads();
  for (int b = gwarp; b < B; b += warps) {
    if (!ended(b)) continue;
    const int hold = held(a.kv_len[b]);
    const int32_t* own = a.page_table + static_cast<int64_t>(b) * MP;
    int at = fresh[b];
    for (int i0 = 0; i0 < hold; i0 += 32) {
      const bool mine = claimed(own, b, i0 + lane, hold);
      const uint32_t who = __ballot_sync(0xffffffffu, mine);
      if (mine) {
        const int page = own[i0 + lane], to = at + __popc(who & ((1u << lane) - 1));
        if (to < a.free_capacity) a.new_free_pages[to] = page;
        a.new_shares[page] = 0;
      }
      at += __popc(who);
    }
  }
  cluster_sync();
  // ---- what may have been read until here ----
  if (p.stage)
    for (int b = gwarp; b < B; b += warps) {
      bool bad;
      if (source(b, &bad) == b) continue;
      for (int i = lane; i < MP; i += 32) a.new_table[static_cast<int64_t>(b) * MP + i] = p.stage[static_cast<int64_t>(b) * MP + i];
    }
  cluster_sync();
  if (rank == 0) {
    for (int b = tid; b < B; b += kForkThreads) {
      bool bad;
      const bool stays = source(b, &bad) == b;
      length[b] = stays ? a.kv_len[b] : length[b];
    }
    __syncthreads();
    for (int b = tid; b < B; b += kForkThreads) a.new_kv_len[b] = length[b];
    if (tid == 0) *a.new_free_count = min(base, a.free_capacity);
  }
}

// ---------------------------------------------------------------------------------
// Copies
// ---------------------------------------------------------------------------------
constexpr int kCopyThreads = 256;
constexpr int kCopyLoads = 4;  // 16-byte loads in flight per thread
constexpr int kCopyChunk = kCopyThreads * kCopyLoads * 16;

struct CopyParams {
  int num_pages;
  const int32_t* pairs;
  uint32_t* status;
  char* base[SPEC_COPY_MAX_BUFFERS];
  int64_t bytes[SPEC_COPY_MAX_BUFFERS];
};

template <typename T>
__device__ __forceinline__ void copy_piece(char* base, int64_t src, int64_t dst, int64_t from, int64_t bytes) {
  constexpr int N = 16 / sizeof(T) * kCopyLoads;
  const T* s = reinterpret_cast<const T*>(base + src + from);
  T* d = reinterpret_cast<T*>(base + dst + from);
  const int n = static_cast<int>(min(bytes - from, static_cast<int64_t>(kCopyChunk)) / static_cast<int64_t>(sizeof(T)));
  for (int i0 = threadIdx.x; i0 < n; i0 += kCopyThreads * kCopyLoads) {
    T x[kCopyLoads];
#pragma unroll
    for (int i = 0; i < kCopyLoads; ++i)
      if (i0 + i * kCopyThreads < n) x[i] = s[i0 + i * kCopyThreads];
#pragma unroll
    for (int i = 0; i < kCopyLoads; ++i)
      if (i0 + i * kCopyThreads < n) d[i0 + i * kCopyThreads] = x[i];
  }
  (void)N;
}

__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyParams p) {
  pdl_wait_prior();
  const int src = p.pairs[2 * blockIdx.x], dst = p.pairs[2 * blockIdx.x + 1];
  if (src < 0 && dst < 0) return;
  if (src < 0 || dst < 0 || src >= p.num_pages || dst >= p.num_pages) {
    if (p.status && threadIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) set_status(p.status, SPEC_FLAG_BAD_PAGE);
    return;
  }
  const int64_t bytes = p.bytes[blockIdx.y];
  char* base = p.base[blockIdx.y];
  const bool wide = ((reinterpret_cast<uintptr_t>(base) | static_cast<uintptr_t>(bytes)) & 15u) == 0;
  for (int64_t at = static_cast<int64_t>(blockIdx.z) * kCopyChunk; at < bytes; at += static_cast<int64_t>(gridDim.z) * kCopyChunk) {
    if (wide) copy_piece<uint4>(base, src * bytes, dst * bytes, at, bytes);
    else copy_piece<uint32_t>(base, src * bytes, dst * bytes, at, bytes);
  }
}

}  // namespace

size_t fork_smem(int batch) { return static_cast<size_t>(batch) * 3 * sizeof(int32_t); }

cudaError_t launch_fork(const spec_fork_args_t& a, char* ws, cudaStream_t stream) {
  ForkParams p;
  p.a = a;
  p.freed = reinterpret_cast<int32_t*>(ws + kWsHeader);
  p.stage = a.new_table == a.page_table
                ? reinterpret_cast<int32_t*>(ws + kWsHeader + ws_round(sizeof(int32_t) * static_cast<size_t>(a.batch)))
                : nullptr;
  const size_t smem = fork_smem(a.batch);
  // the limit belongs to the function, for all host threads: it is always the largest batch's
  const cudaError_t e = cudaFuncSetAttribute(fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(fork_smem(SPEC_SLOTS_MAX_BATCH)));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kForkBlocks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kForkBlocks);
  cfg.blockDim = dim3(kForkThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, fork_kernel, p);
}

cudaError_t launch_copy(const spec_copy_args_t& a, cudaStream_t stream) {
  CopyParams p = {};
  p.num_pages = a.num_pages;
  p.pairs = a.pairs;
  p.status = a.status;
  int64_t most = 1;
  for (int i = 0; i < a.num_buffers; ++i) {
    p.base[i] = static_cast<char*>(a.buffers[i]);
    p.bytes[i] = a.page_bytes[i];
    if (p.bytes[i] > most) most = p.bytes[i];
  }
  const int64_t pieces = (most + kCopyChunk - 1) / kCopyChunk;
  const dim3 grid(a.num_pairs, a.num_buffers, static_cast<unsigned>(pieces < 1024 ? pieces : 1024));
  return launch_overlapped(copy_kernel, grid, kCopyThreads, 0, stream, p);
}

}  // namespace specv
