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
constexpr int kForkBlocks = 16;    // of a cluster, at most
constexpr int kForkEntries = 4096; // table entries that a block takes before there are more blocks
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

// The ids of up to 32 * kAhead entries of a table row, a lane's in a register each.
constexpr int kAhead = 8;
template <typename F>
__device__ __forceinline__ void for_entries(const int32_t* row, int n, F f) {
  const int lane = threadIdx.x & 31;
  for (int i0 = 0; i0 < n; i0 += 32 * kAhead) {
    int id[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) id[k] = i0 + 32 * k + lane < n ? row[i0 + 32 * k + lane] : -1;
    f(i0, id);
  }
}

// One cluster. Each block works out for itself who goes on from whom and which pages the forks
// get (the same in all of them); rows of the table and pages are shared out by warps. Freed
// pages keep one order whatever the order of the blocks: a page goes to the last place that
// held it, by a minimum over the places, and places are counted in order.
//
// What bounds it is latency: a chain of passes (who goes on and the scan, the rows, claims, counts, the list),
// each a round trip or two to L2, and four barriers of the cluster between them (five in place). 512 sequences
// of up to 8,192 tokens, a quarter of which fork or end: 23.6 us; when up to 16 blocks were first taken 29,
// where 8 took 41 and a load at a time 78.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const __grid_constant__ ForkParams p) {
  extern __shared__ int32_t smem[];
  const spec_fork_args_t& a = p.a;
  const int B = a.batch, P = a.page_size, MP = a.max_pages_per_seq, N = a.num_pages;
  int32_t* keeper = smem;          // [B]: who goes on with a sequence's pages
  int32_t* fresh = smem + B;       // [B]: new pages before a fork's, -1: not a fork, -2: refused
  int32_t* source = smem + 2 * B;  // [B]: whom it goes on from (-1: nobody; itself where it stays)
  int32_t* length = smem + 3 * B;  // [B]: tokens it holds so far (-1: out of range)
  uint8_t* refused = reinterpret_cast<uint8_t*>(smem + 4 * B);  // [B]
  __shared__ int sh[32];
  __shared__ int s_taken;
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = blockIdx.x, blocks = gridDim.x;
  const int gwarp = (tid >> 5) * blocks + rank, warps = blocks * (kForkThreads / 32);
  pdl_wait_prior();
  const int count0 = min(max(*a.free_count, 0), a.free_capacity);
  auto held = [&](int n) { return static_cast<int>((static_cast<int64_t>(n) + a.reserved + P - 1) / P); };
  auto row_of = [&](int b) { return a.page_table + static_cast<int64_t>(b) * MP; };

  for (int b = tid; b < B; b += kForkThreads) {
    const int n = a.kv_len[b];
    keeper[b] = kNobody;
    source[b] = a.parent[b];
    length[b] = n >= 0 && static_cast<int64_t>(n) + a.reserved <= static_cast<int64_t>(MP) * P ? n : -1;
  }
  // (holders and the free list, while that is on its way)
  auto copy = [&](int32_t* to, const int32_t* from, int n) {
    const int64_t step = static_cast<int64_t>(blocks) * kForkThreads;
    for (int64_t i0 = rank * kForkThreads + tid; to != from && i0 < n; i0 += kAhead * step) {
      int x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + k * step < n) x[k] = from[i0 + k * step];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (i0 + k * step < n) to[i0 + k * step] = x[k];
    }
  };
  copy(a.new_shares, a.shares, N);
  copy(a.new_free_pages, a.free_pages, a.free_capacity);
  if (tid == 0) s_taken = 0;
  __syncthreads();
  // requests and lengths out of range: the sequence stays as it is (flag 1)
  for (int b = tid; b < B; b += kForkThreads) {
    const int q = source[b];
    const bool ok = q >= -1 && q < B && length[b] >= 0 && (q < 0 || length[q] >= 0);
    fresh[b] = ok ? -1 : -3;
  }
  __syncthreads();
  for (int b = tid; b < B; b += kForkThreads) {
    if (fresh[b] == -3) source[b] = b;
    const int q = source[b];
    if (q >= 0) atomicMin(&keeper[q], q == b ? -1 : b);
  }
  __syncthreads();
  int64_t carry = 0;
  for (int b0 = 0; b0 < B; b0 += kForkThreads) {
    const int b = b0 + tid;
    int need = 0, q = -1;
    bool bad = false, fork = false;
    if (b < B) {
      q = source[b];
      bad = fresh[b] == -3;
      fork = q >= 0 && q != b && keeper[q] != b;
      if (fork) need = held(length[q]) - length[q] / P;
    }
    int all;
    const int64_t before = carry + scan_block(need, sh, &all);
    if (b < B) {
      const bool none_left = fork && need > 0 && before + need > count0;
      if (fork && need > 0 && !none_left) atomicMax(&s_taken, static_cast<int>(before) + need);
      refused[b] = none_left;
      fresh[b] = !fork ? -1 : (none_left ? -2 : static_cast<int>(min(before, static_cast<int64_t>(kNobody))));
      if (rank == 0 && a.flags) a.flags[b] = bad ? 1 : (none_left ? 2 : 0);
    }
    carry += all;
  }
  __syncthreads();
  const int taken = s_taken;
  cluster_sync();  // holders are copied, the free count is read by all

  // ---- tables, copies, holders ----
  auto ended = [&](int b) { return keeper[b] == kNobody && length[b] >= 0; };  // nobody goes on with b's pages
  int32_t* rows_out = p.stage ? p.stage : a.new_table;
  for (int b = gwarp; b < B; b += warps) {
    const int q = source[b];
    int32_t* out = rows_out + static_cast<int64_t>(b) * MP;
    if (q == b) {
      if (!p.stage)
        for_entries(row_of(b), MP, [&](int i0, const int* id) {
#pragma unroll
          for (int k = 0; k < kAhead; ++k)
            if (i0 + 32 * k + lane < MP) out[i0 + 32 * k + lane] = id[k];
        });
      if (lane == 0) a.copies[2 * b] = a.copies[2 * b + 1] = -1;
    } else {
      const bool none = q < 0 || fresh[b] == -2, fork = fresh[b] >= 0;
      const int n = none ? 0 : length[q], hold = none ? 0 : held(n);
      const int whole = fork ? n / P : hold;  // pages held together with others, or taken over
      for_entries(row_of(q < 0 ? 0 : q), none ? 0 : whole, [&](int i0, const int* id) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (i0 + 32 * k + lane < whole) {
            out[i0 + 32 * k + lane] = id[k];
            if (fork && id[k] >= 0 && id[k] < N) atomicAdd(&a.new_shares[id[k]], 1);
          }
      });
      for (int i = whole + lane; i < MP; i += 32)
        out[i] = i < hold ? a.free_pages[count0 - 1 - fresh[b] - (i - whole)] : -1;
      if (lane == 0) {
        const bool copy = !none && fork && n % P != 0;
        a.copies[2 * b] = copy ? row_of(q)[whole] : -1;
        a.copies[2 * b + 1] = copy ? a.free_pages[count0 - 1 - fresh[b]] : -1;
      }
    }
    if (ended(b))
      for_entries(row_of(b), held(length[b]), [&](int, const int* id) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (id[k] >= 0 && id[k] < N) atomicSub(&a.new_shares[id[k]], 1);
      });
  }
  cluster_sync();
  // ---- pages that nobody holds any more: the last place claims each ----
  for (int b = gwarp; b < B; b += warps)
    if (ended(b))
      for_entries(row_of(b), held(length[b]), [&](int i0, const int* id) {
        int left[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) left[k] = id[k] >= 0 && id[k] < N ? __ldcg(&a.new_shares[id[k]]) : 0;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (left[k] < 0) atomicMin(&a.new_shares[id[k]], -kClaim - (b * MP + i0 + 32 * k + lane));
      });
  cluster_sync();
  for (int b = gwarp; b < B; b += warps) {
    int n = 0;
    if (ended(b))
      for_entries(row_of(b), held(length[b]), [&](int i0, const int* id) {
        int claim[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) claim[k] = id[k] >= 0 && id[k] < N ? __ldcg(&a.new_shares[id[k]]) : 0;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          n += __popc(__ballot_sync(0xffffffffu, claim[k] == -kClaim - (b * MP + i0 + 32 * k + lane)));
      });
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
    int at = fresh[b];
    for_entries(row_of(b), held(length[b]), [&](int i0, const int* id) {
      int claim[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) claim[k] = id[k] >= 0 && id[k] < N ? __ldcg(&a.new_shares[id[k]]) : 0;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const bool mine = claim[k] == -kClaim - (b * MP + i0 + 32 * k + lane);
        const uint32_t who = __ballot_sync(0xffffffffu, mine);
        if (mine) {
          const int to = at + __popc(who & ((1u << lane) - 1));
          if (to < a.free_capacity) a.new_free_pages[to] = id[k];
          a.new_shares[id[k]] = 0;
        }
        at += __popc(who);
      }
    });
  }
  if (p.stage) cluster_sync();  // the rows have been read
  // ---- what has been read until here ----
  if (p.stage)
    for (int b = gwarp; b < B; b += warps)
      if (source[b] != b)
        for_entries(p.stage + static_cast<int64_t>(b) * MP, MP, [&](int i0, const int* id) {
#pragma unroll
          for (int k = 0; k < kAhead; ++k)
            if (i0 + 32 * k + lane < MP) a.new_table[static_cast<int64_t>(b) * MP + i0 + 32 * k + lane] = id[k];
        });
  if (rank == 0) {
    // (every block has read the lengths and the count before its first barrier)
    for (int b = tid; b < B; b += kForkThreads) {
      const int q = source[b];
      if (q != b) a.new_kv_len[b] = q < 0 || refused[b] ? 0 : length[q];
      else if (a.new_kv_len != a.kv_len) a.new_kv_len[b] = a.kv_len[b];
    }
    if (tid == 0) *a.new_free_count = min(base, a.free_capacity);
  }
}

// ---------------------------------------------------------------------------------
// Copies
// ---------------------------------------------------------------------------------
// Blocks: (pair, buffer, piece of 16 KB), four loads in flight per thread before the stores. Bound by
// memory: 64 pairs in 64 buffers of 32 KB pages, 268 MB, take 37 us, 7.2 TB/s, because sources of several
// pairs are read from L2; eight pages of one layer take 1.6 us in a graph, a launch.
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

size_t fork_smem(int batch) { return static_cast<size_t>(batch) * (4 * sizeof(int32_t) + 1); }

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
  const cudaError_t wide = cudaFuncSetAttribute(fork_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);  // 16 blocks
  if (wide != cudaSuccess) return wide;
  const int64_t entries = static_cast<int64_t>(a.batch) * a.max_pages_per_seq;
  const int blocks = static_cast<int>(entries / kForkEntries < 1 ? 1 : entries / kForkEntries > kForkBlocks ? kForkBlocks : entries / kForkEntries);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = blocks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
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
