// Pages of a paged cache handed out and taken back on the GPU, from the requests' lengths.
//
// A step's needs are sums over sequences, so every CTA adds up what the sequences before its own share need (lengths are
// 8 bytes a sequence and come from L2) instead of waiting for other CTAs.  The step's outputs lie on one axis on which
// sequence s takes 1 + n_s places, its length first and then its tokens: x(s) = seq_offsets[s] + s rises strictly even
// through empty sequences, CTAs take equal stretches of it, and whoever holds the first token of a page writes its column.
// What a step writes is a few bytes per token, so that calls are bound by launch and a chain of dependent loads (lengths,
// stack or table): 4.2 us each for 256 requests, and for 20480 tokens of prompts next to 230 other requests.
#include "packed.cuh"

namespace samkv {

constexpr int kPageThreads = 512;
constexpr int kPageWarps = kPageThreads / 32;
constexpr int kPagesTicketInt = 62;            // of the status block: finished CTAs of a call, zero between calls

struct PageArgs {
  Seqs seqs;                   // limit: table_width * page_size
  int32_t* table;
  const int32_t* free_pages;
  const int32_t* n_free;
  int32_t *n_free_out, *slots, *positions, *total_len;
  int width, n_pages, shift;
};

struct ReleaseArgs {
  const int32_t* table;
  const int32_t* lengths;
  const uint8_t* done;
  int32_t* free_pages;
  const int32_t* n_free;
  int32_t* n_free_out;
  int n_seq, width, n_pages, shift;
};

__device__ __forceinline__ int read_n_free(const int32_t* p, int n_pages, int* d_status) {
  const int n = *p, m = min(max(n, 0), n_pages);
  if (m != n) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
  return m;
}

// *n_free_out may be the word that the other CTAs read first: the last one to arrive writes it.
__device__ __forceinline__ void write_n_free(int32_t* out, int value, int* d_status, int tid) {
  __syncthreads();                             // (this CTA has read it)
  if (tid != 0) return;
  if (gridDim.x > 1) {
    __threadfence();
    if (atomicAdd(d_status + kPagesTicketInt, 1) != (int)gridDim.x - 1) return;
    atomicExch(d_status + kPagesTicketInt, 0);
  }
  *out = value;
}

// Numbers of pages stop here: more than any pool has (page size * pages < 2^31 and a page has 16 slots at least), and two of
// them add up in 32 bits.
constexpr int kManyPages = 1 << 28;
__device__ __forceinline__ int add_pages(int a, int b) { return min(a + b, kManyPages); }

// Sum of non-negative values over the block, for every thread.
__device__ __forceinline__ int block_sum(int v, int* sh, int tid) {
  const int lane = tid & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = add_pages(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();                             // (sh may still be read from before)
  if (lane == 0) sh[tid >> 5] = v;
  __syncthreads();
  v = lane < kPageWarps ? sh[lane] : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = add_pages(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// Exclusive prefix sum over the block; *total is the sum.
__device__ __forceinline__ int block_scan(int v, int* sh, int tid, int* total) {
  const int lane = tid & 31, warp = tid >> 5;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl = add_pages(incl, x);
  }
  __syncthreads();
  if (lane == 31) sh[warp] = incl;
  __syncthreads();
  int w = lane < kPageWarps ? sh[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w = add_pages(w, x);
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);          // of the warps before this one
  const int own = __shfl_up_sync(0xffffffffu, incl, 1);
  return add_pages(warp > 0 ? before : 0, lane > 0 ? own : 0);
}
// Last of `count` ascending values in shared memory that is not above x; the first one is not.
template <typename T>
__device__ __forceinline__ int last_not_above(const T* values, int count, T x) {
  int lo = 0, hi = count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (values[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Pages that hold n slots.
__device__ __forceinline__ int pages_of(unsigned n, int shift) { return (int)((n + ((1u << shift) - 1u)) >> shift); }
// Pages of a sequence's new tokens (base <= 2^30, n < 2^31).
__device__ __forceinline__ int new_pages(const Seq& q, int width, int shift) {
  return min(pages_of((unsigned)q.base + (unsigned)q.n, shift), width) - pages_of((unsigned)q.base, shift);
}

__global__ void __launch_bounds__(kPageThreads)
page_tables_kernel(const __grid_constant__ PageArgs a, int* __restrict__ d_status) {
  __shared__ int sums[32];
  __shared__ unsigned s_x[kPageThreads];       // the chunk's sequences: place on the axis,
  __shared__ int s_base[kPageThreads], s_n[kPageThreads], s_pre[kPageThreads];   // slots before, new ones, pages handed out before
  __shared__ int s_end;
  const int tid = threadIdx.x, shift = a.shift, page = 1 << shift;
  pdl_launch_dependents();
  if (tid == 0) s_end = a.seqs.n_seq;
  __syncthreads();
  pdl_wait();
  const int n_free = read_n_free(a.n_free, a.n_pages, d_status);
  // the first sequence that ends before it starts ends the list
  for (int s = tid; s < a.seqs.n_seq; s += kPageThreads)
    if (a.seqs.off[s + 1] < a.seqs.off[s]) atomicMin(&s_end, s);
  __syncthreads();
  const int n_seq = s_end;
  unsigned x0 = 0, x1 = 0;                     // this CTA's stretch of the axis (n_tokens + n_seq places fit 32 bits)
  int row0 = 0, row1 = 0;                      // rows that belong to sequences
  if (n_seq > 0) {
    row0 = load_seq(a.seqs, 0).first;
    const Seq l = load_seq(a.seqs, n_seq - 1);
    row1 = l.first + l.n;
    const unsigned all = (unsigned)(row1 - row0) + (unsigned)n_seq, per = (all - 1) / gridDim.x + 1;
    x0 = (unsigned)row0 + (unsigned)min((unsigned long long)per * blockIdx.x, (unsigned long long)all);
    x1 = (unsigned)row0 + (unsigned)min((unsigned long long)per * (blockIdx.x + 1), (unsigned long long)all);
  }
  // pages handed out before the first sequence of the stretch, and by the whole step; that sequence's number
  int before = 0, total = 0, s0 = 0;
  bool clamped = false;
#pragma unroll 4
  for (int s = tid; s < n_seq; s += kPageThreads) {
    const Seq q = load_seq(a.seqs, s);
    const int need = new_pages(q, a.width, shift);
    clamped |= q.clamped;
    total = add_pages(total, need);
    if ((unsigned)q.first + (unsigned)s + (unsigned)q.n < x0) {
      before = add_pages(before, need);
      ++s0;
    }
  }
  if (blockIdx.x == 0 && (clamped || (tid == 0 && n_seq < a.seqs.n_seq))) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
  before = block_sum(before, sums, tid);
  total = block_sum(total, sums, tid);
  s0 = block_sum(s0, sums, tid);
  if (blockIdx.x == 0 && tid == 0 && total > n_free) atomicMax(d_status, (int)CHECK_NO_PAGES);

  for (; s0 < n_seq && x0 < x1; s0 += kPageThreads) {
    const int count = min(kPageThreads, n_seq - s0);
    Seq q = {0, 0, 0, false, false};
    int need = 0, chunk_need;
    if (tid < count) {
      q = load_seq(a.seqs, s0 + tid);
      need = new_pages(q, a.width, shift);
    }
    s_pre[tid] = add_pages(before, block_scan(need, sums, tid, &chunk_need));
    s_x[tid] = (unsigned)q.first + (unsigned)(s0 + tid);
    s_base[tid] = q.base;
    s_n[tid] = q.n;
    __syncthreads();
    const unsigned c0 = max(x0, s_x[0]), c1 = min(x1, s_x[count - 1] + (unsigned)s_n[count - 1] + 1u);
    for (unsigned long long x = (unsigned long long)c0 + tid; x < c1; x += kPageThreads) {
      const int i = last_not_above(s_x, count, (unsigned)x), s = s0 + i, base = s_base[i], pre = s_pre[i];
      const int t = (int)((unsigned)x - s_x[i]) - 1, have = pages_of((unsigned)base, shift);
      if (t < 0) {                             // the sequence itself
        if (a.total_len == nullptr) continue;
        const unsigned end = (unsigned)base + (unsigned)s_n[i];
        const int want = min(pages_of(end, shift), a.width) - have, got = min(want, max(n_free - pre, 0));
        a.total_len[s] = (int)min(end, (unsigned)(have + got) << shift);
        continue;
      }
      const int tok = (int)((unsigned)x - (unsigned)s) - 1;
      const unsigned pos = (unsigned)base + (unsigned)t;
      const int col = (int)(pos >> shift), row = (int)(pos & (unsigned)(page - 1));
      int id = -1;
      if (col >= a.width) {
        atomicMax(d_status, (int)CHECK_APPEND_CAPACITY);
      } else {
        int32_t* entry = a.table + ((size_t)s * a.width + col);
        const int k = pre + (col - have);      // (an old page: k < pre)
        const bool given = col < have || k < n_free;
        if (given) id = col < have ? *entry : a.free_pages[n_free - 1 - k];
        if (given && (unsigned)id >= (unsigned)a.n_pages) {
          atomicMax(d_status, (int)CHECK_PAGE_RANGE);
          id = -1;
        }
        if (col >= have && row == 0) *entry = id;
      }
      if (a.slots != nullptr) a.slots[tok] = id < 0 ? -1 : (id << shift) + row;
      if (a.positions != nullptr) a.positions[tok] = (int)min(pos, 0x7fffffffu);
    }
    before = add_pages(before, chunk_need);
    if (c1 >= x1) break;
    __syncthreads();                           // the chunk's description is used up
  }

  // rows and sequences outside the list
  const int stride = gridDim.x * kPageThreads, first = blockIdx.x * kPageThreads + tid;
  const int outside = row0 + (a.seqs.n_tokens - row1);
  for (long long i = first; i < outside; i += stride) {
    const int tok = i < row0 ? (int)i : row1 + ((int)i - row0);
    if (a.slots != nullptr) a.slots[tok] = -1;
    if (a.positions != nullptr) a.positions[tok] = 0;
  }
  if (a.total_len != nullptr)
    for (int s = n_seq + first; s < a.seqs.n_seq; s += stride) a.total_len[s] = load_seq(a.seqs, s).base;
  write_n_free(a.n_free_out, max(n_free - total, 0), d_status, tid);
}

// Pages that a finished sequence gives back.
__device__ __forceinline__ int released(const ReleaseArgs& a, int s, int* d_status) {
  if (a.done[s] == 0) return 0;
  const int n = a.lengths[s], m = min(max(n, 0), a.width << a.shift);
  if (m != n) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
  return pages_of((unsigned)m, a.shift);
}

__global__ void __launch_bounds__(kPageThreads)
release_pages_kernel(const __grid_constant__ ReleaseArgs a, int* __restrict__ d_status) {
  __shared__ int sums[32];
  __shared__ int s_at[kPageThreads];           // pages of the chunk's sequences before this one
  const int tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  const int n_free = read_n_free(a.n_free, a.n_pages, d_status);
  const int per = (a.n_seq + gridDim.x - 1) / gridDim.x;
  const int s0 = min((int)blockIdx.x * per, a.n_seq), s1 = min(s0 + per, a.n_seq);
  int behind = 0, total = 0;                   // pages behind this CTA's sequences, and of all
#pragma unroll 4
  for (int s = tid; s < a.n_seq; s += kPageThreads) {
    const int n = released(a, s, d_status);
    total = add_pages(total, n);
    if (s >= s1) behind = add_pages(behind, n);
  }
  behind = block_sum(behind, sums, tid);
  total = block_sum(total, sums, tid);
  // place n_free + (pages behind this one): the last sequence's last page comes first, so the last chunk does, too
  for (int end = s1; end > s0; end -= kPageThreads) {
    const int c0 = max(end - kPageThreads, s0), count = end - c0;
    int chunk;
    const int n = tid < count ? released(a, c0 + tid, d_status) : 0;
    s_at[tid] = block_scan(n, sums, tid, &chunk);
    __syncthreads();
    for (int i = tid; i < chunk; i += kPageThreads) {
      const int k = last_not_above(s_at, count, i);            // (the last that starts there: one that has pages)
      const int id = a.table[(size_t)(c0 + k) * a.width + (i - s_at[k])];
      const int at = n_free + add_pages(behind, chunk - 1 - i);
      if ((unsigned)id >= (unsigned)a.n_pages) atomicMax(d_status, (int)CHECK_PAGE_RANGE);
      if (at < a.n_pages) a.free_pages[at] = id;
      else atomicMax(d_status, (int)CHECK_LIST_CAPACITY);
    }
    behind = add_pages(behind, chunk);
    __syncthreads();
  }
  write_n_free(a.n_free_out, min(add_pages(n_free, total), a.n_pages), d_status, tid);
}

namespace {
template <typename Args>
cudaError_t launch_pages(void (*kern)(Args, int*), const Args& a, long long work, int sm_count, int* d_status,
                         cudaStream_t stream) {
  long long ctas = (work + 2 * kPageThreads - 1) / (2 * kPageThreads);
  if (ctas > sm_count) ctas = sm_count;
  if (ctas < 1) ctas = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kPageThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, a, d_status);
}
}  // namespace

cudaError_t launch_page_tables(const Seqs& seqs, const PageTable& t, const int32_t* free_pages, const int32_t* n_free,
                               int32_t* n_free_out, int32_t* slots, int32_t* positions, int32_t* total_len, int sm_count,
                               int* d_status, cudaStream_t stream) {
  const PageArgs a = {seqs, t.table, free_pages, n_free, n_free_out, slots, positions, total_len, t.width, t.n_pages, t.shift};
  return launch_pages(page_tables_kernel, a, (long long)seqs.n_tokens + seqs.n_seq, sm_count, d_status, stream);
}

cudaError_t launch_release_pages(int n_seq, const PageTable& t, const int32_t* lengths, const uint8_t* done,
                                 int32_t* free_pages, const int32_t* n_free, int32_t* n_free_out, int sm_count, int* d_status,
                                 cudaStream_t stream) {
  const ReleaseArgs a = {t.table, lengths, done, free_pages, n_free, n_free_out, n_seq, t.width, t.n_pages, t.shift};
  // (how many pages come back is not known here: 16 sequences a CTA)
  return launch_pages(release_pages_kernel, a, 64LL * n_seq, sm_count, d_status, stream);
}

}  // namespace samkv
