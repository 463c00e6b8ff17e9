// The pages and the token lists of a step, decided on the device (snap_paged_plan).
//
// Requests are served as if one after the other; the prefix sums of what each of them wants (pages it gives back, tokens,
// pages it misses) tell which are served and where each one's pages lie in the stack, so that all of it is parallel but for one scan.
// One thread-block cluster does the call, its phases apart by cluster barriers: count, scan (one CTA), move (pages given back,
// table rows, lists of tokens), fill (the granted pages, read from a stack that is then complete).
#include <climits>

#include "snap_internal.cuh"

namespace snap {
namespace {

constexpr int NT = 1024, NW = NT / 32;
constexpr int MAX_HELD = 2048;                  // requests whose sums a CTA keeps in shared memory for the lists

struct Head { int n0, there, tokens; };         // stack before the call, with what was given back; tokens granted
struct Scratch {
  int* owner;                                   // [max_seqs]: the first request that lists the slot
  int4* rec;                                    // [n]: slot (-1: skipped), n, rows, pages missing or given back
  int* last;                                    // [n]: of a sequence that ends, the last entry that holds a page
  int4* res;                                    // [n]: pages given back before, pages granted before, tokens granted (-1: refused), tokens granted before
  Head* head;
};
__host__ __device__ inline size_t up(size_t x) { return (x + 255) / 256 * 256; }
__host__ __device__ inline size_t carve(char* base, int max_seqs, int n, Scratch* s) {
  size_t off = 0;
  const size_t at[5] = {0, up(sizeof(int) * (size_t)max_seqs), up(sizeof(int4) * (size_t)n), up(sizeof(int) * (size_t)n), up(sizeof(int4) * (size_t)n)};
  char* p[5];
  for (int i = 0; i < 5; ++i) { off += at[i]; p[i] = base + off; }
  if (s) {
    s->owner = reinterpret_cast<int*>(p[0]); s->rec = reinterpret_cast<int4*>(p[1]); s->last = reinterpret_cast<int*>(p[2]);
    s->res = reinterpret_cast<int4*>(p[3]); s->head = reinterpret_cast<Head*>(p[4]);
  }
  return off + up(sizeof(Head));
}

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_rank() { int r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ int cluster_size() { int r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }

// Sum over the block's threads before this one, and of all; every thread calls it.
__device__ __forceinline__ long long block_exclusive(long long v, long long* part /* shared, NW + 1 */, long long& total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
  __syncthreads();                                                       // what was there has been read
  if (lane == 31) part[w] = x;
  __syncthreads();
  if (w == 0) {
    const long long p = part[lane];
    long long q = p;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, q, o); if (lane >= o) q += y; }
    part[lane] = q - p;
    if (lane == 31) part[NW] = q;
  }
  __syncthreads();
  total = part[NW];
  return part[w] + x - v;
}

__device__ __forceinline__ bool held(const PlanArgs& a, int entry) { return entry >= 0 && entry < a.n_pages; }
__device__ __forceinline__ int pages_of(const PlanArgs& a, long long rows) { return (int)((rows + a.page - 1) / a.page); }

__global__ void __launch_bounds__(NT) paged_plan_kernel(const __grid_constant__ PlanArgs a) {
  __shared__ long long part[NW + 1];
  __shared__ int sums[NW], lasts[NW];
  __shared__ int cu_s[MAX_HELD + 1], slot_s[MAX_HELD], row_s[MAX_HELD];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, rank = cluster_rank(), C = cluster_size();
  Scratch s;
  carve(a.scratch, a.max_seqs, a.n, &s);
  pdl_wait();
  const auto report = [&](unsigned bad) { if (bad && a.status) atomicOr(a.status, bad); };

  // ---- who lists a slot first ----
  for (int i = rank * NT + tid; i < a.n; i += C * NT) {
    const int slot = a.slots[i];
    if (slot >= 0 && slot < a.max_seqs) s.owner[slot] = INT_MAX;
    else if (slot != -1) report(SNAP_DEV_BAD_SLOT);
  }
  cluster_barrier();
  for (int i = rank * NT + tid; i < a.n; i += C * NT) {
    const int slot = a.slots[i];
    if (slot >= 0 && slot < a.max_seqs) atomicMin(&s.owner[slot], i);
  }
  cluster_barrier();

  // ---- pages that each request misses, or gives back: `group` warps to a request ----
  int group = 1;
  while (group < NW && (long long)a.n * group * 2 <= (long long)C * NW) group *= 2;
  const int groups = NW / group, mine = w / group, gt = tid % (group * 32);   // groups of a CTA, this thread's and its place in it
  for (int i0 = rank * groups; i0 < a.n; i0 += C * groups) {
    const int i = i0 + mine;
    int count = 0, last = -1;
    int4 rec = make_int4(-1, 0, 0, 0);
    if (i < a.n) {
      const int slot = a.slots[i];
      if (slot >= 0 && slot < a.max_seqs) {
        if (__ldcg(&s.owner[slot]) == i) rec.x = slot;
        else if (gt == 0) report(SNAP_DEV_BAD_SLOT);
      }
      if (rec.x >= 0) {
        rec.y = a.new_tokens[i];
        rec.z = rec.y < 0 ? 0 : max(a.seq_len[slot], 0);
        const int* row = a.table_in + (long long)slot * a.max_pages;
        const long long rows = (long long)rec.z + rec.y;
        if (rec.y < 0) {
#pragma unroll 4
          for (int j = gt; j < a.max_pages; j += group * 32)
            if (held(a, row[j])) { ++count; last = j; }
        } else if (rows <= (long long)a.page * a.max_pages) {
          const int j1 = pages_of(a, rows);
#pragma unroll 4
          for (int j = pages_of(a, rec.z) + gt; j < j1; j += group * 32) count += !held(a, row[j]);
        } else {
          count = -1;                                                    // past the table
        }
      }
    }
    const bool past = count < 0;                                         // (of all the group's threads)
    count = __reduce_add_sync(0xffffffffu, past ? 0 : count);
    last = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) { sums[w] = count; lasts[w] = last; }
    __syncthreads();
    if (gt == 0 && i < a.n) {
      for (int k = 1; k < group; ++k) { count += sums[w + k]; last = max(last, lasts[w + k]); }
      rec.w = past ? -1 : count;
      s.rec[i] = rec;
      s.last[i] = last;
      if (past) report(SNAP_DEV_BAD_PAGE);
    }
    __syncthreads();
  }
  cluster_barrier();

  // ---- the scan ----
  if (rank == 0) {
    const int per = (a.n + NT - 1) / NT, i0 = min(tid * per, a.n), i1 = min(i0 + per, a.n);
    long long back = 0, want = 0, miss = 0, all_back, all_want, all_miss;
    const auto tokens = [](const int4& r) { return r.x >= 0 && r.y > 0 && r.w >= 0 ? r.y : 0; };
    for (int i = i0; i < i1; ++i) {
      const int4 r = __ldcg(&s.rec[i]);
      if (r.x < 0) continue;
      if (r.y < 0) back += r.w;
      else if (r.w > 0) miss += r.w;
      want += tokens(r);
    }
    back = block_exclusive(back, part, all_back);
    want = block_exclusive(want, part, all_want);
    miss = block_exclusive(miss, part, all_miss);
    const int given = *a.n_free_in, n0 = min(max(given, 0), a.n_pages);
    const int there = (int)min(n0 + all_back, (long long)a.n_pages);
    if (tid == 0 && (given != n0 || n0 + all_back > a.n_pages)) report(SNAP_DEV_BAD_PAGE);
    long long got = 0, taken = 0, all_got, all_taken;
    unsigned bad = 0;
    {
      long long wn = want, ms = miss;
      for (int i = i0; i < i1; ++i) {
        const int4 r = __ldcg(&s.rec[i]);
        if (r.x < 0 || r.y < 0 || r.w < 0) continue;
        wn += r.y;
        ms += r.w;
        if (wn <= a.n_tokens_max && (r.w == 0 || ms <= there)) { got += r.y; taken += r.w; }
        else bad = SNAP_DEV_NO_ROOM;
      }
    }
    report(bad);
    long long at = block_exclusive(got, part, all_got);
    block_exclusive(taken, part, all_taken);
    for (int i = i0; i < i1; ++i) {
      const int4 r = __ldcg(&s.rec[i]);
      int4 res = make_int4((int)min(back, (long long)INT_MAX), 0, -1, (int)at);
      if (r.x >= 0 && r.y < 0) back += r.w;
      else if (r.x >= 0 && r.w >= 0) {
        want += r.y;
        res.y = (int)min(miss, (long long)INT_MAX);
        miss += r.w;
        if (want <= a.n_tokens_max && (r.w == 0 || miss <= there)) { res.z = r.y; at += r.y; }
      }
      s.res[i] = res;
      a.cu[i] = res.w;
      a.first_rows[i] = r.z;
      if (a.granted) a.granted[i] = max(res.z, 0);
    }
    if (tid == 0) {
      a.cu[a.n] = (int)all_got;
      *a.n_free_out = there - (int)all_taken;
      *s.head = {n0, there, (int)all_got};
    }
  }
  cluster_barrier();

  // ---- pages given back; table rows ----
  const int n0 = __ldcg(&s.head->n0), there = __ldcg(&s.head->there), all = __ldcg(&s.head->tokens);
  const bool apart = a.table_in != a.table_out;
  for (int i = rank * groups + mine; i < a.n; i += C * groups) {
    const int4 r = __ldcg(&s.rec[i]);
    if (r.x < 0) continue;
    const int* row = a.table_in + (long long)r.x * a.max_pages;
    int* out = a.table_out + (long long)r.x * a.max_pages;
    if (r.y >= 0) {
      if (apart)
#pragma unroll 4
        for (int j = gt; j < a.max_pages; j += group * 32) out[j] = row[j];
      continue;
    }
    const long long at = (long long)n0 + __ldcg(&s.res[i]).x;
    if (__ldcg(&s.last[i]) + 1 == r.w) {                                 // they are the row's first entries
#pragma unroll 4
      for (int j = gt; j < a.max_pages; j += group * 32) {
        const int e = row[j];
        if (j < r.w && at + j < a.n_pages) a.stack[at + j] = e;
        out[j] = -1;
      }
    } else if (gt < 32) {
      int k = 0;
      for (int j0 = 0; j0 < a.max_pages; j0 += 32) {
        const int j = j0 + lane, e = j < a.max_pages ? row[j] : -1;
        const unsigned some = __ballot_sync(0xffffffffu, held(a, e));
        const long long to = at + k + __popc(some & ((1u << lane) - 1u));
        if (held(a, e) && to < a.n_pages) a.stack[to] = e;
        if (j < a.max_pages) out[j] = -1;
        k += __popc(some);
      }
    }
    if (gt == 0) a.seq_len[r.x] = 0;
  }
  // ---- the lists of tokens, four at a time ----
  const bool in_smem = a.n <= MAX_HELD;
  if (in_smem) {
    for (int i = tid; i < a.n; i += NT) {
      const int4 r = __ldcg(&s.rec[i]);
      cu_s[i] = __ldcg(&s.res[i]).w; slot_s[i] = r.x; row_s[i] = r.z;
    }
    if (tid == 0) cu_s[a.n] = all;
  }
  __syncthreads();
  const auto cu = [&](int i) { return in_smem ? cu_s[i] : i < a.n ? __ldcg(&s.res[i]).w : all; };
  for (long long t0 = 4LL * (rank * NT + tid); t0 < a.n_tokens_max; t0 += 4LL * C * NT) {
    alignas(16) int slot[4] = {-1, -1, -1, -1}, row[4] = {0, 0, 0, 0};
    if (t0 < all) {
      int lo = 0, hi = a.n;                                              // cu(lo) <= t0 < cu(hi)
      while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (cu(mid) <= t0) lo = mid; else hi = mid; }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const long long t = t0 + x;
        if (t >= all) break;
        while (cu(lo + 1) <= t) ++lo;
        slot[x] = in_smem ? slot_s[lo] : __ldcg(&s.rec[lo]).x;
        row[x] = (in_smem ? row_s[lo] : __ldcg(&s.rec[lo]).z) + (int)(t - cu(lo));
      }
    }
    if (t0 + 4 <= a.n_tokens_max) {
      *reinterpret_cast<int4*>(a.token_slots + t0) = *reinterpret_cast<const int4*>(slot);
      *reinterpret_cast<int4*>(a.token_rows + t0) = *reinterpret_cast<const int4*>(row);
    } else {
      for (int x = 0; x < 4 && t0 + x < a.n_tokens_max; ++x) { a.token_slots[t0 + x] = slot[x]; a.token_rows[t0 + x] = row[x]; }
    }
  }
  cluster_barrier();

  // ---- the granted pages ----
  for (int i = rank * groups + mine; i < a.n; i += C * groups) {
    const int4 r = __ldcg(&s.rec[i]), res = __ldcg(&s.res[i]);
    if (res.z < 0 || r.w <= 0) continue;
    const int* row = a.table_in + (long long)r.x * a.max_pages;
    int* out = a.table_out + (long long)r.x * a.max_pages;
    const int j0 = pages_of(a, r.z), j1 = pages_of(a, (long long)r.z + r.y), top = there - 1 - res.y;
    if (r.w == j1 - j0) {                                                // none of them holds a page
#pragma unroll 4
      for (int j = j0 + gt; j < j1; j += group * 32) out[j] = __ldcg(&a.stack[top - (j - j0)]);
    } else if (gt < 32) {
      int k = 0;
      for (int b = j0; b < j1; b += 32) {
        const int j = b + lane;
        const bool need = j < j1 && !held(a, row[j]);
        const unsigned some = __ballot_sync(0xffffffffu, need);
        if (need) out[j] = __ldcg(&a.stack[top - k - __popc(some & ((1u << lane) - 1u))]);
        k += __popc(some);
      }
    }
  }
}

}  // namespace

size_t paged_plan_scratch_bytes(int max_seqs, int n_seqs) { return carve(nullptr, max_seqs, n_seqs, nullptr); }

cudaError_t launch_paged_plan(const PlanArgs& a, cudaStream_t st) {
  const int cluster = 8;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(cluster);
  lc.blockDim = dim3(NT);
  lc.stream = st;
  lc.attrs = attr;
  lc.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&lc, paged_plan_kernel, a);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
