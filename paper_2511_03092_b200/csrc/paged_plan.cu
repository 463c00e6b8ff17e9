// The pages and the token lists of a step, decided on the device (snap_paged_plan).
//
// Requests are served as if one after the other; the prefix sums of what each of them wants (pages it gives back, tokens,
// pages it misses) tell which are served and where each one's pages lie in the stack, so that all of it is parallel but for one scan.
// A small call is one CTA's, its phases apart by barriers: count (and copy table rows), scan, move (pages given back, lists of tokens), fill
// (the granted pages, read from a stack that is then complete).  Of a larger one a thread-block cluster counts, scans and gives back, and a
// second launch writes table rows and lists with the whole GPU.
//
// What bounds it: the way of a few numbers through memory, phase after phase, and the launches.  32 requests of a token each take 9.4 us, 6.8 of
// them without lists, rows and pages; 75 requests of up to 60000 rows and 614405 tokens 22.2 (33.7 in one launch of 16 CTAs), for 10 MB, which
// HBM brings in 1.5.
#include <algorithm>
#include <climits>

#include "snap_internal.cuh"

namespace snap {
namespace {

constexpr int MAX_HELD = 2048;                  // requests whose sums a CTA keeps in shared memory for the lists
constexpr int NT = 1024, NW = NT / 32;
constexpr int RNT = 256, PIECE = 4 * RNT;       // threads of the second launch; tokens or entries of a table row that a CTA writes at a time
constexpr int SMALL_N = 256;                    // a call of few requests: one CTA, which keeps all that phases leave each other in shared memory

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

// Sums over the block's threads before this one, and of all, of three numbers at once; every thread calls it.
struct Three { long long x[3]; };
__device__ __forceinline__ Three block_exclusive(Three v, long long (*part)[NW + 1] /* shared, three rows */, Three& total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  Three s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int k = 0; k < 3; ++k) { const long long y = __shfl_up_sync(0xffffffffu, s.x[k], o); if (lane >= o) s.x[k] += y; }
  __syncthreads();                                                       // what was there has been read
  if (lane == 31)
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][w] = s.x[k];
  __syncthreads();
  if (w < 3) {
    const long long p = lane < NW ? part[w][lane] : 0;
    long long q = p;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, q, o); if (lane >= o) q += y; }
    if (lane < NW) part[w][lane] = q - p;
    if (lane == 31) part[w][NW] = q;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) { total.x[k] = part[k][NW]; s.x[k] += part[k][w] - v.x[k]; }
  return s;
}

__device__ __forceinline__ bool held(const PlanArgs& a, int entry) { return entry >= 0 && entry < a.n_pages; }
__device__ __forceinline__ int granted_page(const PlanArgs& a, int at) { return index_ok(at, a.n_pages, a.status) ? __ldcg(&a.stack[at]) : -1; }
__device__ __forceinline__ int pages_of(const PlanArgs& a, long long rows) { return (int)((rows + a.page - 1) / a.page); }

// What one phase leaves the next is read past the first-level cache, which keeps no order between CTAs.
template <typename V> __device__ __forceinline__ V left(const V* p) { return __isShared(p) ? *p : __ldcg(p); }

// A group's threads over `count` entries from `from` on, four at a time where the row is on a 16-byte boundary: f(entry's number, entry)
template <typename F>
__device__ __forceinline__ void over(const int* row, int from, int count, int t, int threads, F f) {
  if (((reinterpret_cast<uintptr_t>(row + from) & 15) == 0) && count % 4 == 0) {
#pragma unroll 4
    for (int j = 4 * t; j < count; j += 4 * threads) {
      const int4 e = *reinterpret_cast<const int4*>(row + from + j);
      f(from + j, e.x); f(from + j + 1, e.y); f(from + j + 2, e.z); f(from + j + 3, e.w);
    }
  } else {
#pragma unroll 8
    for (int j = t; j < count; j += threads) f(from + j, row[from + j]);
  }
}

// The lists of tokens, four at a time, from what a CTA keeps of the requests in shared memory, or from the scratch.
struct Lists {
  int* cu_s; int* slot_s; int* row_s; const Scratch& s; int n, all; bool held;
  __device__ __forceinline__ void take(int threads) const {
    for (int i = threadIdx.x; held && i < n; i += threads) {
      const int4 r = left(&s.rec[i]);
      cu_s[i] = left(&s.res[i]).w; slot_s[i] = r.x; row_s[i] = r.z;
    }
    if (held && threadIdx.x == 0) cu_s[n] = all;
  }
  __device__ __forceinline__ int cu(int i) const { return held ? cu_s[i] : i < n ? __ldcg(&s.res[i]).w : all; }
  __device__ __forceinline__ void write(const PlanArgs& a, long long t0) const {
    alignas(16) int slot[4] = {-1, -1, -1, -1}, row[4] = {0, 0, 0, 0};
    if (t0 < all) {
      int lo = 0, hi = n;                                                // cu(lo) <= t0 < cu(hi)
      while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (cu(mid) <= t0) lo = mid; else hi = mid; }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const long long t = t0 + x;
        if (t >= all) break;
        while (cu(lo + 1) <= t) ++lo;
        slot[x] = held ? slot_s[lo] : __ldcg(&s.rec[lo]).x;
        row[x] = (held ? row_s[lo] : __ldcg(&s.rec[lo]).z) + (int)(t - cu(lo));
      }
    }
    if (t0 + 4 <= a.n_tokens_max) {
      *reinterpret_cast<int4*>(a.token_slots + t0) = *reinterpret_cast<const int4*>(slot);
      *reinterpret_cast<int4*>(a.token_rows + t0) = *reinterpret_cast<const int4*>(row);
    } else {
      for (int x = 0; x < 4 && t0 + x < a.n_tokens_max; ++x) { a.token_slots[t0 + x] = slot[x]; a.token_rows[t0 + x] = row[x]; }
    }
  }
};

// Entries of a row can go four at a time
__device__ __forceinline__ bool fours(const PlanArgs& a, const int* row, const int* out) {
  return a.max_pages % 4 == 0 && ((reinterpret_cast<uintptr_t>(row) | reinterpret_cast<uintptr_t>(out)) & 15) == 0;
}

// One warp: the granted pages of a row some of whose entries [j0, j1) hold a page already
__device__ __forceinline__ void fill_gaps(const PlanArgs& a, const int* row, int* out, int j0, int j1, int top) {
  const int lane = threadIdx.x & 31;
  int k = 0;
  for (int b = j0; b < j1; b += 32) {
    const int j = b + lane, e = j < j1 ? row[j] : 0;
    const bool need = j < j1 && !held(a, e);
    const unsigned some = __ballot_sync(0xffffffffu, need);
    if (j < j1) out[j] = need ? granted_page(a, top - k - __popc(some & ((1u << lane) - 1u))) : e;
    k += __popc(some);
  }
}

// SMALL: one CTA, at most SMALL_N requests
template <bool SMALL>
__global__ void __launch_bounds__(NT) paged_plan_kernel(const __grid_constant__ PlanArgs a) {
  constexpr int HELD = SMALL ? SMALL_N : 1;
  __shared__ long long part[3][NW + 1];
  __shared__ int sums[NW], lasts[NW];
  __shared__ int cu_s[HELD + 1], slot_s[HELD], row_s[HELD];
  __shared__ int new_s[SMALL ? SMALL_N : 1], len_s[SMALL ? SMALL_N : 1];
  __shared__ int4 rec_s[SMALL ? SMALL_N : 1], res_s[SMALL ? SMALL_N : 1];
  __shared__ int last_s[SMALL ? SMALL_N : 1];
  __shared__ Head head_s;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, rank = SMALL ? 0 : cluster_rank(), C = SMALL ? 1 : cluster_size();
  Scratch s;
  carve(a.scratch, a.max_seqs, a.n, &s);
  if (SMALL) { s.rec = rec_s; s.res = res_s; s.last = last_s; s.head = &head_s; }
  const auto phase = [&]() { if (SMALL) __syncthreads(); else cluster_barrier(); };
  pdl_wait();
  const auto report = [&](unsigned bad) { if (bad && a.status) atomicOr(a.status, bad); };

  // ---- who lists a slot first ----
  if (SMALL) {
    if (tid < a.n) {
      const int slot = a.slots[tid], fresh = a.new_tokens[tid];
      const bool valid = slot >= 0 && slot < a.max_seqs;
      slot_s[tid] = slot; new_s[tid] = fresh; len_s[tid] = valid ? a.seq_len[slot] : 0;
      if (!valid && slot != -1) report(SNAP_DEV_BAD_SLOT);
    }
    __syncthreads();
  } else {
    for (int i = rank * NT + tid; i < a.n; i += C * NT) {
      const int slot = a.slots[i];
      if (slot >= 0 && slot < a.max_seqs) s.owner[slot] = INT_MAX;
      else if (slot != -1) report(SNAP_DEV_BAD_SLOT);
    }
    phase();
    for (int i = rank * NT + tid; i < a.n; i += C * NT) {
      const int slot = a.slots[i];
      if (slot >= 0 && slot < a.max_seqs) atomicMin(&s.owner[slot], i);
    }
    phase();
  }

  const bool apart = a.table_in != a.table_out;
  // ---- pages that each request misses, or gives back: `group` warps to a request.  Table rows that go on are copied alongside ----
  int group = 1;
  while (group < NW && (long long)a.n * group * 2 <= (long long)C * NW) group *= 2;
  const int groups = NW / group, mine = w / group, gt = tid % (group * 32), gn = group * 32;   // groups of a CTA, this thread's and its place in it
  for (int i0 = rank * groups; i0 < a.n; i0 += C * groups) {
    const int i = i0 + mine;
    int count = 0, last = -1;
    int4 rec = make_int4(-1, 0, 0, 0);
    if (i < a.n) {
      const int slot = SMALL ? slot_s[i] : a.slots[i];
      if (slot >= 0 && slot < a.max_seqs) {
        bool first = true;
        if (SMALL) {
          for (int x = lane; x < i; x += 32) first = first && slot_s[x] != slot;
          first = __all_sync(0xffffffffu, first);
        } else {
          first = __ldcg(&s.owner[slot]) == i;
        }
        if (first) rec.x = slot;
        else if (gt == 0) report(SNAP_DEV_BAD_SLOT);
      }
      if (rec.x >= 0) {
        rec.y = SMALL ? new_s[i] : a.new_tokens[i];
        rec.z = max(SMALL ? len_s[i] : a.seq_len[slot], 0);
        if (rec.y < 0) rec.z = 0;
        const int* row = a.table_in + (long long)slot * a.max_pages;
        const long long rows = (long long)rec.z + rec.y;
        if (SMALL && rec.y >= 0 && apart) {                              // (what is granted is written over it, phases later)
          int* out = a.table_out + (long long)slot * a.max_pages;
          if (fours(a, row, out)) {
#pragma unroll 4
            for (int j = 4 * gt; j < a.max_pages; j += 4 * gn) *reinterpret_cast<int4*>(out + j) = *reinterpret_cast<const int4*>(row + j);
          } else {
#pragma unroll 8
            for (int j = gt; j < a.max_pages; j += gn) out[j] = row[j];
          }
        }
        if (rec.y < 0) {
          over(row, 0, a.max_pages, gt, gn, [&](int j, int e) { if (held(a, e)) { ++count; last = j; } });
        } else if (rows <= (long long)a.page * a.max_pages) {
          const int j0 = pages_of(a, rec.z);
          over(row, j0, pages_of(a, rows) - j0, gt, gn, [&](int, int e) { count += !held(a, e); });
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
  phase();

  // ---- the scan ----
  if (rank == 0) {
    const int per = (a.n + NT - 1) / NT, i0 = min(tid * per, a.n), i1 = min(i0 + per, a.n);
    const int given = *a.n_free_in, n0 = min(max(given, 0), a.n_pages);
    Three sum = {{0, 0, 0}}, all;                                        // pages given back, tokens wanted, pages missing
    for (int i = i0; i < i1; ++i) {
      const int4 r = left(&s.rec[i]);
      if (r.x < 0 || r.w < 0) continue;
      if (r.y < 0) sum.x[0] += r.w;
      else { sum.x[1] += r.y; sum.x[2] += r.w; }
    }
    const Three before = block_exclusive(sum, part, all);
    const int there = (int)min(n0 + all.x[0], (long long)a.n_pages);
    if (tid == 0 && (given != n0 || n0 + all.x[0] > a.n_pages)) report(SNAP_DEV_BAD_PAGE);
    const auto fits = [&](long long wanted, long long missing, int own) { return wanted <= a.n_tokens_max && (own == 0 || missing <= there); };
    Three got = {{0, 0, 0}}, all_got;                                    // tokens and pages granted
    unsigned bad = 0;
    long long want = before.x[1], miss = before.x[2];
    for (int i = i0; i < i1; ++i) {
      const int4 r = left(&s.rec[i]);
      if (r.x < 0 || r.y < 0 || r.w < 0) continue;
      want += r.y;
      miss += r.w;
      if (fits(want, miss, r.w)) { got.x[0] += r.y; got.x[1] += r.w; }
      else bad = SNAP_DEV_NO_ROOM;
    }
    report(bad);
    long long at = block_exclusive(got, part, all_got).x[0], back = before.x[0];
    want = before.x[1];
    miss = before.x[2];
    for (int i = i0; i < i1; ++i) {
      const int4 r = left(&s.rec[i]);
      int4 res = make_int4((int)min(back, (long long)INT_MAX), 0, -1, (int)at);
      if (r.x >= 0 && r.y < 0) back += r.w;
      else if (r.x >= 0 && r.w >= 0) {
        want += r.y;
        res.y = (int)min(miss, (long long)INT_MAX);
        miss += r.w;
        if (fits(want, miss, r.w)) { res.z = r.y; at += r.y; }
      }
      s.res[i] = res;
      a.cu[i] = res.w;
      a.first_rows[i] = r.z;
      if (a.granted) a.granted[i] = max(res.z, 0);
    }
    if (tid == 0) {
      a.cu[a.n] = (int)all_got.x[0];
      *a.n_free_out = there - (int)all_got.x[1];
      *s.head = {n0, there, (int)all_got.x[0]};
    }
  }
  phase();

  // ---- pages given back ----
  const Head head = {left(&s.head->n0), left(&s.head->there), left(&s.head->tokens)};
  for (int i = rank * groups + mine; i < a.n; i += C * groups) {
    const int4 r = left(&s.rec[i]);
    if (r.x < 0 || r.y >= 0) continue;
    const int* row = a.table_in + (long long)r.x * a.max_pages;
    int* out = a.table_out + (long long)r.x * a.max_pages;
    const long long at = (long long)head.n0 + left(&s.res[i]).x;
    if (left(&s.last[i]) + 1 == r.w) {                                   // they are the row's first entries
      const auto back = [&](int j, int e) { if (j < r.w && at + j < a.n_pages) a.stack[at + j] = e; };
      if (fours(a, row, out)) {
#pragma unroll 4
        for (int j = 4 * gt; j < a.max_pages; j += 4 * gn) {
          if (j < r.w) {
            const int4 e = *reinterpret_cast<const int4*>(row + j);
            back(j, e.x); back(j + 1, e.y); back(j + 2, e.z); back(j + 3, e.w);
          }
          *reinterpret_cast<int4*>(out + j) = make_int4(-1, -1, -1, -1);
        }
      } else {
#pragma unroll 8
        for (int j = gt; j < a.max_pages; j += gn) {
          if (j < r.w) back(j, row[j]);
          out[j] = -1;
        }
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
  // ---- the lists of tokens ----
  if (!SMALL) return;
  const Lists lists = {cu_s, slot_s, row_s, s, a.n, head.tokens, true};
  lists.take(NT);
  __syncthreads();
  for (long long t0 = 4LL * tid; t0 < a.n_tokens_max; t0 += 4LL * NT) lists.write(a, t0);
  __syncthreads();

  // ---- the granted pages ----
  for (int i = rank * groups + mine; i < a.n; i += C * groups) {
    const int4 r = left(&s.rec[i]), res = left(&s.res[i]);
    if (res.z < 0 || r.w <= 0) continue;
    const int* row = a.table_in + (long long)r.x * a.max_pages;
    int* out = a.table_out + (long long)r.x * a.max_pages;
    const int j0 = pages_of(a, r.z), j1 = pages_of(a, (long long)r.z + r.y), top = head.there - 1 - res.y;
    if (r.w == j1 - j0) {                                                // none of them holds a page
#pragma unroll 4
      for (int j = j0 + gt; j < j1; j += gn) out[j] = granted_page(a, top - (j - j0));
    } else if (gt < 32) {
      fill_gaps(a, row, out, j0, j1, top);
    }
  }
}

// The second launch of a larger call: lists, and table rows with what is granted.  A CTA takes PIECE tokens or PIECE entries of a row at a time.
__global__ void __launch_bounds__(RNT) paged_plan_rows_kernel(const __grid_constant__ PlanArgs a) {
  __shared__ int cu_s[MAX_HELD + 1], slot_s[MAX_HELD], row_s[MAX_HELD];
  const int tid = threadIdx.x;
  Scratch s;
  carve(a.scratch, a.max_seqs, a.n, &s);
  pdl_wait();
  const Head head = {left(&s.head->n0), left(&s.head->there), left(&s.head->tokens)};
  const Lists lists = {cu_s, slot_s, row_s, s, a.n, head.tokens, a.n <= MAX_HELD};
  lists.take(RNT);
  __syncthreads();
  const bool apart = a.table_in != a.table_out;
  const int pieces = a.pieces;                                           // of a request's row, or, in place, of the entries it is granted
  const long long of_lists = ((long long)a.n_tokens_max + PIECE - 1) / PIECE, items = of_lists + (long long)a.n * pieces;
  for (long long x = blockIdx.x; x < items; x += gridDim.x) {
    if (x < of_lists) {
      const long long t0 = x * PIECE + 4 * tid;
      if (t0 < a.n_tokens_max) lists.write(a, t0);
      continue;
    }
    const int i = (int)((x - of_lists) / pieces), piece = (int)((x - of_lists) - (long long)i * pieces);
    const int4 r = left(&s.rec[i]), res = left(&s.res[i]);
    if (r.x < 0 || r.y < 0) continue;
    const int* row = a.table_in + (long long)r.x * a.max_pages;
    int* out = a.table_out + (long long)r.x * a.max_pages;
    const bool granted = res.z >= 0 && r.w > 0;
    const int j0 = granted ? pages_of(a, r.z) : 0, j1 = granted ? pages_of(a, (long long)r.z + r.y) : 0, top = head.there - 1 - res.y;
    const int b0 = (apart ? 0 : j0) + piece * PIECE, b1 = min(b0 + PIECE, apart ? a.max_pages : j1);
    const bool gaps = granted && r.w != j1 - j0;                         // some of them hold a page: one warp, after the copy
    if (apart && fours(a, row, out)) {
      const int j = b0 + 4 * tid;
      if (j < b1) {
        int4 e = *reinterpret_cast<const int4*>(row + j);
        if (!gaps && j < j1 && j + 4 > j0) {
          if (j >= j0) e.x = granted_page(a, top - (j - j0));
          if (j + 1 >= j0 && j + 1 < j1) e.y = granted_page(a, top - (j + 1 - j0));
          if (j + 2 >= j0 && j + 2 < j1) e.z = granted_page(a, top - (j + 2 - j0));
          if (j + 3 >= j0 && j + 3 < j1) e.w = granted_page(a, top - (j + 3 - j0));
        }
        if (!gaps) *reinterpret_cast<int4*>(out + j) = e;
        else if (j + 4 <= j0 || j >= j1) *reinterpret_cast<int4*>(out + j) = e;
        else {
          if (j < j0) out[j] = e.x;
          if (j + 1 < j0 || j + 1 >= j1) out[j + 1] = e.y;
          if (j + 2 < j0 || j + 2 >= j1) out[j + 2] = e.z;
          if (j + 3 >= j1) out[j + 3] = e.w;
        }
      }
    } else {
      for (int j = b0 + tid; j < b1; j += RNT) {
        const bool here = j >= j0 && j < j1;
        if (here && !gaps) out[j] = granted_page(a, top - (j - j0));
        else if (!here && apart) out[j] = row[j];
      }
    }
    if (gaps && piece == 0 && tid < 32) fill_gaps(a, row, out, j0, j1, top);
  }
}

}  // namespace

size_t paged_plan_scratch_bytes(int max_seqs, int n_seqs) { return carve(nullptr, max_seqs, n_seqs, nullptr); }

// One CTA where there is little to do, else a cluster of 16 (8 where the device takes no more) and the second launch.  (One CTA against
// two launches: 32 requests, rows of 512 entries 9.3 / 12.8 us; 64 13.1 / 13.9; 128 19.3 / 14.0; 32 of 1024 tokens each 15.9 / 13.3; 8 of
// 4096 13.9 / 13.1.  Clusters of 16 / 8 / 4: 75 requests of 614405 tokens, rows of 8192 entries 22.3 / 25.9 / 31.9; 2000 requests 34.9 / 43.3
// / 59.1; no call was shorter with fewer.)
// In place a request reads few entries unless it ends, and then the whole row, 5.8 us of one CTA for 8192 entries; the rule takes one in a hundred to
// end.  (One CTA / two launches, in place: nobody ends, 16 requests 7.4 / 12.3, 32 with rows of 8192 entries 7.0 / 13.9, 128 of 512 12.3 / 14.8, 250
// of 512 21.4 / 17.2, 250 of 8192 21.3 / 17.6; one in fifty ends, 250 of 8192 51 / 21; one in ten, 64 of 8192 26 / 15.5, 128 of 4096 37 / 17.8, 128
// of 512 15.2 / 15.6; three in ten, 32 of 8192 27 / 17.6, 250 of 512 27.5 / 20.9, 250 of 8192 182 / 28; all, 200 of 15000 501 / 54, one of 15000 9.8 / 14.7.)
cudaError_t launch_paged_plan(const PlanArgs& a, cudaStream_t st) {
  const long long entries = (long long)a.n * (a.table_in != a.table_out ? a.max_pages : 160 + a.max_pages / 48) + a.n_tokens_max;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc = {};
  lc.stream = st;
  lc.attrs = attr;
  lc.numAttrs = 1;
  cudaError_t e;
  if (a.n <= SMALL_N && entries <= 32768) {
    lc.gridDim = dim3(1);
    lc.blockDim = dim3(NT);
    e = cudaLaunchKernelEx(&lc, paged_plan_kernel<true>, a);
  } else {
    const auto kernel = paged_plan_kernel<false>;
    static int widest[kMaxDevices] = {};                                 // CTAs of a cluster that the device takes
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 16; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    lc.blockDim = dim3(NT);
    lc.gridDim = dim3(16);
    lc.numAttrs = 2;
    if (widest[dev] == 0) {
      int fit = 0;
      const bool wide = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                        cudaOccupancyMaxActiveClusters(&fit, kernel, &lc) == cudaSuccess && fit > 0;
      (void)cudaGetLastError();
      widest[dev] = wide ? 16 : 8;
    }
    const int cluster = widest[dev];
    attr[1].val.clusterDim.x = cluster;
    lc.gridDim = dim3(cluster);
    if ((e = cudaLaunchKernelEx(&lc, kernel, a)) != cudaSuccess) return e;
    count_launch();
    // (in place no row is granted more entries than the list's tokens begin, and one that the first ends in)
    PlanArgs rows = a;
    const long long wide = a.table_in != a.table_out ? a.max_pages : std::min<long long>(a.max_pages, a.n_tokens_max / a.page + 2);
    rows.pieces = (int)((wide + PIECE - 1) / PIECE);
    const long long items = ((long long)a.n_tokens_max + PIECE - 1) / PIECE + (long long)a.n * rows.pieces, most = 4LL * sm_count();
    e = launch_pdl(paged_plan_rows_kernel, dim3((unsigned)(items < most ? items : most)), dim3(RNT), 0, st, rows);
  }
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
