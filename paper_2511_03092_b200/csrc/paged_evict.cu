// Eviction from a paged cache by accumulated attention weight (snap_paged_evict): per (sequence, KV head) the
// sinks, the topk rows of the middle with the largest weight and the last l_recent rows move, in order, to the
// pages of another slot.
//
// Selection: one CTA per (sequence, KV head), or a cluster of up to eight for long middles, with its slice of the
// middle's weights in shared memory as order-preserving integers.  The topk-th largest is found by radix steps of
// 11 bits over the range that the keys really span (weights of one layer lie within a few octaves, so the digits
// of the raw bit pattern would fall into a handful of bins and the counting atomics would queue on them); the CTAs
// of a cluster read each other's counts through distributed shared memory.  Equal keys at the threshold go to the
// lower rows; the chosen rows leave in ascending order by counting ranks per CTA, warp and lane (nothing depends on
// timing).
//
// Copy: bound by HBM (each kept row read and written once).  A lane looks up one row's pages, then the warp moves
// its rows with eight 16-byte loads per lane in flight.  The rows that stay whatever the selection says (sinks, last
// rows, sequences within the budget) are copied while the selection, which leaves most SMs idle, is still running: the
// blocks are in the order that starts with the last rows, and a warp waits only where it has rows of the middle.
#include <cooperative_groups.h>

#include "snap_internal.cuh"

namespace snap {
namespace {

namespace cg = cooperative_groups;

constexpr int ENT = 1024, NB = 2048, NB_BITS = 11;      // threads of a selection CTA, bins of a radix step
constexpr int LOADS = 16;                                // loads of a thread in flight
constexpr int MAX_KEYS = 45000;                          // keys of a slice that are kept in shared memory (180 KB)

struct EvictArgs {
  const int* src; const int* dst;
  int n, Hkv, Ls, Lr, K, max_seqs;
  PageMap map;
  int* seq_len;
  const float* w_in; float* w_out;
  int* idx;                            // [n][Hkv][K] selected rows, ascending
  int* kept;                           // NULL or [n][Hkv][Ls + K + Lr]
  char* kp; char* vp;
  int k_vecs, v_vecs, eb;              // 16-byte pieces of a row; bytes of an element
  unsigned k_magic, v_magic;           // p / k_vecs = p * k_magic >> 20 for the pieces of a warp
  uint32_t* status;
  int keys_cap;                        // keys of a slice that fit the launch's shared memory (0: read from global every time)
};

// Larger weight, larger key; -0 counts as 0, NaN below everything.
__device__ __forceinline__ unsigned key_of(float w) {
  if (isnan(w)) return 0u;
  const unsigned u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// May sequence i be moved?  (All threads of the block.)  Its destination must be no source and no earlier destination.
template <int NT>
__device__ bool entry_ok(const EvictArgs& a, int i, int& src, int& dst) {
  src = a.src[i];
  dst = a.dst[i];
  int clash = src < 0 || src >= a.max_seqs || dst < 0 || dst >= a.max_seqs;
  for (int e = threadIdx.x; e < a.n; e += NT) clash |= a.src[e] == dst || (e < i && a.dst[e] == dst);
  return !__syncthreads_or(clash);
}

// CLUSTER: two to eight CTAs share a middle; otherwise one has it all and the cluster's barriers and reads fall away.
template <bool CLUSTER>
__global__ void __launch_bounds__(ENT) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ unsigned keys[];                     // [keys_cap]
  __shared__ __align__(16) int hist[2][NB];
  __shared__ int warp_s[ENT / 32], warp_e[ENT / 32];
  __shared__ unsigned s_red[2][ENT / 32], s_range[2];
  __shared__ int s_bin, s_above, s_in, s_cnt[2], s_len;
  cg::cluster_group cl = cg::this_cluster();
  const int CL = CLUSTER ? (int)cl.num_blocks() : 1, rank = CLUSTER ? (int)cl.block_rank() : 0;
  const auto barrier = [&]() { if (CLUSTER) cl.sync(); else __syncthreads(); };
  const int kvh = blockIdx.y, i = blockIdx.z, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  for (int b = tid; b < 2 * NB; b += ENT) (&hist[0][0])[b] = 0;
  pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int src = 0, dst;
  const bool ok = entry_ok<ENT>(a, i, src, dst);
  if (rank == 0 && tid == 0) {                           // one reading of the length for the whole cluster
    const int len = ok ? a.seq_len[src] : -1;
    s_len = ok ? min(max(len, 0), a.map.cap) : -1;
    if (kvh == 0) {
      const unsigned bad = (ok ? 0u : SNAP_DEV_BAD_SLOT) | (len > a.map.cap ? SNAP_DEV_BAD_PAGE : 0u);
      if (bad && a.status) atomicOr(a.status, bad);
    }
  }
  barrier();
  const int len = CLUSTER ? *cl.map_shared_rank(&s_len, 0) : s_len;
  const int keep = a.Ls + a.K + a.Lr;
  if (len <= keep || a.K == 0) {                         // uniform over the cluster: nothing to select
    if (CLUSTER) cl.sync();                              // (the length has been read everywhere)
    return;
  }
  const int m = len - a.Ls - a.Lr;                       // candidates: more than K
  const int per = (m + CL - 1) / CL, c0 = min(rank * per, m), mine = min(c0 + per, m) - c0;
  const float* wt = a.w_in + ((long long)src * a.Hkv + kvh) * a.map.cap + a.Ls + c0;
  const bool held = per <= a.keys_cap;
  const auto key = [&](int e) { return held ? keys[e] : key_of(wt[e]); };

  // ---- the range the keys span ----
  unsigned lo = 0xffffffffu, hi = 0u;
  for (int e0 = tid; e0 < mine; e0 += LOADS * ENT) {     // (one CTA's loads in flight are all there is to hide the latency)
    float x[LOADS];
#pragma unroll
    for (int u = 0; u < LOADS; ++u)
      if (e0 + u * ENT < mine) x[u] = __ldcg(wt + e0 + u * ENT);
#pragma unroll
    for (int u = 0; u < LOADS; ++u)
      if (e0 + u * ENT < mine) {
        const unsigned k = key_of(x[u]);
        if (held) keys[e0 + u * ENT] = k;
        lo = min(lo, k);
        hi = max(hi, k);
      }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) { s_red[0][w] = lo; s_red[1][w] = hi; }
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, s_red[0][lane]);   // 32 warps: every warp reduces them all
  hi = __reduce_max_sync(0xffffffffu, s_red[1][lane]);
  if (CLUSTER) {
    if (tid == 0) { s_range[0] = lo; s_range[1] = hi; }
    cl.sync();
    lo = __reduce_min_sync(0xffffffffu, lane < CL ? cl.map_shared_rank(s_range, lane)[0] : 0xffffffffu);
    hi = __reduce_max_sync(0xffffffffu, lane < CL ? cl.map_shared_rank(s_range, lane)[1] : 0u);
  }

  // ---- the K-th largest key: it lies in [base, base + 2^bits), `need` keys of that range are wanted ----
  unsigned base = lo;
  int bits = lo == hi ? 0 : 32 - __clz(hi - lo);
  int need = a.K;
  bool all = false;                                      // every key of the range is wanted
  for (int step = 0; bits > 0 && !all; ++step) {
    int* h = hist[step & 1];
    const int shift = max(bits - NB_BITS, 0);
    const unsigned span = bits == 32 ? 0xffffffffu : (1u << bits) - 1u;
#pragma unroll 4
    for (int e = tid; e < mine; e += ENT) {
      const unsigned k = key(e);
      if (k >= base && k - base <= span) atomicAdd(&h[(k - base) >> shift], 1);
    }
    barrier();                                           // every CTA's counts are there
    // thread t has bins NB - 1 - 2 t and the one below: descending order over threads
    constexpr int BPT = NB / ENT;
    static_assert(BPT == 2, "a thread reads its two bins as one int2");
    int cnt[BPT] = {0, 0};
    if (CLUSTER) {
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < CL) {
          const int2 v = *reinterpret_cast<const int2*>(cl.map_shared_rank(h, r) + NB - BPT * (tid + 1));
          cnt[0] += v.y; cnt[1] += v.x;
        }
    } else {
      const int2 v = *reinterpret_cast<const int2*>(h + NB - BPT * (tid + 1));
      cnt[0] = v.y; cnt[1] = v.x;
    }
    const int sum = cnt[0] + cnt[1];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += x; }
    if (lane == 31) warp_s[w] = incl;
    // the other buffer is free again: every CTA has read it before the barrier above
    for (int b = tid; b < NB; b += ENT) hist[(step + 1) & 1][b] = 0;
    __syncthreads();
    int above = incl - sum + __reduce_add_sync(0xffffffffu, lane < w ? warp_s[lane] : 0);
#pragma unroll
    for (int b = 0; b < BPT; ++b) {
      if (above < need && above + cnt[b] >= need) { s_bin = NB - 1 - BPT * tid - b; s_above = above; s_in = cnt[b]; }   // one thread
      above += cnt[b];
    }
    __syncthreads();
    base += (unsigned)s_bin << shift;
    need -= s_above;
    all = s_in == need;
    bits = shift;
  }
  // keys in [base, base + 2^bits) are at the threshold: `need` of them are taken, the lower rows first; above: all
  const unsigned span = bits == 32 ? 0xffffffffu : (1u << bits) - 1u;

  // ---- emission in row order: a thread has a run of consecutive candidates (an odd number of them, so that the threads
  // of a warp read different banks), counts them, and learns from a scan where its rows go ----
  const int run = ((mine + ENT - 1) / ENT) | 1, e0 = min(tid * run, mine), e1 = min(e0 + run, mine);
  int gt = 0, eq = 0;
  for (int e = e0; e < e1; ++e) {
    const unsigned k = key(e);
    const bool at = k >= base && k - base <= span;
    gt += k >= base && !at;
    eq += at;
  }
  const auto scan = [&](int v, int* warps) {             // exclusive over the CTA
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += x; }
    if (lane == 31) warps[w] = incl;
    return incl - v;
  };
  __syncthreads();                                       // warp_s has been read
  int gt_before = scan(gt, warp_s), eq_before = scan(eq, warp_e);
  __syncthreads();
  gt_before += __reduce_add_sync(0xffffffffu, lane < w ? warp_s[lane] : 0);
  eq_before += __reduce_add_sync(0xffffffffu, lane < w ? warp_e[lane] : 0);
  if (CLUSTER) {
    if (tid == ENT - 1) { s_cnt[0] = gt_before + gt; s_cnt[1] = eq_before + eq; }
    cl.sync();
    gt_before += __reduce_add_sync(0xffffffffu, lane < rank ? cl.map_shared_rank(s_cnt, lane)[0] : 0);
    eq_before += __reduce_add_sync(0xffffffffu, lane < rank ? cl.map_shared_rank(s_cnt, lane)[1] : 0);
  }
  int* out = a.idx + ((long long)i * a.Hkv + kvh) * a.K;
  int pos = gt_before + min(eq_before, need);
  for (int e = e0; e < e1; ++e) {
    const unsigned k = key(e);
    if (k < base) continue;
    const bool at = k - base <= span, take = !at || eq_before < need;
    eq_before += at;
    if (take) {
      if (index_ok(pos, a.K, a.status)) out[pos] = a.Ls + c0 + e;
      ++pos;
    }
  }
  if (CLUSTER) cl.sync();                                // no CTA leaves while another may read its counts
}

constexpr int CNT = 256;                                 // threads of a copy CTA

// Grid: row groups x (sequence, KV head), the last row group of all of those first; a warp moves CROWS rows.  SAME: keys and
// values are laid out alike, so that one offset serves both.  What is read before the wait was written before the
// selection kernel started; it is read past L1.  (Except the slots, which all blocks go through and which L1 therefore serves: past
// it 4 sequences of 6148 to 8000 rows take 36.5 us instead of 35.4, 12 of them with 4 KV heads of 64 dims 38.7 instead of 37.0.  A launch
// finds nothing older in L1: replayed evictions whose slots a kernel had rewritten right before them go by the new ones.)
template <int CROWS, bool SAME>
__global__ void __launch_bounds__(CNT, 4) evict_copy_kernel(const __grid_constant__ EvictArgs a, int groups) {
  const int units = a.n * a.Hkv, group = groups - 1 - (int)(blockIdx.x / units), unit = blockIdx.x % units;
  const int i = unit / a.Hkv, kvh = unit - i * a.Hkv, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int keep = a.Ls + a.K + a.Lr, r0 = (group * (CNT / 32) + w) * CROWS;
  int src, dst;
  const bool ok = entry_ok<CNT>(a, i, src, dst);
  const int len = ok ? min(max(__ldcg(a.seq_len + src), 0), a.map.cap) : -1, rows = len < keep ? len : keep;
  const bool selected = len > keep && r0 < a.Ls + a.K && r0 + CROWS > a.Ls;      // rows of the middle among the warp's
  if (selected) pdl_wait();
  // lane l < CROWS: row r0 + l of the destination; byte offsets of its source and destination, ks < 0: nothing to copy
  long long ks = -1, kd = 0, vs = 0, vd = 0;
  if (lane < CROWS && r0 + lane < keep) {
    const int r = r0 + lane;
    int from = -1;
    if (r < rows) {
      if (len <= keep || r < a.Ls) from = r;
      else if (r < a.Ls + a.K) from = __ldcg(a.idx + ((long long)i * a.Hkv + kvh) * a.K + r - a.Ls);
      else from = len - keep + r;
      if (!index_ok(from, len, a.status)) from = -1;
    }
    if (a.kept) a.kept[((long long)i * a.Hkv + kvh) * keep + r] = from;
    if (from >= 0) {
      const int sp = from / a.map.page, dp = r / a.map.page;
      const int s_page = __ldcg(a.map.table + (long long)src * a.map.max_pages + sp);
      const int d_page = dp < a.map.max_pages ? __ldcg(a.map.table + (long long)dst * a.map.max_pages + dp) : -1;
      if (s_page < 0 || s_page >= a.map.n_pages || d_page < 0 || d_page >= a.map.n_pages) {
        if (a.status) atomicOr(a.status, SNAP_DEV_BAD_PAGE);
      } else {
        const int so = from - sp * a.map.page, dof = r - dp * a.map.page;
        ks = (s_page * a.map.kp + kvh * a.map.kh + so * a.map.kr) * a.eb;
        kd = (d_page * a.map.kp + kvh * a.map.kh + dof * a.map.kr) * a.eb;
        vs = (s_page * a.map.vp + kvh * a.map.vh + so * a.map.vr) * a.eb;
        vd = (d_page * a.map.vp + kvh * a.map.vh + dof * a.map.vr) * a.eb;
        if (a.w_out) {
          const long long b = (long long)kvh * a.map.cap, per = (long long)a.Hkv * a.map.cap;
          a.w_out[dst * per + b + r] = __ldcg(a.w_in + src * per + b + from);
        }
      }
    }
  }
  // the rows' 16-byte pieces, U per lane and tensor in flight
  const auto move = [&](int vecs, unsigned magic, long long s_off, long long d_off, char* p0, char* p1) {
    constexpr int U = 4;
    for (int b = 0; b < CROWS * vecs; b += 32 * U) {
      uint4 x[U], y[SAME ? U : 1];
      long long to[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const unsigned p = b + 32 * u + lane, row = p * magic >> 20, c = p - row * vecs;
        const int from = row < CROWS ? (int)row : 0;
        const long long s = __shfl_sync(0xffffffffu, s_off, from), d = __shfl_sync(0xffffffffu, d_off, from);
        to[u] = row < CROWS && s >= 0 ? d + 16 * c : -1;
        if (to[u] >= 0) {
          x[u] = __ldcg(reinterpret_cast<const uint4*>(p0 + s + 16 * c));
          if (SAME) y[SAME ? u : 0] = __ldcg(reinterpret_cast<const uint4*>(p1 + s + 16 * c));
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (to[u] >= 0) {
          *reinterpret_cast<uint4*>(p0 + to[u]) = x[u];
          if (SAME) *reinterpret_cast<uint4*>(p1 + to[u]) = y[SAME ? u : 0];
        }
    }
  };
  move(a.k_vecs, a.k_magic, ks, kd, a.kp, a.vp);
  if (!SAME) move(a.v_vecs, a.v_magic, ks < 0 ? -1 : vs, vd, a.vp, nullptr);
  pdl_wait();                                              // nobody leaves before the selection has ended
  if (ok && kvh == 0 && group == 0 && threadIdx.x == 0) a.seq_len[dst] = rows;
}

template <int CROWS>
cudaError_t launch_copy(const EvictArgs& a, int keep, bool same, cudaStream_t st) {
  constexpr int per = CNT / 32 * CROWS;
  const int groups = (keep + per - 1) / per;
  const dim3 grid((unsigned)((long long)groups * a.n * a.Hkv));
  return same ? launch_pdl(evict_copy_kernel<CROWS, true>, grid, dim3(CNT), 0, st, a, groups)
              : launch_pdl(evict_copy_kernel<CROWS, false>, grid, dim3(CNT), 0, st, a, groups);
}

}  // namespace

size_t paged_evict_scratch_bytes(const Shape& s, int n_seqs) {
  return align_up((size_t)n_seqs * s.Hkv * (s.K > 0 ? s.K : 1) * sizeof(int));
}

cudaError_t launch_paged_evict(int dtype, const Shape& s, const PageMap& m, const int* src, const int* dst, int n_seqs,
                               void* k_pages, void* v_pages, int* seq_len, const float* w_in, float* w_out, int* kept,
                               char* scratch, uint32_t* status, cudaStream_t st) {
  EvictArgs a;
  a.src = src; a.dst = dst; a.n = n_seqs; a.Hkv = s.Hkv; a.Ls = s.Ls; a.Lr = s.Lr; a.K = s.K; a.max_seqs = s.max_seqs;
  a.map = m; a.seq_len = seq_len; a.w_in = w_in; a.w_out = w_out; a.kept = kept; a.status = status;
  a.idx = reinterpret_cast<int*>(scratch);
  a.kp = static_cast<char*>(k_pages); a.vp = static_cast<char*>(v_pages);
  a.eb = elt_bytes(dtype);
  a.k_vecs = s.d_qk * a.eb / 16; a.v_vecs = s.d_v * a.eb / 16;
  a.k_magic = ((1u << 20) + a.k_vecs - 1) / a.k_vecs;       // exact below 2^20 / vecs: a warp has 32 rows of 64 pieces at most
  a.v_magic = ((1u << 20) + a.v_vecs - 1) / a.v_vecs;
  const int most = m.cap - s.Ls - s.Lr;                    // candidates there can be
  // CTAs of a middle: as many as bring a slice down to 8192 keys while each has an SM to itself (96 middles of 32k on one
  // CTA each take 20 us, on two 25), more where a slice would not fit shared memory.
  int CL = 1;
  while (CL < 8 && (most / CL > MAX_KEYS || (most / CL > 8192 && 2LL * CL * n_seqs * s.Hkv <= (long long)sm_count()))) CL *= 2;
  const bool cluster = CL > 1;
  const int per = most > 0 ? (most + CL - 1) / CL : 0;
  a.keys_cap = per <= MAX_KEYS ? per : 0;
  const size_t smem = (size_t)a.keys_cap * sizeof(unsigned);
  cudaError_t e;
  if (cluster) {
    static SmemLimit limit = {};
    if ((e = ensure_dyn_smem(evict_select_kernel<true>, smem < 1024 ? 1024 : smem, limit)) != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)CL;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(CL, s.Hkv, n_seqs);
    lc.blockDim = dim3(ENT);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    lc.attrs = attr;
    lc.numAttrs = 2;
    e = cudaLaunchKernelEx(&lc, evict_select_kernel<true>, a);
  } else {
    static SmemLimit limit = {};
    if ((e = ensure_dyn_smem(evict_select_kernel<false>, smem < 1024 ? 1024 : smem, limit)) != cudaSuccess) return e;
    e = launch_pdl(evict_select_kernel<false>, dim3(1, s.Hkv, n_seqs), dim3(ENT), smem, st, a);
  }
  count_launch();
  if (e != cudaSuccess) return e;
  const bool same = m.kp == m.vp && m.kh == m.vh && m.kr == m.vr && a.k_vecs == a.v_vecs;
  // Many rows: 32 per warp, so that a warp's look-ups serve four batches of loads; few: 8, to have more warps.  (us with 32 / 8, 8 KV
  // heads of 128 dims, 5124 rows stay: 1 sequence 18.4 / 16.0, 4 35.5 / 35.3, 6 48.3 / 49.5, 8 61.1 / 63.1, 12 88.0 / 91.5.)
  const bool many = (long long)n_seqs * s.Hkv * s.Sc >= 2048LL * sm_count();
  e = many ? launch_copy<32>(a, s.Sc, same, st) : launch_copy<8>(a, s.Sc, same, st);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
