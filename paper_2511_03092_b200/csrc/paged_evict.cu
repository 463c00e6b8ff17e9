// Eviction from a paged cache by accumulated attention weight (snap_paged_evict): per (sequence, KV head) the
// sinks, the topk rows of the middle with the largest weight and the last l_recent rows move, in order, to the
// pages of another slot.
//
// Selection: a cluster of CTAs per (sequence, KV head), each with a slice of the middle's weights in shared
// memory as order-preserving integers.  The topk-th largest is found by radix steps of 11 bits over the range
// that the keys really span (weights of one layer lie within a few octaves, so the digits of the raw bit pattern
// would fall into a handful of bins and the counting atomics would queue on them); each CTA counts its slice and
// reads the others' counts through distributed shared memory.  Equal keys at the threshold go to the lower rows;
// the chosen rows leave in ascending order by counting ranks per CTA, warp and lane (nothing depends on timing).
//
// Copy: bound by HBM (each kept row read and written once).  A warp moves eight rows with all their loads in
// flight; page numbers and source rows are looked up by one lane per row.
#include <cooperative_groups.h>

#include "snap_internal.cuh"

namespace snap {
namespace {

namespace cg = cooperative_groups;

constexpr int ENT = 512, NB = 2048, NB_BITS = 11;       // threads of a selection CTA, bins of a radix step
constexpr int MAX_KEYS = 45000;                          // keys of a slice that are kept in shared memory (180 KB)

struct EvictArgs {
  const int* src; const int* dst;
  int n, Hkv, Ls, Lr, K, max_seqs;
  PageMap map;
  int* seq_len;
  const float* w_in; float* w_out;
  int* idx;                            // [n][Hkv][K] selected rows, ascending
  int* len;                            // [n] rows of each sequence, -1: skipped
  int* kept;                           // NULL or [n][Hkv][Ls + K + Lr]
  char* kp; char* vp;
  int k_vecs, v_vecs, eb;              // 16-byte pieces of a row; bytes of an element
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

__global__ void __launch_bounds__(ENT) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ unsigned keys[];                     // [keys_cap]
  __shared__ __align__(16) int hist[2][NB];
  __shared__ int warp_s[ENT / 32];
  __shared__ unsigned s_lo, s_hi, s_red[2][ENT / 32];
  __shared__ int s_bin, s_above, s_in, s_cnt[2], s_len;
  cg::cluster_group cl = cg::this_cluster();
  const int CL = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int kvh = blockIdx.y, i = blockIdx.z, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
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
      a.len[i] = s_len;
    }
  }
  cl.sync();
  const int len = *cl.map_shared_rank(&s_len, 0);
  const int keep = a.Ls + a.K + a.Lr;
  if (len <= keep || a.K == 0) {                         // uniform over the cluster: nothing to select
    cl.sync();                                           // (the length has been read everywhere)
    return;
  }
  const int m = len - a.Ls - a.Lr;                       // candidates: more than K
  const int per = (m + CL - 1) / CL, c0 = min(rank * per, m), mine = min(c0 + per, m) - c0;
  const float* wt = a.w_in + ((long long)src * a.Hkv + kvh) * a.map.cap + a.Ls + c0;
  const bool held = per <= a.keys_cap;
  const auto key = [&](int e) { return held ? keys[e] : key_of(wt[e]); };

  // ---- the range the keys span ----
  unsigned lo = 0xffffffffu, hi = 0u;
#pragma unroll 4
  for (int e = tid; e < mine; e += ENT) {
    const unsigned k = key_of(wt[e]);
    if (held) keys[e] = k;
    lo = min(lo, k);
    hi = max(hi, k);
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) { s_red[0][w] = lo; s_red[1][w] = hi; }
  for (int b = tid; b < 2 * NB; b += ENT) (&hist[0][0])[b] = 0;
  __syncthreads();
  if (w == 0) {
    lo = lane < ENT / 32 ? s_red[0][lane] : 0xffffffffu;
    hi = lane < ENT / 32 ? s_red[1][lane] : 0u;
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) { s_lo = lo; s_hi = hi; }
  }
  cl.sync();
  lo = 0xffffffffu; hi = 0u;
  for (int r = 0; r < CL; ++r) {
    lo = min(lo, *cl.map_shared_rank(&s_lo, r));
    hi = max(hi, *cl.map_shared_rank(&s_hi, r));
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
    for (int e = tid; e < mine; e += ENT) {
      const unsigned k = key(e);
      if (k >= base && k - base <= span) atomicAdd(&h[(k - base) >> shift], 1);
    }
    cl.sync();                                           // every CTA's counts are there
    // thread t has bins NB - 1 - 4 t and the three below: descending order over threads
    constexpr int BPT = NB / ENT;
    int cnt[BPT], sum = 0;
#pragma unroll
    for (int b = 0; b < BPT; ++b) cnt[b] = 0;
    for (int r = 0; r < CL; ++r) {
      const int* hr = cl.map_shared_rank(h, r);
      const int4 v = *reinterpret_cast<const int4*>(hr + NB - BPT * (tid + 1));
      cnt[0] += v.w; cnt[1] += v.z; cnt[2] += v.y; cnt[3] += v.x;
    }
#pragma unroll
    for (int b = 0; b < BPT; ++b) sum += cnt[b];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += x; }
    if (lane == 31) warp_s[w] = incl;
    __syncthreads();
    int above = incl - sum;
    for (int x = 0; x < w; ++x) above += warp_s[x];
#pragma unroll
    for (int b = 0; b < BPT; ++b) {
      if (above < need && above + cnt[b] >= need) { s_bin = NB - 1 - BPT * tid - b; s_above = above; s_in = cnt[b]; }   // one thread
      above += cnt[b];
    }
    // the other buffer is free again: every CTA has read it before the barrier above
    for (int b = tid; b < NB; b += ENT) hist[(step + 1) & 1][b] = 0;
    __syncthreads();
    base += (unsigned)s_bin << shift;
    need -= s_above;
    all = s_in == need;
    bits = shift;
  }
  // keys in [base, base + 2^bits) are at the threshold: `need` of them are taken, the lower rows first; above: all
  const unsigned span = bits == 32 ? 0xffffffffu : (1u << bits) - 1u;

  // ---- emission in row order: counts per CTA, then per warp ----
  const int seg = ((mine + ENT / 32 - 1) / (ENT / 32) + 31) & ~31, e0 = min(w * seg, mine), e1 = min(e0 + seg, mine);
  int gt = 0, eq = 0;
  for (int e = e0 + lane; e < e1; e += 32) {
    const unsigned k = key(e);
    const bool at = k >= base && k - base <= span;
    gt += k >= base && !at;
    eq += at;
  }
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  __syncthreads();                                       // warp_s has been read
  if (lane == 0) { warp_s[w] = gt; s_red[0][w] = (unsigned)eq; }
  __syncthreads();
  int gt_before = 0, eq_before = 0;
  for (int x = 0; x < w; ++x) { gt_before += warp_s[x]; eq_before += (int)s_red[0][x]; }
  if (tid == ENT - 1) { s_cnt[0] = gt_before + gt; s_cnt[1] = eq_before + eq; }
  cl.sync();
  for (int r = 0; r < rank; ++r) {
    gt_before += *cl.map_shared_rank(&s_cnt[0], r);
    eq_before += *cl.map_shared_rank(&s_cnt[1], r);
  }
  int* out = a.idx + ((long long)i * a.Hkv + kvh) * a.K;
  const unsigned below = (1u << lane) - 1u;
  for (int e = e0; e < e1; e += 32) {
    const int x = e + lane;
    const unsigned k = x < e1 ? key(x) : 0u;
    const bool at = x < e1 && k >= base && k - base <= span, up = x < e1 && k >= base && !at;
    const unsigned m_gt = __ballot_sync(0xffffffffu, up), m_eq = __ballot_sync(0xffffffffu, at);
    const int my_eq = eq_before + __popc(m_eq & below), pos = gt_before + __popc(m_gt & below) + min(my_eq, need);
    if ((up || (at && my_eq < need)) && index_ok(pos, a.K, a.status)) out[pos] = a.Ls + c0 + x;
    gt_before += __popc(m_gt);
    eq_before += __popc(m_eq);
  }
  cl.sync();                                             // no CTA leaves while another may read its counts
}

constexpr int CNT = 256, CROWS = 8, CTA_ROWS = CNT / 32 * CROWS;      // rows of a warp, of a CTA

// grid (row groups, KV heads, sequences)
__global__ void __launch_bounds__(CNT) evict_copy_kernel(const __grid_constant__ EvictArgs a) {
  pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int kvh = blockIdx.y, i = blockIdx.z, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int len = a.len[i], keep = a.Ls + a.K + a.Lr, rows = len < keep ? len : keep;
  const int r0 = (blockIdx.x * (CNT / 32) + w) * CROWS;
  if (r0 >= keep) return;
  const int src = len >= 0 ? a.src[i] : 0, dst = len >= 0 ? a.dst[i] : 0;
  if (len >= 0 && kvh == 0 && blockIdx.x == 0 && threadIdx.x == 0) a.seq_len[dst] = rows;
  // lane l < CROWS: row r0 + l of the destination
  long long ks = -1, vs = 0, kd = 0, vd = 0;             // byte offsets; ks < 0: nothing to copy
  if (lane < CROWS) {
    const int r = r0 + lane;
    int from = -1;
    if (r < rows) {
      if (len <= keep || r < a.Ls) from = r;
      else if (r < a.Ls + a.K) from = a.idx[((long long)i * a.Hkv + kvh) * a.K + r - a.Ls];
      else from = len - keep + r;
      if (!index_ok(from, len, a.status)) from = -1;
    }
    if (a.kept && r < keep) a.kept[((long long)i * a.Hkv + kvh) * keep + r] = from;
    if (from >= 0) {
      const int sp = from / a.map.page, dp = r / a.map.page;
      const int s_page = a.map.table[(long long)src * a.map.max_pages + sp];
      const int d_page = dp < a.map.max_pages ? a.map.table[(long long)dst * a.map.max_pages + dp] : -1;
      if (s_page < 0 || s_page >= a.map.n_pages || d_page < 0 || d_page >= a.map.n_pages) {
        if (a.status) atomicOr(a.status, SNAP_DEV_BAD_PAGE);
      } else {
        const int so = from - sp * a.map.page, dof = r - dp * a.map.page;
        ks = (s_page * a.map.kp + kvh * a.map.kh + so * a.map.kr) * a.eb;
        vs = (s_page * a.map.vp + kvh * a.map.vh + so * a.map.vr) * a.eb;
        kd = (d_page * a.map.kp + kvh * a.map.kh + dof * a.map.kr) * a.eb;
        vd = (d_page * a.map.vp + kvh * a.map.vh + dof * a.map.vr) * a.eb;
        if (a.w_out) {
          const long long b = (long long)kvh * a.map.cap, per = (long long)a.Hkv * a.map.cap;
          a.w_out[dst * per + b + r] = a.w_in[src * per + b + from];
        }
      }
    }
  }
  // rows of 16-byte pieces, key pieces then value pieces of a row; U pieces per lane in flight
  constexpr int U = 8;
  const int vecs = a.k_vecs + a.v_vecs, total = CROWS * vecs;
  for (int b = 0; b < total; b += 32 * U) {
    uint4 x[U];
    char* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = b + 32 * u + lane, row = p / vecs, c = p - row * vecs;
      const int from = row < CROWS ? row : 0;
      const long long s_k = __shfl_sync(0xffffffffu, ks, from), s_v = __shfl_sync(0xffffffffu, vs, from);
      const long long d_k = __shfl_sync(0xffffffffu, kd, from), d_v = __shfl_sync(0xffffffffu, vd, from);
      to[u] = nullptr;
      if (row < CROWS && s_k >= 0) {
        const bool isk = c < a.k_vecs;
        x[u] = *reinterpret_cast<const uint4*>(isk ? a.kp + s_k + 16 * c : a.vp + s_v + 16 * (c - a.k_vecs));
        to[u] = isk ? a.kp + d_k + 16 * c : a.vp + d_v + 16 * (c - a.k_vecs);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) *reinterpret_cast<uint4*>(to[u]) = x[u];
  }
}

}  // namespace

size_t paged_evict_scratch_bytes(const Shape& s, int n_seqs) {
  return align_up((size_t)n_seqs * s.Hkv * (s.K > 0 ? s.K : 1) * sizeof(int)) + align_up((size_t)n_seqs * sizeof(int));
}

cudaError_t launch_paged_evict(int dtype, const Shape& s, const PageMap& m, const int* src, const int* dst, int n_seqs,
                               void* k_pages, void* v_pages, int* seq_len, const float* w_in, float* w_out, int* kept,
                               char* scratch, uint32_t* status, cudaStream_t st) {
  EvictArgs a;
  a.src = src; a.dst = dst; a.n = n_seqs; a.Hkv = s.Hkv; a.Ls = s.Ls; a.Lr = s.Lr; a.K = s.K; a.max_seqs = s.max_seqs;
  a.map = m; a.seq_len = seq_len; a.w_in = w_in; a.w_out = w_out; a.kept = kept; a.status = status;
  a.idx = reinterpret_cast<int*>(scratch);
  a.len = reinterpret_cast<int*>(scratch + align_up((size_t)n_seqs * s.Hkv * (s.K > 0 ? s.K : 1) * sizeof(int)));
  a.kp = static_cast<char*>(k_pages); a.vp = static_cast<char*>(v_pages);
  a.eb = elt_bytes(dtype);
  a.k_vecs = s.d_qk * a.eb / 16; a.v_vecs = s.d_v * a.eb / 16;
  // A short middle fits one CTA; longer ones are cut over eight.
  const int most = m.cap - s.Ls - s.Lr;                    // candidates there can be
  const int CL = most <= 4096 ? 1 : 8;
  const int per = most > 0 ? (most + CL - 1) / CL : 0;
  a.keys_cap = per <= MAX_KEYS ? per : 0;
  const size_t smem = (size_t)a.keys_cap * sizeof(unsigned);
  static SmemLimit limit = {};
  cudaError_t e = ensure_dyn_smem(evict_select_kernel, smem < 1024 ? 1024 : smem, limit);
  if (e != cudaSuccess) return e;
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
  e = cudaLaunchKernelEx(&lc, evict_select_kernel, a);
  count_launch();
  if (e != cudaSuccess) return e;
  e = launch_pdl(evict_copy_kernel, dim3((s.Sc + CTA_ROWS - 1) / CTA_ROWS, s.Hkv, n_seqs), dim3(CNT), 0, st, a);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
