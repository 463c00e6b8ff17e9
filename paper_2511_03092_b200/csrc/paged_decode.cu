// Attention of one token per sequence over a cache in pages (snap_paged_decode_attn).
//
//     out[i][h] = sum_r p_r V_r / sum_r p_r,   p_r = exp(scale q.K_r - max),   r over the sequence's rows
//
// Every cache row is read once and serves the whole head group, so HBM bounds the call: 16 sequences of 8192 to 65536
// rows (32 heads on 8, 128 dims, 2.2 GB) take 322 to 328 us, 6.7 TB/s.  One sequence of 5124 rows takes 11.7 to 12.1 us for 21 MB,
// and 45 of up to 333 rows 14.4 to 15.0: there the chain of slot, length, page, tile, join is what counts.
//
// (sequence, KV head, head block) is a unit; its rows are cut into tiles.  The units in a row form one line, each as
// long as its tiles plus a fixed share for what a unit costs however short it is (its queries, its joining), and the line
// is divided evenly between the CTAs: sequences of any lengths load the GPU evenly and the host need not know the
// lengths.  A CTA walks over its stretch, which holds whole units and at most one cut one at either end; units of a few
// tiles are never cut.  A whole unit's output is written at once; a cut one leaves the sum, the maximum and the
// unnormalised output of its piece, which the second launch joins in a fixed order (no atomics: equal inputs give equal
// bits).
//
// Tensor-core kernel: the group's heads are the N side of mma.sync.m16n8k16, S^T = K tile . Q^T and
// O^T += V tile^T . P^T, so the cost of a row does not grow with the group.  It is built for heads of up to 64, 128 and
// 256 dims; what a head lacks is neither read nor multiplied.  Each warp runs a pipeline of its own over tiles of 16
// rows that TMA fetches (four-dimensional map: dim, row of a page, KV head, page) with the 128-byte swizzle, or, where a
// page holds no whole boxes of eight rows, that the lanes copy piece by piece; the pipeline runs ahead over unit borders,
// and the pages of the tiles after next are looked up while a tile is computed.  The probabilities enter the second
// product as two bf16 numbers (p and what its rounding left), which keeps their rounding out of the result: 2^-17
// instead of 2^-9 a row.
//
// In single precision it multiplies with m16n8k8 on numbers split into parts of 11 bits.  Keys, queries and probabilities have
// two (off by 2^-23 at most; the exponential is good to 2^-22) and a logit's product is three, together within 2^-20 of the exact one,
// less than summing a few dozen of them in single precision may lose.  Values have three parts and lose nothing: with two, a
// sequence of one row did not return its value row, at 1 to 7 % less time (8 sequences of 2000 to 6000 rows, 64 dims, 4 KV heads,
// groups of 1, 4, 16: 20.3 / 20.7, 21.3 / 21.6, 27.0 / 28.0 us; 128 dims, 8, 16: 35.3 / 36.2, 45.7 / 48.5; 256 dims, 8: 68.7 / 72.9).
// Groups of up to four wide heads are faster on the portable kernel.
//
// Portable kernel: the same pipelines per warp over tiles of 8 KB, brought in through tensor maps or by a bulk copy per
// row; a lane holds four dims of a row.  Four rows at a time, the 4 x heads partial dot products are reduced by halving
// exchanges, after which a lane owns one (row, head) pair: one shuffle per pair instead of five, one exponential per lane.
// (Eight rows at a time need twice the code for the same work; a step of short sequences runs through it once, at the speed
// at which instructions arrive.)  4 sequences of 2001 to 4100 rows, 8 heads on 2, take 15.2 to 16.1 us (latency); 28 of 1324 to 2196, 8
// on 4, 41.6 us, 74 % of the HBM rate.
//
// With weights, the split kernel also stores the logits, and CTAs of the second launch turn them into the group's
// attention weight of each row once the unit's maximum and sum are known: 8 sequences of 9000 to 16384 rows take 85 us
// with weights, 72 without.
#include <cuda.h>

#include "mma_helpers.cuh"
#include "packed_f32.cuh"
#include "snap_internal.cuh"
#include "umma_helpers.cuh"

namespace snap {
namespace {

using namespace mmasync;
using umma::mbar_expect_tx;
using umma::mbar_init;
using umma::mbar_try_wait;
using umma::smem_u32;

constexpr int TR = 16;                          // rows of a tile of the tensor-core kernel
__host__ __device__ constexpr int simt_rows(bool wide) { return wide ? 4 : 8; }   // ... of the portable kernel: 8 KB of single precision either way
constexpr int UNIT_TILES = 6;                   // what a unit costs besides its tiles, in tiles; units of at most that many stay whole
constexpr int MIN_TILES = 1;                    // a CTA gets at least that much beyond one unit's share (at least one: no stretch is empty)
// (Measured over 40 calls of all sizes: 4 and 4 take 8 % longer, 8 and 1 2 %, 4 and 1 as long but 4 % longer for many short sequences.)
constexpr int MAX_CTAS = 1024, MAX_HELD = 128;  // sequences whose slot and length a CTA keeps in shared memory
// (Held against looked up in the batch's arrays: 17 sequences of up to 400 rows 14.4 / 14.95 us, 45 of 333 14.75 / 15.0, 100 of 500 35.7 /
// 35.8, 128 of 2000 96.7 / 97.0: the more sequences, the less it is worth.)
constexpr unsigned kPagedWaitLimit = 1u << 22;

struct PagedArgs {
  const void* q; void* out;
  const void* kp; const void* vp;
  const int* slots; const int* seq_len;
  int n, Hq, Hkv, g, gb, nhb, U, d_qk, d_v, max_seqs;    // U = Hkv * nhb units per sequence, gb heads each (the last block fewer)
  int gs;                                       // logits of a row: gb, or up to the next multiple of 4
  float scale_log2;
  PageMap map;
  int tr;                                       // rows of a tile
  int4* entry;                                  // [n + 1]: (the line before sequence i, per unit of a sequence; its slot, rows, tiles)
  float2* ml_unit;                              // [n * U][gb]: (max, sum), log2 domain, of units that one CTA did whole
  float2* ml_part; float* o_part;               // [2 * CTAs][gb], [2 * CTAs][gb][d_v]: pieces of cut units; CTA c's is 2 c, or
                                                // 2 c + 1 when it holds the unit's first tile (it has one of either at most)
  float* scores;                                // NULL, or [n * U][cap][gs] logits in the log2 domain
  const float* w_in; float* w_out;
  uint32_t* status;
  int ctas;
  int stages, tiled;                            // portable kernel: stages of a warp; tiles come through the tensor maps
};

__device__ __forceinline__ int rows_of(const PagedArgs& a, int slot) {
  if (slot < 0 || slot >= a.max_seqs) return 0;
  return min(max(a.seq_len[slot], 0), a.map.cap);
}
template <int ROWS> __device__ __forceinline__ int tiles_of(int rows) { return (int)(((unsigned)rows + ROWS - 1) / ROWS); }
__device__ __forceinline__ int length_of(int nt) { return nt > 0 ? nt + UNIT_TILES : 0; }           // on the line
// Where tile t of a unit begins on the line, counted from the unit: the first tile carries the unit's share, and all
// tiles of a short unit begin (and so stay) with the first.
__device__ __forceinline__ int begin_of(int t, int nt) { return t == 0 || nt <= UNIT_TILES ? 0 : UNIT_TILES + t; }

// CTAs that share a line of length W, where CTA c's stretch begins, and whose stretch position x lies in.  (32-bit
// arithmetic where it suffices: 64-bit divisions are long instruction sequences.)
__device__ __forceinline__ int active_ctas(long long W, int ctas) {
  if (W >= (long long)ctas * (MIN_TILES + UNIT_TILES)) return ctas;
  return W > 0 ? max((int)W / (MIN_TILES + UNIT_TILES), 1) : 0;
}
__device__ __forceinline__ long long stretch_begin(long long W, int active, int c) {
  return W < (1 << 21) ? (long long)((unsigned)W * (unsigned)c / (unsigned)active) : W * c / active;
}
__device__ __forceinline__ int owner_of(long long x, long long W, int active) {
  return W < (1 << 21) ? (int)((((unsigned)x + 1) * (unsigned)active - 1) / (unsigned)W) : (int)(((x + 1) * active - 1) / W);
}

// Slots and lengths of the call's sequences, in shared memory when they fit.
struct Held { int2 e[MAX_HELD]; };
// A place on the line.  pos: where its unit begins, from the CTA's first unit on.
struct Place { int e, u, t, nt, slot, len, pos; };   // sequence, unit, tile of the unit, tiles per unit, slot, rows
template <int ROWS> __device__ __forceinline__ void load_entry(const PagedArgs& a, const Held& held, Place& p) {
  if (p.e >= a.n) {                             // the end of the line
    p.slot = -1; p.len = 0; p.nt = 1 << 29; p.e = a.n;
    return;
  }
  if (a.n <= MAX_HELD) { const int2 v = held.e[p.e]; p.slot = v.x; p.len = v.y; }
  else { p.slot = a.slots[p.e]; p.len = rows_of(a, p.slot); }
  p.nt = tiles_of<ROWS>(p.len);
}
template <int ROWS> __device__ __forceinline__ void next_unit(const PagedArgs& a, const Held& held, Place& p) {
  p.pos += length_of(p.nt);
  if (++p.u == a.U) {
    p.u = 0;
    do { ++p.e; load_entry<ROWS>(a, held, p); } while (p.nt == 0);
  }
}
// `step` tiles on, or (false) past `end`, the end of the CTA's stretch
template <int ROWS> __device__ __forceinline__ bool advance(const PagedArgs& a, const Held& held, Place& p, int step, int end) {
  p.t += step;
  while (p.t >= p.nt) {
    p.t -= p.nt;
    next_unit<ROWS>(a, held, p);
    if (p.e >= a.n || p.pos >= end) return false;
  }
  return p.pos + begin_of(p.t, p.nt) < end;
}

__device__ __forceinline__ int warp_inclusive(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += x; }
  return v;
}
// Slot and rows of sequence e; conditions to report
__device__ __forceinline__ int2 read_entry(const PagedArgs& a, int e, unsigned& bad) {
  const int slot = a.slots[e];
  int len = 0;
  if (slot >= 0 && slot < a.max_seqs) {
    len = a.seq_len[slot];
    if (len > a.map.cap) { bad |= SNAP_DEV_BAD_PAGE; len = a.map.cap; }
    len = max(len, 0);
  } else if (slot != -1) {
    bad |= SNAP_DEV_BAD_SLOT;
  }
  return make_int2(slot, len);
}

// All threads of the CTA: the place of its first tile and the end of its stretch (both counted from that tile's unit).
// Returns false (to all) when it has none.  CTA 0 also writes the entries and reports bad slots and lengths.
// Up to MAX_HELD sequences the first warp does it (its result handed over in shared memory: a dozen warps of an SM doing
// the same would wait for one another), with more the CTA together.
template <int ROWS, int NT, bool SMALL>
__device__ __forceinline__ bool locate_part(const PagedArgs& a, Place& p, int& end, Held& held, int* scan /* shared, NT / 32 + 2 */) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = blockIdx.x;
  unsigned bad = 0;
  int total = 0, e_at = 0, before_at = 0;
  long long W = 0, x0 = 0, x1 = 0;
  int active = 0;
  const auto stretch = [&]() {
    W = (long long)total * a.U;
    active = active_ctas(W, a.ctas);
    if (c >= active) return false;
    x0 = stretch_begin(W, active, c);
    x1 = stretch_begin(W, active, c + 1);
    return true;
  };
  if (SMALL) {
    const int per = (a.n + 31) / 32, e0 = min(lane * per, a.n), e1 = min(e0 + per, a.n);   // a lane's sequences
    int mine = 0;
#pragma unroll 1
    for (int e = e0; e < e1; ++e) {
      const int2 v = read_entry(a, e, bad);
      held.e[e] = v;
      mine += length_of(tiles_of<ROWS>(v.y));
    }
    const int incl = warp_inclusive(mine, lane);
    int before = incl - mine;
    total = __shfl_sync(0xffffffffu, incl, 31);
    if (c == 0) {
      int at = before;
#pragma unroll 1
      for (int e = e0; e < e1; ++e) {
        const int2 v = held.e[e];
        const int nt = tiles_of<ROWS>(v.y);
        a.entry[e] = make_int4(at, v.x, v.y, nt);
        at += length_of(nt);
      }
      if (lane == 0) a.entry[a.n] = make_int4(total, -1, 0, 0);
      if (bad && a.status) atomicOr(a.status, bad);
    }
    __syncwarp();
    if (!stretch()) return false;
    int e = e0;
    const bool here = x0 >= (long long)before * a.U && x0 < (long long)incl * a.U;       // one lane
    if (here) {
#pragma unroll 1
      for (; e < e1 - 1; ++e) {
        const int len = length_of(tiles_of<ROWS>(held.e[e].y));
        if (x0 < (long long)(before + len) * a.U) break;
        before += len;
      }
    }
    const int from = max(__ffs(__ballot_sync(0xffffffffu, here)) - 1, 0);
    e_at = __shfl_sync(0xffffffffu, e, from);
    before_at = __shfl_sync(0xffffffffu, before, from);
  } else {
    const int per = (a.n + NT - 1) / NT, e0 = min(tid * per, a.n), e1 = min(e0 + per, a.n);
    int mine = 0;
    for (int e = e0; e < e1; ++e) mine += length_of(tiles_of<ROWS>(read_entry(a, e, bad).y));
    const int incl = warp_inclusive(mine, lane);
    if (lane == 31) scan[warp] = incl;
    if (tid == 0) scan[NT / 32] = scan[NT / 32 + 1] = 0;
    __syncthreads();
    int before = incl - mine;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) { const int x = scan[w]; total += x; if (w < warp) before += x; }
    if (c == 0) {
      int at = before;
      for (int e = e0; e < e1; ++e) {
        const int2 v = read_entry(a, e, bad);
        const int nt = tiles_of<ROWS>(v.y);
        a.entry[e] = make_int4(at, v.x, v.y, nt);
        at += length_of(nt);
      }
      if (tid == 0) a.entry[a.n] = make_int4(total, -1, 0, 0);
      if (bad && a.status) atomicOr(a.status, bad);
    }
    if (!stretch()) return false;
    if (x0 >= (long long)before * a.U && x0 < (long long)(before + mine) * a.U) {        // one thread
      for (int e = e0; e < e1; ++e) {
        const int len = length_of(tiles_of<ROWS>(read_entry(a, e, bad).y));
        if (x0 < (long long)(before + len) * a.U) { scan[NT / 32] = e; scan[NT / 32 + 1] = before; break; }
        before += len;
      }
    }
    __syncthreads();
    e_at = scan[NT / 32];
    before_at = scan[NT / 32 + 1];
  }
  p.e = e_at;
  load_entry<ROWS>(a, held, p);
  p.nt = max(p.nt, 1);                          // (only if another stream changes the lengths during the call: stay in bounds)
  const long long rel = x0 - (long long)before_at * a.U;
  const int unit = length_of(p.nt);
  p.u = (int)min(rel < (1LL << 31) ? (long long)((unsigned)rel / (unsigned)unit) : rel / unit, (long long)a.U - 1);
  const int o = (int)(rel - (long long)p.u * unit);
  // the first tile that begins at or after x0
  p.t = o <= 0 ? 0 : p.nt <= UNIT_TILES ? p.nt : max(1, o - UNIT_TILES);
  p.pos = 0;
  end = (int)min(x1 - x0 + max(o, 0), (long long)(1 << 30));
  if (p.t >= p.nt) {
    p.t = 0;
    next_unit<ROWS>(a, held, p);
    end -= p.pos;
    p.pos = 0;
    if (p.e >= a.n || end <= 0) return false;
  }
  return true;
}
struct Found { Place p; int end, any; };
template <int ROWS, int NT>
__device__ __forceinline__ bool locate(const PagedArgs& a, Place& p, int& end, Held& held, int* scan, Found& found /* shared */) {
  if (a.n > MAX_HELD) return locate_part<ROWS, NT, false>(a, p, end, held, scan);
  if (threadIdx.x < 32) {
    const bool any = locate_part<ROWS, NT, true>(a, p, end, held, scan);
    if (threadIdx.x == 0) { found.any = any; found.p = p; found.end = end; }
  }
  __syncthreads();
  p = found.p;
  end = found.end;
  return found.any;
}
// Tiles of the unit at p, from p.t on, that begin before the end of the stretch: the end of that range of tiles
__device__ __forceinline__ int segment_end(const Place& p, int end) {
  return p.nt <= UNIT_TILES ? p.nt : min(p.nt, max(end - p.pos - UNIT_TILES, 1));
}

// The CTA's result of a segment, the sum of NBUF buffers [cols][ld] in shared memory, leaves for the output (a whole unit) or the
// scratch of pieces.  L, M: per column in shared memory.
template <typename T, int NT, int NBUF>
__device__ __forceinline__ void write_segment(const PagedArgs& a, const float* buf, int ld, int buf_stride, const float* M, const float* L,
                                              int e, int u, int nh, bool whole, int piece) {
  const int tid = threadIdx.x, d4 = a.d_v / 4;
  if (!index_ok(e, a.n, a.status) || !index_ok(u, a.U, a.status) || !(whole || index_ok(piece, 2LL * a.ctas, a.status))) return;
  const int kvh = u / a.nhb, hb = u - kvh * a.nhb;
  T* out = static_cast<T*>(a.out) + ((long long)e * a.Hq + kvh * a.g + hb * a.gb) * a.d_v;
  float* part = a.o_part + (long long)piece * a.gb * a.d_v;
#pragma unroll 2
  for (int x = tid; x < nh * d4; x += NT) {
    const int h = x / d4, c = (x - h * d4) * 4;
    float4 o = *reinterpret_cast<const float4*>(buf + h * ld + c);
#pragma unroll
    for (int b = 1; b < NBUF; ++b) {
      const float4 y = *reinterpret_cast<const float4*>(buf + b * buf_stride + h * ld + c);
      o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
    }
    if (whole) {
      const float inv = L[h] > 0.f ? 1.f / L[h] : L[h];                    // no row: zero; NaN stays
      alignas(16) T r[4] = {from_f32<T>(o.x * inv), from_f32<T>(o.y * inv), from_f32<T>(o.z * inv), from_f32<T>(o.w * inv)};
      if (sizeof(T) == 4) *reinterpret_cast<uint4*>(out + h * a.d_v + c) = *reinterpret_cast<const uint4*>(r);
      else *reinterpret_cast<uint2*>(out + h * a.d_v + c) = *reinterpret_cast<const uint2*>(r);
    } else {
      *reinterpret_cast<float4*>(part + h * a.d_v + c) = o;
    }
  }
  if (tid < nh && (!whole || a.scores))
    (whole ? a.ml_unit + ((long long)e * a.U + u) * a.gb : a.ml_part + (long long)piece * a.gb)[tid] = make_float2(M[tid], L[tid]);
}

__device__ __forceinline__ bool wait_bounded(uint32_t bar, unsigned parity) {
  for (unsigned it = 0; it < kPagedWaitLimit; ++it)
    if (mbar_try_wait(bar, parity)) return true;
  return false;
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
// byte offset of row r, 16-byte chunk c (0..7) inside a 128-byte-swizzled slab
__device__ __forceinline__ uint32_t swz(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

// ---------------------------------------------------------------------------------------------------------------
// tensor-core kernel
// ---------------------------------------------------------------------------------------------------------------
constexpr int SLAB_B = TR * 128;                 // one 128-byte-wide slab of a tile
template <typename T> __host__ __device__ constexpr int slab_dims() { return 128 / (int)sizeof(T); }

template <typename T, int D, int NWARP, int NSTAGE, int NG> struct MmaShape {
  static constexpr int NT = NWARP * 32, NSL = D / slab_dims<T>(), KS = D / 16, NCOL = 8 * NG;
  static constexpr int TENS_B = NSL * SLAB_B, STAGE_B = 2 * TENS_B;
  static constexpr int LD = D + 4;               // column stride of the exchange buffers: fragments store without bank conflicts
  static constexpr size_t stages_b = (size_t)NWARP * NSTAGE * STAGE_B;
  static constexpr size_t bars_b = NWARP * NSTAGE * 8;
  static constexpr size_t smem = 1024 + stages_b + bars_b + (size_t)(NWARP / 2 * NCOL * LD + 2 * NWARP * NCOL + 2 * NCOL) * sizeof(float);
};

// A single-precision number as two of the tensor cores' 11 bits: x = hi + lo within 2^-21 of x, hi rounded and lo cut off.
// (In integer arithmetic: with the conversion instruction, which has a fraction of its rate, 8 sequences of 2000 to 6000
// rows and 8 heads on each of 4 took 40.6 us instead of 35.3, both with values in two parts.)  A NaN leaves one part NaN at least; above
// 2^128 (1 - 2^-12) x counts as infinite.
struct Tf32 { uint32_t hi, lo; };
__device__ __forceinline__ Tf32 tf32_of(float x) {
  Tf32 t;
  t.hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
  t.lo = __float_as_uint(x - __uint_as_float(t.hi)) & 0xffffe000u;
  return t;
}
__device__ __forceinline__ void mma1688(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// A value as three, exactly: x = hi + lo + rest, hi and lo cut off (so that nothing finite becomes infinite).  Outputs are
// averages of value rows: a row whose weight is 1 comes out unrounded.  (Below some 1e-31 the last part leaves the normal numbers.)
struct Tf32x3 { uint32_t hi, lo, rest; };
__device__ __forceinline__ Tf32x3 tf32x3_of(float x) {
  Tf32x3 t;
  t.hi = __float_as_uint(x) & 0xffffe000u;
  const float r = x - __uint_as_float(t.hi);
  t.lo = __float_as_uint(r) & 0xffffe000u;
  t.rest = __float_as_uint(r - __uint_as_float(t.lo));
  return t;
}
// c += a . b in single precision: hi hi + hi lo + lo hi; what is left out is 2^-22 of a product
__device__ __forceinline__ void mma_3tf32(float (&c)[4], const Tf32* a, const Tf32& b0, const Tf32& b1) {
  mma1688(c, a[0].lo, a[1].lo, a[2].lo, a[3].lo, b0.hi, b1.hi);
  mma1688(c, a[0].hi, a[1].hi, a[2].hi, a[3].hi, b0.lo, b1.lo);
  mma1688(c, a[0].hi, a[1].hi, a[2].hi, a[3].hi, b0.hi, b1.hi);
}
// ... with a exact; lo lo, 2^-21 of a product, is left out
__device__ __forceinline__ void mma_3tf32(float (&c)[4], const Tf32x3* a, const Tf32& b0, const Tf32& b1) {
  mma1688(c, a[0].rest, a[1].rest, a[2].rest, a[3].rest, b0.hi, b1.hi);
  mma1688(c, a[0].lo, a[1].lo, a[2].lo, a[3].lo, b0.hi, b1.hi);
  mma1688(c, a[0].hi, a[1].hi, a[2].hi, a[3].hi, b0.lo, b1.lo);
  mma1688(c, a[0].hi, a[1].hi, a[2].hi, a[3].hi, b0.hi, b1.hi);
}

// How a tile comes in.  EXACT: through the tensor maps, heads of D dims and pages of a multiple of 16 rows, without the
// tests that other shapes need in the inner loops (with them a 128-wide call takes 4 to 15 % longer, a 256-wide one half
// as long again).  BOXES: through the tensor maps, pages of a multiple of 8 rows.  ROWS: any pages; the lanes copy a
// row's 16-byte pieces themselves (cp.async), each from the page of its row.
enum class Tiles { EXACT, BOXES, ROWS };
template <typename T, int D, int NWARP, int NSTAGE, int NG, int CTAS, Tiles MODE>
__global__ void __launch_bounds__(NWARP * 32, CTAS)
paged_mma_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v) {
  using S = MmaShape<T, D, NWARP, NSTAGE, NG>;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int SD = slab_dims<T>();
  constexpr int KS = S::KS, NCOL = S::NCOL, LD = S::LD;
  constexpr bool EXACT = MODE == Tiles::EXACT, BY_ROWS = MODE == Tiles::ROWS;
  constexpr int LOOK = BY_ROWS ? 32 / TR : 32;                           // tiles that a warp looks up at once
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(stages + S::stages_b);
  float* buf = reinterpret_cast<float*>(bars + NWARP * NSTAGE);          // [NWARP / 2][NCOL][LD]
  float* wm = buf + NWARP / 2 * NCOL * LD;                                       // [NWARP][NCOL] maxima, then sums
  float* wl = wm + NWARP * NCOL;
  float* jm = wl + NWARP * NCOL;                                         // [NCOL] joined maxima, then sums
  float* jl = jm + NCOL;
  __shared__ int scan[S::NT / 32 + 2];
  __shared__ Held held;
  __shared__ Found found;

  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, gq = lane >> 2, tq = lane & 3;
  unsigned char* wstages = stages + w * NSTAGE * S::STAGE_B;
  const uint32_t stage0 = smem_u32(wstages), bar0 = smem_u32(bars + w * NSTAGE);
  if (lane == 0) {
    for (int s = 0; s < NSTAGE; ++s) mbar_init(bar0 + 8 * s, BY_ROWS ? 32 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (w == 0 && !BY_ROWS) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_k) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_v) : "memory");
    }
  }
  __syncwarp();
  pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  Place at;
  int end;
  if (!locate<TR, S::NT>(a, at, end, held, scan, found)) return;

  // ---- the warp's producer: runs NSTAGE tiles ahead of the consumer, over unit borders; warp w takes the CTA's tiles
  // w, w + NWARP, ... ----
  // Lane l looks up the page of the warp's tile l, l + 32, ...: one look-up's latency for 32 tiles.  (ROWS: of row l % 16
  // of tile l / 16, l / 16 + 2, ...)
  Place pr = at;
  bool valid = advance<TR>(a, held, pr, w + NWARP * (lane / (32 / LOOK)), end);
  // BOXES: where a page is no multiple of 16 rows, the tile's halves are looked up apart (one box each).
  const bool halves = MODE == Tiles::BOXES && a.map.page % TR != 0;
  int pid = -1, pid_hi = -1, n_issued = 0;
  unsigned bad_stage = 0, todo = 0;                                      // bits 2 s, 2 s + 1: the halves of stage s are on a bad page; lanes with a tile to issue
  unsigned long long rows_stage = 0;                                     // ROWS: 16 bits per stage, the rows that are there
  int kvh_of = 0, row_of = 0, row_hi = 0;
  const auto fetch = [&]() {
    todo = __ballot_sync(0xffffffffu, valid);
    if (BY_ROWS) {
      pid = -1;
      const int row = pr.t * TR + lane % TR;
      if (valid && row < pr.len) {
        const int pg = row / a.map.page;
        row_of = row - pg * a.map.page;
        kvh_of = pr.u / a.nhb;
        if (index_ok(pg, a.map.max_pages, a.status)) pid = a.map.table[(long long)pr.slot * a.map.max_pages + pg];
        if (pid < 0) pid = a.map.n_pages;                                // (bad, not absent)
      }
      return;
    }
    if (valid && pr.len > 0) {
      const int* table = a.map.table + (long long)pr.slot * a.map.max_pages;
      const int row = pr.t * TR, pg = row / a.map.page;
      pid = index_ok(pg, a.map.max_pages, a.status) ? table[pg] : -1;
      row_of = row - pg * a.map.page;
      kvh_of = pr.u / a.nhb;
      if (halves) {
        const int pg_hi = (row + TR / 2) / a.map.page;
        pid_hi = row + TR / 2 < pr.len && index_ok(pg_hi, a.map.max_pages, a.status) ? table[pg_hi] : 0;   // (no row there: any page will do)
        row_hi = row + TR / 2 - pg_hi * a.map.page;
      }
    }
  };
  fetch();
  const T* q_all = static_cast<const T*>(a.q);
  // B fragments of Q^T.  bf16: column 8 gi + gq, dims 16 ks + 2 tq (+1), + 8 (+9).  Single precision: dims 16 ks + 4 tq .. + 3
  uint32_t qb[NG][KS][F32 ? 4 : 2];
  const auto load_q = [&]() {
    const int kvh = at.u / a.nhb, hb = at.u - kvh * a.nhb, nh = min(a.gb, a.g - hb * a.gb);
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      const int col = 8 * gi + gq;
      const T* qp = q_all + ((long long)at.e * a.Hq + kvh * a.g + hb * a.gb + (col < nh ? col : 0)) * (EXACT ? D : a.d_qk) + (F32 ? 4 : 2) * tq;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bool there = col < nh && (EXACT || 16 * ks < a.d_qk);
        if constexpr (F32) {
          const uint4 x = there ? *reinterpret_cast<const uint4*>(qp + 16 * ks) : make_uint4(0, 0, 0, 0);
          qb[gi][ks][0] = x.x; qb[gi][ks][1] = x.y; qb[gi][ks][2] = x.z; qb[gi][ks][3] = x.w;
        } else {
          qb[gi][ks][0] = there ? *reinterpret_cast<const uint32_t*>(qp + 16 * ks) : 0u;
          qb[gi][ks][1] = there ? *reinterpret_cast<const uint32_t*>(qp + 16 * ks + 8) : 0u;
        }
      }
    }
  };
  load_q();                                                              // (the first tiles' look-ups wait alongside)
  const int d_qk = EXACT ? D : a.d_qk, d_v = EXACT ? D : a.d_v;
  const unsigned tile_b = (unsigned)((d_qk + SD - 1) / SD + (d_v + SD - 1) / SD) * SLAB_B;   // the slabs that hold anything
  const auto issue_rows = [&]() {                                        // the tile of the lower or upper half of the lanes
    const int s = n_issued % NSTAGE, l = (n_issued % LOOK) * TR;
    const unsigned okay = (__ballot_sync(0xffffffffu, pid >= 0 && pid < a.map.n_pages) >> l) & 0xffffu;
    rows_stage = (rows_stage & ~(0xffffull << (16 * s))) | (unsigned long long)okay << (16 * s);
    if (lane / TR == l / TR && pid >= a.map.n_pages && a.status) atomicOr(a.status, SNAP_DEV_BAD_PAGE);
    const long long k_off = pid * a.map.kp + kvh_of * a.map.kh + row_of * a.map.kr, v_off = pid * a.map.vp + kvh_of * a.map.vh + row_of * a.map.vr;
    // CPR lanes to a row (of a narrower head some have nothing to copy)
    constexpr int EPC = 16 / (int)sizeof(T), CPR = D / EPC;
    const T* kp = static_cast<const T*>(a.kp);
    const T* vp = static_cast<const T*>(a.vp);
#pragma unroll
    for (int x0 = 0; x0 < TR * CPR; x0 += 32) {
      const int r = (x0 + lane) / CPR, c = (x0 + lane) % CPR;
      const long long ko = __shfl_sync(0xffffffffu, k_off, l + r), vo = __shfl_sync(0xffffffffu, v_off, l + r);
      const uint32_t dst = stage0 + s * S::STAGE_B + (c >> 3) * SLAB_B + swz(r, c & 7);
      if ((okay >> r) & 1u) {
        if (EPC * c < d_qk) cp_async16(dst, kp + ko + EPC * c, 16);
        if (EPC * c < d_v) cp_async16(dst + S::TENS_B, vp + vo + EPC * c, 16);
      }
    }
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar0 + 8 * s) : "memory");
    todo &= ~(0xffffu << l);
    if (++n_issued % LOOK == 0) {
      if (valid) valid = advance<TR>(a, held, pr, LOOK * NWARP, end);
      fetch();
    }
  };
  const auto issue = [&]() {                                             // the lowest lane's tile of `todo`
    if (BY_ROWS) { issue_rows(); return; }
    const int s = n_issued % NSTAGE, l = n_issued & 31;
    const unsigned lo = __ballot_sync(0xffffffffu, pid < 0 || pid >= a.map.n_pages);
    const unsigned hi = halves ? __ballot_sync(0xffffffffu, pid_hi < 0 || pid_hi >= a.map.n_pages) : lo;
    const unsigned bad = ((lo >> l) & 1u) | ((hi >> l) & 1u) << 1;
    bad_stage = (bad_stage & ~(3u << (2 * s))) | bad << (2 * s);
    if (lane == l) {
      const uint32_t dst = stage0 + s * S::STAGE_B, bar = bar0 + 8 * s;
      mbar_expect_tx(bar, tile_b);
#pragma unroll 1
      for (int half = 0; half <= (int)halves; ++half) {
        const int page = (bad >> half) & 1u ? 0 : half ? pid_hi : pid, row = half ? row_hi : row_of;
        const uint32_t at = dst + half * (SLAB_B / 2);
#pragma unroll
        for (int h = 0; h < S::NSL; ++h) {
          if (SD * h < d_qk) tma_load_4d(at + h * SLAB_B, &tmap_k, SD * h, row, kvh_of, page, bar);
          if (SD * h < d_v) tma_load_4d(at + S::TENS_B + h * SLAB_B, &tmap_v, SD * h, row, kvh_of, page, bar);
        }
      }
      if (bad && a.status) atomicOr(a.status, SNAP_DEV_BAD_PAGE);
    }
    todo &= todo - 1;
    if ((++n_issued & 31) == 0) {                                        // 32 tiles issued: the next 32
      if (valid) valid = advance<TR>(a, held, pr, 32 * NWARP, end);
      fetch();
    }
  };
#pragma unroll 1
  for (int s = 0; s < NSTAGE && todo; ++s) issue();

  // ldmatrix lane roles: K (plain): row (lane & 7) + 8 * bit3, chunk + bit4; V (transposed): row (lane & 7) + 8 * bit4, chunk + bit3
  const int k_row = (lane & 7) + ((lane >> 3) & 1) * 8, k_cadd = lane >> 4;
  const int v_row = (lane & 7) + ((lane >> 4) & 1) * 8, v_cadd = (lane >> 3) & 1;

  bool dead = false;                                                     // a bounded wait ran out: nothing more is read
  int n = 0, done = 0;                                                   // tiles done by this warp; by the CTA before this segment
  while (true) {
    // ---- a segment: the CTA's tiles [at.t, tb) of one unit ----
    const int tb = segment_end(at, end), cnt = tb - at.t;
    const int hb = at.u % a.nhb, nh = min(a.gb, a.g - hb * a.gb);
    const bool whole = cnt == at.nt;
    float oacc[NG][KS][4], m_ref[NG][2], l_part[NG][2];                  // O^T: dims 16 db + gq (+8), columns 8 gi + 2 tq (+1)
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      m_ref[gi][0] = m_ref[gi][1] = -INFINITY;
      l_part[gi][0] = l_part[gi][1] = 0.f;
#pragma unroll
      for (int db = 0; db < KS; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x) oacc[gi][db][x] = 0.f;
    }
    float* srow = a.scores ? a.scores + ((long long)at.e * a.U + at.u) * a.map.cap * a.gs : nullptr;

    for (; w + n * NWARP < done + cnt && !dead; ++n) {
      const int s = n % NSTAGE;
      const bool landed = wait_bounded(bar0 + 8 * s, (unsigned)(n / NSTAGE) & 1u);
      if (__any_sync(0xffffffffu, !landed)) { dead = true; break; }
      const int row0 = (at.t + (w + n * NWARP - done)) * TR;
      const int nrows = min(at.len - row0, TR);
      const unsigned bad = BY_ROWS ? ~(unsigned)(rows_stage >> (16 * s)) & 0xffffu : (bad_stage >> (2 * s)) & 3u;
      const auto there = [&](int r) { return BY_ROWS ? !((bad >> r) & 1u) : r < nrows && !((bad >> (r >> 3)) & 1u); };
      const uint32_t sK = stage0 + s * S::STAGE_B, sV = sK + S::TENS_B;
      if (nrows < TR || bad) {
        // rows past the end, or on a bad page, may hold anything, and a zero probability does not silence a NaN in V: clear them
        constexpr int CPR = D * (int)sizeof(T) / 16;
        for (int x = lane; x < TR * CPR; x += 32) {
          const int r = x / CPR, c = x % CPR;
          if (!there(r))
            *reinterpret_cast<uint4*>(wstages + s * S::STAGE_B + S::TENS_B + (c >> 3) * SLAB_B + swz(r, c & 7)) = make_uint4(0, 0, 0, 0);
        }
        __syncwarp();
      }
      // ---- S^T = K tile . Q^T ----
      // one column group: two accumulators, of even and odd steps, make the chain of dependent products half as long
      constexpr int CH = NG == 1 ? 2 : 1;
      float vc[CH][NG][4];
#pragma unroll
      for (int ch = 0; ch < CH; ++ch)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int x = 0; x < 4; ++x) vc[ch][gi][x] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (!EXACT && 16 * ks >= d_qk) break;
        if constexpr (F32) {
          // (the queries are split anew for every tile: their two parts would take the registers of two more blocks)
#pragma unroll
          for (int gi = 0; gi < NG; ++gi)
#pragma unroll
            for (int x = 0; x < 4; ++x) asm volatile("" : "+r"(qb[gi][ks][F32 ? x : 0]));
          // two steps of eight dims: of the 16, a thread's four are k = tq, tq + 4 of the first step, then of the second
          const unsigned char* sk = wstages + s * S::STAGE_B + (ks >> 1) * SLAB_B;
          const float4 lo8 = *reinterpret_cast<const float4*>(sk + swz(gq, (ks & 1) * 4 + tq));
          const float4 hi8 = *reinterpret_cast<const float4*>(sk + swz(gq + 8, (ks & 1) * 4 + tq));
          const Tf32 kx[8] = {tf32_of(lo8.x), tf32_of(hi8.x), tf32_of(lo8.y), tf32_of(hi8.y), tf32_of(lo8.z), tf32_of(hi8.z), tf32_of(lo8.w), tf32_of(hi8.w)};
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int gi = 0; gi < NG; ++gi)
              mma_3tf32(vc[CH == 2 ? st : 0][gi], kx + 4 * st, tf32_of(__uint_as_float(qb[gi][ks][2 * st])), tf32_of(__uint_as_float(qb[gi][ks][2 * st + 1])));
        } else {
          uint32_t af[4];
          ldsm4(sK + (ks >> 2) * SLAB_B + swz(k_row, (ks & 3) * 2 + k_cadd), af);
#pragma unroll
          for (int gi = 0; gi < NG; ++gi) mma16816(vc[ks % CH][gi], af, qb[gi][ks][0], qb[gi][ks][1]);
        }
      }
      float v[NG][4];
#pragma unroll
      for (int gi = 0; gi < NG; ++gi)
#pragma unroll
        for (int x = 0; x < 4; ++x) v[gi][x] = CH == 2 ? vc[0][gi][x] + vc[CH - 1][gi][x] : vc[0][gi][x];
      bool refresh = false;
#pragma unroll
      for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
          v[gi][x] = there(gq + (x >> 1) * 8) ? v[gi][x] * a.scale_log2 : -INFINITY;
        refresh = refresh || fmaxf(v[gi][0], v[gi][2]) > m_ref[gi][0] + 8.f || fmaxf(v[gi][1], v[gi][3]) > m_ref[gi][1] + 8.f;
      }
      if (srow) {
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
          const int col = 8 * gi + 2 * tq;
#pragma unroll
          for (int r8 = 0; r8 < 2; ++r8) {
            const int row = row0 + gq + 8 * r8;
            if (row >= at.len || !index_ok(row, a.map.cap, a.status)) continue;   // (a bad page's rows are written: as -inf)
            float* sp = srow + (long long)row * a.gs + col;
            if (a.gs % 2 == 0 && col < nh) *reinterpret_cast<float2*>(sp) = make_float2(v[gi][2 * r8], v[gi][2 * r8 + 1]);   // (nh may end between them)
            else {
              if (col < nh) sp[0] = v[gi][2 * r8];
              if (col + 1 < nh) sp[1] = v[gi][2 * r8 + 1];
            }
          }
        }
      }
      // The reference of the exponentials follows the maximum lazily: it moves (and the sums are rescaled) only when
      // a logit lies 8 above it, i.e. before a probability passes 2^8.
      if (__any_sync(0xffffffffu, refresh)) {
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
          float mx0 = fmaxf(v[gi][0], v[gi][2]), mx1 = fmaxf(v[gi][1], v[gi][3]);
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1) {
            mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o));
            mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o));
          }
          const float n0 = fmaxf(m_ref[gi][0], mx0), n1 = fmaxf(m_ref[gi][1], mx1);
          const float a0 = m_ref[gi][0] == -INFINITY ? 0.f : exp2f(m_ref[gi][0] - n0);
          const float a1 = m_ref[gi][1] == -INFINITY ? 0.f : exp2f(m_ref[gi][1] - n1);
          m_ref[gi][0] = n0; m_ref[gi][1] = n1;
          l_part[gi][0] *= a0; l_part[gi][1] *= a1;
#pragma unroll
          for (int db = 0; db < KS; ++db) {
            oacc[gi][db][0] *= a0; oacc[gi][db][1] *= a1; oacc[gi][db][2] *= a0; oacc[gi][db][3] *= a1;
          }
        }
      }
      if constexpr (F32) {
        Tf32 pb[NG][2][2];                                                 // P^T as B operands: [k block of 8 rows][k = tq: row 2 tq, k = tq + 4: row 2 tq + 1]
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
          const float r0 = m_ref[gi][0] == -INFINITY ? 0.f : m_ref[gi][0], r1 = m_ref[gi][1] == -INFINITY ? 0.f : m_ref[gi][1];
#pragma unroll
          for (int r8 = 0; r8 < 2; ++r8) {
            const float p0 = fast_exp2(v[gi][2 * r8] - r0), p1 = fast_exp2(v[gi][2 * r8 + 1] - r1);
            l_part[gi][0] += p0;
            l_part[gi][1] += p1;
            // transposed as two matrices of 16-bit halves
            const uint32_t up = movmatrix_t(__byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632));
            const uint32_t dn = movmatrix_t(__byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x5410));
            pb[gi][r8][0] = tf32_of(__uint_as_float(__byte_perm(dn, up, 0x5410)));
            pb[gi][r8][1] = tf32_of(__uint_as_float(__byte_perm(dn, up, 0x7632)));
          }
        }
        // ---- O^T += V tile^T . P^T ----  (even rows first: the threads of a warp then read different banks)
#pragma unroll
        for (int db = 0; db < KS; ++db) {
          if (!EXACT && 16 * db >= d_v) break;
          const unsigned char* sv = wstages + s * S::STAGE_B + S::TENS_B + (db >> 1) * SLAB_B + (gq & 3) * 4;
          const int c = (db & 1) * 4 + (gq >> 2);
#pragma unroll
          for (int r8 = 0; r8 < 2; ++r8) {
            const int r = 8 * r8 + 2 * tq;
            const auto val = [&](int row, int chunk) { return tf32x3_of(*reinterpret_cast<const float*>(sv + swz(row, chunk))); };
            const Tf32x3 vx[4] = {val(r, c), val(r, c + 2), val(r + 1, c), val(r + 1, c + 2)};
#pragma unroll
            for (int gi = 0; gi < NG; ++gi) mma_3tf32(oacc[gi][db], vx, pb[gi][r8][0], pb[gi][r8][1]);
          }
        }
      } else {
        uint32_t ph[NG][2], pl[NG][2];                                     // P^T as B operands: the rounded p and the rest
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) {
          const float r0 = m_ref[gi][0] == -INFINITY ? 0.f : m_ref[gi][0], r1 = m_ref[gi][1] == -INFINITY ? 0.f : m_ref[gi][1];
#pragma unroll
          for (int r8 = 0; r8 < 2; ++r8) {
            const float p0 = fast_exp2(v[gi][2 * r8] - r0), p1 = fast_exp2(v[gi][2 * r8 + 1] - r1);
            l_part[gi][0] += p0;
            l_part[gi][1] += p1;
            const uint32_t hi = pack_bf16(p0, p1);
            const float h0 = __uint_as_float(hi << 16), h1 = __uint_as_float(hi & 0xffff0000u);
            ph[gi][r8] = movmatrix_t(hi);
            pl[gi][r8] = movmatrix_t(pack_bf16(p0 - h0, p1 - h1));
          }
        }
        // ---- O^T += V tile^T . P^T ----
#pragma unroll
        for (int db = 0; db < KS; ++db) {
          if (!EXACT && 16 * db >= d_v) break;
          uint32_t af[4];
          ldsm4t(sV + (db >> 2) * SLAB_B + swz(v_row, (db & 3) * 2 + v_cadd), af);
#pragma unroll
          for (int gi = 0; gi < NG; ++gi) {
            mma16816(oacc[gi][db], af, ph[gi][0], ph[gi][1]);
            mma16816(oacc[gi][db], af, pl[gi][0], pl[gi][1]);
          }
        }
      }
      __syncwarp();
      if (todo) {
        // the stage was read, and possibly cleared, through the generic proxy; the copy that refills it is of the async proxy
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        issue();
      }
    }

    // ---- join the warps: maxima first, then the outputs pairwise through two buffers ----
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
      for (int o = 4; o <= 16; o <<= 1) {
        l_part[gi][0] += __shfl_xor_sync(0xffffffffu, l_part[gi][0], o);
        l_part[gi][1] += __shfl_xor_sync(0xffffffffu, l_part[gi][1], o);
      }
      if (gq == 0) {
        const int c = w * NCOL + 8 * gi + 2 * tq;
        wm[c] = m_ref[gi][0]; wm[c + 1] = m_ref[gi][1];
        wl[c] = l_part[gi][0]; wl[c + 1] = l_part[gi][1];
      }
    }
    __syncthreads();
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      float f[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float M = -INFINITY;
#pragma unroll
        for (int ww = 0; ww < NWARP; ++ww) M = fmaxf(M, wm[ww * NCOL + 8 * gi + 2 * tq + x]);
        f[x] = m_ref[gi][x] == -INFINITY ? 0.f : exp2f(m_ref[gi][x] - M);
      }
#pragma unroll
      for (int db = 0; db < KS; ++db) {
        oacc[gi][db][0] *= f[0]; oacc[gi][db][1] *= f[1]; oacc[gi][db][2] *= f[0]; oacc[gi][db][3] *= f[1];
      }
    }
    if (tid < NCOL) {
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int ww = 0; ww < NWARP; ++ww) M = fmaxf(M, wm[ww * NCOL + tid]);
#pragma unroll
      for (int ww = 0; ww < NWARP; ++ww) {
        const float lw = wl[ww * NCOL + tid];
        L += lw == 0.f ? 0.f : lw * exp2f(wm[ww * NCOL + tid] - M);
      }
      jm[tid] = M; jl[tid] = L;
    }
    // the upper half of the warps leave their outputs in a buffer each, the lower half add theirs there
#pragma unroll 1
    for (int lower = 0; lower < 2; ++lower) {
      if ((w < NWARP / 2) == (lower == 1)) {
        float* b = buf + (w % (NWARP / 2)) * NCOL * LD + 2 * tq * LD + gq;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int db = 0; db < KS; ++db)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              float* p = b + (8 * gi + (x & 1)) * LD + 16 * db + 8 * (x >> 1);
              *p = lower ? *p + oacc[gi][db][x] : oacc[gi][db][x];
            }
      }
      __syncthreads();
    }
    write_segment<T, S::NT, NWARP / 2>(a, buf, LD, NCOL * LD, jm, jl, at.e, at.u, nh, whole, 2 * blockIdx.x + (at.t == 0));

    if (tb < at.nt) break;
    done += cnt;
    at.t = 0;
    next_unit<TR>(a, held, at);
    if (at.e >= a.n || at.pos >= end) break;
    load_q();
  }
  if (dead) {
    if (a.status) atomicOr(a.status, SNAP_DEV_WAIT_TIMEOUT);
    for (int x = n; x < n_issued; ++x) (void)wait_bounded(bar0 + 8 * (x % NSTAGE), (unsigned)(x / NSTAGE) & 1u);
  }
}

// ---------------------------------------------------------------------------------------------------------------
// portable kernel
// ---------------------------------------------------------------------------------------------------------------
struct Four { F2 a, b; };                          // four consecutive elements
__device__ __forceinline__ Four four(const float* p) {
  const ulonglong2 r = *reinterpret_cast<const ulonglong2*>(p);
  return {r.x, r.y};
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, unsigned bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

constexpr int SNW = 4, SNT = SNW * 32;            // warps and threads of a CTA
constexpr int MAX_STAGES = 6;                     // of a warp

// NV: 128-dim chunks of a row, HB: heads of a unit (a power of two)
template <int NV, int HB, int CTAS>
__global__ void __launch_bounds__(SNT, CTAS) paged_simt_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v) {
  constexpr int LD = 128 * NV + 4, STR = simt_rows(NV > 1), TPL = 32 / STR;   // tiles that a warp looks up at once, a lane per row
  constexpr int NVAL = 4 * HB, HL = 8 / HB;                              // (row, head) pairs of four rows; lanes that hold the same pair
  extern __shared__ unsigned char smem_dyn[];
  // [SNW][a.stages][STR key rows | STR value rows], on a 128-byte boundary as every part of it is (rows are multiples of 32 bytes)
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 127) & ~uintptr_t(127));
  __shared__ __align__(16) float buf[2 * HB * LD];
  __shared__ float wm[SNW * HB], wl[SNW * HB], jm[HB], jl[HB];
  __shared__ uint64_t bars[SNW * MAX_STAGES];
  __shared__ int scan[SNT / 32 + 2];
  __shared__ Held held;
  __shared__ Found found;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const unsigned krow_b = a.d_qk * sizeof(float), vrow_b = a.d_v * sizeof(float), stage_b = STR * (krow_b + vrow_b);
  const unsigned char* wstages = stages + w * a.stages * stage_b;
  const uint32_t stage0 = smem_u32(wstages), bar0 = smem_u32(bars + w * MAX_STAGES);
  if (lane == 0) {
    for (int s = 0; s < a.stages; ++s) mbar_init(bar0 + 8 * s, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  Place at;
  int end;
  if (!locate<STR, SNT>(a, at, end, held, scan, found)) return;
  const int my_head = (lane & 7) / HL;                                   // after the exchange lane l owns row l / 8 and this head

  // ---- the warp's producer: lane l looks up row l % STR of the warp's tile l / STR, l / STR + TPL, ... ----
  Place pr = at;
  bool valid = advance<STR>(a, held, pr, w + SNW * (lane / STR), end);
  int pid = -1, prow = 0, kvh_of = 0, s_in = 0, in_flight = 0, next = 0;  // next: which of the TPL tiles is issued next
  constexpr unsigned ROWS = (1u << STR) - 1u;
  unsigned todo = 0;                                                     // bit STR j: tile j is there
  unsigned long long okay_of = 0;                                        // 8 bits per stage: the rows that are there
  const auto fetch = [&]() {
    todo = __ballot_sync(0xffffffffu, valid);
    pid = -1;
    const int row = pr.t * STR + lane % STR;
    if (valid && row < pr.len) {
      const int pg = row / a.map.page;
      prow = row - pg * a.map.page;
      if (index_ok(pg, a.map.max_pages, a.status)) pid = a.map.table[(long long)pr.slot * a.map.max_pages + pg];
      kvh_of = pr.u / a.nhb;
    }
  };
  const auto issue = [&]() {
    const bool mine = lane / STR == next, bad = mine && valid && pr.t * STR + lane % STR < pr.len && (pid < 0 || pid >= a.map.n_pages);
    if (bad) {
      pid = -1;
      if (a.status) atomicOr(a.status, SNAP_DEV_BAD_PAGE);
    }
    const unsigned okay = (__ballot_sync(0xffffffffu, pid >= 0) >> (STR * next)) & ROWS;
    okay_of = (okay_of & ~(0xffull << (8 * s_in))) | ((unsigned long long)okay << (8 * s_in));
    const uint32_t bar = bar0 + 8 * s_in, dst = stage0 + s_in * stage_b;
    const int r = lane % STR;
    if (a.tiled) {                                                       // one copy each for the tile's keys and values
      if (mine && r == 0) {
        mbar_expect_tx(bar, okay ? stage_b : 0u);
        if (okay) {
          tma_load_4d(dst, &tmap_k, 0, prow, kvh_of, pid, bar);
          tma_load_4d(dst + STR * krow_b, &tmap_v, 0, prow, kvh_of, pid, bar);
        }
      }
    } else {                                                             // a copy per row
      if (lane == 0) mbar_expect_tx(bar, __popc(okay) * (krow_b + vrow_b));
      __syncwarp();
      if (mine && pid >= 0) {
        bulk_load(dst + r * krow_b, static_cast<const float*>(a.kp) + pid * a.map.kp + kvh_of * a.map.kh + prow * a.map.kr, krow_b, bar);
        bulk_load(dst + STR * krow_b + r * vrow_b, static_cast<const float*>(a.vp) + pid * a.map.vp + kvh_of * a.map.vh + prow * a.map.vr, vrow_b, bar);
      }
    }
    ++in_flight;
    if (++s_in == a.stages) s_in = 0;
    todo &= ~(ROWS << (STR * next));
    if (++next == TPL) {
      next = 0;
      if (valid) valid = advance<STR>(a, held, pr, TPL * SNW, end);
      fetch();
    }
  };
  fetch();
  F2 q[HB][NV][2];
  const auto load_q = [&]() {
    const int kvh = at.u / a.nhb, hb = at.u - kvh * a.nhb, nh = min(a.gb, a.g - hb * a.gb);
    const float* qp = static_cast<const float*>(a.q) + ((long long)at.e * a.Hq + kvh * a.g + hb * a.gb) * a.d_qk + 4 * lane;
#pragma unroll
    for (int h = 0; h < HB; ++h)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        Four f = {0, 0};
        if (h < nh && 4 * lane + 128 * j < a.d_qk) f = four(qp + h * a.d_qk + 128 * j);
        q[h][j][0] = f.a; q[h][j][1] = f.b;
      }
  };
  load_q();                                                              // (the first tiles' look-ups wait alongside)
#pragma unroll 1
  for (int s = 0; s < a.stages && todo; ++s) issue();

  bool dead = false;                                                     // a bounded wait ran out: nothing more is read
  int n = 0, done = 0, s_out = 0;
  unsigned parity = 0;
  while (true) {
    const int tb = segment_end(at, end), cnt = tb - at.t;
    const int hb = at.u % a.nhb, nh = min(a.gb, a.g - hb * a.gb);
    const bool whole = cnt == at.nt;
    F2 o[HB][NV][2];
    float m_ref = -INFINITY, l_part = 0.f;
#pragma unroll
    for (int h = 0; h < HB; ++h)
#pragma unroll
      for (int j = 0; j < NV; ++j) o[h][j][0] = o[h][j][1] = 0;
    float* srow = a.scores ? a.scores + ((long long)at.e * a.U + at.u) * a.map.cap * a.gs : nullptr;

    for (; w + n * SNW < done + cnt && !dead; ++n) {
      const bool landed = wait_bounded(bar0 + 8 * s_out, parity);
      if (__any_sync(0xffffffffu, !landed)) { dead = true; break; }
      --in_flight;
      const int row0 = (at.t + (w + n * SNW - done)) * STR;
      const unsigned okay = (unsigned)(okay_of >> (8 * s_out)) & 0xffu;
#pragma unroll 1
      for (int r0 = 0; r0 < STR; r0 += 4) {
        const unsigned there = (okay >> r0) & 0xfu;
        if (there == 0u && !srow) continue;
        const float* kx = reinterpret_cast<const float*>(wstages + s_out * stage_b) + r0 * a.d_qk + 4 * lane;
        const float* vx = reinterpret_cast<const float*>(wstages + s_out * stage_b + STR * krow_b) + r0 * a.d_v + 4 * lane;
        float s[NVAL];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          Four f[NV];
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            f[j] = {0, 0};
            if (4 * lane + 128 * j < a.d_qk) f[j] = four(kx + r * a.d_qk + 128 * j);
          }
#pragma unroll
          for (int h = 0; h < HB; ++h) {
            F2 x = mul2(f[0].a, q[h][0][0]);
            x = fma2(f[0].b, q[h][0][1], x);
#pragma unroll
            for (int j = 1; j < NV; ++j) {
              x = fma2(f[j].a, q[h][j][0], x);
              x = fma2(f[j].b, q[h][j][1], x);
            }
            const float2 y = unpack2(x);
            s[r * HB + h] = y.x + y.y;
          }
        }
        // halving exchange: each step sums over one lane bit and leaves a lane half of the values
        int left = NVAL;
#pragma unroll
        for (int b = 16; b > 0; b >>= 1) {
          if (left > 1) {
            left >>= 1;
#pragma unroll
            for (int x = 0; x < NVAL / 2; ++x)
              if (x < left) {
                const bool up = lane & b;
                const float give = up ? s[x] : s[x + left], keep = up ? s[x + left] : s[x];
                s[x] = keep + __shfl_xor_sync(0xffffffffu, give, b);
              }
          } else {
            s[0] += __shfl_xor_sync(0xffffffffu, s[0], b);
          }
        }
        // rows that are not there hold anything
        const float v = (there >> (lane >> 3)) & 1u ? s[0] * a.scale_log2 : -INFINITY;
        const int row = row0 + r0 + (lane >> 3);
        if (srow && row < at.len && my_head < nh && index_ok(row, a.map.cap, a.status)) srow[(long long)row * a.gs + my_head] = v;   // (lanes of one pair write the same)
        if (__any_sync(0xffffffffu, v > m_ref + 8.f)) {                    // the reference moves lazily, as in the kernel above
          float mx = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          const float nm = fmaxf(m_ref, mx), al = m_ref == -INFINITY ? 0.f : exp2f(m_ref - nm);
          m_ref = nm;
          l_part *= al;
#pragma unroll
          for (int h = 0; h < HB; ++h) {
            const float f = __shfl_sync(0xffffffffu, al, h * HL);
            const F2 f2 = pack2(f, f);
#pragma unroll
            for (int j = 0; j < NV; ++j) { o[h][j][0] = mul2(o[h][j][0], f2); o[h][j][1] = mul2(o[h][j][1], f2); }
          }
        }
        const float p = fast_exp2(v - (m_ref == -INFINITY ? 0.f : m_ref));
        l_part += p;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (!((there >> r) & 1u)) continue;                              // a zero probability does not silence a NaN
          Four f[NV];
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            f[j] = {0, 0};
            if (4 * lane + 128 * j < a.d_v) f[j] = four(vx + r * a.d_v + 128 * j);
          }
#pragma unroll
          for (int h = 0; h < HB; ++h) {
            const float x = __shfl_sync(0xffffffffu, p, 8 * r + h * HL);
            const F2 x2 = pack2(x, x);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
              o[h][j][0] = fma2(x2, f[j].a, o[h][j][0]);
              o[h][j][1] = fma2(x2, f[j].b, o[h][j][1]);
            }
          }
        }
      }
      if (++s_out == a.stages) { s_out = 0; parity ^= 1u; }
      __syncwarp();                                                      // the stage has been read
      if (todo) issue();
    }

    // ---- join the warps ----
    l_part += __shfl_xor_sync(0xffffffffu, l_part, 8);
    l_part += __shfl_xor_sync(0xffffffffu, l_part, 16);
    if (lane < 8) { wm[w * HB + my_head] = m_ref; wl[w * HB + my_head] = l_part; }   // (equal values where lanes share a head)
    __syncthreads();
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      float M = -INFINITY;
#pragma unroll
      for (int ww = 0; ww < SNW; ++ww) M = fmaxf(M, wm[ww * HB + h]);
      const float mw = wm[w * HB + h], f = mw == -INFINITY ? 0.f : fast_exp2(mw - M);
      const F2 f2 = pack2(f, f);
#pragma unroll
      for (int j = 0; j < NV; ++j) { o[h][j][0] = mul2(o[h][j][0], f2); o[h][j][1] = mul2(o[h][j][1], f2); }
    }
    if (tid < HB) {
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int ww = 0; ww < SNW; ++ww) M = fmaxf(M, wm[ww * HB + tid]);
#pragma unroll
      for (int ww = 0; ww < SNW; ++ww) {
        const float lw = wl[ww * HB + tid];
        L += lw == 0.f ? 0.f : lw * fast_exp2(wm[ww * HB + tid] - M);
      }
      jm[tid] = M; jl[tid] = L;
    }
#pragma unroll 1
    for (int lower = 0; lower < 2; ++lower) {
      if ((w < SNW / 2) == (lower == 1)) {
        float* b = buf + (w % (SNW / 2)) * HB * LD + 4 * lane;
#pragma unroll
        for (int h = 0; h < HB; ++h)
#pragma unroll
          for (int j = 0; j < NV; ++j) {
            float4* x = reinterpret_cast<float4*>(b + h * LD + 128 * j);
            const float2 f0 = unpack2(o[h][j][0]), f1 = unpack2(o[h][j][1]);
            float4 f = make_float4(f0.x, f0.y, f1.x, f1.y);
            if (lower) { const float4 y = *x; f.x += y.x; f.y += y.y; f.z += y.z; f.w += y.w; }
            *x = f;
          }
      }
      __syncthreads();
    }
    write_segment<float, SNT, SNW / 2>(a, buf, LD, HB * LD, jm, jl, at.e, at.u, nh, whole, 2 * blockIdx.x + (at.t == 0));
    if (tb < at.nt) break;
    done += cnt;
    at.t = 0;
    next_unit<STR>(a, held, at);
    if (at.e >= a.n || at.pos >= end) break;
    load_q();
  }
  if (dead) {
    if (a.status) atomicOr(a.status, SNAP_DEV_WAIT_TIMEOUT);
    for (; in_flight > 0; --in_flight) {
      (void)wait_bounded(bar0 + 8 * s_out, parity);
      if (++s_out == a.stages) { s_out = 0; parity ^= 1u; }
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------
// second launch: joins the pieces of cut units, zeroes the outputs of empty sequences, sums the weights
// ---------------------------------------------------------------------------------------------------------------
constexpr int JNT = 256;
__host__ __device__ constexpr int join_rows(int quads) { return quads == 1 ? 2 : 1; }   // of a thread at a time
constexpr int MAX_MU = 2048;                       // heads of a KV head whose weights are summed (in the shared memory that a join's outputs take)

struct Pieces { int np, c0; };                     // pieces of a unit; np <= 1: done whole
__device__ __forceinline__ Pieces pieces_of(const PagedArgs& a, int u, int before, int total, int nt) {
  Pieces p;
  const long long W = (long long)total * a.U, x = (long long)before * a.U + (long long)u * length_of(nt);
  const int active = active_ctas(W, a.ctas);
  p.c0 = owner_of(x, W, active);
  p.np = owner_of(x + begin_of(nt - 1, nt), W, active) - p.c0 + 1;
  return p;
}
__device__ __forceinline__ int piece_at(const Pieces& p, int k) { return 2 * (p.c0 + k) + (k == 0); }

// Weights of (sequence, KV head) id / per: the rows of batches id mod per, + per, ...  line: the line's length; mu_s:
// shared, [nhb][gb], p = 2^(logit - mu)
template <int Q>
__device__ __forceinline__ void join_weights(const PagedArgs& a, int id, int per, int line, float* mu_s) {
  constexpr int R = join_rows(Q), BATCH = R * JNT;                         // rows of a thread, of the CTA
  __shared__ float piece_m[JNT], piece_l[JNT];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int part = id % per, kvh = (id / per) % a.Hkv, e = id / per / a.Hkv;
  const int4 at = a.entry[e];
  const int before = at.x, slot = at.y, len = at.z, nt = at.w;
  if ((long long)part * BATCH >= len) return;
  const long long base = ((long long)slot * a.Hkv + kvh) * a.map.cap;
  float4 v[R][Q], ahead[R][Q];                                            // logits of this and of the next step
  float old[R], old_ahead[R];
  const auto load = [&](int row0, int hb, float4 (&to)[R][Q]) {
    const float* sc = a.scores + ((long long)e * a.U + kvh * a.nhb + hb) * a.map.cap * a.gs;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int row = row0 + j * JNT + tid;
      const float* sr = sc + (long long)row * a.gs;
#pragma unroll
      for (int c = 0; c < Q; ++c) {
        to[j][c] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row >= len || 4 * c >= a.gs) continue;
        if (a.gs >= 4) to[j][c] = *reinterpret_cast<const float4*>(sr + 4 * c);
        else {
          to[j][c].x = sr[0];
          if (a.gs == 2) to[j][c].y = sr[1];
        }
      }
    }
  };
  const auto load_old = [&](int row0, float (&to)[R]) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int row = row0 + j * JNT + tid;
      to[j] = a.w_in && row < len ? a.w_in[base + row] : 0.f;
    }
  };
  load(part * BATCH, 0, v);                                               // under way while the maxima and sums are put together
  load_old(part * BATCH, old);
  int again = 0;                                                         // the slot was listed before: its first entry counts
  for (int x = tid; x < e; x += JNT) again |= a.slots[x] == slot;
  if (__syncthreads_or(again)) {
    if (tid == 0 && a.status) atomicOr(a.status, SNAP_DEV_BAD_SLOT);
    return;
  }
  const int npar = JNT / a.gb, mine = tid % a.gb, k0 = tid / a.gb;         // pieces read at once, this thread's column and first piece
  for (int hb = 0; hb < a.nhb; ++hb) {
    const int u = kvh * a.nhb + hb, nh = min(a.gb, a.g - hb * a.gb);
    const Pieces p = pieces_of(a, u, before, line, nt);
    float m = -INFINITY, l = 0.f;
    if (mine < nh && k0 < npar) {
      if (p.np <= 1) {
        if (k0 == 0) {
          const float2 ml = a.ml_unit[((long long)e * a.U + u) * a.gb + mine];
          m = ml.x; l = ml.y;
        }
      } else {
#pragma unroll 4
        for (int k = k0; k < p.np; k += npar) {
          if (!index_ok(piece_at(p, k), 2LL * a.ctas, a.status)) continue;
          const float2 ml = a.ml_part[(long long)piece_at(p, k) * a.gb + mine];
          if (ml.y == 0.f) continue;                                       // a piece without rows
          const float nm = fmaxf(m, ml.x);
          l = (l == 0.f ? 0.f : l * exp2f(m - nm)) + ml.y * exp2f(ml.x - nm);   // (a NaN stays, also of a piece with no other maximum)
          m = nm;
        }
      }
    }
    __syncthreads();                                                       // the block before has been read
    piece_m[tid] = m;
    piece_l[tid] = l;
    __syncthreads();
    for (int col = w; col < nh; col += JNT / 32) {
      float M = -INFINITY, L = 0.f;
      for (int k = lane; k < npar; k += 32) M = fmaxf(M, piece_m[k * a.gb + col]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      for (int k = lane; k < npar; k += 32) {
        const float pl = piece_l[k * a.gb + col];
        L += pl == 0.f ? 0.f : pl * exp2f(piece_m[k * a.gb + col] - M);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
      if (lane == 0) mu_s[hb * a.gb + col] = L == 0.f ? INFINITY : M + log2f(L);   // no valid row: all weights 0
    }
  }
  __syncthreads();
  for (int row0 = part * BATCH; row0 < len;) {
    const int next = (int)min((long long)row0 + (long long)per * BATCH, (long long)len);
    float sum[R];                                                          // (the old weight is added last: one rounding at the size of the total)
#pragma unroll
    for (int j = 0; j < R; ++j) sum[j] = 0.f;
    // A row on a page that is not there was left out: its entry stays.  Its logits are -infinity, which those of a row that
    // counts may be too, so the page table decides (looked up for such rows only).
    bool stays[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int row = row0 + j * JNT + tid;
      stays[j] = row >= len;
      if (!stays[j] && v[j][0].x == -INFINITY) {
        const int page = a.map.table[(long long)slot * a.map.max_pages + row / a.map.page];
        stays[j] = page < 0 || page >= a.map.n_pages;
      }
    }
    for (int hb = 0; hb < a.nhb; ++hb) {
      const int nh = min(a.gb, a.g - hb * a.gb);
      const float* mu = mu_s + hb * a.gb;
      if (hb + 1 < a.nhb) load(row0, hb + 1, ahead);
      else { load(next, 0, ahead); load_old(next, old_ahead); }
#pragma unroll
      for (int c = 0; c < Q; ++c)
#pragma unroll
        for (int j = 0; j < R; ++j) {
          if (4 * c < nh) sum[j] += fast_exp2(v[j][c].x - mu[4 * c]);
          if (4 * c + 1 < nh) sum[j] += fast_exp2(v[j][c].y - mu[4 * c + 1]);
          if (4 * c + 2 < nh) sum[j] += fast_exp2(v[j][c].z - mu[4 * c + 2]);
          if (4 * c + 3 < nh) sum[j] += fast_exp2(v[j][c].w - mu[4 * c + 3]);
          v[j][c] = ahead[j][c];
        }
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int row = row0 + j * JNT + tid;
      if (!stays[j] && index_ok(row, a.map.cap, a.status)) a.w_out[base + row] = old[j] + sum[j];
      old[j] = old_ahead[j];
    }
    row0 = next;
  }
}

// Grid: `first` CTAs for the weights, which take longer, then the outputs'.  The outputs go either by query head (a CTA
// each: the shorter way to the pieces), or, where there are many heads, by the borders between the stretches of the first
// launch: the unit that a border cuts is joined by the CTAs of the borders that cut it, which take its heads in turn, so
// that no more CTAs than borders are started however many units there are.  (By heads against by borders: one sequence
// of 5124 rows, 32 heads 11.9 / 12.9 us a call; 16 of up to 6000 rows, 512 heads 41.9 / 43.7; 24, 768 heads 55.8 / 57.3; 48 of up
// to 400 rows, 1536 heads 24.6 / 23.3, 20 of them, 640 heads 13.9 / 14.2.)
//
// This kernel lets the next one start only when it ends: blocks of the split kernel that start beside blocks of this
// one get the registers in between them, and once these end the rest of an SM's registers is in pieces too small for
// the third block, which then waits for a whole stretch to end (16 long sequences: 366 instead of 332 us a call).
//
// Weights: `per` CTAs for each (sequence, KV head) put together the maximum and sum of every head of the group (thread t
// reads the pieces of column t mod gb: all of them in one latency), then walk over the rows, a thread to a row and all of
// a row's logits at once, the next rows' on their way meanwhile.  Q: 16-byte pieces of a row's logits (0: no weights).
template <typename T, int Q>
__global__ void __launch_bounds__(JNT, 3) paged_join_kernel(const __grid_constant__ PagedArgs a, int first, int by_heads, int per) {
  __shared__ __align__(16) float acc_s[JNT / 32][256];
  __shared__ float red_m[JNT / 32], red_l[JNT / 32];
  __shared__ int s_e;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  if (tid == 0) s_e = -1;
  pdl_wait();
  const int line = a.entry[a.n].x;
  const int joins = gridDim.x - first, id = (int)blockIdx.x - first;       // of the outputs
  if (Q == 0 || id >= 0) {
    int e, u, nt, col0, step;
    Pieces p;
    const auto zero = [&](int row, int rows) {                             // outputs of a sequence without rows
      T* out = static_cast<T*>(a.out) + (long long)row * a.d_v;
      for (int x = tid; x < rows * a.d_v; x += JNT) out[x] = from_f32<T>(0.f);
    };
    if (by_heads) {
      e = id / a.Hq;
      const int head = id - e * a.Hq, kvh = head / a.g, x = head - kvh * a.g, hb = x / a.gb;
      u = kvh * a.nhb + hb;
      col0 = x - hb * a.gb;
      step = a.gb;
      const int4 at = a.entry[e];
      const int before = at.x;
      nt = at.w;
      if (nt == 0) { zero(id, 1); return; }
      p = pieces_of(a, u, before, line, nt);
      if (p.np <= 1) return;                                               // written by the split kernel
    } else {
      for (int i = id; i < a.n; i += joins)
        if (a.entry[i].w == 0) zero(i * a.Hq, a.Hq);
      const long long W = (long long)line * a.U;
      const int active = active_ctas(W, a.ctas), c = id + 1;
      if (c >= active) return;
      const long long x = stretch_begin(W, active, c);
      __syncthreads();
      for (int i = tid; i < a.n; i += JNT) {                               // one thread has it
        const int4 at = a.entry[i];
        if ((long long)at.x * a.U <= x && x < (long long)(at.x + length_of(at.w)) * a.U) s_e = i;
      }
      __syncthreads();
      e = s_e;
      if (e < 0) return;                                                   // (only if the lengths change during the call)
      const int4 at = a.entry[e];
      const int before = at.x, unit = length_of(at.w);
      const long long rel = x - (long long)before * a.U;
      nt = at.w;
      u = rel < (1LL << 31) ? (int)((unsigned)rel / (unsigned)unit) : (int)(rel / unit);
      p = pieces_of(a, u, before, line, nt);
      // the unit's pieces are those of the CTAs c0 .. c0 + np - 1: the border before CTA c0 + k is its k-th
      const int kth = c - p.c0;
      if (p.np <= 1 || kth < 1 || kth >= p.np) return;                     // not cut, or cut elsewhere
      col0 = kth - 1;
      step = p.np - 1;
    }
    const int kvh = u / a.nhb, hb = u - kvh * a.nhb, nh = min(a.gb, a.g - hb * a.gb);
    for (int col = col0; col < nh; col += step) {
      // a warp takes every eighth piece, four at a time: their (max, sum) and outputs come in together
      float m = -INFINITY, l = 0.f;
      float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
      for (int k0 = w; k0 < p.np; k0 += 4 * (JNT / 32)) {
        float2 ml[4];
        float4 v[4][2];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int k = k0 + y * (JNT / 32);
          const bool there = k < p.np && index_ok(piece_at(p, k), 2LL * a.ctas, a.status);
          ml[y] = make_float2(-INFINITY, 0.f);
          if (there) ml[y] = a.ml_part[(long long)piece_at(p, k) * a.gb + col];
          const float* o = a.o_part + ((long long)piece_at(p, there ? k : 0) * a.gb + col) * a.d_v + 4 * lane;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            v[y][j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (there && 4 * lane + 128 * j < a.d_v) v[y][j] = *reinterpret_cast<const float4*>(o + 128 * j);
          }
        }
        const float nm = fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), m);
        const float f = m == -INFINITY ? 0.f : fast_exp2(m - nm);
        m = nm;
        l *= f;
#pragma unroll
        for (int j = 0; j < 2; ++j) { acc[j].x *= f; acc[j].y *= f; acc[j].z *= f; acc[j].w *= f; }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          if (ml[y].y == 0.f) continue;                                    // a piece without rows
          const float g = fast_exp2(ml[y].x - m);
          l = fmaf(ml[y].y, g, l);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            acc[j].x = fmaf(g, v[y][j].x, acc[j].x); acc[j].y = fmaf(g, v[y][j].y, acc[j].y);
            acc[j].z = fmaf(g, v[y][j].z, acc[j].z); acc[j].w = fmaf(g, v[y][j].w, acc[j].w);
          }
        }
      }
      __syncthreads();                                                     // the column before has been read
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (4 * lane + 128 * j < a.d_v) *reinterpret_cast<float4*>(&acc_s[w][4 * lane + 128 * j]) = acc[j];
      if (lane == 0) { red_m[w] = m; red_l[w] = l; }
      __syncthreads();
      float M = -INFINITY, L = 0.f, f_w[JNT / 32];
#pragma unroll
      for (int k = 0; k < JNT / 32; ++k) M = fmaxf(M, red_m[k]);
#pragma unroll
      for (int k = 0; k < JNT / 32; ++k) {
        f_w[k] = red_l[k] == 0.f ? 0.f : fast_exp2(red_m[k] - M);
        L = fmaf(red_l[k], f_w[k], L);
      }
      const float inv = L > 0.f ? 1.f / L : L;
      T* out = static_cast<T*>(a.out) + ((long long)e * a.Hq + kvh * a.g + hb * a.gb + col) * a.d_v;
      for (int x2 = tid; x2 < a.d_v; x2 += JNT) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < JNT / 32; ++k) s = fmaf(acc_s[k][x2], f_w[k], s);
        out[x2] = from_f32<T>(s * inv);
      }
    }
    return;
  }
  if constexpr (Q > 0) join_weights<Q>(a, blockIdx.x, per, line, &acc_s[0][0]);
}

// ---------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------
template <typename T, int D, int NWARP, int NSTAGE, int NG, int CTAS, Tiles MODE>
cudaError_t launch_mma_as(const PagedArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  using S = MmaShape<T, D, NWARP, NSTAGE, NG>;
  static_assert(CTAS * (S::smem + sizeof(Held) + 1280) <= 228 * 1024, "all CTAs of the grid are resident at once");
  static SmemLimit limit = {};
  if (cudaError_t e = ensure_dyn_smem(paged_mma_kernel<T, D, NWARP, NSTAGE, NG, CTAS, MODE>, S::smem, limit)) return e;
  const cudaError_t e = launch_pdl(paged_mma_kernel<T, D, NWARP, NSTAGE, NG, CTAS, MODE>, dim3(a.ctas), dim3(S::NT), S::smem, st, a, tk, tv);
  count_launch();
  return e;
}

template <typename T, int D, int NWARP, int NSTAGE, int NG, int CTAS>
cudaError_t launch_mma(const PagedArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  if (!a.tiled) return launch_mma_as<T, D, NWARP, NSTAGE, NG, CTAS, Tiles::ROWS>(a, tk, tv, st);
  return a.d_qk == D && a.d_v == D && a.map.page % TR == 0 ? launch_mma_as<T, D, NWARP, NSTAGE, NG, CTAS, Tiles::EXACT>(a, tk, tv, st)
                                                           : launch_mma_as<T, D, NWARP, NSTAGE, NG, CTAS, Tiles::BOXES>(a, tk, tv, st);
}

// CTAs per SM that the kernels are built for (launch bounds, and the shared memory of the tensor-core ones)
constexpr int kMmaCtas = 3, kMmaCtasWide = 2;
constexpr int simt_ctas(bool wide) { return wide ? 2 : 3; }
// Stages of a warp of the portable kernel: what the CTAs of an SM leave each other of its shared memory.
int simt_stages(const Shape& s, int eb, int ctas, bool wide) {
  const int stage = simt_rows(wide) * (s.d_qk + s.d_v) * eb, n = (228 * 1024 / ctas - 11500) / (SNW * stage);   // 11.5 KB: static and reserved
  return n < 1 ? 1 : n > MAX_STAGES ? MAX_STAGES : n;
}

template <int NV, int HB>
cudaError_t launch_simt_hb(const PagedArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  constexpr int C = simt_ctas(NV > 1);
  static SmemLimit limit = {};
  const size_t smem = (size_t)SNW * a.stages * a.tr * (a.d_qk + a.d_v) * sizeof(float) + 128;
  if (cudaError_t e = ensure_dyn_smem(paged_simt_kernel<NV, HB, C>, smem, limit)) return e;
  const cudaError_t e = launch_pdl(paged_simt_kernel<NV, HB, C>, dim3(a.ctas), dim3(SNT), smem, st, a, tk, tv);
  count_launch();
  return e;
}
template <int NV>
cudaError_t launch_simt(const PagedArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  if (a.gb <= 1) return launch_simt_hb<NV, 1>(a, tk, tv, st);
  if (a.gb <= 2) return launch_simt_hb<NV, 2>(a, tk, tv, st);
  return launch_simt_hb<NV, 4>(a, tk, tv, st);
}

// Logits stored of a row: vectors of four, when there are more than two.
int logits_of(int gb) { return gb <= 2 ? gb : (gb + 3) / 4 * 4; }

}  // namespace

int paged_decode_plan(int dtype, const Shape& s, const PageMap& m, int n_active, bool weights, int sms, PagedDecodePlan* p) {
  // Single precision: on the tensor cores a group of any size costs the same, but a tile's numbers have to be split.  8
  // sequences of 2000 to 6000 rows, 4 KV heads, portable against tensor cores in us: 64 dims, groups of 1, 4, 16: 26.9 / 20.7,
  // 33.5 / 21.6, 66.4 / 28.0; 128 dims, 1, 4, 8, 16: 29.2 / 34.5, 32.8 / 35.1, 38.9 / 36.1, 66.9 / 48.5; 256 dims, 4, 8: 50.6 /
  // 71.9, 79.7 / 72.9.
  p->mma = dtype == SNAP_BF16 || s.g > 4 || (s.d_qk <= 64 && s.d_v <= 64);
  const bool wide = s.d_qk > 128 || s.d_v > 128;
  const int most = p->mma ? (dtype == SNAP_F32 && wide ? 8 : 16) : 4;     // heads of a unit
  p->nhb = (s.g + most - 1) / most;
  p->gb = (s.g + p->nhb - 1) / p->nhb;
  const int per_sm = p->mma ? (p->gb > 8 || (dtype == SNAP_BF16 && wide) ? kMmaCtasWide : kMmaCtas) : simt_ctas(wide);
  p->ctas = sms * per_sm < MAX_CTAS ? sms * per_sm : MAX_CTAS;
  const long long units = (long long)n_active * s.Hkv * p->nhb;
  // grid and index limits; a line of tiles and the scratch have to be countable
  if (units > (1LL << 30) || (long long)n_active * s.Hq > 0x7fffffffLL || (weights && p->nhb * p->gb > MAX_MU) ||
      units * (m.cap / 4LL + 1 + UNIT_TILES) > (1LL << 37) || n_active * (m.cap / 4LL + 1 + UNIT_TILES) > 0x7fffffffLL)
    return SNAP_ERR_UNSUPPORTED;
  size_t off = 0;
  p->entry_off = off; off += align_up((size_t)(n_active + 1) * sizeof(int4));
  p->ml_off = off;     off += align_up(((size_t)units + 2 * (size_t)p->ctas) * p->gb * sizeof(float2));
  p->o_off = off;      off += align_up(2 * (size_t)p->ctas * p->gb * s.d_v * sizeof(float));
  p->score_off = off;
  if (weights) off += align_up((size_t)units * m.cap * logits_of(p->gb) * sizeof(float));
  p->bytes = off;
  return SNAP_OK;
}

cudaError_t launch_paged_decode(int dtype, const Shape& s, const PageMap& m, const PagedDecodePlan& p, const void* q,
                                const int* slots, int n_active, const void* k_pages, const void* v_pages, const int* seq_len,
                                const float* w_in, float* w_out, void* out, char* scratch, uint32_t* status, cudaStream_t st) {
  PagedArgs a;
  a.q = q; a.out = out; a.kp = k_pages; a.vp = v_pages; a.slots = slots; a.seq_len = seq_len;
  a.n = n_active; a.Hq = s.Hq; a.Hkv = s.Hkv; a.g = s.g; a.gb = p.gb; a.nhb = p.nhb; a.U = s.Hkv * p.nhb;
  a.d_qk = s.d_qk; a.d_v = s.d_v; a.max_seqs = s.max_seqs;
  a.scale_log2 = s.scale * 1.4426950408889634f;
  a.map = m;
  a.entry = reinterpret_cast<int4*>(scratch + p.entry_off);
  a.ml_unit = reinterpret_cast<float2*>(scratch + p.ml_off);
  a.ml_part = a.ml_unit + (size_t)n_active * a.U * p.gb;
  a.o_part = reinterpret_cast<float*>(scratch + p.o_off);
  a.scores = w_out ? reinterpret_cast<float*>(scratch + p.score_off) : nullptr;
  a.gs = logits_of(p.gb);
  a.w_in = w_in; a.w_out = w_out; a.status = status; a.ctas = p.ctas;
  const bool wide = s.d_qk > 128 || s.d_v > 128;
  a.tr = p.mma ? TR : simt_rows(wide);
  a.stages = simt_stages(s, elt_bytes(dtype), simt_ctas(wide), wide);
  // Tiles come through tensor maps where a page holds whole ones: 64 dims wide with the 128-byte swizzle for the
  // tensor-core kernel, whole rows for the portable one.  (Encoding both takes the host under a microsecond.)
  CUtensorMap tk = {}, tv = {};
  const umma::EncodeTiledFn enc = umma::encode_tiled_fn();
  const int rows = p.mma && m.page % TR ? TR / 2 : a.tr;       // of a box
  const auto encode = [&](CUtensorMap* t, const void* base, int d, long long ps, long long hs, long long rs) {
    const cuuint64_t eb = (cuuint64_t)elt_bytes(dtype);
    const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)m.page, (cuuint64_t)s.Hkv, (cuuint64_t)m.n_pages};
    // a stride that is never applied (one KV head, one page) may be anything: the map gets one that it takes
    const cuuint64_t strides[3] = {(cuuint64_t)rs * eb, (cuuint64_t)(s.Hkv > 1 ? hs : d) * eb, (cuuint64_t)(m.n_pages > 1 ? ps : d) * eb};
    const cuuint32_t box[4] = {(cuuint32_t)(p.mma ? 128 / elt_bytes(dtype) : d), (cuuint32_t)rows, 1, 1}, estr[4] = {1, 1, 1, 1};
    return enc(t, dtype == SNAP_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims,
               strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, p.mma ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  a.tiled = m.page % rows == 0 && enc && encode(&tk, k_pages, s.d_qk, m.kp, m.kh, m.kr) && encode(&tv, v_pages, s.d_v, m.vp, m.vh, m.vr);
  cudaError_t e;
  if (p.mma) {
    const bool two = p.gb > 8;
    const int d = s.d_qk > s.d_v ? s.d_qk : s.d_v;
    // Warps, stages of a warp and CTAs per SM share out its memory and registers.  Where a stage takes 16 KB or more, four
    // warps with one stage each beat two with two: 256 dims, 16 heads on each of 8, 8 sequences of 4000 to 8000 rows 93.9 /
    // 86.0 us; 4 heads on 4, 10 of 2158 to 21298 89.8 / 84.5.
    using BF = __nv_bfloat16;
    if (dtype == SNAP_F32) {
      if (d <= 64) e = two ? launch_mma<float, 64, 4, 2, 2, kMmaCtasWide>(a, tk, tv, st) : launch_mma<float, 64, 4, 2, 1, kMmaCtas>(a, tk, tv, st);
      else if (d <= 128) e = two ? launch_mma<float, 128, 4, 1, 2, kMmaCtasWide>(a, tk, tv, st) : launch_mma<float, 128, 4, 1, 1, kMmaCtas>(a, tk, tv, st);
      else e = launch_mma<float, 256, 2, 1, 1, kMmaCtas>(a, tk, tv, st);
    }
    else if (d <= 64) e = two ? launch_mma<BF, 64, 4, 4, 2, kMmaCtasWide>(a, tk, tv, st) : launch_mma<BF, 64, 4, 4, 1, kMmaCtas>(a, tk, tv, st);
    else if (d <= 128) e = two ? launch_mma<BF, 128, 4, 2, 2, kMmaCtasWide>(a, tk, tv, st) : launch_mma<BF, 128, 4, 2, 1, kMmaCtas>(a, tk, tv, st);
    else e = two ? launch_mma<BF, 256, 4, 1, 2, kMmaCtasWide>(a, tk, tv, st) : launch_mma<BF, 256, 4, 1, 1, kMmaCtasWide>(a, tk, tv, st);
  } else {
    e = wide ? launch_simt<2>(a, tk, tv, st) : launch_simt<1>(a, tk, tv, st);
  }
  if (e != cudaSuccess) return e;
  const int sms = sm_count(), heads = n_active * s.Hq, by_heads = heads <= 512 || p.ctas < 2;
  const int joins = by_heads ? heads : p.ctas - 1, pairs = n_active * s.Hkv;
  // CTAs of a (sequence, KV head)'s weights: as many as run at once beside half of the outputs' (which end sooner), and no
  // more than it can have batches of rows.  (A CTA per 1024 rows instead, each with the maxima and sums to put together:
  // 3 sequences of 22670 to 49189 rows, 16 heads on one, 35.7 us a call against 27.9; 8 heads 28.0 / 24.2; 8 sequences,
  // 4 heads on each of 8 the same.)
  const int quads = (p.gb + 3) / 4, batch = join_rows(quads) * JNT, most = (m.cap + batch - 1) / batch;
  const int room = 3 * sms, want = (joins < room ? room - joins / 2 : room / 2) / pairs, per = want < 1 ? 1 : want < most ? want : most;
  const int first = w_out ? pairs * per : 0;
  const dim3 grid((unsigned)(first + joins));
  const auto join = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(JNT), 0, st, a, first, by_heads, per); };
  if (dtype == SNAP_F32) {
    e = !w_out ? join(paged_join_kernel<float, 0>) : quads == 1 ? join(paged_join_kernel<float, 1>)
        : quads == 2 ? join(paged_join_kernel<float, 2>) : join(paged_join_kernel<float, 4>);
  } else {
    e = !w_out ? join(paged_join_kernel<__nv_bfloat16, 0>) : quads == 1 ? join(paged_join_kernel<__nv_bfloat16, 1>)
        : quads == 2 ? join(paged_join_kernel<__nv_bfloat16, 2>) : join(paged_join_kernel<__nv_bfloat16, 4>);
  }
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
