// Attention over caches in pages: how the tiles of all sequences are divided between CTAs, and how what they leave is joined.
// Shared by the kernels over full-precision pages (paged_decode.cu) and over 8-bit ones (q8_decode.cu).
//
// (sequence, KV head, block of its columns) is a unit; its rows are cut into tiles.  The units in a row form one line, each as
// long as its tiles plus a fixed share for what a unit costs however short it is (its queries, its joining), and the line
// is divided evenly between the CTAs: sequences of any lengths load the GPU evenly and the host need not know the
// lengths.  A CTA walks over its stretch, which holds whole units and at most one cut one at either end; units of a few
// tiles are never cut.  A whole unit's output is written at once; a cut one leaves the sum, the maximum and the
// unnormalised output of its piece, which the second launch joins in a fixed order (no atomics: equal inputs give equal
// bits).  A column is a query head of the KV head's group, of one of its tokens where there are several.
#pragma once

#include <cuda.h>

#include "mma_helpers.cuh"
#include "snap_internal.cuh"
#include "umma_helpers.cuh"

namespace snap {
namespace paged {

using mmasync::fast_exp2;
using umma::mbar_try_wait;

constexpr int UNIT_TILES = 6;                   // what a unit costs besides its tiles, in tiles; units of at most that many stay whole
                                                // (a kernel's arguments may have other numbers: share(), whole())
constexpr int MIN_TILES = 1;                    // a CTA gets at least that much beyond one unit's share (at least one: no stretch is empty)
// (Over full-precision pages, 40 calls of all sizes: 4 and 4 take 8 % longer, 8 and 1 2 %, 4 and 1 as long but 4 % longer for many short sequences.)
constexpr int MAX_CTAS = 1024, MAX_HELD = 128;  // sequences whose slot and length a CTA keeps in shared memory
// (Held against looked up in the batch's arrays: 17 sequences of up to 400 rows 14.4 / 14.95 us, 45 of 333 14.75 / 15.0, 100 of 500 35.7 /
// 35.8, 128 of 2000 96.7 / 97.0: the more sequences, the less it is worth.)
constexpr unsigned kPagedWaitLimit = 1u << 22;

// What the functions below take of a kernel's arguments, which also have out_row(e, kvh, x): the row of `out` that column x of a
// KV head of sequence e goes to.
struct LineArgs {
  void* out;
  const int* slots; const int* seq_len;
  int n, Hkv, g, gb, nhb, U, d_v, max_seqs;     // g columns of a KV head in U / Hkv = nhb units of gb columns (the last fewer)
  int rows_seq;                                 // rows of `out` of a sequence: Hkv * g
  PageMap map;
  int4* entry;                                  // [n + 1]: (the line before sequence i, per unit of a sequence; its slot, rows, tiles)
  float2* ml_unit;                              // [n * U][gb]: (max, sum), log2 domain, of units that one CTA did whole
  float2* ml_part; float* o_part;               // [2 * CTAs][gb], [2 * CTAs][gb][d_v]: pieces of cut units; CTA c's is 2 c, or
                                                // 2 c + 1 when it holds the unit's first tile (it has one of either at most)
  bool keep_ml;                                 // ml_unit is wanted
  uint32_t* status;
  int ctas;
  __device__ __forceinline__ constexpr int share() const { return UNIT_TILES; }
  __device__ __forceinline__ constexpr int whole() const { return UNIT_TILES; }
};

template <typename A> __device__ __forceinline__ int rows_of(const A& a, int slot) {
  if (slot < 0 || slot >= a.max_seqs) return 0;
  return min(max(a.seq_len[slot], 0), a.map.cap);
}
template <int ROWS> __device__ __forceinline__ int tiles_of(int rows) { return (int)(((unsigned)rows + ROWS - 1) / ROWS); }
template <typename A> __device__ __forceinline__ int length_of(const A& a, int nt) { return nt > 0 ? nt + a.share() : 0; }   // on the line
// Where tile t of a unit begins on the line, counted from the unit: the first tile carries the unit's share, and all
// tiles of a short unit begin (and so stay) with the first.
template <typename A> __device__ __forceinline__ int begin_of(const A& a, int t, int nt) { return t == 0 || nt <= a.whole() ? 0 : a.share() + t; }

// CTAs that share a line of length W, where CTA c's stretch begins, and whose stretch position x lies in.  (32-bit
// arithmetic where it suffices: 64-bit divisions are long instruction sequences.)
template <typename A> __device__ __forceinline__ int active_ctas(const A& a, long long W) {
  const int least = MIN_TILES + a.share();
  if (W >= (long long)a.ctas * least) return a.ctas;
  return W > 0 ? max((int)W / least, 1) : 0;
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
template <int ROWS, typename A> __device__ __forceinline__ void load_entry(const A& a, const Held& held, Place& p) {
  if (p.e >= a.n) {                             // the end of the line
    p.slot = -1; p.len = 0; p.nt = 1 << 29; p.e = a.n;
    return;
  }
  if (a.n <= MAX_HELD) { const int2 v = held.e[p.e]; p.slot = v.x; p.len = v.y; }
  else { p.slot = a.slots[p.e]; p.len = rows_of(a, p.slot); }
  p.nt = tiles_of<ROWS>(p.len);
}
template <int ROWS, typename A> __device__ __forceinline__ void next_unit(const A& a, const Held& held, Place& p) {
  p.pos += length_of(a, p.nt);
  if (++p.u == a.U) {
    p.u = 0;
    do { ++p.e; load_entry<ROWS>(a, held, p); } while (p.nt == 0);
  }
}
// `step` tiles on, or (false) past `end`, the end of the CTA's stretch
template <int ROWS, typename A> __device__ __forceinline__ bool advance(const A& a, const Held& held, Place& p, int step, int end) {
  p.t += step;
  while (p.t >= p.nt) {
    p.t -= p.nt;
    next_unit<ROWS>(a, held, p);
    if (p.e >= a.n || p.pos >= end) return false;
  }
  return p.pos + begin_of(a, p.t, p.nt) < end;
}

__device__ __forceinline__ int warp_inclusive(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += x; }
  return v;
}
// Slot and rows of the sequence in a slot; conditions to report
template <typename A> __device__ __forceinline__ int2 read_entry(const A& a, int slot, unsigned& bad) {
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
template <int ROWS, int NT, bool SMALL, typename A>
__device__ __forceinline__ bool locate_part(const A& a, Place& p, int& end, Held& held, int* scan /* shared, NT / 32 + 2 */) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = blockIdx.x;
  unsigned bad = 0;
  int total = 0, e_at = 0, before_at = 0;
  long long W = 0, x0 = 0, x1 = 0;
  int active = 0;
  const auto stretch = [&]() {
    W = (long long)total * a.U;
    active = active_ctas(a, W);
    if (c >= active) return false;
    x0 = stretch_begin(W, active, c);
    x1 = stretch_begin(W, active, c + 1);
    return true;
  };
  if (SMALL) {
    const int per = (a.n + 31) / 32, e0 = min(lane * per, a.n), e1 = min(e0 + per, a.n);   // a lane's sequences
    int mine = 0;
    constexpr int MOST = (MAX_HELD + 31) / 32;
    int slots[MOST];                                                     // (all slots on their way at once, then all lengths)
#pragma unroll
    for (int x = 0; x < MOST; ++x) slots[x] = e0 + x < e1 ? a.slots[e0 + x] : -1;
    int2 v[MOST];
#pragma unroll
    for (int x = 0; x < MOST; ++x) v[x] = read_entry(a, slots[x], bad);
#pragma unroll
    for (int x = 0; x < MOST; ++x)
      if (e0 + x < e1) {
        held.e[e0 + x] = v[x];
        mine += length_of(a, tiles_of<ROWS>(v[x].y));
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
        at += length_of(a, nt);
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
        const int len = length_of(a, tiles_of<ROWS>(held.e[e].y));
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
    for (int e = e0; e < e1; ++e) mine += length_of(a, tiles_of<ROWS>(read_entry(a, a.slots[e], bad).y));
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
        const int2 v = read_entry(a, a.slots[e], bad);
        const int nt = tiles_of<ROWS>(v.y);
        a.entry[e] = make_int4(at, v.x, v.y, nt);
        at += length_of(a, nt);
      }
      if (tid == 0) a.entry[a.n] = make_int4(total, -1, 0, 0);
      if (bad && a.status) atomicOr(a.status, bad);
    }
    if (!stretch()) return false;
    if (x0 >= (long long)before * a.U && x0 < (long long)(before + mine) * a.U) {        // one thread
      for (int e = e0; e < e1; ++e) {
        const int len = length_of(a, tiles_of<ROWS>(read_entry(a, a.slots[e], bad).y));
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
  const int unit = length_of(a, p.nt);
  p.u = (int)min(rel < (1LL << 31) ? (long long)((unsigned)rel / (unsigned)unit) : rel / unit, (long long)a.U - 1);
  const int o = (int)(rel - (long long)p.u * unit);
  // the first tile that begins at or after x0
  p.t = o <= 0 ? 0 : p.nt <= a.whole() ? p.nt : max(1, o - a.share());
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
template <int ROWS, int NT, typename A>
__device__ __forceinline__ bool locate(const A& a, Place& p, int& end, Held& held, int* scan, Found& found /* shared */) {
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
template <typename A> __device__ __forceinline__ int segment_end(const A& a, const Place& p, int end) {
  return p.nt <= a.whole() ? p.nt : min(p.nt, max(end - p.pos - a.share(), 1));
}

// The CTA's result of a segment, the sum of NBUF buffers [cols][ld] in shared memory, leaves for the output (a whole unit) or the
// scratch of pieces.  L, M: per column in shared memory.
template <typename T, int NT, int NBUF, typename A>
__device__ __forceinline__ void write_segment(const A& a, const float* buf, int ld, int buf_stride, const float* M, const float* L,
                                              int e, int u, int nh, bool whole, int piece) {
  const int tid = threadIdx.x, d4 = a.d_v / 4;
  if (!index_ok(e, a.n, a.status) || !index_ok(u, a.U, a.status) || !(whole || index_ok(piece, 2LL * a.ctas, a.status))) return;
  const int kvh = u / a.nhb, hb = u - kvh * a.nhb;
  T* const all = static_cast<T*>(a.out);
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
      T* out = all + a.out_row(e, kvh, hb * a.gb + h) * a.d_v + c;
      if (sizeof(T) == 4) *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(r);
      else *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(r);
    } else {
      *reinterpret_cast<float4*>(part + h * a.d_v + c) = o;
    }
  }
  if (tid < nh && (!whole || a.keep_ml))
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
// second launch: joins the pieces of cut units, zeroes the outputs of empty sequences
// ---------------------------------------------------------------------------------------------------------------
constexpr int JNT = 256;

struct Pieces { int np, c0; };                     // pieces of a unit; np <= 1: done whole
template <typename A> __device__ __forceinline__ Pieces pieces_of(const A& a, int u, int before, int total, int nt) {
  Pieces p;
  const long long W = (long long)total * a.U, x = (long long)before * a.U + (long long)u * length_of(a, nt);
  const int active = active_ctas(a, W);
  p.c0 = owner_of(x, W, active);
  p.np = owner_of(x + begin_of(a, nt - 1, nt), W, active) - p.c0 + 1;
  return p;
}
__device__ __forceinline__ int piece_at(const Pieces& p, int k) { return 2 * (p.c0 + k) + (k == 0); }

// CTA `id` of `joins`, line: the line's length.  The outputs go either by query head (a CTA
// each: the shorter way to the pieces), or, where there are many heads, by the borders between the stretches of the first
// launch: the unit that a border cuts is joined by the CTAs of the borders that cut it, which take its heads in turn, so
// that no more CTAs than borders are started however many units there are.  (By heads against by borders: one sequence
// of 5124 rows, 32 heads 11.9 / 12.9 us a call; 16 of up to 6000 rows, 512 heads 41.9 / 43.7; 24, 768 heads 55.8 / 57.3; 48 of up
// to 400 rows, 1536 heads 24.6 / 23.3, 20 of them, 640 heads 13.9 / 14.2.)
//
// This kernel lets the next one start only when it ends: blocks of the split kernel that start beside blocks of this
// one get the registers in between them, and once these end the rest of an SM's registers is in pieces too small for
// the third block, which then waits for a whole stretch to end (16 long sequences: 366 instead of 332 us a call).
struct JoinShared { float acc_s[JNT / 32][256]; float red_m[JNT / 32], red_l[JNT / 32]; int s_e; };
template <typename T, typename A>
__device__ __forceinline__ void join_outputs(const A& a, int id, int joins, int by_heads, int line, JoinShared& sh) {
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  auto& acc_s = sh.acc_s;
  auto& red_m = sh.red_m;
  auto& red_l = sh.red_l;
  auto& s_e = sh.s_e;
  int e, u, nt, col0, step;
  Pieces p;
  const auto zero = [&](long long row, int rows) {                       // outputs of a sequence without rows
    T* out = static_cast<T*>(a.out) + row * a.d_v;
    for (long long x = tid; x < (long long)rows * a.d_v; x += JNT) out[x] = from_f32<T>(0.f);
  };
  if (by_heads) {
    e = id / a.rows_seq;
    const int head = id - e * a.rows_seq, kvh = head / a.g, x = head - kvh * a.g, hb = x / a.gb;
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
      if (a.entry[i].w == 0) zero((long long)i * a.rows_seq, a.rows_seq);
    const long long W = (long long)line * a.U;
    const int active = active_ctas(a, W), c = id + 1;
    if (c >= active) return;
    const long long x = stretch_begin(W, active, c);
    __syncthreads();
    for (int i = tid; i < a.n; i += JNT) {                               // one thread has it
      const int4 at = a.entry[i];
      if ((long long)at.x * a.U <= x && x < (long long)(at.x + length_of(a, at.w)) * a.U) s_e = i;
    }
    __syncthreads();
    e = s_e;
    if (e < 0) return;                                                   // (only if the lengths change during the call)
    const int4 at = a.entry[e];
    const int before = at.x, unit = length_of(a, at.w);
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
    T* out = static_cast<T*>(a.out) + a.out_row(e, kvh, hb * a.gb + col) * a.d_v;
    for (int x2 = tid; x2 < a.d_v; x2 += JNT) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < JNT / 32; ++k) s = fmaf(acc_s[k][x2], f_w[k], s);
      out[x2] = from_f32<T>(s * inv);
    }
  }
}

}  // namespace paged
}  // namespace snap
