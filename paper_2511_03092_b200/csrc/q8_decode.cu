// Attention of the last tokens of each sequence over a cache in pages of 8-bit numbers (snap_paged_q8_decode_attn).
//
//     out[i][u][h] = sum_r p_r s'_r V_r / sum_r p_r,   p_r = exp(scale s_r q.K_r - max),   r < len - q_len + 1 + u
//
// with K_r, V_r the codes of row r and s_r, s'_r the scales of its block.  A row that is read serves all columns of a unit at once: the
// group's query heads, of each token, up to 16 (heads wider than 128 dims: 8); of more columns every 16 read the rows again and convert them
// again.  How the work is divided and joined: paged_line.cuh.
//
// A warp's tile is 32 rows, S^T = K tile . Q^T and O^T += V tile^T . P^T with m16n8k16 on half-precision numbers, the columns on
// the N side: a code is one exactly, and converting two takes one instruction.  (Products of 8-bit numbers, m16n8k32, with queries and weights
// split in two such numbers, take longer: four tokens a step 112 us where one half-precision number took 60.)  The order of the inner dims of a product is free, so codes are used as ldmatrix delivers them: four
// neighbouring dims of a key row are positions 2t, 2t + 1, 2t + 8, 2t + 9 of a step of 16, and the queries are read in that order;
// four rows of a value dim, transposed by bytes, are those positions as well, the rows being addressed in the order that
// movmatrix leaves of the weights.
//
// Queries are brought to a largest number of 2^14 to 2^15 by a power of two, which leaves a bf16 query exact down to 2^-29 of its
// largest number (cut off 2^-39 below it); single-precision ones enter as two such numbers.  The scale of a key row multiplies its logits, that
// of a value row its weight.  The products of weight and scale are brought to the range of half precision by a power of two per column, which is
// taken off again when a tile's outputs are added to the sums: these are of single precision, in the numbers' own size, so that no tile
// depends on what another one held.  The power moves when a tile's largest product leaves [1, 2^15], the reference of the exponentials when
// one passes 2^15 or weights pass 2^6.  A tile whose value scales lie more than 2^6 apart (a block keeps the scale of a row that was given up)
// goes through several times, the rows of the largest scales first.  (Sums held on the columns' powers, which lose the rows of smaller scales:
// calls of all kinds 0.8 % less, 16 long sequences 181 us instead of 188, four tokens a step 58.6 instead of 61.4.  A loop around a tile's rounds
// instead of a second way through the loop over tiles: 4 % more.)
//
// A weight is two half-precision numbers, 21 bits; what lies far below the tile's largest rounds to multiples of 2^-24 of it (of 2^-36 where the
// second numbers are summed apart, times 2^11: single precision, and two heads side by side).  One number of 11 bits, an eighth of a bf16
// output's own rounding, puts one output in 30 on the other side of a border between two bf16 numbers.  The second costs 3 % where a side's spare
// columns take it (185 -> 190 us), else 2 to 9 %, 14 % with sixteen columns (63 -> 72 us).
//
// Where a row's heads lie side by side (pages stored rows first), two warps of a CTA take one head and two the next, over the same rows: HBM
// then delivers twice as much in a row (128-byte heads, 16 long sequences, with sums on the columns' powers: 208 us without, 172 with; heads first 168).
//
// What bounds it: 16 sequences of 8192 to 65536 rows, 32 heads on 8 of 128 dims, HBM (1.04 GB 179 us, 89 % of the copy rate); four tokens a step (16
// columns), some 950 instructions per tile and warp, which wait for one another's results, two warps to a scheduler: 8 sequences of 9000 to 16384 rows
// 72 us; small calls, the chain of look-up, first tiles, exchange and join, in two launches: one sequence of 5124 rows 12.1 us, 45 of up to 333 16.
// (The two sides at the shares, the CTAs per SM and the columns of a unit below were measured with weights of one number.)
#include <type_traits>

#include "e4m3.cuh"
#include "paged_line.cuh"

namespace snap {
namespace {

using namespace mmasync;
using namespace paged;
using umma::mbar_expect_tx;
using umma::mbar_init;
using umma::smem_u32;

constexpr int TR = 32;                          // rows of a tile, a lane each
constexpr float NOTHING = -3.402823466e38f;     // the reference of a column that has seen no row: every logit lies far above it
// What a unit costs besides its tiles, in tiles; units of at most WHOLE tiles stay whole, since a call that cuts none has nothing to join.
// (48 calls of 1 to 100 sequences of up to 20000 rows: 6 and 6 take 7 % longer, 4 and 6 4 %, 4 and 8 4 %, 3 and 12 2 %, 6 and 12 2 %, 4 and
// 24 0.5 %; 45 sequences of up to 333 rows, 8 KV heads of 128 dims 16.2 us, with 6 and 6 22.1.)
constexpr int SHARE = 4, WHOLE = 12;
constexpr int LOOK = 2;                         // tiles whose pages are looked up ahead of their copies

// n / d for 0 <= n < 2^31 by a multiplication: division by invariant integers (Granlund and Montgomery, 1994), with a reciprocal rounded up.
// With L = ceil(log2 d) and m = floor(2^(31 + L) / d) + 1 (below 2^32, as d > 2^(L - 1)), d m = 2^(31 + L) + e with 0 < e <= d <= 2^L, so
// n m / 2^(31 + L) = n / d + n e / (d 2^(31 + L)) lies less than 1 / d above n / d and has the same whole part.
struct Divisor {
  uint32_t m; int L;
  __device__ __forceinline__ int quotient(int n) const { return (int)(__umulhi(2u * (uint32_t)n, m) >> L); }
};
Divisor divisor(uint32_t d) {
  int L = 0;
  while (L < 31 && (1u << L) < d) ++L;
  return {(uint32_t)((1ull << (31 + L)) / d + 1), L};
}

struct Q8Args : LineArgs {
  const void* q;
  const uint8_t* kp; const uint8_t* vp; const float* ks; const float* vs;
  int Hq, q_len, gq, gc, d_qk;                  // gq query heads of a KV head, gc = gq * q_len columns
  int heads, sc;                                // KV heads of a unit, a side each; columns of a side
  float scale_log2;
  Divisor by_page, by_block, by_gq, by_gc, by_nhb;
  int blocks;                                   // scales of a page and KV head
  int box;                                      // rows of a copy, 0: rows are copied by the lanes
  __device__ __forceinline__ constexpr int share() const { return SHARE; }
  __device__ __forceinline__ constexpr int whole() const { return WHOLE; }
  __device__ __forceinline__ long long out_row(int e, int k, int x) const {
    const int h = heads > 1 ? by_gc.quotient(x) : 0, y = x - h * gc, u = by_gq.quotient(y);
    return ((long long)e * q_len + u) * Hq + (k * heads + h) * gq + (y - u * gq);
  }
  __device__ __forceinline__ int token_of(int x) const { return by_gq.quotient(heads > 1 ? x - by_gc.quotient(x) * gc : x); }
};

template <int D, int NWARP, int NSTAGE, int NG, int SIDES> struct Q8Shape {
  static constexpr int NT = NWARP * 32, KS = D / 16, NCOL = 8 * NG;      // columns of a unit, of both sides together
  static constexpr int SW = D < 128 ? D : 128, NSL = D / SW;             // bytes of a slab's rows; slabs
  static constexpr int SLAB_B = TR * SW, TENS_B = NSL * SLAB_B, STAGE_B = 2 * TENS_B;
  // column stride of the exchange buffers: fragments store without bank conflicts; as many buffers as leave room for the CTAs of an SM
  static constexpr int LD = D + 4, NBUF = SIDES == 1 && D * NG <= 128 ? NWARP / 2 : 1;
  static constexpr size_t stages_b = (size_t)NWARP * NSTAGE * STAGE_B;
  static constexpr size_t rows_b = (size_t)NWARP * NSTAGE * 2 * TR * sizeof(float);     // the rows' scales
  static constexpr size_t bars_b = NWARP * NSTAGE * 8;
  static constexpr size_t smem = 1024 + stages_b + rows_b + bars_b +
                                 (size_t)(NBUF * NCOL * LD + 2 * NWARP * NCOL + 2 * NCOL) * sizeof(float);
};

// byte offset of row r, 16-byte chunk c inside a slab swizzled as the copies do it
template <int SW> __device__ __forceinline__ uint32_t swizzled(int r, int c) {
  return SW == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)) : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same on a sum of zero
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Two 16 x 16 matrices of bytes, transposed: lane (g, t) gets rows 4 t .. 4 t + 3 of columns g and g + 8 of each
__device__ __forceinline__ void ldsm_bytes_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// x as two half-precision numbers: what rounding leaves of it, times `by`
__device__ __forceinline__ uint32_t rest_f16(float lo, float hi, uint32_t rounded, float by = 1.f) {
  const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&rounded));
  return pack_f16((lo - r.x) * by, (hi - r.y) * by);
}
// Of four codes, a one for each that is a NaN, in the lowest bit of its byte
__device__ __forceinline__ uint32_t nan_codes(uint32_t four) { return ((four & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u; }
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }
__device__ __forceinline__ float one_over(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }   // x a power of two from 2^-126 to 2^126
__device__ __forceinline__ float power_of(int e) { return exp2_of(min(max(e, -126), 127)); }

// How a tile comes in: through the tensor maps, heads of exactly D dims (EXACT) or fewer; or, where a page is no multiple of
// 8 rows, copied by the lanes in 16-byte pieces (ROWS).
enum class Tiles { EXACT, BOXES, ROWS };
template <typename T, int D, int NWARP, int NSTAGE, int NG, int SIDES, int CTAS, Tiles MODE>
__global__ void __launch_bounds__(NWARP * 32, CTAS)
q8_mma_kernel(const __grid_constant__ Q8Args a, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v) {
  using S = Q8Shape<D, NWARP, NSTAGE, NG, SIDES>;
  constexpr bool F32 = sizeof(T) == 4, EXACT = MODE == Tiles::EXACT, BY_ROWS = MODE == Tiles::ROWS;
  constexpr int KS = S::KS, NCOL = S::NCOL, WPS = NWARP / SIDES, LD = S::LD, SW = S::SW, PARTS = F32 ? 2 : 1, MT = TR / 16;
  // Weights times scales, by column: a tile's largest one is brought to 2^TARGET or more, and again when a later tile's leaves [LEAST, LIMIT]; value
  // scales that lie further than 2^NEAR apart do not meet.
  constexpr float LEAST = 1.f, LIMIT = 32768.f;
  constexpr int TARGET = 9, NEAR = 6;
  // A weight is two half-precision numbers.  Where a side has four columns at most, its other four are the same ones over again, and take the second
  // numbers; else the values are multiplied twice.
  constexpr bool PAIR = SIDES == 2;
  constexpr int NUM = PAIR ? 1 : 2;                                      // products of a tile's values
  constexpr float REST = 2048.f;                                         // where a second number is summed apart: times this, it has the first one's range
  constexpr unsigned ALL = NG == 1 ? 0xffu : 0xffffu;                    // a bit for each of the warp's columns
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  float* row_scales = reinterpret_cast<float*>(stages + S::stages_b);    // [NWARP][NSTAGE][keys, values][TR]
  uint64_t* bars = reinterpret_cast<uint64_t*>(row_scales + S::rows_b / sizeof(float));
  float* buf = reinterpret_cast<float*>(bars + NWARP * NSTAGE);          // [NBUF][NCOL][LD]
  float* wm = buf + S::NBUF * NCOL * LD;                                 // [NWARP][NCOL] references, then sums
  float* wl = wm + NWARP * NCOL;
  float* jm = wl + NWARP * NCOL;                                         // [NCOL] joined maxima, then sums
  float* jl = jm + NCOL;
  __shared__ int scan[S::NT / 32 + 2];
  __shared__ Held held;
  __shared__ Found found;
  __shared__ int some_nan;                                               // a NaN among a segment's values that not every column sees

  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, gq = lane >> 2, tq = lane & 3, side = w % SIDES, ws = w / SIDES;
  unsigned char* wstages = stages + w * NSTAGE * S::STAGE_B;
  float* wscales = row_scales + w * NSTAGE * 2 * TR;
  const uint32_t stage0 = smem_u32(wstages), scale0 = smem_u32(wscales), bar0 = smem_u32(bars + w * NSTAGE);
  if (tid == 0) some_nan = 0;
  if (lane == 0) {
    for (int s = 0; s < NSTAGE; ++s) mbar_init(bar0 + 8 * s, BY_ROWS ? 32 : 33);
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
  const int d_qk = EXACT ? D : a.d_qk, d_v = EXACT ? D : a.d_v;

  // ---- the warp's producer: NSTAGE tiles ahead of the consumer, over unit borders; of a side's WPS warps the ws-th takes the CTA's
  // tiles ws, ws + WPS, ...; lane l looks up the page of the tile's row l ----
  const auto head_of = [&](int u) { return SIDES == 1 ? a.by_nhb.quotient(u) : 2 * u + side; };
  Place pr = at;
  int pr_stop = segment_end(a, pr, end), pr_head = head_of(pr.u);           // the CTA's tiles of pr's unit end there
  const int* pr_table = a.map.table + (long long)max(pr.slot, 0) * a.map.max_pages;
  bool more = true;
  const auto settle = [&]() {                                            // pr.t may have passed its unit's tiles: the unit that has it
    while (pr.t >= pr_stop) {
      if (pr_stop < pr.nt) { more = false; return; }
      pr.t -= pr.nt;
      next_unit<TR>(a, held, pr);
      if (pr.e >= a.n || pr.pos >= end) { more = false; return; }
      pr_stop = segment_end(a, pr, end);
      pr_head = head_of(pr.u);
      pr_table = a.map.table + (long long)pr.slot * a.map.max_pages;
    }
  };
  pr.t += ws;
  settle();
  struct Look { int page, off, kvh; bool tile; };                        // off: row of the page, -1 no row
  const auto look_up = [&]() {                                           // (nothing waits here for what the table says)
    Look r = {-1, -1, pr_head, more};
    const int row = pr.t * TR + lane;
    if (more && row < pr.len) {
      const int pg = a.by_page.quotient(row);
      r.off = row - pg * a.map.page;
      if (index_ok(pg, a.map.max_pages, a.status)) r.page = pr_table[pg];
    }
    pr.t += WPS;
    if (pr.t >= pr_stop && more) settle();
    return r;
  };
  // B fragments of Q^T, column 8 gi + gq, dims 16 ks + 4 tq .. + 3; of single precision the rounded number, then what it leaves
  const T* q_all = static_cast<const T*>(a.q);
  uint32_t qb[NG][KS][PARTS][2];
  float q_scale[NG][2];                                                  // of this thread's two columns of the logits
  using Four = std::conditional_t<F32, uint4, uint2>;                    // four numbers' bits
  const auto load_q = [&]() {                                            // the numbers themselves, to begin with
    const int k = a.by_nhb.quotient(at.u), hb = at.u - k * a.nhb, x0 = hb * a.gb + side * a.sc, nh = min(a.sc, a.g - x0);
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      const int col = PAIR ? gq & 3 : 8 * gi + gq;
      const T* qp = q_all + a.out_row(at.e, k, col < nh ? x0 + col : 0) * d_qk + 4 * tq;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Four v = {};
        if (col < nh && (EXACT || 16 * ks < d_qk)) v = *reinterpret_cast<const Four*>(qp + 16 * ks);
        qb[gi][ks][0][0] = v.x; qb[gi][ks][0][1] = v.y;
        if constexpr (F32) { qb[gi][ks][PARTS - 1][0] = v.z; qb[gi][ks][PARTS - 1][1] = v.w; }
      }
    }
  };
  const auto make_q = [&]() {
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      float x[KS][4], big = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          x[ks][c] = __uint_as_float(F32 ? qb[gi][ks][F32 ? c / 2 : 0][c % 2] : c % 2 ? qb[gi][ks][0][c / 2] & 0xffff0000u : qb[gi][ks][0][c / 2] << 16);
#pragma unroll
        for (int c = 0; c < 4; ++c) big = fmaxf(big, fabsf(x[ks][c]));
      }
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
      // 2^up in two factors: a query of subnormal numbers needs more than one can hold
      const int up = 14 - exponent_of(big);
      const float f0 = power_of(up / 2), f1 = power_of(up - up / 2);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float lo = x[ks][2 * c] * f0 * f1, hi = x[ks][2 * c + 1] * f0 * f1;
          qb[gi][ks][0][c] = pack_f16(lo, hi);
          if constexpr (F32) qb[gi][ks][PARTS - 1][c] = rest_f16(lo, hi, qb[gi][ks][0][c]);
        }
      const float back = a.scale_log2 * power_of(-(up / 2)) * power_of(up / 2 - up);
#pragma unroll
      for (int c = 0; c < 2; ++c) q_scale[gi][c] = __shfl_sync(0xffffffffu, back, (2 * tq + c) * 4);
    }
  };
  // A step: the copy of the tile looked up LOOK steps before, the look-up of another.  (The steps before the first copy are no
  // code of their own: a call of short sequences runs through the kernel about once, at the speed at which instructions arrive.)
  const int page_scales = a.Hkv * a.blocks;
  const unsigned copy_b = (unsigned)(((d_qk + SW - 1) / SW + (d_v + SW - 1) / SW) * a.box * SW);
  int n_issued = 0, steps = 0;
  unsigned there_of[NSTAGE];                                             // of each stage, the rows that are there
#pragma unroll
  for (int s = 0; s < NSTAGE; ++s) there_of[s] = 0;
  Look look[LOOK];
#pragma unroll
  for (int x = 0; x < LOOK; ++x) look[x] = {-1, -1, 0, false};
  const auto step = [&]() {
    const int s = n_issued % NSTAGE;
    const Look l = look[0];
#pragma unroll
    for (int x = 0; x + 1 < LOOK; ++x) look[x] = look[x + 1];
    look[LOOK - 1] = look_up();
    ++steps;
    if (!l.tile) return;
    const bool okay = l.off >= 0 && (unsigned)l.page < (unsigned)a.map.n_pages;
    const unsigned rows = __ballot_sync(0xffffffffu, okay);
#pragma unroll
    for (int y = 0; y < NSTAGE; ++y) there_of[y] = y == s ? rows : there_of[y];
    const uint32_t dst = stage0 + s * S::STAGE_B, bar = bar0 + 8 * s, sc = scale0 + (s * 2 * TR + lane) * 4;
    if (okay) {
      const long long x = (long long)l.page * page_scales + (l.kvh * a.blocks + a.by_block.quotient(l.off));
      cp_async4(sc, a.ks + x);
      cp_async4(sc + TR * 4, a.vs + x);
    } else {
      wscales[s * 2 * TR + lane] = 0.f;
      wscales[s * 2 * TR + TR + lane] = 0.f;
      if (l.off >= 0 && a.status) atomicOr(a.status, SNAP_DEV_BAD_PAGE);
    }
    if constexpr (BY_ROWS) {
      const long long k_off = l.page * a.map.kp + l.kvh * a.map.kh + l.off * a.map.kr, v_off = l.page * a.map.vp + l.kvh * a.map.vh + l.off * a.map.vr;
      constexpr int CPR = D / 16;                                        // lanes to a row
#pragma unroll
      for (int x0 = 0; x0 < TR * CPR; x0 += 32) {
        const int r = (x0 + lane) / CPR, c = (x0 + lane) % CPR;
        const long long ko = __shfl_sync(0xffffffffu, k_off, r), vo = __shfl_sync(0xffffffffu, v_off, r);
        const uint32_t to = dst + c / (SW / 16) * S::SLAB_B + swizzled<SW>(r, c % (SW / 16));
        if ((rows >> r) & 1u) {
          // (a step of products is 32 dims: zeros behind a head of an odd number of 16)
          if (16 * c < d_qk + 16) cp_async16(to, a.kp + ko + (16 * c < d_qk ? 16 * c : 0), 16 * c < d_qk ? 16 : 0);
          if (16 * c < d_v) cp_async16(to + S::TENS_B, a.vp + vo + 16 * c, 16);
        }
      }
    } else {
      const bool first = okay && (lane & (a.box - 1)) == 0;              // of a copy's rows
      const unsigned copies = __ballot_sync(0xffffffffu, first);
      if (lane == 0) mbar_expect_tx(bar, __popc(copies) * copy_b);
      if (first) {
#pragma unroll
        for (int h = 0; h < S::NSL; ++h) {
          if (SW * h < d_qk) tma_load_4d(dst + h * S::SLAB_B + lane * SW, &tmap_k, SW * h, l.off, l.kvh, l.page, bar);
          if (SW * h < d_v) tma_load_4d(dst + S::TENS_B + h * S::SLAB_B + lane * SW, &tmap_v, SW * h, l.off, l.kvh, l.page, bar);
        }
      }
    }
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
    ++n_issued;
  };
  // ldmatrix lane roles.  Keys: row (lane & 7) + 8 * bit3, chunk + bit4; values, by bytes: row 4 t + j of 16 is row 2 t + j % 2 + 8 (j / 2) of the tile's
  const int l_row = (lane & 7) + ((lane >> 3) & 1) * 8, l_cadd = lane >> 4;
  const int b_row = (lane & 16) + ((lane >> 1) & 6) + (lane & 1) + (lane & 2) * 4;
  const uint32_t l_at = stage0 + swizzled<SW>(l_row, l_cadd), b_at = stage0 + S::TENS_B + swizzled<SW>(b_row, 0);   // (other chunks: exclusive or)

  bool dead = false;                                                     // a bounded wait ran out: nothing more is read
  int n = 0, done = 0;                                                   // tiles done by this warp; by the CTA before this segment
  while (true) {
    // ---- a segment: the CTA's tiles [at.t, tb) of one unit ----
    const int tb = segment_end(a, at, end), cnt = tb - at.t;
    const int hb = at.u - a.by_nhb.quotient(at.u) * a.nhb, nh = min(a.gb, a.g - hb * a.gb);
    const bool whole = cnt == at.nt;
    const int all_see = at.len - a.q_len + 1;                            // rows that every column sees
    // O^T: dims 16 db + gq (+ 8: the upper two), columns 8 gi + 2 tq (+ 1)
    float oacc[NG][KS][4];
    // per column: reference of the exponentials, sum of the weights, the power of two on a tile's products of weight and scale
    float ref[NG][2], l_part[NG][2], f[NG][2];
    // value scales from lowest to highest may meet; no power of two above `most`, which none of them turns into an infinity
    float lowest = INFINITY, highest = 0.f, most = 1.f;
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
      for (int c = 0; c < 2; ++c) { ref[gi][c] = NOTHING; l_part[gi][c] = 0.f; f[gi][c] = 1.f; }
#pragma unroll
      for (int db = 0; db < KS; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x) oacc[gi][db][x] = 0.f;
    }

    load_q();                                                            // on its way while the first copies are looked up
    bool fresh = true;
    unsigned rest = 0;                                                   // rows of the tile at hand that are left for another round
    for (;; n += rest == 0) {
      while (steps < LOOK || (look[0].tile && n_issued < n + NSTAGE)) step();
      if (fresh) make_q();
      if (ws + n * WPS >= done + cnt || dead) break;
      const int s = n % NSTAGE;
      const bool landed = wait_bounded(bar0 + 8 * s, (unsigned)(n / NSTAGE) & 1u);
      if (__any_sync(0xffffffffu, !landed)) { dead = true; break; }
      const int row0 = (at.t + (ws + n * WPS - done)) * TR;
      unsigned rows = there_of[0];
#pragma unroll
      for (int y = 1; y < NSTAGE; ++y) rows = y == s ? there_of[y] : rows;
      const uint32_t l_K = l_at + s * S::STAGE_B, b_V = b_at + s * S::STAGE_B;
      if (rows != 0xffffffffu || row0 + TR > all_see) {
        // Rows past the end, or on a bad page, may hold anything, and a zero weight does not silence a NaN in V: clear them.  Of a row that only
        // some columns see a NaN becomes a code of zero; those columns get theirs at the segment's end.
        constexpr int CPR = D / 16;
        const int from = min(rows != 0xffffffffu ? __ffs(~rows) - 1 : TR, max(all_see - row0, 0));
#pragma unroll 1
        for (int x = from * CPR + lane; x < TR * CPR; x += 32) {
          const int r = x / CPR, c = x % CPR;
          if (((rows >> r) & 1u) && row0 + r < all_see) continue;
          uint4* at = reinterpret_cast<uint4*>(wstages + s * S::STAGE_B + S::TENS_B + c / (SW / 16) * S::SLAB_B + swizzled<SW>(r, c % (SW / 16)));
          uint4 w = make_uint4(0, 0, 0, 0);
          if ((rows >> r) & 1u) {
            w = *at;
            const uint4 n = make_uint4(nan_codes(w.x), nan_codes(w.y), nan_codes(w.z), nan_codes(w.w));
            if (!(n.x | n.y | n.z | n.w)) continue;
            w = make_uint4(w.x & ~(n.x * 255u), w.y & ~(n.y * 255u), w.z & ~(n.z * 255u), w.w & ~(n.w * 255u));
            some_nan = 1;
          }
          *at = w;
        }
        __syncwarp();
      }
      // ---- S^T = K tile . Q^T ----
      float v[MT][NG][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int x = 0; x < 4; ++x) v[mt][gi][x] = 0.f;
#pragma unroll
      for (int k2 = 0; k2 < KS / 2; ++k2) {                              // 32 dims
        if (!EXACT && 32 * k2 >= d_qk) break;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t c[4];
          ldsm4((l_K ^ (k2 * 2 % (SW / 16) << 4)) + k2 * 32 / SW * S::SLAB_B + 16 * mt * SW, c);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!EXACT && 32 * k2 + 16 * h >= d_qk) break;
            const uint32_t a0 = halves_of_codes(c[2 * h] & 0xffffu), a2 = halves_of_codes(c[2 * h] >> 16);
            const uint32_t a1 = halves_of_codes(c[2 * h + 1] & 0xffffu), a3 = halves_of_codes(c[2 * h + 1] >> 16);
#pragma unroll
            for (int gi = 0; gi < NG; ++gi)
#pragma unroll
              for (int y = PARTS - 1; y >= 0; --y) mma_f16(v[mt][gi], a0, a1, a2, a3, qb[gi][2 * k2 + h][y][0], qb[gi][2 * k2 + h][y][1]);
          }
        }
      }
      // ---- logits; rows that are not there, or that a column does not see ----
      const auto row_of = [&](int mt, int r8) { return 16 * mt + 8 * r8 + gq; };
      const float* sc = wscales + s * 2 * TR;
      if (rest) rows = rest;
      rest = 0;
      float v_scale[MT][2];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r8 = 0; r8 < 2; ++r8) v_scale[mt][r8] = sc[TR + row_of(mt, r8)];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r8 = 0; r8 < 2; ++r8) {
          const float k_scale = sc[row_of(mt, r8)];
#pragma unroll
          for (int gi = 0; gi < NG; ++gi)
#pragma unroll
            for (int c = 0; c < 2; ++c) v[mt][gi][2 * r8 + c] *= fminf(q_scale[gi][c] * k_scale, -NOTHING);   // (0 times infinity is no logit)
        }
      if (rows != 0xffffffffu || row0 + TR > all_see) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int r8 = 0; r8 < 2; ++r8)
            if (!((rows >> row_of(mt, r8)) & 1u)) v_scale[mt][r8] = lowest;  // (it meets a weight of zero)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int c = 0; c < 2; ++c) {                                  // (a column that is not there may see anything)
            const int sees = all_see + (a.q_len > 1 ? a.token_of(hb * a.gb + side * a.sc + (PAIR ? 2 * (tq & 1) : 8 * gi + 2 * tq) + c) : 0) - row0;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int r8 = 0; r8 < 2; ++r8)
                if (!(((rows >> row_of(mt, r8)) & 1u) && row_of(mt, r8) < sees)) v[mt][gi][2 * r8 + c] = -INFINITY;
          }
      }
      // ---- weights, and weights times scales: in range with the reference and the power as they are? ----
      float p[MT][NG][4], add[NG][2];
#pragma unroll 1
      for (int pass = 0;; ++pass) {                                      // (a unit's first tile has no reference yet)
        float largest = 0.f;
        unsigned good = 0;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) add[gi][0] = add[gi][1] = 0.f;
        if (!fresh || pass > 0) {
#pragma unroll
          for (int gi = 0; gi < NG; ++gi)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float big = 0.f;
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r8 = 0; r8 < 2; ++r8) {
                  const float e = fast_exp2(v[mt][gi][2 * r8 + c] - ref[gi][c]);
                  add[gi][c] += e;
                  p[mt][gi][2 * r8 + c] = e * (v_scale[mt][r8] * f[gi][c]);
                  big = fmaxf(big, p[mt][gi][2 * r8 + c]);
                }
              good |= (unsigned)(big >= LEAST) << (2 * gi + c);
              largest = fmaxf(largest, big);
            }
        }
        if (pass > 0) break;
        // (weights of 2^6 above the reference are a reason as well, however small the scales they meet: sums have to stay within single precision)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi) largest = fmaxf(largest, (add[gi][0] + add[gi][1]) * 512.f);
        const float least = fminf(fminf(v_scale[0][0], v_scale[0][1]), fminf(v_scale[1][0], v_scale[1][1]));
        const float greatest = fmaxf(fmaxf(v_scale[0][0], v_scale[0][1]), fmaxf(v_scale[1][0], v_scale[1][1]));
        const bool near = least >= lowest && greatest <= highest;
        const unsigned said = __reduce_or_sync(0xffffffffu, good << (2 * NG * tq) | (unsigned)(largest > LIMIT) << 31 | (unsigned)!near << 30);
        if (said == ALL) break;
        if (!(said >> 30)) {
          // some columns lie below the range: their power moves, and nothing else
#pragma unroll
          for (int gi = 0; gi < NG; ++gi)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float big = 0.f;
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) big = fmaxf(big, fmaxf(p[mt][gi][c], p[mt][gi][2 + c]));
#pragma unroll
              for (int o = 4; o <= 16; o <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
              if (((said >> (2 * NG * tq + 2 * gi + c)) & 1u) || big == 0.f) continue;
              const int was = exponent_of(f[gi][c]), now = min(min(was + TARGET - exponent_of(big), was + 127), exponent_of(most));
              const float by = exp2_of(now - was);
              f[gi][c] = exp2_of(now);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) { p[mt][gi][c] *= by; p[mt][gi][2 + c] *= by; }
            }
          break;
        }
        fresh = false;
        if ((said >> 30) & 1u) {
          // lane r has row r: those whose scale lies within 2^NEAR below the largest are taken in now, the others in another round
          const bool left = (rows >> lane) & 1u;
          const unsigned power = left ? __float_as_uint(sc[TR + lane]) >> 23 : 0u, top = __reduce_max_sync(0xffffffffu, power);
          const unsigned now = __ballot_sync(0xffffffffu, left && power + NEAR >= top);
          lowest = __uint_as_float((unsigned)max((int)top - NEAR / 2 - 1, 0) << 23);
          highest = __uint_as_float(min(top + NEAR / 2 - 1, 254u) << 23 | 0x7fffffu);
          most = exp2_of(min(126, 247 - (int)min(top + NEAR / 2 - 1, 254u)));
          rest = rows & ~now;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r8 = 0; r8 < 2; ++r8)
              if (!((now >> row_of(mt, r8)) & 1u)) {
                v_scale[mt][r8] = 0.f;
#pragma unroll
                for (int gi = 0; gi < NG; ++gi) v[mt][gi][2 * r8] = v[mt][gi][2 * r8 + 1] = -INFINITY;
              }
        }
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float mx = -INFINITY, big = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int r8 = 0; r8 < 2; ++r8) {
                mx = fmaxf(mx, v[mt][gi][2 * r8 + c]);
                big = fmaxf(big, v[mt][gi][2 * r8 + c] + (float)exponent_of(v_scale[mt][r8]));
              }
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) {
              mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
              big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
            }
            const float to = fmaxf(ref[gi][c], mx), al = exp2f(ref[gi][c] - to);
            const int k = (int)fminf(fmaxf(TARGET - floorf(big - to), -126.f), 126.f);
            l_part[gi][c] *= al;
            ref[gi][c] = to;
            f[gi][c] = fminf(exp2_of(k), most);
#pragma unroll
            for (int db = 0; db < KS; ++db) { oacc[gi][db][c] *= al; oacc[gi][db][2 + c] *= al; }
          }
      }
#pragma unroll
      for (int gi = 0; gi < NG; ++gi) { l_part[gi][0] += add[gi][0]; l_part[gi][1] += add[gi][1]; }
      // ---- O^T += V tile^T . P^T, the power of two taken off again ----
      uint32_t pb[MT][NG][NUM][2];                                       // P^T as B operands: rows 16 mt + 2 tq, + 1, then + 8, + 9, of column 8 gi + gq
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int r8 = 0; r8 < 2; ++r8) {
            const float p0 = p[mt][gi][2 * r8], p1 = p[mt][gi][2 * r8 + 1];
            if constexpr (PAIR || F32) {
              const uint32_t hi = pack_f16(p0, p1), lo = rest_f16(p0, p1, hi, REST);
              pb[mt][gi][0][r8] = movmatrix_t(PAIR && tq >= 2 ? lo : hi);
              if constexpr (!PAIR) pb[mt][gi][NUM - 1][r8] = movmatrix_t(lo);
            } else {                                                     // cut, not rounded: what is cut off needs no conversion back
              const float h0 = __uint_as_float(__float_as_uint(p0) & 0xffffe000u), h1 = __uint_as_float(__float_as_uint(p1) & 0xffffe000u);
              pb[mt][gi][0][r8] = movmatrix_t(pack_f16(h0, h1));
              pb[mt][gi][NUM - 1][r8] = movmatrix_t(pack_f16(p0 - h0, p1 - h1));
            }
          }
#pragma unroll
      for (int db = 0; db < KS; ++db) {
        if (!EXACT && 16 * db >= d_v) break;
        uint32_t c[4];                                                   // dims gq and + 8, of the tile's first 16 rows, then of the others
        ldsm_bytes_t((b_V ^ (db % (SW / 16) << 4)) + db * 16 / SW * S::SLAB_B, c);
        constexpr int SUMS = NUM == 2 && F32 ? 2 : 1;
        float o[NG][SUMS][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const uint32_t a0 = halves_of_codes(c[2 * mt] & 0xffffu), a2 = halves_of_codes(c[2 * mt] >> 16);
          const uint32_t a1 = halves_of_codes(c[2 * mt + 1] & 0xffffu), a3 = halves_of_codes(c[2 * mt + 1] >> 16);
#pragma unroll
          for (int gi = 0; gi < NG; ++gi)
#pragma unroll
            for (int y = NUM - 1; y >= 0; --y) {
              if (mt == 0 && (SUMS == 2 || y == NUM - 1)) mma_f16_first(o[gi][SUMS == 2 ? y : 0], a0, a1, a2, a3, pb[mt][gi][y][0], pb[mt][gi][y][1]);
              else mma_f16(o[gi][SUMS == 2 ? y : 0], a0, a1, a2, a3, pb[mt][gi][y][0], pb[mt][gi][y][1]);
            }
        }
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float sum = SUMS == 2 ? fmaf(o[gi][SUMS - 1][x], 1.f / REST, o[gi][0][x]) : o[gi][0][x];
            oacc[gi][db][x] = fmaf(sum, one_over(f[gi][x & 1]), oacc[gi][db][x]);
          }
      }
      __syncwarp();
      // the stage was read, and possibly cleared, through the generic proxy; the copy that refills it is of the async proxy
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }

    // ---- join the warps: references first, then the outputs ----
#pragma unroll
    for (int gi = 0; gi < NG; ++gi)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int o = 4; o <= 16; o <<= 1) l_part[gi][c] += __shfl_xor_sync(0xffffffffu, l_part[gi][c], o);
        if (gq == 0) {
          wm[w * NCOL + 8 * gi + 2 * tq + c] = ref[gi][c];
          wl[w * NCOL + 8 * gi + 2 * tq + c] = l_part[gi][c];
        }
      }
    __syncthreads();
    const bool marked = some_nan != 0;
#pragma unroll
    for (int gi = 0; gi < NG; ++gi)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float M = -INFINITY;
#pragma unroll
        for (int ww = side; ww < NWARP; ww += SIDES) M = fmaxf(M, wm[ww * NCOL + 8 * gi + 2 * tq + c]);
        const float y = exp2f(ref[gi][c] - M);
#pragma unroll
        for (int db = 0; db < KS; ++db)
#pragma unroll
          for (int up = 0; up < 4; up += 2) {
            float& o = oacc[gi][db][up + c];
            if (PAIR) o = fmaf(__shfl_xor_sync(0xffffffffu, o, 2), 1.f / REST, o);
            o *= y;
          }
      }
    if (tid < NCOL) {
      const int of = SIDES > 1 && tid >= a.sc, col = tid - of * a.sc;    // its side, and the column there
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int ww = 0; ww < WPS; ++ww) M = fmaxf(M, wm[(ww * SIDES + of) * NCOL + col]);
#pragma unroll
      for (int ww = 0; ww < WPS; ++ww) {
        const float lw = wl[(ww * SIDES + of) * NCOL + col];
        L += lw == 0.f ? 0.f : lw * exp2f(wm[(ww * SIDES + of) * NCOL + col] - M);
      }
      jm[tid] = M; jl[tid] = L;
    }
    // the last warps leave their outputs in a buffer each, those before add theirs there, in turns
#pragma unroll 1
    for (int turn = WPS / S::NBUF - 1; turn >= 0; --turn) {
      if (ws / S::NBUF == turn) {
        const bool add = turn < WPS / S::NBUF - 1;
        float* b = buf + (ws % S::NBUF * NCOL + side * a.sc + 2 * tq) * LD + gq;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            if (SIDES > 1 && 2 * tq + c >= a.sc) continue;               // (the other side's)
            float* to = b + (8 * gi + c) * LD;
            if (add) {                                                   // (all loads before the first store, which they might wait for)
#pragma unroll
              for (int db = 0; db < KS; ++db) {
                oacc[gi][db][c] += to[16 * db];
                oacc[gi][db][2 + c] += to[16 * db + 8];
              }
            }
#pragma unroll
            for (int db = 0; db < KS; ++db) {
              to[16 * db] = oacc[gi][db][c];
              to[16 * db + 8] = oacc[gi][db][2 + c];
            }
          }
      }
      __syncthreads();
    }
    if (marked) {
      // the segment's rows that only later tokens see, looked at once more: a NaN goes to the columns that see it
#pragma unroll 1
      for (int r = max(all_see, at.t * TR); r < min(at.len, tb * TR); ++r) {
        const int pg = a.by_page.quotient(r), page = index_ok(pg, a.map.max_pages, a.status) ? a.map.table[(long long)at.slot * a.map.max_pages + pg] : -1;
        if (page < 0 || page >= a.map.n_pages) continue;
#pragma unroll 1
        for (int x = tid; x < nh * d_v; x += S::NT) {
          const int col = x / d_v, dim = x - col * d_v, column = hb * a.gb + col;
          if (r >= all_see + a.token_of(column)) continue;
          const int kvh = a.by_nhb.quotient(at.u) * a.heads + (a.heads > 1 ? a.by_gc.quotient(column) : 0);
          const uint8_t code = a.vp[page * a.map.vp + kvh * a.map.vh + (r - pg * a.map.page) * a.map.vr + dim];
          if ((code & 0x7f) == 0x7f) buf[col * LD + dim] = NAN;
        }
      }
      if (tid == 0) some_nan = 0;
      __syncthreads();
    }
    write_segment<T, S::NT, S::NBUF>(a, buf, LD, NCOL * LD, jm, jl, at.e, at.u, nh, whole, 2 * blockIdx.x + (at.t == 0));

    if (tb < at.nt) break;
    done += cnt;
    at.t = 0;
    next_unit<TR>(a, held, at);
    if (at.e >= a.n || at.pos >= end) break;
  }
  if (dead) {
    if (a.status) atomicOr(a.status, SNAP_DEV_WAIT_TIMEOUT);
    for (int x = n; x < n_issued; ++x) (void)wait_bounded(bar0 + 8 * (x % NSTAGE), (unsigned)(x / NSTAGE) & 1u);
  }
}

template <typename T>
__global__ void __launch_bounds__(JNT, 3) q8_join_kernel(const __grid_constant__ Q8Args a, int by_heads) {
  __shared__ __align__(16) JoinShared sh;
  if (threadIdx.x == 0) sh.s_e = -1;
  pdl_wait();
  join_outputs<T>(a, (int)blockIdx.x, (int)gridDim.x, by_heads, a.entry[a.n].x, sh);
}

// ---------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------
template <typename T, int D, int NWARP, int NSTAGE, int NG, int SIDES, int CTAS, Tiles MODE>
cudaError_t launch_as(const Q8Args& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  using S = Q8Shape<D, NWARP, NSTAGE, NG, SIDES>;
  static_assert(CTAS * (S::smem + sizeof(Held) + 1280) <= 228 * 1024, "all CTAs of the grid are resident at once");
  static SmemLimit limit = {};
  const auto kernel = q8_mma_kernel<T, D, NWARP, NSTAGE, NG, SIDES, CTAS, MODE>;
  if (cudaError_t e = ensure_dyn_smem(kernel, S::smem, limit)) return e;
  const cudaError_t e = launch_pdl(kernel, dim3(a.ctas), dim3(S::NT), S::smem, st, a, tk, tv);
  count_launch();
  return e;
}
template <typename T, int D, int NWARP, int NSTAGE, int NG, int SIDES, int CTAS>
cudaError_t launch_split(const Q8Args& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  if (!a.box) return launch_as<T, D, NWARP, NSTAGE, NG, SIDES, CTAS, Tiles::ROWS>(a, tk, tv, st);
  return a.d_qk == D && a.d_v == D ? launch_as<T, D, NWARP, NSTAGE, NG, SIDES, CTAS, Tiles::EXACT>(a, tk, tv, st)
                                   : launch_as<T, D, NWARP, NSTAGE, NG, SIDES, CTAS, Tiles::BOXES>(a, tk, tv, st);
}

// CTAs per SM: heads of up to 64 dims and eight columns; else.  (128 dims with three CTAs of two stages a warp instead of two of three: the
// 16 long sequences 188.7 us instead of 173.8.)
constexpr int kCtas = 3, kCtasWide = 2;

template <typename T>
cudaError_t launch_type(const Q8Args& a, int d, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  if (d <= 64)
    return a.heads > 1 ? launch_split<T, 64, 4, 2, 1, 2, kCtas>(a, tk, tv, st)
         : a.gb > 8    ? launch_split<T, 64, 4, 3, 2, 1, kCtasWide>(a, tk, tv, st)
                       : launch_split<T, 64, 4, 2, 1, 1, kCtas>(a, tk, tv, st);
  if (d <= 128)
    return a.heads > 1 ? launch_split<T, 128, 4, 3, 1, 2, kCtasWide>(a, tk, tv, st)
         : a.gb > 8    ? launch_split<T, 128, 4, 3, 2, 1, kCtasWide>(a, tk, tv, st)
                       : launch_split<T, 128, 4, 3, 1, 1, kCtasWide>(a, tk, tv, st);
  if (a.heads > 1) return launch_split<T, 256, 4, 1, 1, 2, kCtasWide>(a, tk, tv, st);
  return launch_split<T, 256, 4, 1, 1, 1, kCtasWide>(a, tk, tv, st);
}

}  // namespace

int q8_decode_plan(const Shape& s, const Q8Map& m, int n_active, int q_len, int sms, Q8DecodePlan* p) {
  const bool wide = s.d_qk > 128 || s.d_v > 128;
  const long long cols = (long long)s.g * q_len;
  // Two KV heads to a unit, as its two sides: where they lie side by side and eight columns hold both.
  p->heads = s.Hkv % 2 == 0 && 2 * cols <= 8 && m.pages.kh < m.pages.kr ? 2 : 1;
  // Columns of a unit.  (Sixteen of more than 128 dims take more registers than there are: 32 heads of 256 dims on 2, 8 sequences of 4000 to
  // 8000 rows 43.2 us instead of 28.4 in two units.)
  const int most = wide ? 8 : 16;
  p->nhb = (int)((cols + most - 1) / most);
  p->gb = p->heads > 1 ? 2 * (int)cols : (int)((cols + p->nhb - 1) / p->nhb);
  const int per_sm = p->gb > 8 || s.d_qk > 64 || s.d_v > 64 ? kCtasWide : kCtas;
  p->ctas = sms * per_sm < MAX_CTAS ? sms * per_sm : MAX_CTAS;
  const long long units = (long long)n_active * s.Hkv * p->nhb, tiles = m.pages.cap / (long long)TR + 1 + SHARE;
  // grid and index limits; a line of tiles and the scratch have to be countable
  if (cols > (1 << 20) || units > (1LL << 30) || n_active * (long long)s.Hq * q_len > 0x7fffffffLL || units * tiles > (1LL << 37) ||
      n_active * tiles > 0x7fffffffLL)
    return SNAP_ERR_UNSUPPORTED;
  size_t off = 0;
  p->entry_off = off; off += align_up((size_t)(n_active + 1) * sizeof(int4));
  p->ml_off = off;    off += align_up(2 * (size_t)p->ctas * p->gb * sizeof(float2));
  p->o_off = off;     off += align_up(2 * (size_t)p->ctas * p->gb * s.d_v * sizeof(float));
  p->bytes = off;
  return SNAP_OK;
}

cudaError_t launch_q8_decode(int dtype, const Shape& s, const Q8Map& m, const Q8DecodePlan& p, const void* q, const int* slots,
                             int n_active, int q_len, const void* k_pages, const void* v_pages, const float* k_scales,
                             const float* v_scales, const int* seq_len, void* out, char* scratch, uint32_t* status, cudaStream_t st) {
  const PageMap& pm = m.pages;
  Q8Args a;
  a.out = out; a.slots = slots; a.seq_len = seq_len;
  a.n = n_active; a.Hkv = s.Hkv; a.g = s.g * q_len * p.heads; a.gb = p.gb; a.nhb = p.nhb; a.U = s.Hkv / p.heads * p.nhb;
  a.d_v = s.d_v; a.max_seqs = s.max_seqs; a.rows_seq = s.Hq * q_len;
  a.map = pm;
  a.entry = reinterpret_cast<int4*>(scratch + p.entry_off);
  a.ml_unit = nullptr; a.keep_ml = false;
  a.ml_part = reinterpret_cast<float2*>(scratch + p.ml_off);
  a.o_part = reinterpret_cast<float*>(scratch + p.o_off);
  a.status = status; a.ctas = p.ctas;
  a.q = q; a.kp = static_cast<const uint8_t*>(k_pages); a.vp = static_cast<const uint8_t*>(v_pages); a.ks = k_scales; a.vs = v_scales;
  a.Hq = s.Hq; a.q_len = q_len; a.gq = s.g; a.gc = s.g * q_len; a.d_qk = s.d_qk; a.heads = p.heads; a.sc = p.gb / p.heads;
  a.scale_log2 = s.scale * 1.4426950408889634f;
  a.by_page = divisor((uint32_t)pm.page); a.by_block = divisor((uint32_t)m.block); a.blocks = m.blocks;
  a.by_gq = divisor((uint32_t)a.gq); a.by_gc = divisor((uint32_t)a.gc); a.by_nhb = divisor((uint32_t)a.nhb);
  // Tiles come through tensor maps of boxes 64 or 128 bytes wide, as many rows at once as a page always holds whole.
  const int d = s.d_qk > s.d_v ? s.d_qk : s.d_v, sw = d <= 64 ? 64 : 128, rows = pm.page % 32 == 0 ? 32 : pm.page % 16 == 0 ? 16 : 8;
  CUtensorMap tk = {}, tv = {};
  const umma::EncodeTiledFn enc = umma::encode_tiled_fn();
  const auto encode = [&](CUtensorMap* t, const void* base, int dims_of, long long ps, long long hs, long long rs) {
    const cuuint64_t dims[4] = {(cuuint64_t)dims_of, (cuuint64_t)pm.page, (cuuint64_t)s.Hkv, (cuuint64_t)pm.n_pages};
    // a stride that is never applied (one KV head, one page) may be anything: the map gets one that it takes
    const cuuint64_t strides[3] = {(cuuint64_t)rs, (cuuint64_t)(s.Hkv > 1 ? hs : dims_of), (cuuint64_t)(pm.n_pages > 1 ? ps : dims_of)};
    const cuuint32_t box[4] = {(cuuint32_t)sw, (cuuint32_t)rows, 1, 1}, estr[4] = {1, 1, 1, 1};
    return enc(t, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               sw == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  a.box = pm.page % 8 == 0 && enc && encode(&tk, k_pages, s.d_qk, pm.kp, pm.kh, pm.kr) && encode(&tv, v_pages, s.d_v, pm.vp, pm.vh, pm.vr) ? rows : 0;
  cudaError_t e;
  using BF = __nv_bfloat16;
  e = dtype == SNAP_F32 ? launch_type<float>(a, d, tk, tv, st) : launch_type<BF>(a, d, tk, tv, st);
  if (e != cudaSuccess) return e;
  // Joined by heads unless there is a unit for every CTA: then few are cut.  (By heads / by borders: 192 units on 296 CTAs, 24 sequences of 2000
  // to 9000 rows 63.5 / 65.2 us; 48, six of 300 to 1000 26.8 / 28.7; 128, 16 of 3000 to 9000 51.8 / 55.7; 384, 48 of 300 to 700 31.3 / 30.8; 540
  // on 444, 45 of up to 333 18.4 / 18.4.)
  const int heads = n_active * a.rows_seq, by_heads = ((long long)n_active * a.U <= p.ctas && heads <= 4096) || p.ctas < 2;
  const dim3 grid((unsigned)(by_heads ? heads : p.ctas - 1));
  e = dtype == SNAP_F32 ? launch_pdl(q8_join_kernel<float>, grid, dim3(JNT), 0, st, a, by_heads)
                        : launch_pdl(q8_join_kernel<BF>, grid, dim3(JNT), 0, st, a, by_heads);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
