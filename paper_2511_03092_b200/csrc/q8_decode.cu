// Attention of the last tokens of each sequence over a cache in pages of 8-bit numbers (snap_paged_q8_decode_attn).
//
//     out[i][u][h] = sum_r p_r s'_r V_r / sum_r p_r,   p_r = exp(scale s_r q.K_r - max),   r < len - q_len + 1 + u
//
// with K_r, V_r the codes of row r and s_r, s'_r the scales of its block.  Every row is read once and serves all columns (the
// group's query heads, of each token) at once, so HBM bounds the call.  How the work is divided and joined: paged_line.cuh.
//
// A warp's tile is 32 rows, S^T = K tile . Q^T and O^T += V tile^T . P^T with m16n8k16 on half-precision numbers: a code is
// one exactly, and converting two takes one instruction.  The order of the products' inner dims is free, so codes are used as ldmatrix
// delivers them: four neighbouring dims of a key row are positions 2t, 2t + 1, 2t + 8, 2t + 9 of a step of 16, and the queries
// are read in that order; the transposed 16-bit units of two value rows hold two dims each, which become rows g and g + 8 of the product.
//
// Queries are brought to a largest number of 2^14 to 2^15 by a power of two, which leaves a bf16 query exact down to 2^-29 of its
// largest number (cut off 2^-39 below it); single-precision ones enter as two such numbers.  The scale of a key row multiplies its logits, that
// of a value row its weight.  Weights times scales are brought to the range of half precision by another power of two per
// column, `f`, which follows the largest of them (scales may lie far apart); they round to 11 bits (bf16: an eighth of the
// output's own rounding) or are two numbers (single precision).
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
constexpr int LOOK = 2;                         // tiles whose pages are looked up ahead of their copies

// n / d for 0 <= n < 2^31 by a multiplication
struct Divisor {
  uint32_t d, m; int s;
  __device__ __forceinline__ int quotient(int n) const { return (int)((__umulhi(m, (uint32_t)n) + (uint32_t)n) >> s); }
};
Divisor divisor(uint32_t d) {
  Divisor r;
  r.d = d;
  for (r.s = 0; (1ull << r.s) < d; ++r.s) {}
  r.m = (uint32_t)(((1ull << 32) * ((1ull << r.s) - d)) / d + 1);
  return r;
}

struct Q8Args : LineArgs {
  const void* q;
  const uint8_t* kp; const uint8_t* vp; const float* ks; const float* vs;
  int Hq, q_len, gq, d_qk;                      // gq query heads of a KV head; g = gq * q_len
  float scale_log2;
  Divisor by_page, by_block;
  int blocks;                                   // scales of a page and KV head
  int box;                                      // rows of a copy, 0: rows are copied by the lanes
  __device__ __forceinline__ long long out_row(int e, int kvh, int x) const {
    const int u = x / gq;
    return ((long long)e * q_len + u) * Hq + kvh * gq + (x - u * gq);
  }
};

template <int D, int NWARP, int NSTAGE, int NG> struct Q8Shape {
  static constexpr int NT = NWARP * 32, KS = D / 16, NCOL = 8 * NG;
  static constexpr int SW = D < 128 ? D : 128, NSL = D / SW;             // bytes of a slab's rows; slabs
  static constexpr int SLAB_B = TR * SW, TENS_B = NSL * SLAB_B, STAGE_B = 2 * TENS_B;
  static constexpr int LD = D + 4, NBUF = D * NG < 128 ? NWARP / 2 : 1;  // exchange buffers: as many as leave room for the CTAs of an SM
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
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// x as two half-precision numbers: what rounding leaves of it
__device__ __forceinline__ uint32_t rest_f16(float lo, float hi, uint32_t rounded) {
  const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&rounded));
  return pack_f16(lo - r.x, hi - r.y);
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ int exponent_of(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }
__device__ __forceinline__ float power_of(int e) { return exp2_of(min(max(e, -126), 127)); }

// How a tile comes in: through the tensor maps, heads of exactly D dims (EXACT) or fewer; or, where a page is no multiple of
// 8 rows, copied by the lanes in 16-byte pieces (ROWS).
enum class Tiles { EXACT, BOXES, ROWS };
template <typename T, int D, int NWARP, int NSTAGE, int NG, int CTAS, Tiles MODE>
__global__ void __launch_bounds__(NWARP * 32, CTAS)
q8_mma_kernel(const __grid_constant__ Q8Args a, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v) {
  using S = Q8Shape<D, NWARP, NSTAGE, NG>;
  constexpr bool F32 = sizeof(T) == 4, EXACT = MODE == Tiles::EXACT, BY_ROWS = MODE == Tiles::ROWS;
  constexpr int KS = S::KS, NCOL = S::NCOL, LD = S::LD, SW = S::SW, PARTS = F32 ? 2 : 1, MT = TR / 16;
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  float* row_scales = reinterpret_cast<float*>(stages + S::stages_b);    // [NWARP][NSTAGE][keys, values][TR]
  uint64_t* bars = reinterpret_cast<uint64_t*>(row_scales + S::rows_b / sizeof(float));
  float* buf = reinterpret_cast<float*>(bars + NWARP * NSTAGE);          // [NBUF][NCOL][LD]
  float* wm = buf + S::NBUF * NCOL * LD;                                 // [NWARP][NCOL] maxima, then sums
  float* wl = wm + NWARP * NCOL;
  float* jm = wl + NWARP * NCOL;                                         // [NCOL] joined maxima, then sums
  float* jl = jm + NCOL;
  __shared__ int scan[S::NT / 32 + 2];
  __shared__ Held held;
  __shared__ Found found;

  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, gq = lane >> 2, tq = lane & 3;
  unsigned char* wstages = stages + w * NSTAGE * S::STAGE_B;
  float* wscales = row_scales + w * NSTAGE * 2 * TR;
  const uint32_t stage0 = smem_u32(wstages), scale0 = smem_u32(wscales), bar0 = smem_u32(bars + w * NSTAGE);
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

  // ---- the warp's producer: NSTAGE tiles ahead of the consumer, over unit borders; warp w takes the CTA's tiles w, w + NWARP, ...;
  // lane l looks up the page of the tile's row l ----
  Place pr = at;
  bool more = advance<TR>(a, held, pr, w, end);
  struct Look { int page, off, kvh; bool tile; };                        // off: row of the page, -1 no row
  const auto look_up = [&]() {                                           // (nothing waits here for what the table says)
    Look r = {-1, -1, 0, more};
    if (more) {
      const int row = pr.t * TR + lane;
      r.kvh = pr.u / a.nhb;
      if (row < pr.len) {
        const int pg = a.by_page.quotient(row);
        r.off = row - pg * a.map.page;
        if (index_ok(pg, a.map.max_pages, a.status)) r.page = a.map.table[(long long)pr.slot * a.map.max_pages + pg];
      }
      more = advance<TR>(a, held, pr, NWARP, end);
    }
    return r;
  };
  Look look[LOOK];
#pragma unroll
  for (int x = 0; x < LOOK; ++x) look[x] = look_up();

  // B fragments of Q^T, column 8 gi + gq, dims 16 ks + 4 tq .. + 3; of single precision the rounded number, then what it leaves
  const T* q_all = static_cast<const T*>(a.q);
  uint32_t qb[NG][KS][PARTS][2];
  float q_scale[NG][2];                                                  // of this thread's two columns of the logits
  int sees[NG][2];                                                       // rows that these columns see
  const auto load_q = [&]() {
    const int kvh = at.u / a.nhb, hb = at.u - kvh * a.nhb, nh = min(a.gb, a.g - hb * a.gb);
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
      const int col = 8 * gi + gq;
      const T* qp = q_all + a.out_row(at.e, kvh, hb * a.gb + (col < nh ? col : 0)) * d_qk + 4 * tq;
      float x[KS][4], big = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bool there = col < nh && (EXACT || 16 * ks < d_qk);
        if constexpr (F32) {
          const float4 v = there ? *reinterpret_cast<const float4*>(qp + 16 * ks) : make_float4(0.f, 0.f, 0.f, 0.f);
          x[ks][0] = v.x; x[ks][1] = v.y; x[ks][2] = v.z; x[ks][3] = v.w;
        } else {
          const uint2 v = there ? *reinterpret_cast<const uint2*>(qp + 16 * ks) : make_uint2(0, 0);
          x[ks][0] = __uint_as_float(v.x << 16); x[ks][1] = __uint_as_float(v.x & 0xffff0000u);
          x[ks][2] = __uint_as_float(v.y << 16); x[ks][3] = __uint_as_float(v.y & 0xffff0000u);
        }
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
          if constexpr (F32) qb[gi][ks][1][c] = rest_f16(lo, hi, qb[gi][ks][0][c]);
        }
      const float back = a.scale_log2 / f0 / f1;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        q_scale[gi][c] = __shfl_sync(0xffffffffu, back, (2 * tq + c) * 4);
        const int mine = 8 * gi + 2 * tq + c;
        sees[gi][c] = mine < nh ? at.len - a.q_len + 1 + (hb * a.gb + mine) / a.gq : at.len;
      }
    }
  };
  load_q();                                                              // (the first tiles' look-ups wait alongside)

  int n_issued = 0;
  unsigned long long there_of = 0;                                       // 32 bits for each of two stages: the rows that are there
  static_assert(NSTAGE <= 2, "the rows of two stages fit");
  const auto issue = [&]() {
    const int s = n_issued % NSTAGE;
    const Look l = look[0];
#pragma unroll
    for (int x = 0; x + 1 < LOOK; ++x) look[x] = look[x + 1];
    look[LOOK - 1] = look_up();
    const bool okay = l.off >= 0 && l.page >= 0 && l.page < a.map.n_pages;
    const unsigned rows = __ballot_sync(0xffffffffu, okay);
    there_of = (there_of & ~(0xffffffffull << (32 * s))) | (unsigned long long)rows << (32 * s);
    if (!okay && l.off >= 0 && a.status) atomicOr(a.status, SNAP_DEV_BAD_PAGE);
    const uint32_t dst = stage0 + s * S::STAGE_B, bar = bar0 + 8 * s, sc = scale0 + (s * 2 * TR + lane) * 4;
    if (okay) {
      const long long x = ((long long)l.page * a.Hkv + l.kvh) * a.blocks + a.by_block.quotient(l.off);
      cp_async4(sc, a.ks + x);
      cp_async4(sc + TR * 4, a.vs + x);
    } else {
      wscales[s * 2 * TR + lane] = 0.f;
      wscales[s * 2 * TR + TR + lane] = 0.f;
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
          if (16 * c < d_qk) cp_async16(to, a.kp + ko + 16 * c, 16);
          if (16 * c < d_v) cp_async16(to + S::TENS_B, a.vp + vo + 16 * c, 16);
        }
      }
    } else {
      const bool first = okay && lane % a.box == 0;                      // of a copy's rows
      const unsigned copies = __popc(__ballot_sync(0xffffffffu, first));
      const unsigned slabs = (unsigned)((d_qk + SW - 1) / SW + (d_v + SW - 1) / SW);
      if (lane == 0) mbar_expect_tx(bar, copies * slabs * (unsigned)(a.box * SW));
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
#pragma unroll 1
  for (int s = 0; s < NSTAGE && look[0].tile; ++s) issue();

  // ldmatrix lane roles: K (plain): row (lane & 7) + 8 * bit3, chunk + bit4; V (transposed): the same
  const int l_row = (lane & 7) + ((lane >> 3) & 1) * 8, l_cadd = lane >> 4;

  bool dead = false;                                                     // a bounded wait ran out: nothing more is read
  int n = 0, done = 0;                                                   // tiles done by this warp; by the CTA before this segment
  while (true) {
    // ---- a segment: the CTA's tiles [at.t, tb) of one unit ----
    const int tb = segment_end(at, end), cnt = tb - at.t;
    const int hb = at.u % a.nhb, nh = min(a.gb, a.g - hb * a.gb);
    const bool whole = cnt == at.nt;
    const int all_see = at.len - a.q_len + 1;                            // rows that every column sees
    float oacc[NG][KS][4];                                               // O^T: dims 16 db + 2 gq (+ 1: the upper two), columns 8 gi + 2 tq (+ 1)
    // per column: reference of the exponentials, sum of the weights, largest weight times scale, factor on those and where it has to fall
    float m_ref[NG][2], l_part[NG][2], top[NG][2], f[NG][2], most[NG][2];
#pragma unroll
    for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
      for (int c = 0; c < 2; ++c) { m_ref[gi][c] = -INFINITY; l_part[gi][c] = top[gi][c] = most[gi][c] = 0.f; f[gi][c] = 1.f; }
#pragma unroll
      for (int db = 0; db < KS; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x) oacc[gi][db][x] = 0.f;
    }

    for (; w + n * NWARP < done + cnt && !dead; ++n) {
      const int s = n % NSTAGE;
      const bool landed = wait_bounded(bar0 + 8 * s, (unsigned)(n / NSTAGE) & 1u);
      if (__any_sync(0xffffffffu, !landed)) { dead = true; break; }
      const int row0 = (at.t + (w + n * NWARP - done)) * TR;
      const unsigned rows = (unsigned)(there_of >> (32 * s));
      const uint32_t sK = stage0 + s * S::STAGE_B, sV = sK + S::TENS_B;
      if (rows != 0xffffffffu) {
        // rows past the end, or on a bad page, may hold anything, and a zero weight does not silence a NaN in V: clear them
        constexpr int CPR = D / 16;
        for (int x = lane; x < TR * CPR; x += 32) {
          const int r = x / CPR, c = x % CPR;
          if (!((rows >> r) & 1u))
            *reinterpret_cast<uint4*>(wstages + s * S::STAGE_B + S::TENS_B + c / (SW / 16) * S::SLAB_B + swizzled<SW>(r, c % (SW / 16))) = make_uint4(0, 0, 0, 0);
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
          ldsm4(sK + k2 * 32 / SW * S::SLAB_B + swizzled<SW>(16 * mt + l_row, k2 * 2 % (SW / 16) + l_cadd), c);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!EXACT && 32 * k2 + 16 * h >= d_qk) break;
            const uint32_t a0 = halves_of_codes(c[2 * h] & 0xffffu), a2 = halves_of_codes(c[2 * h] >> 16);
            const uint32_t a1 = halves_of_codes(c[2 * h + 1] & 0xffffu), a3 = halves_of_codes(c[2 * h + 1] >> 16);
#pragma unroll
            for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
              for (int p = PARTS - 1; p >= 0; --p) mma_f16(v[mt][gi], a0, a1, a2, a3, qb[gi][2 * k2 + h][p][0], qb[gi][2 * k2 + h][p][1]);
            }
          }
        }
      }
      // ---- logits; rows that are not there, or that a column does not see ----
      const float* sc = wscales + s * 2 * TR;
      const bool masked = rows != 0xffffffffu || row0 + TR > all_see;
      bool refresh = false;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r8 = 0; r8 < 2; ++r8) {
          const int r = 16 * mt + 8 * r8 + gq;
          const float k_scale = sc[r];
#pragma unroll
          for (int gi = 0; gi < NG; ++gi)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float& x = v[mt][gi][2 * r8 + c];
              x *= q_scale[gi][c] * k_scale;
              if (masked && !(((rows >> r) & 1u) && row0 + r < sees[gi][c])) x = -INFINITY;
              refresh = refresh || x > m_ref[gi][c] + 8.f;
            }
        }
      // The reference of the exponentials follows the maximum lazily: it moves (and the sums are rescaled) only when
      // a logit lies 8 above it, i.e. before a weight passes 2^8.
      refresh = __any_sync(0xffffffffu, refresh);
      if (refresh) {
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float mx = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) mx = fmaxf(mx, fmaxf(v[mt][gi][c], v[mt][gi][2 + c]));
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float nm = fmaxf(m_ref[gi][c], mx), al = m_ref[gi][c] == -INFINITY ? 0.f : exp2f(m_ref[gi][c] - nm);
            m_ref[gi][c] = nm;
            l_part[gi][c] *= al;
            top[gi][c] *= al;
#pragma unroll
            for (int db = 0; db < KS; ++db) { oacc[gi][db][c] *= al; oacc[gi][db][2 + c] *= al; }
          }
      }
      // ---- weights, and weights times scales ----
      bool lower = refresh;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r8 = 0; r8 < 2; ++r8) {
          const float v_scale = sc[TR + 16 * mt + 8 * r8 + gq];
#pragma unroll
          for (int gi = 0; gi < NG; ++gi)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float& x = v[mt][gi][2 * r8 + c];
              x = fast_exp2(x - (m_ref[gi][c] == -INFINITY ? 0.f : m_ref[gi][c]));
              l_part[gi][c] += x;
              x *= v_scale;
              lower = lower || x > most[gi][c];
            }
        }
      if (__any_sync(0xffffffffu, lower)) {                              // the factor goes by the largest so far: 2^6 to 2^7 after it
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float mx = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) mx = fmaxf(mx, fmaxf(v[mt][gi][c], v[mt][gi][2 + c]));
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            top[gi][c] = fmaxf(top[gi][c], mx);
            const int e = min(max(6 - exponent_of(top[gi][c]), -120), 120);
            const float ratio = power_of(e - exponent_of(f[gi][c]));
            f[gi][c] = exp2_of(e);
            most[gi][c] = power_of(15 - e);
#pragma unroll
            for (int db = 0; db < KS; ++db) { oacc[gi][db][c] *= ratio; oacc[gi][db][2 + c] *= ratio; }
          }
      }
      uint32_t pb[MT][NG][PARTS][2];                                     // P^T as B operands
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int r8 = 0; r8 < 2; ++r8) {
            const float p0 = v[mt][gi][2 * r8] * f[gi][0], p1 = v[mt][gi][2 * r8 + 1] * f[gi][1];
            const uint32_t hi = pack_f16(p0, p1);
            pb[mt][gi][0][r8] = movmatrix_t(hi);
            if constexpr (F32) pb[mt][gi][PARTS - 1][r8] = movmatrix_t(rest_f16(p0, p1, hi));
          }
      // ---- O^T += V tile^T . P^T ----
#pragma unroll
      for (int d2 = 0; d2 < KS / 2; ++d2) {                              // 32 dims
        if (!EXACT && 32 * d2 >= d_v) break;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          uint32_t c[4];
          ldsm4t(sV + d2 * 32 / SW * S::SLAB_B + swizzled<SW>(16 * mt + l_row, d2 * 2 % (SW / 16) + l_cadd), c);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!EXACT && 32 * d2 + 16 * h >= d_v) break;
            const uint32_t x = __byte_perm(c[2 * h], 0, 0x3120), y = __byte_perm(c[2 * h + 1], 0, 0x3120);   // two rows of a dim, then of the next
            const uint32_t a0 = halves_of_codes(x & 0xffffu), a1 = halves_of_codes(x >> 16);
            const uint32_t a2 = halves_of_codes(y & 0xffffu), a3 = halves_of_codes(y >> 16);
#pragma unroll
            for (int gi = 0; gi < NG; ++gi) {
#pragma unroll
              for (int p = PARTS - 1; p >= 0; --p) mma_f16(oacc[gi][2 * d2 + h], a0, a1, a2, a3, pb[mt][gi][p][0], pb[mt][gi][p][1]);
            }
          }
        }
      }
      __syncwarp();
      if (look[0].tile) {
        // the stage was read, and possibly cleared, through the generic proxy; the copy that refills it is of the async proxy
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        issue();
      }
    }

    // ---- join the warps: maxima first, then the outputs ----
#pragma unroll
    for (int gi = 0; gi < NG; ++gi)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int o = 4; o <= 16; o <<= 1) l_part[gi][c] += __shfl_xor_sync(0xffffffffu, l_part[gi][c], o);
        if (gq == 0) {
          wm[w * NCOL + 8 * gi + 2 * tq + c] = m_ref[gi][c];
          wl[w * NCOL + 8 * gi + 2 * tq + c] = l_part[gi][c];
        }
      }
    __syncthreads();
#pragma unroll
    for (int gi = 0; gi < NG; ++gi)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float M = -INFINITY;
#pragma unroll
        for (int ww = 0; ww < NWARP; ++ww) M = fmaxf(M, wm[ww * NCOL + 8 * gi + 2 * tq + c]);
        const float y = m_ref[gi][c] == -INFINITY ? 0.f : exp2f(m_ref[gi][c] - M) / f[gi][c];
#pragma unroll
        for (int db = 0; db < KS; ++db) { oacc[gi][db][c] *= y; oacc[gi][db][2 + c] *= y; }
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
    // the last warps leave their outputs in a buffer each, those before add theirs there, in turns
#pragma unroll 1
    for (int turn = NWARP / S::NBUF - 1; turn >= 0; --turn) {
      if (w / S::NBUF == turn) {
        const bool add = turn < NWARP / S::NBUF - 1;
        float* b = buf + w % S::NBUF * NCOL * LD + 2 * tq * LD + 2 * gq;
#pragma unroll
        for (int gi = 0; gi < NG; ++gi)
#pragma unroll
          for (int db = 0; db < KS; ++db)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float2* p = reinterpret_cast<float2*>(b + (8 * gi + c) * LD + 16 * db);
              float2 x = make_float2(oacc[gi][db][c], oacc[gi][db][2 + c]);
              if (add) { const float2 y = *p; x.x += y.x; x.y += y.y; }
              *p = x;
            }
      }
      __syncthreads();
    }
    write_segment<T, S::NT, S::NBUF>(a, buf, LD, NCOL * LD, jm, jl, at.e, at.u, nh, whole, 2 * blockIdx.x + (at.t == 0));

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
template <typename T, int D, int NWARP, int NSTAGE, int NG, int CTAS, Tiles MODE>
cudaError_t launch_as(const Q8Args& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  using S = Q8Shape<D, NWARP, NSTAGE, NG>;
  static_assert(CTAS * (S::smem + sizeof(Held) + 1280) <= 228 * 1024, "all CTAs of the grid are resident at once");
  static SmemLimit limit = {};
  const auto kernel = q8_mma_kernel<T, D, NWARP, NSTAGE, NG, CTAS, MODE>;
  if (cudaError_t e = ensure_dyn_smem(kernel, S::smem, limit)) return e;
  const cudaError_t e = launch_pdl(kernel, dim3(a.ctas), dim3(S::NT), S::smem, st, a, tk, tv);
  count_launch();
  return e;
}
template <typename T, int D, int NWARP, int NSTAGE, int NG, int CTAS>
cudaError_t launch_split(const Q8Args& a, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  if (!a.box) return launch_as<T, D, NWARP, NSTAGE, NG, CTAS, Tiles::ROWS>(a, tk, tv, st);
  return a.d_qk == D && a.d_v == D ? launch_as<T, D, NWARP, NSTAGE, NG, CTAS, Tiles::EXACT>(a, tk, tv, st)
                                   : launch_as<T, D, NWARP, NSTAGE, NG, CTAS, Tiles::BOXES>(a, tk, tv, st);
}

constexpr int kCtas = 3, kCtasWide = 2;         // per SM: one group of eight columns and heads of up to 128 dims; else

}  // namespace

int q8_decode_plan(int dtype, const Shape& s, const Q8Map& m, int n_active, int q_len, int sms, Q8DecodePlan* p) {
  const bool wide = s.d_qk > 128 || s.d_v > 128;
  const long long cols = (long long)s.g * q_len;
  const int most = wide && dtype == SNAP_F32 ? 8 : 16;                    // columns of a unit
  p->nhb = (int)((cols + most - 1) / most);
  p->gb = (int)((cols + p->nhb - 1) / p->nhb);
  const int per_sm = p->gb > 8 || wide ? kCtasWide : kCtas;
  p->ctas = sms * per_sm < MAX_CTAS ? sms * per_sm : MAX_CTAS;
  const long long units = (long long)n_active * s.Hkv * p->nhb, tiles = m.pages.cap / (long long)TR + 1 + UNIT_TILES;
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
  a.n = n_active; a.Hkv = s.Hkv; a.g = s.g * q_len; a.gb = p.gb; a.nhb = p.nhb; a.U = s.Hkv * p.nhb;
  a.d_v = s.d_v; a.max_seqs = s.max_seqs; a.rows_seq = s.Hq * q_len;
  a.map = pm;
  a.entry = reinterpret_cast<int4*>(scratch + p.entry_off);
  a.ml_unit = nullptr; a.keep_ml = false;
  a.ml_part = reinterpret_cast<float2*>(scratch + p.ml_off);
  a.o_part = reinterpret_cast<float*>(scratch + p.o_off);
  a.status = status; a.ctas = p.ctas;
  a.q = q; a.kp = static_cast<const uint8_t*>(k_pages); a.vp = static_cast<const uint8_t*>(v_pages); a.ks = k_scales; a.vs = v_scales;
  a.Hq = s.Hq; a.q_len = q_len; a.gq = s.g; a.d_qk = s.d_qk;
  a.scale_log2 = s.scale * 1.4426950408889634f;
  a.by_page = divisor((uint32_t)pm.page); a.by_block = divisor((uint32_t)m.block); a.blocks = m.blocks;
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
               sw == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  a.box = pm.page % 8 == 0 && enc && encode(&tk, k_pages, s.d_qk, pm.kp, pm.kh, pm.kr) && encode(&tv, v_pages, s.d_v, pm.vp, pm.vh, pm.vr) ? rows : 0;
  const bool two = p.gb > 8;
  cudaError_t e;
  using BF = __nv_bfloat16;
  if (dtype == SNAP_F32) {
    if (d <= 64) e = two ? launch_split<float, 64, 4, 2, 2, kCtasWide>(a, tk, tv, st) : launch_split<float, 64, 4, 2, 1, kCtas>(a, tk, tv, st);
    else if (d <= 128) e = two ? launch_split<float, 128, 4, 2, 2, kCtasWide>(a, tk, tv, st) : launch_split<float, 128, 4, 2, 1, kCtas>(a, tk, tv, st);
    else e = launch_split<float, 256, 4, 1, 1, kCtasWide>(a, tk, tv, st);
  }
  else if (d <= 64) e = two ? launch_split<BF, 64, 4, 2, 2, kCtasWide>(a, tk, tv, st) : launch_split<BF, 64, 4, 2, 1, kCtas>(a, tk, tv, st);
  else if (d <= 128) e = two ? launch_split<BF, 128, 4, 2, 2, kCtasWide>(a, tk, tv, st) : launch_split<BF, 128, 4, 2, 1, kCtas>(a, tk, tv, st);
  else e = two ? launch_split<BF, 256, 4, 1, 2, kCtasWide>(a, tk, tv, st) : launch_split<BF, 256, 4, 1, 1, kCtasWide>(a, tk, tv, st);
  if (e != cudaSuccess) return e;
  const int heads = n_active * a.rows_seq, by_heads = heads <= 512 || p.ctas < 2;
  const dim3 grid((unsigned)(by_heads ? heads : p.ctas - 1));
  e = dtype == SNAP_F32 ? launch_pdl(q8_join_kernel<float>, grid, dim3(JNT), 0, st, a, by_heads)
                        : launch_pdl(q8_join_kernel<BF>, grid, dim3(JNT), 0, st, a, by_heads);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
