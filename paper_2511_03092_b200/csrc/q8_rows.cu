// Rows between dense tensors and pages of 8-bit numbers: the append, which rotates and quantises them on the way in
// (snap_paged_q8_append), and the gather, which brings them back (snap_paged_q8_gather).
//
// The scale of a block (rows of one KV head that share it) goes by the largest of the inputs, not of the rotated keys: a pair
// (a, b) turned and multiplied by m is at most sqrt(2) m max(|a|, |b|) in either place.  So it does not depend on how sines
// are rounded, and the pass that looks for it computes no angles.
#include "e4m3.cuh"
#include "snap_internal.cuh"

namespace snap {
namespace {

constexpr int NT = 256, NW = NT / 32;           // threads of the gather
constexpr int ANT = 128, ANW = ANT / 32;        // ... of the append: four blocks per SM hide each other's look-ups better than two of 256
                                                // (26003 tokens 152 us instead of 160; three without spills 150 instead of 140)
constexpr int SLAB = 16;                        // rows whose angles are held at a time

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { using type = uint4; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<4> { using type = unsigned; };
template <> struct RawOf<2> { using type = unsigned short; };
template <> struct RawOf<1> { using type = unsigned char; };
template <typename E, int V> union Vec {
  typename RawOf<V * (int)sizeof(E)>::type raw;
  E e[V];
  __device__ Vec() {}
};

// The entry that token t belongs to: the last i with cu[i] <= t, -1 when there is none (a whole warp asks).
__device__ __forceinline__ int entry_of(const Q8Rows& r, int t) {
  const int lane = threadIdx.x & 31;
  int lo = -1, hi = r.n_seqs + 1;                                        // cu[lo] <= t; cu[hi] is not looked at
  while (hi - lo > 1) {
    const int step = (hi - lo - 1 + 31) / 32, at = lo + 1 + lane * step;
    const unsigned le = __ballot_sync(0xffffffffu, at < hi && r.cu[at] <= t);
    const int k = 31 - __clz(le);                                        // -1: none
    hi = min(hi, lo + 1 + (k + 1) * step);
    if (k >= 0) lo = lo + 1 + k * step;
  }
  return lo;
}

constexpr int HOLD = 4;                         // pairs of vectors that a lane keeps from the look for the largest number to the rounding

// Where a warp's lanes stand in the rows of a head cut into items (pairs of vectors, 32 at most): in pass k a lane has item j of row
// r0 + k * rpp.
struct Lanes {
  int items, rpp, r0, j;
  __device__ __forceinline__ Lanes(int items_) : items(items_) {
    const int lane = threadIdx.x & 31;
    rpp = 32 / items;
    r0 = lane / items;
    j = lane - r0 * items;
    if (r0 >= rpp) r0 = 1 << 30;                // (a spare lane: no row)
  }
};

// The largest number's size of a vector
template <typename T, int N> __device__ __forceinline__ float largest_of(const Vec<T, N>& v) {
  if constexpr (sizeof(T) == 2) {               // two at a time
    __nv_bfloat162 m = __habs2(reinterpret_cast<const __nv_bfloat162*>(v.e)[0]);
#pragma unroll
    for (int e = 1; e < N / 2; ++e) m = __hmax2(m, __habs2(reinterpret_cast<const __nv_bfloat162*>(v.e)[e]));
    return fmaxf(fmaxf(__low2float(m), __high2float(m)), 0.f);
  } else {
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, fabsf(v.e[e]));
    return m;
  }
}

struct AppendLaunch {
  Q8AppendArgs a;
  int group, blocks, chunk;                     // rows and blocks of a group, tokens of a CTA
  int nj, ni, X;                                // items of a head: those that turn, all; threads on them
};

// V numbers times f as codes
template <int V> __device__ __forceinline__ void put_codes(uint8_t* to, const float (&x)[V], float f) {
  if constexpr (V == 1) *to = (uint8_t)codes_of_floats(x[0] * f, 0.f);
  else if constexpr (V == 2) *reinterpret_cast<unsigned short*>(to) = (unsigned short)codes_of_floats(x[0] * f, x[1] * f);
  else {
    uint32_t w[V / 4];
#pragma unroll
    for (int e = 0; e < V / 4; ++e) w[e] = codes_of_floats(x[4 * e] * f, x[4 * e + 1] * f) | codes_of_floats(x[4 * e + 2] * f, x[4 * e + 3] * f) << 16;
    if constexpr (V == 4) *reinterpret_cast<uint32_t*>(to) = w[0];
    else *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[V / 4 - 1]);
  }
}

// cos and sin of position * f, the angle taken in half turns: its whole turns come off exactly
__device__ __forceinline__ float2 cos_sin(int pos, double f) {
  const double u = (double)pos * f * 0.3183098861837907;                 // 1 / pi
  const double w = fma(-2.0, rint(0.5 * u), u);                          // [-1, 1]
  const float wh = (float)w, wl = (float)(w - (double)wh) * 3.14159265f;
  float s, c;
  sincospif(wh, &s, &c);
  return make_float2(fmaf(-wl, s, c), fmaf(wl, c, s));
}

// A CTA takes the groups (whole blocks, at least SLAB rows) that begin with one of its tokens, and of their heads every
// gridDim.y-th.  First a warp to a head's keys or values: the scales of its blocks; of values, which then only have to be rounded, also the
// codes (up to HOLD pairs of vectors a lane stay in registers for that).  Then keys and queries: a thread keeps the cosines and sines of its
// pairs of one row and walks over the heads, the keys coming in again, mostly from L2.
//
// A step of few tokens is bound by its chain of look-ups (entry, table, scale, rows) and the host's call: 32 sequences 6.6 us.  A large one is
// instructions as much as HBM: conversions, rotations and stores of two or four bytes a lane; 26003 tokens of 32 + 8 heads of 128 dims 141 us
// for 638 MB, 4.5 TB/s (69 % of the measured copy rate).
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(ANT, 4) q8_append_kernel(const __grid_constant__ AppendLaunch L) {
  const Q8AppendArgs& a = L.a;
  const Q8Rows& r = a.r;
  const PageMap& pm = r.map.pages;
  const int B = r.map.block, G = L.group, half = a.rot / 2;
  extern __shared__ float2 table[];                                      // [SLAB][rot / 2]
  float* inv_k = reinterpret_cast<float*>(table + SLAB * half);          // [heads of the CTA][blocks of a group]: 1 / scale of the keys
  __shared__ int page_s[SLAB], blk_s[SLAB], begin_s[SLAB];               // of each block: page (-1: skipped), block of the page, its first row there
  __shared__ unsigned big_s[ANW][SLAB];                                   // of each warp's task and block: the largest number, as its bits
  __shared__ float inv_s[ANW][SLAB];                                      // ... and 1 / scale
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, y = blockIdx.y, ny = gridDim.y;
  const int nk = (r.Hkv - y + ny - 1) / ny, nq = r.Hq > y ? (r.Hq - y + ny - 1) / ny : 0;
  constexpr int EV = 16 / (int)sizeof(T);                                // numbers of a vector of values
  using VT = Vec<T, V>;
  using VV = Vec<T, EV>;
  const Lanes lk(r.d_qk / EV / 2), lv(r.d_v / EV / 2);
  const int per = ANT / L.X, tx = tid % L.X, tq = tid / L.X;              // (row, head) pairs at once; this thread's item and place among those
  const int apart = half ? ANT / half : 1, angle = half ? tid % half : 0, angle_z = half ? tid / half : apart;   // rows of angles at once; this thread's
  pdl_wait();
  const double freq = angle_z < apart ? a.freqs[angle] : 0.0;
  // Up to 32 entries are read once, a lane each, and looked through without memory.
  const bool few = r.n_seqs <= 32;
  int my_cu = 0, my_slot = -1, my_first = 0, total = 0;
  if (few) {
    total = r.cu[r.n_seqs];
    if (lane < r.n_seqs) { my_cu = r.cu[lane]; my_slot = r.slots[lane]; my_first = r.first[lane]; }
  }
  const int t0 = blockIdx.x * L.chunk, t1 = min(t0 + L.chunk, r.n_tokens);
  for (int t = t0; t < t1;) {
    int i, from, to, slot, first;
    if (few) {
      i = total <= t ? r.n_seqs : 31 - __clz(__ballot_sync(0xffffffffu, lane < r.n_seqs && my_cu <= t));
      from = __shfl_sync(0xffffffffu, my_cu, max(i, 0) & 31);
      to = i + 1 < r.n_seqs ? __shfl_sync(0xffffffffu, my_cu, (i + 1) & 31) : total;
      slot = __shfl_sync(0xffffffffu, my_slot, max(i, 0) & 31);
      first = __shfl_sync(0xffffffffu, my_first, max(i, 0) & 31);
      if (i < 0) to = __shfl_sync(0xffffffffu, my_cu, 0);                // (where the first entry's begin)
    } else {
      i = entry_of(r, t);
      const int at = min(max(i, 0), r.n_seqs - 1);
      from = r.cu[at]; to = r.cu[i < 0 ? 0 : at + 1]; slot = r.slots[at]; first = r.first[at];
    }
    if (i >= r.n_seqs) break;
    if (i < 0) { t = min(max(to, t + 1), t1); continue; }
    to = min(to, r.n_tokens);
    if (from > t || to <= t) { ++t; continue; }                          // (sums that decrease: go on all the same)
    const unsigned row = (unsigned)first + (unsigned)t - (unsigned)from; // (neither is negative, or the entry is skipped)
    const bool begins = t == from;
    if (slot < 0 || slot >= r.max_seqs || first < 0) {
      if (begins && tid == 0 && y == 0 && slot != -1 && r.status)
        atomicOr(r.status, slot < 0 || slot >= r.max_seqs ? SNAP_DEV_BAD_SLOT : SNAP_DEV_BAD_PAGE);
      t = to;
      continue;
    }
    const int in_group = (int)(row % (unsigned)G);
    if (!begins && in_group) { t = (int)min((long long)to, (long long)t + (G - in_group)); continue; }
    bool again = false;                                                  // the slot was listed before
    if (few) again = __any_sync(0xffffffffu, lane < i && my_slot == slot);
    else {
      for (int x = tid; x < i; x += ANT) again = again || r.slots[x] == slot;
      again = __syncthreads_or(again);
    }
    if (again) {
      if (begins && tid == 0 && y == 0 && r.status) atomicOr(r.status, SNAP_DEV_BAD_SLOT);
      t = to;
      continue;
    }
    const int n = min(G - in_group, to - t);                             // the run: rows [row, row + n), tokens from t on
    const int in_block = (int)(row % (unsigned)B), n_blocks = (in_block + n - 1) / B + 1;
    int page = -1, off = 0;                                              // of block tid
    if (tid < n_blocks) {
      const unsigned begin = row - in_block + (unsigned)tid * B, pg = begin / (unsigned)pm.page;
      off = (int)(begin - pg * pm.page);
      if (pg < (unsigned)pm.max_pages) page = pm.table[(long long)slot * pm.max_pages + pg];
    }
    const auto angles = [&](int s0, int rows) {
      for (int z = angle_z; angle_z < apart && z < rows; z += apart) {
        const float2 cs = cos_sin(a.positions ? a.positions[t + s0 + z] : (int)(row + s0 + z), freq);
        table[z * half + angle] = make_float2(cs.x * a.magnitude, cs.y * a.magnitude);
      }
    };
    angles(0, min(SLAB, n));                                             // while the table answers
    if (tid < n_blocks) {
      if (!index_ok(off / B, r.map.blocks, r.status) || page < 0 || page >= pm.n_pages) {
        page = -1;
        if (y == 0 && r.status) atomicOr(r.status, SNAP_DEV_BAD_PAGE);
      }
      page_s[tid] = page; blk_s[tid] = off / B; begin_s[tid] = off;
    }
    // The whole warp: the scales of head h's blocks, lane b knowing the largest of the new numbers of block b; 1 / scale for lane b, or -scale of
    // a block that keeps one which is no power of two: there 1 / scale is rounded, and numbers have to be divided.
    bool uneven = false;
    const auto scale_of = [&](bool keys, int h, float largest) {
      const bool mine = lane < n_blocks && page_s[min(lane, SLAB - 1)] >= 0;
      const float need = exp2_of(scale_exponent(keys ? largest * a.growth : largest));
      float* place = nullptr;
      float scale = need, ratio = 1.f;
      if (mine) place = (keys ? r.k_scales : r.v_scales) + ((long long)page_s[lane] * r.Hkv + h) * r.map.blocks + blk_s[lane];
      if (mine && lane == 0 && begins && in_block > 0) {                 // rows of the sequence are there already
        const float old = *place;
        if (need <= old) scale = old;
        else ratio = old / need;
      }
      ratio = __shfl_sync(0xffffffffu, ratio, 0);
      if (ratio != 1.f) {                                                // they move to the new scale
        uint8_t* codes = keys ? r.k_pages + page_s[0] * pm.kp + h * pm.kh + begin_s[0] * pm.kr : r.v_pages + page_s[0] * pm.vp + h * pm.vh + begin_s[0] * pm.vr;
        const long long stride = keys ? pm.kr : pm.vr;
        const int words = (keys ? r.d_qk : r.d_v) / 4;
        for (int z = 0; z < in_block; ++z)
          for (int c = lane; c < words; c += 32) {
            uint32_t* at = reinterpret_cast<uint32_t*>(codes + z * stride) + c;
            const float2 f0 = floats_of_codes(*at & 0xffffu), f1 = floats_of_codes(*at >> 16);
            *at = codes_of_floats(product_to_odd(f0.x, ratio), product_to_odd(f0.y, ratio)) |
                  codes_of_floats(product_to_odd(f1.x, ratio), product_to_odd(f1.y, ratio)) << 16;   // (rounded once, whatever the old scale)
          }
      }
      if (mine) *place = scale;
      if ((__float_as_uint(scale) & 0x7fffffu) == 0) return 1.f / scale;
      uneven = true;
      return -scale;
    };
    __syncthreads();
    // ---- scales, and the codes of values: pairs of neighbouring vectors ----
    for (int task = w; task < 2 * nk; task += ANW) {
      const bool keys = task < nk;
      const Lanes& l = keys ? lk : lv;
      const int hi = keys ? task : task - nk, h = y + ny * hi, passes = (n + l.rpp - 1) / l.rpp;
      const long long tok = keys ? a.k_tok : a.v_tok;
      const T* src = static_cast<const T*>(keys ? a.k : a.v) + t * tok + h * (keys ? a.k_head : a.v_head) + l.j * 2 * EV;
      if (lane < SLAB) big_s[w][lane] = 0u;
      __syncwarp();
      float big = 0.f;
      VV va[HOLD], vb[HOLD];
      const auto row_of = [&](int k) { return l.r0 + k * l.rpp; };
      const auto there = [&](int k) { return l.r0 + k * l.rpp < n; };   // (also false past the last pass)
      const auto load = [&](int k, VV& x, VV& z) {
        const T* p = src + row_of(k) * tok;
        x.raw = *reinterpret_cast<const uint4*>(p);
        z.raw = *reinterpret_cast<const uint4*>(p + EV);
      };
      const auto block_of = [&](int z) { return n_blocks > 1 ? (in_block + z) / B : 0; };
      for (int k0 = (passes - 1) / HOLD * HOLD; k0 >= 0; k0 -= HOLD) {   // the first HOLD last: they stay
#pragma unroll
        for (int u = 0; u < HOLD; ++u)
          if (there(k0 + u)) load(k0 + u, va[u], vb[u]);
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
          if (!there(k0 + u)) continue;
          const float m = fmaxf(largest_of(va[u]), largest_of(vb[u]));
          if (n_blocks > 1) atomicMax(&big_s[w][block_of(row_of(k0 + u))], __float_as_uint(m));
          else big = fmaxf(big, m);
        }
      }
      __syncwarp();
      if (n_blocks > 1) big = __uint_as_float(big_s[w][min(lane, SLAB - 1)]);
      else big = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(big)));
      const float inv = scale_of(keys, h, big);
      if (lane < n_blocks) (keys ? inv_k + hi * L.blocks : inv_s[w])[lane] = inv;
      __syncwarp();
      const bool as_is = !keys || half == 0;                             // (keys that are not rotated are rounded as values are)
      uint8_t* const codes = keys ? r.k_pages + h * pm.kh : r.v_pages + h * pm.vh;
      const long long page_stride = keys ? pm.kp : pm.vp, row_stride = keys ? pm.kr : pm.vr;
      for (int k0 = 0; as_is && k0 < passes; k0 += HOLD) {
        if (k0 > 0)
#pragma unroll
          for (int u = 0; u < HOLD; ++u)
            if (there(k0 + u)) load(k0 + u, va[u], vb[u]);
#pragma unroll
        for (int u = 0; u < HOLD; ++u) {
          if (!there(k0 + u)) continue;
          const int z = row_of(k0 + u), b = block_of(z), page = page_s[b];
          if (page < 0) continue;
          const float f = (keys ? inv_k + hi * L.blocks : inv_s[w])[b];
          uint8_t* c = codes + page * page_stride + (begin_s[b] + in_block + z - b * B) * row_stride + l.j * 2 * EV;
          if (f < 0.f) {
#pragma unroll 1
            for (int e = 0; e < 2 * EV; ++e) c[e] = (uint8_t)codes_of_floats(quotient_to_odd(to_f32<T>(src[z * tok + e]), -f), 0.f);
            continue;
          }
          uint32_t o[EV / 2];
#pragma unroll
          for (int e = 0; e < EV / 4; ++e) {
            o[e] = codes_of_floats(to_f32<T>(va[u].e[4 * e]) * f, to_f32<T>(va[u].e[4 * e + 1]) * f) |
                   codes_of_floats(to_f32<T>(va[u].e[4 * e + 2]) * f, to_f32<T>(va[u].e[4 * e + 3]) * f) << 16;
            o[EV / 4 + e] = codes_of_floats(to_f32<T>(vb[u].e[4 * e]) * f, to_f32<T>(vb[u].e[4 * e + 1]) * f) |
                            codes_of_floats(to_f32<T>(vb[u].e[4 * e + 2]) * f, to_f32<T>(vb[u].e[4 * e + 3]) * f) << 16;
          }
          if constexpr (EV == 8) *reinterpret_cast<uint4*>(c) = make_uint4(o[0], o[1], o[EV / 2 - 2], o[EV / 2 - 1]);
          else *reinterpret_cast<uint2*>(c) = make_uint2(o[0], o[1]);
        }
      }
    }
    // ---- keys and queries, SLAB rows at a time ----
    for (int s0 = 0; s0 < n && (half > 0 || a.q || a.k_out); s0 += SLAB) {
      const int rows = min(SLAB, n - s0);
      if (s0 > 0) angles(s0, rows);
      if (__syncthreads_or(uneven) && s0 == 0 && half > 0) {             // (the keys' scales are there as well)
        // keys of the first block on a scale that is no power of two: nobody below writes their codes
        const int d = r.d_qk, there = min(n, B - in_block);
#pragma unroll 1
        for (int hi = 0; hi < nk; ++hi) {
          const float scale = -inv_k[hi * L.blocks];
          if (scale <= 0.f) continue;
          const int h = y + ny * hi;
#pragma unroll 1
          for (int x = tid; x < there * d; x += ANT) {
            const int z = x / d, c = x - z * d, at = c - a.offset;
            const T* k = static_cast<const T*>(a.k) + (long long)(t + z) * a.k_tok + h * a.k_head;
            float v = to_f32<T>(k[c]);
            if (at >= 0 && at < a.rot) {
              const int j = INTER ? at / 2 : at % half;
              const bool second = INTER ? at % 2 : at >= half;
              const float other = to_f32<T>(k[second ? c - (INTER ? 1 : half) : c + (INTER ? 1 : half)]);
              const float2 cs = cos_sin(a.positions ? a.positions[t + z] : (int)(row + z), a.freqs[j]);
              const float co = cs.x * a.magnitude, si = cs.y * a.magnitude;
              v = second ? fmaf(v, co, other * si) : fmaf(v, co, -(other * si));
            }
            r.k_pages[page_s[0] * pm.kp + h * pm.kh + (begin_s[0] + in_block + z) * pm.kr + c] = (uint8_t)codes_of_floats(quotient_to_odd(v, scale), 0.f);
          }
        }
        __syncthreads();                                                 // (the rotated keys may be written over these)
      }
      // threads as [rows][heads][items]: as many rows at once as there are, unless that leaves threads over
      int Z = 1;
      while (Z < rows && 2 * Z <= per) Z *= 2;
      while (Z > 1 && 8 * (per / Z * Z) < 7 * per) Z /= 2;
      const int Y = per / Z, ty = tq % Y;
      for (int z = tq / Y; z < rows; z += Z) {
        if (tq >= Y * Z) break;                                          // (a spare thread)
        const int b = n_blocks > 1 ? (in_block + s0 + z) / B : 0, page = page_s[b];
        if (page < 0) continue;
        const long long tk = t + s0 + z;
        const T* q = static_cast<const T*>(a.q) + tk * a.q_tok;
        const T* k = static_cast<const T*>(a.k) + tk * a.k_tok;
        T* q_out = static_cast<T*>(a.q_out) + tk * r.Hq * r.d_qk;
        T* k_out = a.k_out ? static_cast<T*>(a.k_out) + tk * r.Hkv * r.d_qk : nullptr;
        uint8_t* codes = r.k_pages + page * pm.kp + (begin_s[b] + in_block + s0 + z - b * B) * pm.kr;
        for (int j = tx; j < L.ni; j += L.X) {
          const bool turn = j < L.nj;
          const auto other = [&](int c) { return c * V < a.offset ? c * V : c * V + a.rot; };
          const int at_a = turn ? a.offset + (INTER ? 2 * j * V : j * V) : other(2 * (j - L.nj));
          const int at_b = turn ? at_a + (INTER ? V : half) : other(2 * (j - L.nj) + 1);
          float2 cs[V];
          if (turn) {
#pragma unroll
            for (int e = 0; e < V; ++e) cs[e] = table[z * half + j * V + e];
          }
          const auto source = [&](int h) { return h < nq ? q + (y + ny * h) * a.q_head : k + (y + ny * (h - nq)) * a.k_head; };
          // Heads at a time.  (bf16, 26003 tokens: 4 140 us, 3 145, 2 155; single precision, 4099 tokens: 4 13.6, 2 11.6.)
          constexpr int U = sizeof(T) == 4 ? 2 : 4;
          for (int h0 = ty; h0 < nq + nk; h0 += U * Y) {
            VT va[U], vb[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (h0 + u * Y < nq + nk) {
                const T* s = source(h0 + u * Y);
                va[u].raw = *reinterpret_cast<const decltype(VT::raw)*>(s + at_a);
                vb[u].raw = *reinterpret_cast<const decltype(VT::raw)*>(s + at_b);
              }
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int h = h0 + u * Y;
              if (h >= nq + nk) break;
              float fa[V], fb[V];
#pragma unroll
              for (int e = 0; e < V; ++e) { fa[e] = to_f32<T>(va[u].e[e]); fb[e] = to_f32<T>(vb[u].e[e]); }
              if (turn) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                  // interleaved: the item's 2 V elements are V neighbouring pairs, else pair e is (fa[e], fb[e])
                  float& p = INTER ? (2 * e < V ? fa[(2 * e) % V] : fb[(2 * e) % V]) : fa[e];
                  float& s = INTER ? (2 * e + 1 < V ? fa[(2 * e + 1) % V] : fb[(2 * e + 1) % V]) : fb[e];
                  const float p1 = fmaf(p, cs[e].x, -(s * cs[e].y)), s1 = fmaf(s, cs[e].x, p * cs[e].y);
                  p = p1; s = s1;
                }
              }
              const bool query = h < nq;
              const int head = y + ny * (query ? h : h - nq);
              T* o = query ? q_out + head * r.d_qk : k_out ? k_out + head * r.d_qk : nullptr;
              if (o) {
#pragma unroll
                for (int e = 0; e < V; ++e) { va[u].e[e] = from_f32<T>(fa[e]); vb[u].e[e] = from_f32<T>(fb[e]); }
                *reinterpret_cast<decltype(VT::raw)*>(o + at_a) = va[u].raw;
                *reinterpret_cast<decltype(VT::raw)*>(o + at_b) = vb[u].raw;
              }
              if (!query && half > 0) {
                const float f = inv_k[(h - nq) * L.blocks + b];
                uint8_t* c = codes + head * pm.kh;
                if (f > 0.f) {
                  put_codes<V>(c + at_a, fa, f);
                  put_codes<V>(c + at_b, fb, f);
                }
              }
            }
          }
        }
      }
      __syncthreads();
    }
    __syncthreads();                                                     // what the run's blocks are has been read
    if (t + n == to && y == 0 && tid == 0 && index_ok(slot, r.max_seqs, r.status)) a.seq_len[slot] = (int)min((long long)row + n, (long long)pm.cap);
    t += n;
  }
}

// ---- gather: a CTA per CHUNK tokens ----
// What a token's numbers need of it comes first (page and row, as offsets); then a thread takes a vector of a head, of every token:
// nothing is divided on the way.  32768 rows of 8 KV heads of 128 dims 46 us for 201 MB, 4.4 TB/s (67 % of the copy rate: a lane's two stores lie
// 16 bytes apart, so that each covers half of its sectors); with divisions on the way 66.  A call of few rows is three dependent reads
// and a launch: 23 sequences of single precision 4.2 us.
constexpr int CHUNK = 16;
struct GatherLaunch {
  Q8GatherArgs a;
  int chunk, k_items, items, lanes;             // tokens of a CTA; 16-code pieces of a token's keys, of both; threads on a token
};

template <typename T>
__global__ void __launch_bounds__(NT, 6) q8_gather_kernel(const __grid_constant__ GatherLaunch L) {
  const Q8GatherArgs& a = L.a;
  const Q8Rows& r = a.r;
  const PageMap& pm = r.map.pages;
  __shared__ long long k_s[CHUNK], v_s[CHUNK], scale_s[CHUNK];           // of each token: its row's offsets, its block's scale (-1: left as it is)
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, t0 = blockIdx.x * L.chunk, n = min(L.chunk, r.n_tokens - t0);
  constexpr int EV = 16 / (int)sizeof(T);
  pdl_wait();
  for (int z = w; z < n; z += NW) {
    const int t = t0 + z, i = entry_of(r, t);
    int page = -1, off = 0;
    if (i >= 0 && i < r.n_seqs) {
      const int slot = r.slots[i], first = r.first[i];
      unsigned bad = 0;
      if (slot >= 0 && slot < r.max_seqs) {
        const unsigned row = (unsigned)first + (unsigned)(t - r.cu[i]);
        if (first >= 0 && row < (unsigned)pm.cap) {
          const int pg = (int)(row / (unsigned)pm.page);
          page = pm.table[(long long)slot * pm.max_pages + pg];
          off = (int)row - pg * pm.page;
        }
        if (page < 0 || page >= pm.n_pages) { page = -1; bad = SNAP_DEV_BAD_PAGE; }
      } else if (slot != -1) {
        bad = SNAP_DEV_BAD_SLOT;
      }
      if (bad && lane == 0 && r.status) atomicOr(r.status, bad);
    }
    if (lane == 0) {
      k_s[z] = page * pm.kp + off * pm.kr;
      v_s[z] = page * pm.vp + off * pm.vr;
      scale_s[z] = page < 0 ? -1 : (long long)page * r.Hkv * r.map.blocks + off / r.map.block;
    }
  }
  __syncthreads();
  const int z0 = tid / L.lanes, step = NT / L.lanes;
  if (z0 >= step) return;
  for (int x = tid - z0 * L.lanes; x < L.items; x += L.lanes) {
    const bool keys = x < L.k_items;
    const int per = (keys ? r.d_qk : r.d_v) / 16, at = keys ? x : x - L.k_items, h = at / per, c = (at - h * per) * 16;
    const uint8_t* codes = (keys ? r.k_pages + h * pm.kh : r.v_pages + h * pm.vh) + c;
    const float* scales = (keys ? r.k_scales : r.v_scales) + h * r.map.blocks;
    const long long tok = keys ? a.k_tok : a.v_tok;
    const long long* offset = keys ? k_s : v_s;
    T* out = (keys ? static_cast<T*>(a.k) + h * a.k_head : static_cast<T*>(a.v) + h * a.v_head) + t0 * tok + c;
    // Tokens at a time, six blocks on an SM.  (Four, as many blocks as that leaves: large calls as long, 23 sequences of single precision 5.9
    // us instead of 4.2; one, eight blocks: 32768 rows 48.7 instead of 46.0.)
    constexpr int U = 2;
    for (int z = z0; z < n; z += U * step) {
      uint4 in[U];
      float f[U];
      bool there[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int zu = z + u * step;
        const long long at_scale = zu < n ? scale_s[zu] : -1;
        there[u] = at_scale >= 0;
        if (there[u]) {
          f[u] = scales[at_scale];
          in[u] = *reinterpret_cast<const uint4*>(codes + offset[zu]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!there[u]) continue;
        const uint32_t words[4] = {in[u].x, in[u].y, in[u].z, in[u].w};
        T* to = out + (z + u * step) * tok;
        if (sizeof(T) == 2 && (__float_as_uint(f[u]) & 0x7fffffu)) {     // a product of more bits than single precision has
          const uint8_t* again = codes + offset[z + u * step];
#pragma unroll 1
          for (int e = 0; e < 16; ++e) to[e] = from_f32<T>(product_to_odd(floats_of_codes(again[e]).x, f[u]));
          continue;
        }
#pragma unroll
        for (int v = 0; v < 16 / EV; ++v) {
          Vec<T, EV> o;
#pragma unroll
          for (int e = 0; e < EV / 4; ++e) {
            const uint32_t word = words[v * (EV / 4) + e];
            const float2 f0 = floats_of_codes(word & 0xffffu), f1 = floats_of_codes(word >> 16);
            o.e[4 * e] = from_f32<T>(f0.x * f[u]); o.e[4 * e + 1] = from_f32<T>(f0.y * f[u]);
            o.e[4 * e + 2] = from_f32<T>(f1.x * f[u]); o.e[4 * e + 3] = from_f32<T>(f1.y * f[u]);
          }
          *reinterpret_cast<uint4*>(to + v * EV) = o.raw;
        }
      }
    }
  }
}

template <typename T, int V>
cudaError_t launch_append_v(const Q8AppendArgs& a, cudaStream_t st) {
  AppendLaunch L;
  L.a = a;
  const Q8Rows& r = a.r;
  L.nj = a.rot / 2 / V;
  L.ni = L.nj + (r.d_qk - a.rot) / V / 2;
  const int B = r.map.block;
  L.blocks = B < SLAB ? SLAB / B : 1;
  L.group = B * L.blocks;
  L.X = L.ni < 64 ? L.ni : 64;
  const int mean = r.n_tokens / r.n_seqs;
  L.chunk = mean < 1 ? 1 : mean < L.group ? mean : L.group;
  // few tokens: several CTAs to a token's heads
  const long long ctas = ((long long)r.n_tokens + L.chunk - 1) / L.chunk;
  int ny = (int)(4LL * sm_count() / ctas);
  ny = ny < 1 ? 1 : ny > r.Hkv ? r.Hkv : ny;
  const int most = 4096 / L.blocks;                                      // (scales of a CTA's heads in shared memory)
  if (ny < (r.Hkv + most - 1) / most) ny = (r.Hkv + most - 1) / most;
  const size_t smem = SLAB * (size_t)(a.rot / 2) * sizeof(float2) + (size_t)L.blocks * ((r.Hkv + ny - 1) / ny) * sizeof(float);
  auto kernel = a.interleaved ? q8_append_kernel<T, V, true> : q8_append_kernel<T, V, false>;
  const cudaError_t e = launch_pdl(kernel, dim3((unsigned)ctas, (unsigned)ny), dim3(ANT), smem, st, L);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// V: the widest vector (16 bytes at most) that neither the rotated part's start nor its half cuts.
cudaError_t launch_q8_append(int dtype, const Q8AppendArgs& a, cudaStream_t st) {
  const int g = a.rot ? (a.offset | (a.rot / 2)) : 16;
  if (dtype == SNAP_F32) {
    if (g % 4 == 0) return launch_append_v<float, 4>(a, st);
    if (g % 2 == 0) return launch_append_v<float, 2>(a, st);
    return launch_append_v<float, 1>(a, st);
  }
  if (g % 8 == 0) return launch_append_v<__nv_bfloat16, 8>(a, st);
  if (g % 4 == 0) return launch_append_v<__nv_bfloat16, 4>(a, st);
  if (g % 2 == 0) return launch_append_v<__nv_bfloat16, 2>(a, st);
  return launch_append_v<__nv_bfloat16, 1>(a, st);
}

cudaError_t launch_q8_gather(int dtype, const Q8GatherArgs& a, cudaStream_t st) {
  const int sms = sm_count();
  GatherLaunch L;
  L.a = a;
  L.k_items = a.r.Hkv * (a.r.d_qk / 16);
  L.items = L.k_items + a.r.Hkv * (a.r.d_v / 16);
  L.lanes = L.items < NT ? L.items : NT;
  // (few tokens: spread over the GPU)
  L.chunk = CHUNK;
  while (L.chunk > 4 && (a.r.n_tokens + L.chunk - 1) / L.chunk < 4 * sms) L.chunk /= 2;
  const dim3 grid((unsigned)((a.r.n_tokens + L.chunk - 1) / L.chunk));
  const cudaError_t e = dtype == SNAP_F32 ? launch_pdl(q8_gather_kernel<float>, grid, dim3(NT), 0, st, L)
                                          : launch_pdl(q8_gather_kernel<__nv_bfloat16>, grid, dim3(NT), 0, st, L);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
