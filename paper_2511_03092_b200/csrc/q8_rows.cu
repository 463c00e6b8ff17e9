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

constexpr int NT = 256, NW = NT / 32;
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

struct AppendLaunch { Q8AppendArgs a; int group, chunk, nj, ni, nhk, nhq; };   // rows of a group, tokens of a CTA; items of a head; heads of a CTA at most

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
// gridDim.y-th.
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(NT) q8_append_kernel(const __grid_constant__ AppendLaunch L) {
  const Q8AppendArgs& a = L.a;
  const Q8Rows& r = a.r;
  const PageMap& pm = r.map.pages;
  const int B = r.map.block, G = L.group;
  extern __shared__ float2 table[];                                      // [SLAB][rot / 2], then the blocks' scales
  float* inv = reinterpret_cast<float*>(table + SLAB * (a.rot / 2));     // [blocks of a group][2 nhk]: 1 / scale of keys, of values
  __shared__ int page_s[SLAB];                                           // of each block, -1: skipped
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, y = blockIdx.y, ny = gridDim.y;
  const int nk = (r.Hkv - y + ny - 1) / ny, nq = r.Hq > y ? (r.Hq - y + ny - 1) / ny : 0, half = a.rot / 2;
  constexpr int EV = 16 / (int)sizeof(T);
  using VT = Vec<T, V>;
  pdl_wait();
  const int t0 = blockIdx.x * L.chunk, t1 = min(t0 + L.chunk, r.n_tokens);
  for (int t = t0; t < t1;) {
    const int i = entry_of(r, t);
    if (i >= r.n_seqs) break;
    if (i < 0) { t = min(max(r.cu[0], t + 1), t1); continue; }
    const int from = r.cu[i], to = min(r.cu[i + 1], r.n_tokens), slot = r.slots[i], first = r.first[i];
    if (from > t || to <= t) { ++t; continue; }                          // (sums that decrease: go on all the same)
    const long long row = (long long)first + (t - from);
    const bool begins = t == from;
    if (slot < 0 || slot >= r.max_seqs || first < 0) {
      if (begins && tid == 0 && y == 0 && slot != -1 && r.status)
        atomicOr(r.status, slot < 0 || slot >= r.max_seqs ? SNAP_DEV_BAD_SLOT : SNAP_DEV_BAD_PAGE);
      t = to;
      continue;
    }
    if (!begins && row % G) { t = (int)min((long long)to, t + (G - row % G)); continue; }
    int again = 0;                                                       // the slot was listed before
    for (int x = tid; x < i; x += NT) again |= r.slots[x] == slot;
    if (__syncthreads_or(again)) {
      if (begins && tid == 0 && y == 0 && r.status) atomicOr(r.status, SNAP_DEV_BAD_SLOT);
      t = to;
      continue;
    }
    const int n = (int)min(G - row % G, (long long)(to - t));            // the run: rows [row, row + n), tokens from t on
    const long long block0 = row / B;
    const int n_blocks = (int)((row + n - 1) / B - block0) + 1;
    if (tid < n_blocks) {
      const long long pg = (block0 + tid) * B / pm.page;
      int page = -1;
      if (pg < pm.max_pages) page = pm.table[(long long)slot * pm.max_pages + pg];
      if (page < 0 || page >= pm.n_pages) {
        page = -1;
        if (y == 0 && r.status) atomicOr(r.status, SNAP_DEV_BAD_PAGE);
      }
      page_s[tid] = page;
    }
    __syncthreads();
    // ---- scales: a warp for each (block, head, keys or values) ----
    for (int task = w; task < n_blocks * 2 * nk; task += NW) {
      const int b = task / (2 * nk), j = task % (2 * nk), kvh = y + ny * (j >> 1), page = page_s[b];
      if (page < 0) continue;
      const bool keys = (j & 1) == 0;
      const int d = keys ? r.d_qk : r.d_v;
      const long long begin = (block0 + b) * B, lo = max(begin, row), hi = min(begin + B, row + n);
      const long long tok = keys ? a.k_tok : a.v_tok;
      const T* src = static_cast<const T*>(keys ? a.k : a.v) + (t + (lo - row)) * tok + kvh * (keys ? a.k_head : a.v_head);
      float big = 0.f;
      const int per = d / EV, total = (int)(hi - lo) * per;
#pragma unroll 4
      for (int x = lane; x < total; x += 32) {
        Vec<T, EV> v;
        v.raw = *reinterpret_cast<const uint4*>(src + x / per * tok + x % per * EV);
#pragma unroll
        for (int e = 0; e < EV; ++e) big = fmaxf(big, fabsf(to_f32<T>(v.e[e])));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
      float scale = exp2_of(scale_exponent(keys ? big * a.growth : big));
      const int blk = (int)(begin % pm.page) / B;
      float* place = (keys ? r.k_scales : r.v_scales) + ((long long)page * r.Hkv + kvh) * r.map.blocks + blk;
      if (begin < first) {                                               // rows of the sequence are there already
        const float old = *place;
        __syncwarp();
        if (scale <= old) scale = old;
        else {
          const float ratio = old / scale;
          uint8_t* codes = keys ? r.k_pages + page * pm.kp + kvh * pm.kh + begin % pm.page * pm.kr
                                : r.v_pages + page * pm.vp + kvh * pm.vh + begin % pm.page * pm.vr;
          const long long stride = keys ? pm.kr : pm.vr;
          const int each = d / 4;
          for (int x = lane; x < (int)(first - begin) * each; x += 32) {
            uint32_t* c = reinterpret_cast<uint32_t*>(codes + x / each * stride) + x % each;
            const uint32_t v = *c;
            const float2 f0 = floats_of_codes(v & 0xffffu), f1 = floats_of_codes(v >> 16);
            *c = codes_of_floats(f0.x * ratio, f0.y * ratio) | codes_of_floats(f1.x * ratio, f1.y * ratio) << 16;
          }
        }
      }
      if (lane == 0) {
        *place = scale;
        inv[b * 2 * L.nhk + j] = 1.f / scale;
      }
    }
    // ---- rows ----
    for (int s0 = 0; s0 < n; s0 += SLAB) {
      const int rows = min(SLAB, n - s0);
      for (int e = tid; e < rows * half; e += NT) {
        const int z = e / half, pos = a.positions ? a.positions[t + s0 + z] : (int)(row + s0 + z);
        const float2 cs = cos_sin(pos, a.freqs[e - z * half]);
        table[e] = make_float2(cs.x * a.magnitude, cs.y * a.magnitude);
      }
      __syncthreads();
      const auto block_of = [&](int z) { return (int)((row + s0 + z) / B - block0); };
      // queries and keys: two vectors of a head, a part of it that turns or two of its other vectors
      for (int x = tid; x < rows * (nq + nk) * L.ni; x += NT) {
        const int j = x % L.ni, h = x / L.ni % (nq + nk), z = x / L.ni / (nq + nk), b = block_of(z), page = page_s[b];
        if (page < 0) continue;
        const bool turn = j < L.nj, query = h < nq;
        const auto other = [&](int c) { return c * V < a.offset ? c * V : c * V + a.rot; };
        const int at_a = turn ? a.offset + (INTER ? 2 * j * V : j * V) : other(2 * (j - L.nj));
        const int at_b = turn ? at_a + (INTER ? V : half) : other(2 * (j - L.nj) + 1);
        const int head = query ? y + ny * h : y + ny * (h - nq);
        const long long tk = t + s0 + z;
        const T* src = query ? static_cast<const T*>(a.q) + tk * a.q_tok + head * a.q_head : static_cast<const T*>(a.k) + tk * a.k_tok + head * a.k_head;
        VT va, vb;
        va.raw = *reinterpret_cast<const decltype(VT::raw)*>(src + at_a);
        vb.raw = *reinterpret_cast<const decltype(VT::raw)*>(src + at_b);
        float fa[V], fb[V];
#pragma unroll
        for (int e = 0; e < V; ++e) { fa[e] = to_f32<T>(va.e[e]); fb[e] = to_f32<T>(vb.e[e]); }
        if (turn) {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            // interleaved: the item's 2 V elements are V neighbouring pairs, else pair e is (fa[e], fb[e])
            float& p = INTER ? (2 * e < V ? fa[(2 * e) % V] : fb[(2 * e) % V]) : fa[e];
            float& q = INTER ? (2 * e + 1 < V ? fa[(2 * e + 1) % V] : fb[(2 * e + 1) % V]) : fb[e];
            const float2 cs = table[z * half + j * V + e];
            const float p1 = fmaf(p, cs.x, -(q * cs.y)), q1 = fmaf(q, cs.x, p * cs.y);
            p = p1; q = q1;
          }
        }
        T* out = query ? static_cast<T*>(a.q_out) + (tk * r.Hq + head) * r.d_qk : a.k_out ? static_cast<T*>(a.k_out) + (tk * r.Hkv + head) * r.d_qk : nullptr;
        if (out) {
          VT oa, ob;
#pragma unroll
          for (int e = 0; e < V; ++e) { oa.e[e] = from_f32<T>(fa[e]); ob.e[e] = from_f32<T>(fb[e]); }
          *reinterpret_cast<decltype(VT::raw)*>(out + at_a) = oa.raw;
          *reinterpret_cast<decltype(VT::raw)*>(out + at_b) = ob.raw;
        }
        if (!query) {
          const float f = inv[b * 2 * L.nhk + 2 * (h - nq)];
          uint8_t* c = r.k_pages + page * pm.kp + head * pm.kh + (row + s0 + z) % pm.page * pm.kr;
          Vec<uint8_t, V> ca, cb;
          if constexpr (V == 1) {
            ca.e[0] = (uint8_t)codes_of_floats(fa[0] * f, 0.f);
            cb.e[0] = (uint8_t)codes_of_floats(fb[0] * f, 0.f);
          } else {
#pragma unroll
            for (int e = 0; e < V; e += 2) {
              const uint32_t u = codes_of_floats(fa[e] * f, fa[e + 1] * f), v = codes_of_floats(fb[e] * f, fb[e + 1] * f);
              ca.e[e] = (uint8_t)u; ca.e[e + 1] = (uint8_t)(u >> 8);
              cb.e[e] = (uint8_t)v; cb.e[e + 1] = (uint8_t)(v >> 8);
            }
          }
          *reinterpret_cast<decltype(ca.raw)*>(c + at_a) = ca.raw;
          *reinterpret_cast<decltype(cb.raw)*>(c + at_b) = cb.raw;
        }
      }
      // values: 16 bytes at a time
      const int per = r.d_v / EV;
      for (int x = tid; x < rows * nk * per; x += NT) {
        const int c = x % per, h = x / per % nk, z = x / per / nk, b = block_of(z), page = page_s[b], head = y + ny * h;
        if (page < 0) continue;
        Vec<T, EV> v;
        v.raw = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + (long long)(t + s0 + z) * a.v_tok + head * a.v_head + c * EV);
        const float f = inv[b * 2 * L.nhk + 2 * h + 1];
        uint32_t o[EV / 4];
#pragma unroll
        for (int e = 0; e < EV / 4; ++e)
          o[e] = codes_of_floats(to_f32<T>(v.e[4 * e]) * f, to_f32<T>(v.e[4 * e + 1]) * f) |
                 codes_of_floats(to_f32<T>(v.e[4 * e + 2]) * f, to_f32<T>(v.e[4 * e + 3]) * f) << 16;
        uint8_t* to_ = r.v_pages + page * pm.vp + head * pm.vh + (row + s0 + z) % pm.page * pm.vr + c * EV;
        if constexpr (EV == 8) *reinterpret_cast<uint2*>(to_) = make_uint2(o[0], o[1]);
        else *reinterpret_cast<uint32_t*>(to_) = o[0];
      }
      __syncthreads();
    }
    if (t + n == to && y == 0 && tid == 0) a.seq_len[slot] = (int)min(row + n, (long long)pm.cap);
    t += n;
  }
}

// ---- gather: a CTA per SLAB tokens ----
template <typename T>
__global__ void __launch_bounds__(NT) q8_gather_kernel(const __grid_constant__ Q8GatherArgs a) {
  const Q8Rows& r = a.r;
  const PageMap& pm = r.map.pages;
  __shared__ int2 place[SLAB];                                           // page (-1: left as it is) and row of the page
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, t0 = blockIdx.x * SLAB;
  constexpr int EV = 16 / (int)sizeof(T);
  pdl_wait();
  for (int z = w; z < SLAB; z += NW) {
    const int t = t0 + z, i = t < r.n_tokens ? entry_of(r, t) : -1;
    int page = -1, off = 0;
    if (i >= 0 && i < r.n_seqs) {
      const int slot = r.slots[i], first = r.first[i];
      unsigned bad = 0;
      if (slot >= 0 && slot < r.max_seqs) {
        const long long row = (long long)first + (t - r.cu[i]);
        if (first >= 0 && row < pm.cap) {
          page = pm.table[(long long)slot * pm.max_pages + row / pm.page];
          off = (int)(row % pm.page);
        }
        if (page < 0 || page >= pm.n_pages) { page = -1; bad = SNAP_DEV_BAD_PAGE; }
      } else if (slot != -1) {
        bad = SNAP_DEV_BAD_SLOT;
      }
      if (bad && lane == 0 && r.status) atomicOr(r.status, bad);
    }
    if (lane == 0) place[z] = make_int2(page, off);
  }
  __syncthreads();
  const auto copy = [&](const uint8_t* pages, long long ps, long long hs, long long rs, const float* scales, int d, T* out, long long tok, long long head) {
    const int per = d / EV;
    for (int x = tid; x < SLAB * r.Hkv * per; x += NT) {
      const int c = x % per, h = x / per % r.Hkv, z = x / per / r.Hkv;
      const int2 p = place[z];
      if (p.x < 0) continue;
      const uint8_t* src = pages + p.x * ps + h * hs + p.y * rs + c * EV;
      const float f = scales[((long long)p.x * r.Hkv + h) * r.map.blocks + p.y / r.map.block];
      uint32_t in[EV / 4];
      if constexpr (EV == 8) { const uint2 v = *reinterpret_cast<const uint2*>(src); in[0] = v.x; in[1] = v.y; }
      else in[0] = *reinterpret_cast<const uint32_t*>(src);
      Vec<T, EV> o;
#pragma unroll
      for (int e = 0; e < EV / 4; ++e) {
        const float2 f0 = floats_of_codes(in[e] & 0xffffu), f1 = floats_of_codes(in[e] >> 16);
        o.e[4 * e] = from_f32<T>(f0.x * f); o.e[4 * e + 1] = from_f32<T>(f0.y * f);
        o.e[4 * e + 2] = from_f32<T>(f1.x * f); o.e[4 * e + 3] = from_f32<T>(f1.y * f);
      }
      *reinterpret_cast<uint4*>(out + (t0 + z) * tok + h * head + c * EV) = o.raw;
    }
  };
  copy(r.k_pages, pm.kp, pm.kh, pm.kr, r.k_scales, r.d_qk, static_cast<T*>(a.k), a.k_tok, a.k_head);
  copy(r.v_pages, pm.vp, pm.vh, pm.vr, r.v_scales, r.d_v, static_cast<T*>(a.v), a.v_tok, a.v_head);
}

template <typename T, int V>
cudaError_t launch_append_v(const Q8AppendArgs& a, cudaStream_t st) {
  AppendLaunch L;
  L.a = a;
  const Q8Rows& r = a.r;
  L.nj = a.rot / 2 / V;
  L.ni = L.nj + (r.d_qk - a.rot) / V / 2;
  const int B = r.map.block;
  L.group = B * (B < SLAB ? SLAB / B : 1);
  const int mean = r.n_tokens / r.n_seqs;
  L.chunk = mean < 1 ? 1 : mean < L.group ? mean : L.group;
  // few tokens: several CTAs to a token's heads
  const long long ctas = (r.n_tokens + L.chunk - 1) / L.chunk;
  int ny = (int)(2LL * sm_count() / ctas);
  ny = ny < 1 ? 1 : ny > r.Hkv ? r.Hkv : ny;
  L.nhk = (r.Hkv + ny - 1) / ny;
  L.nhq = (r.Hq + ny - 1) / ny;
  const size_t smem = SLAB * (size_t)(a.rot / 2) * sizeof(float2) + (size_t)(L.group / B) * 2 * L.nhk * sizeof(float);
  auto kernel = a.interleaved ? q8_append_kernel<T, V, true> : q8_append_kernel<T, V, false>;
  static SmemLimit limit[2] = {};
  if (smem > 48 * 1024)
    if (cudaError_t e = ensure_dyn_smem(kernel, smem, limit[a.interleaved])) return e;
  const cudaError_t e = launch_pdl(kernel, dim3((unsigned)ctas, (unsigned)ny), dim3(NT), smem, st, L);
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
  const dim3 grid((unsigned)((a.r.n_tokens + SLAB - 1) / SLAB));
  const cudaError_t e = dtype == SNAP_F32 ? launch_pdl(q8_gather_kernel<float>, grid, dim3(NT), 0, st, a)
                                          : launch_pdl(q8_gather_kernel<__nv_bfloat16>, grid, dim3(NT), 0, st, a);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
