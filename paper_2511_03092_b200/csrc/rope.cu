// Rotary positions of queries and keys, and the same pass with the keys and values going to the pages of a
// paged cache (snap_rope, snap_paged_append).
//
// Pair i of a head turns by the angle position * f_i: (a, b) -> m (a cos - b sin, b cos + a sin).  The angle and
// its reduction to one turn are in double precision (at position 10^6 a single-precision angle is off by up to
// 0.03), the sine and cosine of the reduced angle in single with its rounding to single put back to first order,
// the rotation in single, and the result is rounded once.
//
// A pass reads and writes every element once and computes next to nothing, so memory bounds it.  A thread keeps
// the cosines and sines of its V pairs (two 16-byte vectors of a head) in registers and walks over the heads of
// its token; the angles of a token are computed once, by the whole block, and handed over in shared memory.  What
// counts is how many warps are resident, not how much each has in flight: one head at a time and five blocks per SM
// turn a 32768-token prompt of 40 heads of 128 dims in 110 to 114 us by the GPU (6.1 to 5.9 TB/s); where that took 110,
// two heads at a time and four blocks took 113 us, three and three 125, and looping over tokens in as many blocks as fit 124 to
// 144.  Appending 26003 tokens of the same layer (queries, keys twice, values) takes 122 to 126 us (5.7 to 5.5 TB/s).  Threads are
// laid out as [tokens][heads][items of
// a head]: consecutive threads are on consecutive vectors, and few tokens spread over more threads per token.
//
// The kernel after it starts when this one ends, not beside its last blocks: attention over the pages comes next, whose
// blocks fill an SM's registers to the last thousand and would find them in pieces.
#include "snap_internal.cuh"

namespace snap {
namespace {

constexpr int NT = 256;

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { using type = uint4; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<4> { using type = unsigned; };
template <> struct RawOf<2> { using type = unsigned short; };

template <typename T, int V> union Vec {
  typename RawOf<V * (int)sizeof(T)>::type raw;
  T e[V];
  __device__ Vec() {}
};

struct RopeLaunch { RopeArgs a; int nj, ni, nc, X, Y, Z; };   // items of a head that turn, all items, copied vectors; thread layout

// cos and sin of position * f, the angle taken in half turns: its whole turns come off exactly
__device__ __forceinline__ float2 cos_sin(int pos, double f) {
  const double u = (double)pos * f * 0.3183098861837907;                 // 1 / pi
  const double r = fma(-2.0, rint(0.5 * u), u);                          // [-1, 1]
  const float rh = (float)r, rl = (float)(r - (double)rh) * 3.14159265f;
  float s, c;
  sincospif(rh, &s, &c);
  return make_float2(fmaf(-rl, s, c), fmaf(rl, c, s));
}

// Which of a head's dims turn: all that this call moves (of an unpaged call in place, the others stay where they are), some, none.
enum class Turns { ALL, SOME, NONE };
template <typename T, int V, bool INTER, bool PAGED, Turns TURNS>
__global__ void __launch_bounds__(NT, 5) rope_kernel(const __grid_constant__ RopeLaunch L) {
  using VT = Vec<T, V>;
  using Raw = decltype(VT::raw);
  const RopeArgs& a = L.a;
  extern __shared__ float2 table[];                                      // [Z][rot / 2]
  __shared__ int dup[NT];
  __shared__ int2 placed[NT];                                             // slot and row of each of the block's tokens, row -1: skipped
  const int tid = threadIdx.x, x = tid % L.X, y = (tid / L.X) % L.Y, z = tid / (L.X * L.Y);
  const int t = blockIdx.x * L.Z + z, half = a.rot / 2;
  const bool mine = z < L.Z && t < a.n_tokens;                            // the block may have spare threads
  constexpr bool paged = PAGED;
  if (tid < L.Z) dup[tid] = 0;
  pdl_wait();

  // ---- where the token goes ----
  bool skip = !mine;
  int slot = 0, row = 0, page = 0, off = 0;
  unsigned bad = 0;
  if (mine && paged) {
    slot = a.slots[t];
    if (slot < 0 || slot >= a.max_seqs) {
      skip = true;
      bad = slot == -1 ? 0u : SNAP_DEV_BAD_SLOT;
    } else {
      row = a.rows ? a.rows[t] : a.seq_len[slot];
      if (row < 0 || row >= a.map.cap) { skip = true; bad = SNAP_DEV_BAD_PAGE; }
      else {
        off = row % a.map.page;
        if (!index_ok(row / a.map.page, a.map.max_pages, a.status)) page = -1;
        else page = a.map.table[(long long)slot * a.map.max_pages + row / a.map.page];
        if (page < 0 || page >= a.map.n_pages) { skip = true; bad = SNAP_DEV_BAD_PAGE; }
      }
    }
  }
  if (paged && !a.rows) {
    // Listed earlier in this call?  Then it is skipped for that alone: its row is the first one's next, or not, as that one's
    // block ends sooner or later, and with it what the page table would say.
    const bool listed = mine && slot >= 0 && slot < a.max_seqs;
    __syncthreads();                                                      // dup is zero
    if (listed)
      for (int e = tid - z * L.X * L.Y; e < t; e += L.X * L.Y)
        if (a.slots[e] == slot) dup[z] = 1;
    __syncthreads();
    if (listed && dup[z]) { skip = true; bad = SNAP_DEV_BAD_SLOT; }
  }

  const T* q = static_cast<const T*>(a.q) + t * a.q_tok;
  const T* k = static_cast<const T*>(a.k) + t * a.k_tok;
  const int H = a.Hq + a.Hkv;
  const auto source = [&](int h) { return h < a.Hq ? q + h * a.q_head : k + (h - a.Hq) * a.k_head; };
  // Item j of a head: two vectors that turn, or, behind those, two neighbours of the head's other dims (whose number is
  // even: heads are multiples of 16 dims, the part that turns of two vectors).  (All of them in
  // one loop: a head's row is read and written as a whole.  With the other dims copied afterwards 28357 tokens of 51 heads of
  // 64 dims, half of them turned, took 115 us instead of 74.)
  int at_a, at_b;
  bool turn;
  const auto item = [&](int j) {
    turn = TURNS == Turns::ALL || j < L.nj;
    const auto other = [&](int c) { return c * V < a.offset ? c * V : c * V + a.rot; };
    at_a = turn ? a.offset + (INTER ? 2 * j * V : j * V) : other(2 * (j - L.nj));
    at_b = turn ? at_a + (INTER ? V : half) : other(2 * (j - L.nj) + 1);
  };
  VT va, vb;
  const auto load = [&](int h) {
    if (PAGED && !index_ok(slot, a.max_seqs, a.status)) return;
    const T* s = source(h);
    va.raw = *reinterpret_cast<const Raw*>(s + at_a);
    vb.raw = *reinterpret_cast<const Raw*>(s + at_b);
  };
  if (TURNS != Turns::NONE) item(x);
  // on their way while the angles (and a paged token's page) are looked up; a token without a slot is padding and has no rows
  if (TURNS != Turns::NONE && mine && (!PAGED || (slot >= 0 && slot < a.max_seqs)) && x < L.ni && y < H) load(y);

  if (paged && x == 0 && y == 0 && z < L.Z) placed[z] = make_int2(slot, skip ? -1 : row);
  // ---- values: copied to the page while the angles are on their way ----
  if (paged && !skip) {
    const T* v = static_cast<const T*>(a.v) + t * a.v_tok;
    T* vp = static_cast<T*>(a.v_pages) + page * a.map.vp + off * a.map.vr;
    const int n = a.d_v / V;
    for (int h = y; h < a.Hkv; h += L.Y)
      for (int c = x; c < n; c += 2 * L.X) {
        Raw r0, r1;
        r0 = *reinterpret_cast<const Raw*>(v + h * a.v_head + c * V);
        if (c + L.X < n) r1 = *reinterpret_cast<const Raw*>(v + h * a.v_head + (c + L.X) * V);
        *reinterpret_cast<Raw*>(vp + h * a.map.vh + c * V) = r0;
        if (c + L.X < n) *reinterpret_cast<Raw*>(vp + h * a.map.vh + (c + L.X) * V) = r1;
      }
  }

  // ---- the angles of the block's tokens ----
  for (int e = tid; e < L.Z * half; e += NT) {
    const int ez = e / half, et = blockIdx.x * L.Z + ez, i = e - ez * half;
    if (et >= a.n_tokens) break;
    const int es = PAGED ? a.slots[et] : 0;
    int pos = 0;
    if (!PAGED || (es >= 0 && es < a.max_seqs)) {                          // (padding has no position)
      if (!index_ok(es, PAGED ? a.max_seqs : 1, a.status)) pos = 0;
      else if (a.positions) pos = a.positions[et];
      else pos = a.rows ? a.rows[et] : a.seq_len[es];
    }
    const float2 cs = cos_sin(pos, a.freqs[i]);
    table[e] = make_float2(cs.x * a.magnitude, cs.y * (a.magnitude * a.sign));
  }
  __syncthreads();                                                        // everyone has read seq_len
  if (mine && paged && x == 0 && y == 0) {
    if (bad && a.status) atomicOr(a.status, bad);
    if (!skip) {
      // of a run of a sequence's rows the last one speaks for all (thousands of tokens share a length)
      if (a.rows) {
        if (!(z + 1 < L.Z && placed[z + 1].x == slot && placed[z + 1].y > row)) atomicMax(&a.seq_len[slot], row + 1);
      }
      else a.seq_len[slot] = row + 1;                                     // this token alone has the slot
    }
  }
  if (skip) return;

  T* qo = static_cast<T*>(a.q_out) + t * a.qo_tok;
  T* ko = a.k_out ? static_cast<T*>(a.k_out) + t * a.ko_tok : nullptr;
  T* kp = paged ? static_cast<T*>(a.k_pages) + page * a.map.kp + off * a.map.kr : nullptr;
  const auto put = [&](int h, int at, Raw v) {
    if (h < a.Hq) *reinterpret_cast<Raw*>(qo + h * a.qo_head + at) = v;
    else {
      if (ko) *reinterpret_cast<Raw*>(ko + (h - a.Hq) * a.ko_head + at) = v;
      if (kp) *reinterpret_cast<Raw*>(kp + (h - a.Hq) * a.map.kh + at) = v;
    }
  };

  for (int j = x; TURNS != Turns::NONE && j < L.ni; j += L.X) {
    if (j != x) item(j);
    float2 cs[V];
    if (turn) {
#pragma unroll
      for (int i = 0; i < V; ++i) cs[i] = table[z * half + j * V + i];
    }
    for (int h = y; h < H; h += L.Y) {
      if (j != x || h != y) load(h);
      if (turn) {
        VT oa, ob;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          // interleaved: the item's 2 V elements are V neighbouring pairs, else pair i is (va[i], vb[i])
          const float p = to_f32<T>(INTER ? (2 * i < V ? va.e[(2 * i) % V] : vb.e[(2 * i) % V]) : va.e[i]);
          const float r = to_f32<T>(INTER ? (2 * i + 1 < V ? va.e[(2 * i + 1) % V] : vb.e[(2 * i + 1) % V]) : vb.e[i]);
          const T c0 = from_f32<T>(fmaf(p, cs[i].x, -(r * cs[i].y))), c1 = from_f32<T>(fmaf(r, cs[i].x, p * cs[i].y));
          if (INTER) {
            if (2 * i < V) oa.e[(2 * i) % V] = c0; else ob.e[(2 * i) % V] = c0;
            if (2 * i + 1 < V) oa.e[(2 * i + 1) % V] = c1; else ob.e[(2 * i + 1) % V] = c1;
          } else {
            oa.e[i] = c0;
            ob.e[i] = c1;
          }
        }
        if (TURNS == Turns::ALL) {                                         // (through va and vb: 113 instead of 110 us for the prompt above)
          put(h, at_a, oa.raw);
          put(h, at_b, ob.raw);
          continue;
        }
        va = oa;
        vb = ob;
      }
      put(h, at_a, va.raw);
      put(h, at_b, vb.raw);
    }
  }
  // ---- no dims that turn: four heads at a time ----
  for (int c = x; TURNS == Turns::NONE && c < L.nc; c += L.X) {
    for (int h0 = y; h0 < H; h0 += 4 * L.Y) {
      Raw r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h0 + u * L.Y < H) r[u] = *reinterpret_cast<const Raw*>(source(h0 + u * L.Y) + c * V);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (h0 + u * L.Y < H) put(h0 + u * L.Y, c * V, r[u]);
    }
  }
  if (paged) {
    if (a.weights && x == 0 && index_ok(row, a.map.cap, a.status))
      for (int h = y; h < a.Hkv; h += L.Y) a.weights[((long long)slot * a.Hkv + h) * a.map.cap + row] = 0.f;
  }
}

template <typename T, int V>
cudaError_t launch_v(const RopeArgs& a, int sms, cudaStream_t st) {
  RopeLaunch L;
  L.a = a;
  const bool in_place = !a.k_pages && (!a.q || a.q == a.q_out) && (!a.k || a.k == a.k_out);
  L.nj = a.rot / 2 / V;
  L.nc = in_place ? 0 : (a.d_qk - a.rot) / V;
  L.ni = L.nj + L.nc / 2;
  const int items = L.nj > 0 ? L.ni : L.nc;
  L.X = items < 64 ? items : 64;
  const int H = a.Hq + a.Hkv, per = NT / L.X;                             // (token, head) pairs of a block
  // As many threads as there is work for, up to what the GPU holds at once; more work: a thread takes several heads of its
  // token, at most four to eight, so that the angles it reads are used that often, in the split that leaves the fewest
  // threads without one.
  L.Y = H < per ? H : per;
  const long long work = (long long)a.n_tokens * H * L.X, full = (work + 5LL * sms * NT - 1) / (5LL * sms * NT);
  if (full > 1) {
    int best = 0;
    const int least = full < 4 ? (int)full : 4, most = full < 4 ? least + 1 : 8;
    for (int its = most; its >= least; --its) {
      const int Y = (H + its - 1) / its, used = Y <= per ? per / Y * H * 64 / its : 0;   // head slots that do work
      if (used > best) { best = used; L.Y = Y; }
    }
  }
  L.Z = per / L.Y;
  if (L.Z > a.n_tokens) L.Z = a.n_tokens;
  const size_t smem = (size_t)L.Z * (a.rot / 2) * sizeof(float2);        // at most 2048 pairs: X covers them or Z is small
  const dim3 grid((a.n_tokens + L.Z - 1) / L.Z);
  const auto launch = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(NT), smem, st, L); };
  cudaError_t e;
  if (L.nj == 0) e = launch(rope_kernel<T, V, false, true, Turns::NONE>);                  // (an append)
  else if (L.nc == 0 && a.k_pages) e = a.interleaved ? launch(rope_kernel<T, V, true, true, Turns::ALL>) : launch(rope_kernel<T, V, false, true, Turns::ALL>);
  else if (L.nc == 0) e = a.interleaved ? launch(rope_kernel<T, V, true, false, Turns::ALL>) : launch(rope_kernel<T, V, false, false, Turns::ALL>);
  else if (a.k_pages) e = a.interleaved ? launch(rope_kernel<T, V, true, true, Turns::SOME>) : launch(rope_kernel<T, V, false, true, Turns::SOME>);
  else e = a.interleaved ? launch(rope_kernel<T, V, true, false, Turns::SOME>) : launch(rope_kernel<T, V, false, false, Turns::SOME>);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// V: the widest vector (16 bytes at most) that neither the rotated part's start nor its half cuts.
cudaError_t launch_rope(int dtype, const RopeArgs& a, cudaStream_t st) {
  const int sms = sm_count();
  const int g = a.rot ? (a.offset | (a.rot / 2)) : 16;
  if (dtype == SNAP_F32) {
    if (g % 4 == 0) return launch_v<float, 4>(a, sms, st);
    if (g % 2 == 0) return launch_v<float, 2>(a, sms, st);
    return launch_v<float, 1>(a, sms, st);
  }
  if (g % 8 == 0) return launch_v<__nv_bfloat16, 8>(a, sms, st);
  if (g % 4 == 0) return launch_v<__nv_bfloat16, 4>(a, sms, st);
  if (g % 2 == 0) return launch_v<__nv_bfloat16, 2>(a, sms, st);
  return launch_v<__nv_bfloat16, 1>(a, sms, st);
}

}  // namespace snap
