// Attention of the last tokens of each sequence over a cache in pages of 8-bit numbers (snap_paged_q8_decode_attn).
//
// A warp to each (sequence, token, query head): eight dims to a lane, one row after the other, with the running maximum and
// sum of the softmax.
#include "e4m3.cuh"
#include "mma_helpers.cuh"
#include "snap_internal.cuh"

namespace snap {
namespace {

constexpr int NW = 4;

struct Q8Args {
  const void* q; void* out;
  const uint8_t* kp; const uint8_t* vp; const float* ks; const float* vs;
  const int* slots; const int* seq_len;
  int n, q_len, Hq, Hkv, g, d_qk, d_v, max_seqs;
  float scale_log2;
  Q8Map map;
  uint32_t* status;
};

template <typename T>
__global__ void __launch_bounds__(NW * 32) q8_decode_kernel(const __grid_constant__ Q8Args a) {
  const PageMap& pm = a.map.pages;
  const int lane = threadIdx.x & 31;
  const long long id = (long long)blockIdx.x * NW + (threadIdx.x >> 5);
  pdl_wait();
  if (id >= (long long)a.n * a.q_len * a.Hq) return;
  const int h = (int)(id % a.Hq), u = (int)(id / a.Hq % a.q_len), i = (int)(id / a.Hq / a.q_len), kvh = h / a.g, c0 = 8 * lane;
  const int slot = a.slots[i];
  int len = 0;
  unsigned bad = 0;
  if (slot >= 0 && slot < a.max_seqs) {
    len = a.seq_len[slot];
    if (len > pm.cap) { len = pm.cap; bad = SNAP_DEV_BAD_PAGE; }
  } else if (slot != -1) {
    bad = SNAP_DEV_BAD_SLOT;
  }
  float q[8], o[8] = {}, m = -INFINITY, l = 0.f;
  const T* qp = static_cast<const T*>(a.q) + id * a.d_qk;
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = c0 < a.d_qk ? to_f32<T>(qp[c0 + e]) : 0.f;
  const int rows = min(len, len - a.q_len + 1 + u);
  for (int row = 0; row < rows; ++row) {
    const int page = pm.table[(long long)slot * pm.max_pages + row / pm.page], off = row % pm.page;
    if (page < 0 || page >= pm.n_pages) { bad |= SNAP_DEV_BAD_PAGE; continue; }
    const auto read = [&](const uint8_t* p, int d, float (&x)[8]) {
      const uint2 c = c0 < d ? *reinterpret_cast<const uint2*>(p + c0) : make_uint2(0, 0);
      const float2 f[4] = {floats_of_codes(c.x & 0xffffu), floats_of_codes(c.x >> 16), floats_of_codes(c.y & 0xffffu), floats_of_codes(c.y >> 16)};
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[2 * e] = f[e].x; x[2 * e + 1] = f[e].y; }
    };
    const long long sc = ((long long)page * a.Hkv + kvh) * a.map.blocks + off / a.map.block;
    float k[8], v[8], x = 0.f;
    read(a.kp + page * pm.kp + kvh * pm.kh + off * pm.kr, a.d_qk, k);
    read(a.vp + page * pm.vp + kvh * pm.vh + off * pm.vr, a.d_v, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) x = fmaf(q[e], k[e], x);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    x *= a.ks[sc] * a.scale_log2;
    const float nm = fmaxf(m, x), f = m == -INFINITY ? 0.f : exp2f(m - nm), p = x == -INFINITY ? 0.f : exp2f(x - nm), pv = p * a.vs[sc];
    m = nm;
    l = fmaf(l, f, p);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(pv, v[e], o[e] * f);
  }
  if (bad && lane == 0 && a.status) atomicOr(a.status, bad);
  const float inv = l > 0.f ? 1.f / l : l;
  T* out = static_cast<T*>(a.out) + id * a.d_v;
  if (c0 < a.d_v)
#pragma unroll
    for (int e = 0; e < 8; ++e) out[c0 + e] = from_f32<T>(o[e] * inv);
}

}  // namespace

int q8_decode_plan(int, const Shape& s, const Q8Map&, int n_active, int q_len, int, Q8DecodePlan* p) {
  if ((long long)n_active * q_len * s.Hq > 0x7fffffffLL) return SNAP_ERR_UNSUPPORTED;
  p->bytes = 256;
  return SNAP_OK;
}

cudaError_t launch_q8_decode(int dtype, const Shape& s, const Q8Map& m, const Q8DecodePlan&, const void* q, const int* slots,
                             int n_active, int q_len, const void* k_pages, const void* v_pages, const float* k_scales,
                             const float* v_scales, const int* seq_len, void* out, char*, uint32_t* status, cudaStream_t st) {
  Q8Args a;
  a.q = q; a.out = out; a.kp = static_cast<const uint8_t*>(k_pages); a.vp = static_cast<const uint8_t*>(v_pages);
  a.ks = k_scales; a.vs = v_scales; a.slots = slots; a.seq_len = seq_len;
  a.n = n_active; a.q_len = q_len; a.Hq = s.Hq; a.Hkv = s.Hkv; a.g = s.g; a.d_qk = s.d_qk; a.d_v = s.d_v; a.max_seqs = s.max_seqs;
  a.scale_log2 = s.scale * 1.4426950408889634f;
  a.map = m; a.status = status;
  const dim3 grid((unsigned)(((long long)n_active * q_len * s.Hq + NW - 1) / NW));
  const cudaError_t e = dtype == SNAP_F32 ? launch_pdl(q8_decode_kernel<float>, grid, dim3(NW * 32), 0, st, a)
                                          : launch_pdl(q8_decode_kernel<__nv_bfloat16>, grid, dim3(NW * 32), 0, st, a);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace snap
