// page_frags.hpp - matrix-core fragments of one 16-token page of one KV head,
// loaded straight from the pools into registers (the decode and draft kernels).
// Internal to libsq; to be included inside a .hip file.
//
// Lane l = n + 16 * kg (n = l & 15, kg = l >> 4):
//   K fragment    K[token n][channels 8 kg + 32 s .. +8]      (A of 16x16x32)
//   V^T fragment  V^T[channel n + 16 jd][tokens 4 kg .. +4]
#pragma once

#include "fp8.hpp"
#include "sq_common.hpp"

namespace sq {
namespace {

template <int D> struct KFrag {
  uint4 k[D / 32];
};
template <int D> struct VFrag {
  uint2 v[D / 16];
};

// A buffer resource over one page of one KV head (the pools are read only
// through these): a page that is not wanted gets num_records 0, so its loads
// return zeros without touching memory and every loop iteration issues the
// same loads - which keeps the hardware's in-order load counter waits exact.
constexpr int kRsrcWord3 = 0x00020000;
__device__ inline __amdgpu_buffer_rsrc_t page_rsrc(const char *page, bool want, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(page), (short)0, want ? bytes : 0,
                                           kRsrcWord3);
}
template <bool NT> constexpr int kAux = NT ? 2 : 0; // nt: streamed once
// K fragment: lane (n, kg) takes channels 8 kg + 32 s .. +8 of token n.
template <int D, bool NT>
__device__ inline void load_k(KFrag<D> &f, __amdgpu_buffer_rsrc_t r, int lane_off) {
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, lane_off + 64 * s, 0, kAux<NT>);
    f.k[s] = make_uint4(x[0], x[1], x[2], x[3]);
  }
}
// V^T fragment: lane (n, kg) takes tokens 4 kg .. +4 of channel n + 16 j.
template <int D, bool NT>
__device__ inline void load_v(VFrag<D> &f, __amdgpu_buffer_rsrc_t r, int lane_off) {
#pragma unroll
  for (int j = 0; j < D / 16; ++j) {
    const auto x = __builtin_amdgcn_raw_buffer_load_b64(r, lane_off + 32 * kPage * j, 0, kAux<NT>);
    f.v[j] = make_uint2(x[0], x[1]);
  }
}

// The same fragments in an 8-bit store (E4M3 codes, half the bytes); they
// become bf16 fragments just before the matrix-core instructions.  A K lane
// loads 16 contiguous codes, channels 16 kg + 64 s' .. +16 of token n, in
// one request (a token's row is read in full-line halves, as in bf16); its
// two 8-channel halves feed QK chunks 2 s' and 2 s' + 1, and the query
// fragments take the same channels, so each chunk still pairs q and k
// channel by channel (the dot product is a sum over a permutation of the
// channels).
template <int D> struct KFrag8 {
  uint4 k[D / 64];
};
template <int D> struct VFrag8 {
  uint32_t v[D / 16];
};
template <int D, bool NT>
__device__ inline void load_k(KFrag8<D> &f, __amdgpu_buffer_rsrc_t r, int lane_off) {
#pragma unroll
  for (int s = 0; s < D / 64; ++s) {
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, lane_off + 64 * s, 0, kAux<NT>);
    f.k[s] = make_uint4(x[0], x[1], x[2], x[3]);
  }
}
// A V lane loads the 16 codes of one channel row, c = 64 J + 16 kg + n, in
// one request (four b32 requests would each carry 4 codes).  Word t of that
// row (tokens 4t .. 4t+3) belongs to the lane with the same n in lane row t,
// for matrix-core instruction 4 J + kg: a 4 x 4 transpose across the wave's
// four lane rows, done as the fragment is converted.
template <int D, bool NT>
__device__ inline void load_v(VFrag8<D> &f, __amdgpu_buffer_rsrc_t r, int lane_off) {
#pragma unroll
  for (int J = 0; J < D / 64; ++J) {
    const auto x = __builtin_amdgcn_raw_buffer_load_b128(r, lane_off + 64 * kPage * J, 0, kAux<NT>);
#pragma unroll
    for (int t = 0; t < 4; ++t) f.v[4 * J + t] = x[t];
  }
}
template <int D> __device__ inline KFrag<D> to_bf16(const KFrag8<D> &f) {
  KFrag<D> o;
#pragma unroll
  for (int s = 0; s < D / 64; ++s) {
    const uint2 a = e4m3x4_to_bf16(f.k[s].x), b = e4m3x4_to_bf16(f.k[s].y);
    const uint2 c = e4m3x4_to_bf16(f.k[s].z), d = e4m3x4_to_bf16(f.k[s].w);
    o.k[2 * s] = make_uint4(a.x, a.y, b.x, b.y);
    o.k[2 * s + 1] = make_uint4(c.x, c.y, d.x, d.y);
  }
  return o;
}
template <int D, bool KV8> struct Frags {
  using K = KFrag<D>;
  using V = VFrag<D>;
};
template <int D> struct Frags<D, true> {
  using K = KFrag8<D>;
  using V = VFrag8<D>;
};
template <int D> __device__ inline const KFrag<D> &to_bf16(const KFrag<D> &f) { return f; }
template <int D> __device__ inline const VFrag<D> &to_bf16(const VFrag<D> &f) { return f; }
// Lane row r holds words w[0..3] of rows c = 64 J + 16 r + n; afterwards it
// holds word r of those rows for r' = 0..3.  Swapping lane rows {0,1} with
// {2,3} across word pairs (0,2) and (1,3) exchanges the off-diagonal 2 x 2
// blocks; swapping odd with even lane rows across pairs (0,1) and (2,3)
// transposes each block.
template <int D> __device__ inline VFrag<D> to_bf16(const VFrag8<D> &f) {
  VFrag<D> o;
#pragma unroll
  for (int J = 0; J < D / 64; ++J) {
    const auto a = __builtin_amdgcn_permlane32_swap(f.v[4 * J], f.v[4 * J + 2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(f.v[4 * J + 1], f.v[4 * J + 3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    o.v[4 * J] = e4m3x4_to_bf16(c[0]);
    o.v[4 * J + 1] = e4m3x4_to_bf16(c[1]);
    o.v[4 * J + 2] = e4m3x4_to_bf16(d[0]);
    o.v[4 * J + 3] = e4m3x4_to_bf16(d[1]);
  }
  return o;
}

} // namespace
} // namespace sq
