// open_kernels.hip - gfx950 kernels for tokens whose slots in the cache are
// taken before their K and V exist: a layered model knows a layer's keys only
// after the layer before it has attended.
//
//   k_open    page-table entries, positions and the plan of the open tokens
//   k_qk      a layer's projections: queries and keys normed per head and
//             rotated, K and V stored in the open tokens' slots
//   k_accept  the accepted path of a drafted tree moves to the front of the
//             draft's slots
//
// Pool layouts as in kv_kernels.hip.
#include <algorithm>
#include <type_traits>

#include "fp8.hpp"
#include "open_args.hpp"

namespace sq {
namespace {

constexpr int P = kPage;

// ---------------------------------------------------------------------------
// One launch per opening: the plan's parts come from pinned host memory by a
// kernel (a copy-engine transfer costs 10 us of hand-over), page-table entries
// and positions go out in the same launch.  Bound by latency: 4 us for a chunk, 7 for
// eight trees of 64 nodes (50 KB).
__global__ __launch_bounds__(256) void k_open(OpenArgs a, int32_t copy_blocks) {
  if ((int)blockIdx.x < copy_blocks) {
    int i = blockIdx.x * 256 + threadIdx.x;
    if (blockIdx.x == 0 && threadIdx.x < sizeof(OpenPlan) / 16)
      reinterpret_cast<uint4 *>(a.dst)[threadIdx.x] = reinterpret_cast<const uint4 *>(&a.plan)[threadIdx.x];
    for (int s = 0; s < a.n_segs; ++s) {
      if (i < a.seg_n16[s]) {
        reinterpret_cast<uint4 *>(a.dst + a.seg_off[s])[i] = reinterpret_cast<const uint4 *>(a.src + a.seg_off[s])[i];
        return;
      }
      i -= a.seg_n16[s];
    }
    return;
  }
  const int u = (blockIdx.x - copy_blocks) * 16 + threadIdx.x / 16, slot = threadIdx.x % 16;
  if (u >= a.plan.n_units) return;
  int e = 0;
  for (int b = 1; b < a.plan.batch; ++b) e += a.plan.unit0[b] <= u;
  const int id = a.ids[u];
  if (id < 0) return;
  const int base = a.plan.base[e], page = base / P + u - a.plan.unit0[e];
  if (slot == 0) a.pt[(int64_t)a.row[e] * a.max_pages + page] = id;
  const int t = page * P + slot - base;
  if (t >= 0 && t < a.plan.n[e])
    a.pos[(int64_t)id * P + slot] = a.pos0[e] + (a.depth ? a.depth[a.plan.tok0[e] + t] : t);
}
static_assert(sizeof(OpenPlan) / 16 <= 256, "the plan is written by one workgroup");

// ---------------------------------------------------------------------------
// Queries and keys.  For a head x of D channels, with r = 1 / sqrt(mean x^2 +
// eps) and its weight w: y = x r w; then the first `rot` channels turn in pairs
// by angle = position * inv_freq[i], (a, b) -> (a cos - b sin, b cos + a sin) *
// mscale: channels (i, i + rot/2), or (2i, 2i + 1).  All in fp32, rounded once
// to bf16 or to the store's E4M3 code.  The angle is taken in 64 bits and
// reduced there to a part of a turn: in fp32 an angle of 1e5 radians would be
// off by 4e-3.
//
// Bound by HBM: each projection is read once, each output written once.  A
// workgroup takes 16 tokens (of a stored chunk: one page), 16 lanes each, and
// `its` iterations over the heads of q, of k or of v: 16 lanes hold a head of 128
// channels (or two of 64), 8 channels a lane, laid out so that a lane holds both
// channels of its pairs (two runs of 4) and nothing but the sum of squares crosses
// lanes.  The angles are taken once per token and workgroup, while the first loads
// are in flight; the loads of an iteration are issued before the one before it is
// stored.  V passes through LDS, since a page holds it channel-major.
// Consecutive workgroups take the same tokens' other heads, and q_out and K are
// stored non-temporally: one layer of 8192 tokens, 32 + 8 + 8 heads of 128
// (201 MB), takes 40.8 us (4.9 TB/s) against 46.6 with neither and 43.0 without
// the stores' hint; 512 tokens 6.1 against 6.8.  (With q, k and v read and V
// written non-temporally too 39.6, but 512 tokens 7.2: they come from the cache.)
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v_t __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){lo, hi}, bf16x2v_t));
}
__device__ inline void unpack4(uint2 w, float *x) {
  x[0] = __uint_as_float(w.x << 16);
  x[1] = __uint_as_float(w.x & 0xffff0000u);
  x[2] = __uint_as_float(w.y << 16);
  x[3] = __uint_as_float(w.y & 0xffff0000u);
}
__device__ inline void store8(uint16_t *p, uint32_t lo, uint32_t hi) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  __builtin_nontemporal_store((u32x2_t){lo, hi}, reinterpret_cast<u32x2_t *>(p));
}
__device__ inline uint32_t codes4(const float *x, float inv) {
  return e4m3_encode2(x[0] * inv, x[1] * inv) | e4m3_encode2(x[2] * inv, x[3] * inv) << 16;
}
__device__ inline uint2 codes8(uint4 w, float inv) { // 8 bf16 -> 8 codes
  float x[8];
  unpack4(make_uint2(w.x, w.y), x);
  unpack4(make_uint2(w.z, w.w), x + 4);
  return make_uint2(codes4(x, inv), codes4(x + 4, inv));
}

// What a lane needs for every head of its token.
struct Turn {
  float c[4], s[4];
  int ca, cb; // its channels: ca .. ca + 3 and cb .. cb + 3
  bool on, next;
};

// Sum over the 8 or 16 lanes of a head; every lane ends with the same bits.
template <int LPH> __device__ inline float sum_lanes(float x) {
  auto moved = [](float y, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  x += moved(x, std::integral_constant<int, 0xB1>{});  // lane ^ 1
  x += moved(x, std::integral_constant<int, 0x4E>{});  // lane ^ 2
  x += moved(x, std::integral_constant<int, 0x141>{}); // mirrored in 8
  if (LPH == 16) x += moved(x, std::integral_constant<int, 0x140>{}); // mirrored in 16
  return x;
}

template <int D> __device__ inline void turn_head(const Turn &t, const float *w, float eps, float *x) {
  if (w) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
    ss = sum_lanes<D / 8>(ss);
    const float r = 1.f / sqrtf(fmaf(ss, 1.f / D, eps));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= r * w[i];
  }
  if (!t.on) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float &a = t.next ? x[2 * i] : x[i];
    float &b = t.next ? x[2 * i + 1] : x[i + 4];
    const float na = a * t.c[i] - b * t.s[i], nb = b * t.c[i] + a * t.s[i];
    a = na;
    b = nb;
  }
}

template <int D, bool STORE, bool KV8, bool NEXT>
__global__ __launch_bounds__(256) void k_qk(QkArgs a) {
  constexpr int LPH = D / 8;      // lanes per head
  constexpr int HPI = 16 / LPH;   // heads per iteration
  __shared__ uint16_t tile[HPI][P][D + 8];
  const int tid = threadIdx.x, row = tid >> 4, j = tid & 15, hs = j / LPH, jj = j % LPH;
  const int u = blockIdx.x / a.blocks;
  int t, page = 0, s0 = 0, s1 = 0;
  if constexpr (STORE) {
    const int lane = tid & 63;
    const OpenPlan *pl = a.plan;
    const int e = __popcll(__ballot(lane < pl->batch && pl->unit0[lane] <= u)) - 1;
    page = a.ids[u];
    if (page < 0) return; // (the whole workgroup)
    const int base = pl->base[e], first = (base / P + u - pl->unit0[e]) * P - base; // entry token of slot 0
    s0 = max(0, -first);
    s1 = min(P, min(pl->n[e], a.n - pl->tok0[e]) - first);
    t = pl->tok0[e] + first + row;
  } else {
    s1 = min(P, a.n - u * P);
    t = u * P + row;
  }
  const bool in = row >= s0 && row < s1;
  const int n_q = (a.hq + HPI - 1) / HPI, n_kv = (a.hkv + HPI - 1) / HPI;
  const int q_blocks = (n_q + a.its - 1) / a.its, kv_blocks = (n_kv + a.its - 1) / a.its;
  int y = blockIdx.x - u * a.blocks;

  if (y < q_blocks + kv_blocks) {
    const bool is_k = y >= q_blocks;
    if (is_k) y -= q_blocks;
    const int lo = y * a.its, hi = min(lo + a.its, is_k ? n_kv : n_q), nh = is_k ? a.hkv : a.hq;
    const uint16_t *src = is_k ? a.k + (int64_t)t * a.k_stride : a.q + (int64_t)t * a.q_stride;
    const float *weight = is_k ? a.k_weight : a.q_weight;
    Turn turn;
    turn.next = NEXT;
    turn.on = a.inv_freq && 8 * jj < a.rot;
    turn.ca = !NEXT && turn.on ? 4 * jj : 8 * jj;
    turn.cb = !NEXT && turn.on ? a.rot / 2 + 4 * jj : 8 * jj + 4;
    constexpr int U = 2;
    uint2 ra[U], rb[U];
    auto load = [&](int i0) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int h = (i0 + i) * HPI + hs;
        if (in && i0 + i < hi && h < nh) {
          ra[i] = *reinterpret_cast<const uint2 *>(src + h * D + turn.ca);
          rb[i] = *reinterpret_cast<const uint2 *>(src + h * D + turn.cb);
        }
      }
    };
#pragma unroll
    for (int i = 0; i < U; ++i) ra[i] = rb[i] = make_uint2(0, 0);
    load(lo);
    float w[8];
    if (weight) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = weight[turn.ca + i];
        w[i + 4] = weight[turn.cb + i];
      }
    }
    if (turn.on) {
      const int pos = !in ? 0 : STORE ? a.pos[(int64_t)page * P + row] : a.pos[t];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        double x = (double)pos * (double)a.inv_freq[4 * jj + i] * 0.15915494309189533577; // in turns
        x -= rint(x);
        sincospif(2.f * (float)x, &turn.s[i], &turn.c[i]);
        turn.s[i] *= a.mscale;
        turn.c[i] *= a.mscale;
      }
    }
    auto put_bf16 = [&](uint16_t *p, const float *x) {
      store8(p + turn.ca, pack2(x[0], x[1]), pack2(x[2], x[3]));
      store8(p + turn.cb, pack2(x[4], x[5]), pack2(x[6], x[7]));
    };
    for (int i0 = lo; i0 < hi; i0 += U) {
      uint2 ca[U], cb[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        ca[i] = ra[i];
        cb[i] = rb[i];
      }
      if (i0 + U < hi) load(i0 + U);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int h = (i0 + i) * HPI + hs;
        float x[8];
        unpack4(ca[i], x);
        unpack4(cb[i], x + 4);
        turn_head<D>(turn, weight ? w : nullptr, a.eps, x);
        if (!(in && i0 + i < hi && h < nh)) continue;
        if (!is_k) {
          put_bf16(a.q_out + ((int64_t)t * a.hq + h) * D, x);
        } else if constexpr (!STORE) {
          put_bf16(a.k_out + ((int64_t)t * a.hkv + h) * D, x);
        } else {
          const int64_t at = h * a.head_stride + page * a.page_stride + row * D;
          if constexpr (KV8) {
            uint8_t *p = reinterpret_cast<uint8_t *>(a.k_pool) + at;
            *reinterpret_cast<uint32_t *>(p + turn.ca) = codes4(x, a.inv_k);
            *reinterpret_cast<uint32_t *>(p + turn.cb) = codes4(x + 4, a.inv_k);
          } else {
            put_bf16(a.k_pool + at, x);
          }
        }
      }
    }
    return;
  }
  if constexpr (STORE) {
    const int lo = (y - q_blocks - kv_blocks) * a.its, hi = min(lo + a.its, n_kv);
    for (int it = lo; it < hi; ++it) {
      const int h = it * HPI + hs;
      uint4 w = make_uint4(0, 0, 0, 0);
      if (in && h < a.hkv) w = *reinterpret_cast<const uint4 *>(a.v + (int64_t)t * a.v_stride + h * D + 8 * jj);
      if (it > lo) __syncthreads(); // the tile of the iteration before is read
      *reinterpret_cast<uint4 *>(&tile[hs][row][8 * jj]) = w;
      __syncthreads();
      // thread: 8 slots of one channel
      const int hh = tid / (2 * D), d = tid / 2 % D, half = tid & 1, ho = it * HPI + hh;
      if (ho >= a.hkv || half * 8 + 8 <= s0 || half * 8 >= s1) continue;
      uint16_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = tile[hh][half * 8 + i][d];
      uint4 o;
      __builtin_memcpy(&o, x, 16);
      const int64_t at = ho * a.head_stride + page * a.page_stride + d * P + half * 8;
      const bool whole = half * 8 >= s0 && half * 8 + 8 <= s1;
      if constexpr (KV8) {
        uint8_t *p = reinterpret_cast<uint8_t *>(a.v_pool) + at;
        const uint2 c = codes8(o, a.inv_v);
        if (whole) {
          *reinterpret_cast<uint2 *>(p) = c;
        } else {
          uint8_t y[8];
          __builtin_memcpy(y, &c, 8);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (half * 8 + i >= s0 && half * 8 + i < s1) p[i] = y[i];
        }
      } else if (whole) {
        *reinterpret_cast<uint4 *>(a.v_pool + at) = o;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (half * 8 + i >= s0 && half * 8 + i < s1) a.v_pool[at + i] = x[i];
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Keeping a path.  Its j-th node lies at draft slot c_j >= j and moves to slot j,
// so a token's source is never a slot that an earlier token of the path goes to
// (i < j <= c_j): passes of 16 tokens in order, each loading all it moves before
// it stores.  A workgroup takes one (layer, head) of one sequence.  Bound by
// latency: a few hundred KB in all (paths of eight 64-node trees, 24 layers of 8
// heads, 18 us; with all 64 slots held in registers in one pass 30).
template <int D, class E>
__global__ __launch_bounds__(256) void k_accept(Pools p, AcceptArgs a) {
  constexpr int U = D * (int)sizeof(E) / 16; // 16-byte units per K row
  constexpr int KR = 16 * U, VR = 16 * D / 256;
  const int e = blockIdx.y;
  uint64_t rest = a.mask[e];
  const int n = __popcll(rest);
  const int layer = blockIdx.x / p.hkv, head = blockIdx.x % p.hkv;
  const int32_t *pt = a.pt + (int64_t)a.row[e] * a.max_pages;
  const int base = a.base[e];
  const int64_t chunk = layer * p.layer_stride + head * p.head_stride;
  E *kp = reinterpret_cast<E *>(p.k) + chunk;
  E *vp = reinterpret_cast<E *>(p.v) + chunk;
  const int tid = threadIdx.x;
  __shared__ int64_t src_page[16], dst_page[16];
  __shared__ int src_slot[16], dst_slot[16], move[16];
  for (int j0 = 0; j0 < n; j0 += 16) {
    const int m = min(16, n - j0);
    __syncthreads();
    if (tid < m) {
      uint64_t w = rest;
      for (int i = 0; i < tid; ++i) w &= w - 1;
      const int c = __ffsll((unsigned long long)w) - 1, s = base + c, t = base + j0 + tid;
      src_page[tid] = pt[s / P] * p.page_stride;
      dst_page[tid] = pt[t / P] * p.page_stride;
      src_slot[tid] = s % P;
      dst_slot[tid] = t % P;
      move[tid] = s != t;
      if (blockIdx.x == 0 && s != t) p.pos[(int64_t)pt[t / P] * P + t % P] = a.pos0[e] + j0 + tid;
    }
    for (int i = 0; i < m; ++i) rest &= rest - 1;
    __syncthreads();
    uint4 kr;
    E vr[VR];
    const int kj = tid / U, ku = tid % U;
    const bool km = tid < KR && kj < m && move[kj];
    if (km) kr = reinterpret_cast<const uint4 *>(kp + src_page[kj] + src_slot[kj] * D)[ku];
#pragma unroll
    for (int i = 0; i < VR; ++i) {
      const int jv = (i * 256 + tid) / D, d = (i * 256 + tid) % D;
      vr[i] = 0;
      if (jv < m && move[jv]) vr[i] = vp[src_page[jv] + d * P + src_slot[jv]];
    }
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory"); // every load of the pass is done before any store
    __syncthreads();
    if (km) reinterpret_cast<uint4 *>(kp + dst_page[kj] + dst_slot[kj] * D)[ku] = kr;
#pragma unroll
    for (int i = 0; i < VR; ++i) {
      const int jv = (i * 256 + tid) / D, d = (i * 256 + tid) % D;
      if (jv < m && move[jv]) vp[dst_page[jv] + d * P + dst_slot[jv]] = vr[i];
    }
  }
}

template <int D, bool STORE, bool KV8> hipError_t qk_dispatch(const QkArgs &a, dim3 grid, hipStream_t s) {
  if (a.interleaved) hipLaunchKernelGGL((k_qk<D, STORE, KV8, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_qk<D, STORE, KV8, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int D> hipError_t qk_dispatch_d(const QkArgs &in, hipStream_t s) {
  constexpr int HPI = 128 / D;
  const bool store = in.plan != nullptr;
  QkArgs a = in;
  const int n_kv = (a.hkv + HPI - 1) / HPI;
  const int n_q = (a.hq + HPI - 1) / HPI, most = std::max(n_q, n_kv);
  const int units = store ? a.n_units : (a.n + kPage - 1) / kPage;
  for (a.its = 4;; a.its += 4) {
    a.blocks = (n_q + a.its - 1) / a.its + (n_kv + a.its - 1) / a.its * (store ? 2 : 1);
    if (a.its >= most || (int64_t)units * a.blocks <= 4096) break;
  }
  const dim3 grid(units * a.blocks); // at most 2^20 units of 2 blocks
  if (!store) return qk_dispatch<D, false, false>(a, grid, s);
  return a.kv8 ? qk_dispatch<D, true, true>(a, grid, s) : qk_dispatch<D, true, false>(a, grid, s);
}

} // namespace

hipError_t launch_open(const OpenArgs &a, hipStream_t s) {
  const int copy = std::max(1, (a.n16 + 255) / 256);
  hipLaunchKernelGGL(k_open, dim3(copy + (a.plan.n_units + 15) / 16), dim3(256), 0, s, a, copy);
  return hipGetLastError();
}

hipError_t launch_qk(int d, const QkArgs &a, hipStream_t s) {
  if (d == 128) return qk_dispatch_d<128>(a, s);
  if (d == 64) return qk_dispatch_d<64>(a, s);
  return hipErrorInvalidValue;
}

hipError_t launch_accept(const Pools &p, const AcceptArgs &a, hipStream_t s) {
  if (a.n <= 0) return hipSuccess;
  const dim3 grid(p.nl * p.hkv, a.n), block(256);
  if (p.kv8) {
    if (p.d == 128) hipLaunchKernelGGL((k_accept<128, uint8_t>), grid, block, 0, s, p, a);
    else hipLaunchKernelGGL((k_accept<64, uint8_t>), grid, block, 0, s, p, a);
  } else if (p.d == 128) hipLaunchKernelGGL((k_accept<128, uint16_t>), grid, block, 0, s, p, a);
  else hipLaunchKernelGGL((k_accept<64, uint16_t>), grid, block, 0, s, p, a);
  return hipGetLastError();
}

} // namespace sq
