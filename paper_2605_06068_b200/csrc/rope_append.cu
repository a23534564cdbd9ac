// rope_kv_append: norm of each query and key head, rotation by the token's position and the way into the paged cache, in
// one pass over the projection's output: bytes (16411 tokens of 32 + 16 heads: 391 MB).
//
// A head's row lies across D / 16 lanes, each with two 16-byte vectors: for the rotation of halves the vectors i and
// i + rot/16, whose elements are each other's partners, so that it needs no exchange between lanes; the elements that are not
// rotated as neighbouring vectors. A warp takes kRows rows of one token at a time for each of its segments: the
// token's cosines and sines are read once for all of them. The rows are asked for first, before anything that they wait for
// is known (slot, position, then angles). The norm's sum goes over the segment by shuffles. All of it is held in 32 bits and
// rounded once.
// e4m3 caches: keys and values go another way, since a row's scale is that of its page's first row. A warp takes one head's
// keys, or values, of kRows tokens a segment one behind the other; of them the first rows of pages give the others their
// scale by shuffles, and only a page that begins before the warp's tokens has its first row read once more.
#include "shaped.cuh"
#include "tma_ptx.cuh"

namespace pda {

namespace {

constexpr int kRopeWarps = 4;
constexpr int kRows = 4;  // rows of each segment of a warp

struct Row {
  float a[8], b[8];
};
__device__ __forceinline__ void unpack(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
  return make_uint4(pack2<false>(x[0], x[1]), pack2<false>(x[2], x[3]), pack2<false>(x[4], x[5]), pack2<false>(x[6], x[7]));
}
__device__ __forceinline__ uint2 pack_e4m3(const float (&x)[8], float scale) {
  uint32_t h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(__fdiv_rn(x[2 * e + 1], scale)), "f"(__fdiv_rn(x[2 * e], scale)));
    h[e] = r;
  }
  return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}

// What a lane has to do with a row: its two vectors, and their cosines and sines.
template <int kLanes, bool kPairs>
struct Lane {
  int i, ca, cb;        // lane of the segment; its vectors of a row
  bool mine, rotated;   // (of the last lanes some have no elements)
  __device__ Lane(const RopeAppendParams& p, int lane) {
    i = lane % kLanes;
    mine = 16 * i < p.geom.head_dim;
    rotated = 16 * i < p.rot_dim;
    ca = rotated ? i : 2 * i;
    cb = rotated ? i + p.rot_dim / 16 : 2 * i + 1;
  }
  // A token's positions; false: one is outside the table.
  __device__ __forceinline__ bool positions(const RopeAppendParams& p, int tok, int (&pos)[4]) const {
    bool good = true;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const bool used = (p.axes_used >> a) & 1;
      pos[a] = used ? __ldg(p.positions + a * p.positions_stride + tok) : 0;
      good &= !used || (pos[a] >= 0 && pos[a] < p.table_len);
    }
    return good;
  }
  // Cosines and sines of this lane's elements: of halves frequency 8 i + e, the same for both vectors; of pairs 4 i + e for the
  // first vector's and rot / 4 + 4 i + e for the second's.
  __device__ __forceinline__ void angles(const RopeAppendParams& p, const int (&pos)[4], bool good, float (&c)[8], float (&s)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
    }
    if (!rotated || !good) return;
    const int half = p.rot_dim / 2;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int f = kPairs ? (v == 0 ? 4 * i : p.rot_dim / 4 + 4 * i) : 8 * i + 4 * v;
      const uchar4 ax = *reinterpret_cast<const uchar4*>(p.freq_axis + f);
      auto row = [&](int axis) {
        return p.cos_sin + static_cast<int64_t>(axis == 0 ? pos[0] : axis == 1 ? pos[1] : axis == 2 ? pos[2] : pos[3]) * p.rot_dim + f;
      };
      if (ax.x == ax.y && ax.x == ax.z && ax.x == ax.w) {
        const float4 c4 = __ldg(reinterpret_cast<const float4*>(row(ax.x))), s4 = __ldg(reinterpret_cast<const float4*>(row(ax.x) + half));
        c[4 * v] = c4.x, c[4 * v + 1] = c4.y, c[4 * v + 2] = c4.z, c[4 * v + 3] = c4.w;
        s[4 * v] = s4.x, s[4 * v + 1] = s4.y, s[4 * v + 2] = s4.z, s[4 * v + 3] = s4.w;
      } else {
        const int axes[4] = {ax.x, ax.y, ax.z, ax.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          c[4 * v + e] = __ldg(row(axes[e]) + e);
          s[4 * v + e] = __ldg(row(axes[e]) + half + e);
        }
      }
    }
  }
  // Norm (weight: nullptr for rows that have none) and rotation (turned) of a row by its whole segment. any_norm: the same in
  // all lanes of the warp.
  __device__ __forceinline__ void turn(const RopeAppendParams& p, Row& x, bool any_norm, const __nv_bfloat16* weight, bool turned,
                                       const float (&c)[8], const float (&s)[8]) const {
    if (any_norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x.a[e], x.a[e], fmaf(x.b[e], x.b[e], ss));
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (weight != nullptr && mine) {
        const float inv = 1.f / sqrtf(ss / static_cast<float>(p.geom.head_dim) + p.eps);
        float wa[8], wb[8];
        unpack(__ldg(reinterpret_cast<const uint4*>(weight) + ca), wa);
        unpack(__ldg(reinterpret_cast<const uint4*>(weight) + cb), wb);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x.a[e] = x.a[e] * inv * wa[e];
          x.b[e] = x.b[e] * inv * wb[e];
        }
      }
    }
    if (turned && rotated) {
      if constexpr (kPairs) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a0 = x.a[2 * e], a1 = x.a[2 * e + 1], b0 = x.b[2 * e], b1 = x.b[2 * e + 1];
          x.a[2 * e] = fmaf(a0, c[e], -(a1 * s[e]));
          x.a[2 * e + 1] = fmaf(a1, c[e], a0 * s[e]);
          x.b[2 * e] = fmaf(b0, c[4 + e], -(b1 * s[4 + e]));
          x.b[2 * e + 1] = fmaf(b1, c[4 + e], b0 * s[4 + e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float a = x.a[e], b = x.b[e];
          x.a[e] = fmaf(a, c[e], -(b * s[e]));
          x.b[e] = fmaf(b, c[e], a * s[e]);
        }
      }
    }
  }
};

// Rows of one token: its queries and, where kKv, keys and values of a bf16 cache.
template <int kLanes, bool kPairs, bool kKv>
__device__ __forceinline__ void token_rows(const RopeAppendParams& p, int64_t item, int lane) {
  constexpr int kSegs = 32 / kLanes, kStep = kSegs * kRows;  // rows of a token that a warp takes
  const Lane<kLanes, kPairs> me(p, lane);
  const int Hkv = p.geom.num_kv_heads, heads = p.num_q_heads + (kKv ? 2 * Hkv : 0), steps = (heads + kStep - 1) / kStep;
  const int64_t tok = item / steps;
  if (tok >= p.n_tokens) return;
  const int t = static_cast<int>(tok), row0 = static_cast<int>(item % steps) * kStep + lane / kLanes;
  uint4 ra[kRows], rb[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int row = row0 + k * kSegs;
    ra[k] = rb[k] = make_uint4(0, 0, 0, 0);
    if (me.mine && row < heads) {
      const __nv_bfloat16* at = row < p.num_q_heads ? p.q + t * p.q_token_stride + row * p.q_head_stride
                                : row < p.num_q_heads + Hkv ? p.k + t * p.k_token_stride + (row - p.num_q_heads) * p.k_head_stride
                                                            : p.v + t * p.v_token_stride + (row - p.num_q_heads - Hkv) * p.v_head_stride;
      const uint4* src = reinterpret_cast<const uint4*>(at);
      ra[k] = src[me.ca];
      rb[k] = src[me.cb];
    }
  }
  const int slot = __ldg(p.slot_map + t);
  int pos[4];
  const bool good = me.positions(p, t, pos);
  if (slot < 0) return;  // a padding entry
  const bool in_cache = slot < static_cast<int64_t>(p.geom.num_pages) * kPageSize;
  if (lane == 0 && row0 == 0 && !good) report(p.status, PDA_DEV_BAD_SEQ_LEN);
  if (lane == 0 && row0 == 0 && !in_cache) report(p.status, PDA_DEV_BAD_PAGE);
  float cs[8], sn[8];
  me.angles(p, pos, good, cs, sn);
  const int page = slot / kPageSize, in_page = slot % kPageSize;
  const bool any_norm = p.q_norm != nullptr || p.k_norm != nullptr;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int row = row0 + k * kSegs;
    Row x;
    unpack(ra[k], x.a);
    unpack(rb[k], x.b);
    const bool is_q = row < p.num_q_heads, is_v = row >= p.num_q_heads + Hkv;
    me.turn(p, x, any_norm, is_q ? p.q_norm : is_v ? nullptr : p.k_norm, !is_v, cs, sn);
    if (!me.mine || row >= heads) continue;
    if (is_q) {
      uint4* dst = reinterpret_cast<uint4*>(p.q_out + t * p.qo_token_stride + row * p.qo_head_stride);
      const uint4 zero = make_uint4(0, 0, 0, 0);
      dst[me.ca] = good ? pack(x.a) : zero;
      dst[me.cb] = good ? pack(x.b) : zero;
    } else if (kKv && in_cache && good) {
      const int g = row - p.num_q_heads - (is_v ? Hkv : 0);
      uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(is_v ? p.v_cache : p.k_cache) + page * p.geom.page_stride +
                                            g * p.geom.head_stride + in_page * p.geom.slot_stride);
      dst[me.ca] = pack(x.a);
      dst[me.cb] = pack(x.b);
    }
  }
}

// Keys, or values, of one head and kRows tokens a segment, into an e4m3 cache.
template <int kLanes, bool kPairs>
__device__ __forceinline__ void quantised_rows(const RopeAppendParams& p, int item, int lane) {
  constexpr int kSegs = 32 / kLanes, kTokens = kSegs * kRows;
  const Lane<kLanes, kPairs> me(p, lane);
  const int Hkv = p.geom.num_kv_heads, seg = lane / kLanes;
  const bool is_v = item & 1;
  const int g = (item >> 1) % Hkv, t0 = (item >> 1) / Hkv * kTokens;
  const __nv_bfloat16* rows = is_v ? p.v + g * p.v_head_stride : p.k + g * p.k_head_stride;
  const int64_t stride = is_v ? p.v_token_stride : p.k_token_stride;
  float* scales = is_v ? p.v_scale : p.k_scale;
  const __nv_bfloat16* weight = is_v ? nullptr : p.k_norm;
  auto load = [&](int t, bool there, uint4& a, uint4& b) {
    a = b = make_uint4(0, 0, 0, 0);
    if (there && me.mine) {
      const uint4* src = reinterpret_cast<const uint4*>(rows + t * stride);
      a = src[me.ca];
      b = src[me.cb];
    }
  };
  auto largest = [&](const Row& x) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(fabsf(x.a[e]), fabsf(x.b[e])));
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    return top;
  };
  uint4 ra[kRows], rb[kRows];
  int slot[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {  // token t0 + k kSegs + seg
    const int t = t0 + k * kSegs + seg;
    load(t, t < p.n_tokens, ra[k], rb[k]);
    slot[k] = t < p.n_tokens ? __ldg(p.slot_map + t) : -1;
  }
  // The page that begins before these tokens: its first row, if this call has it.
  const int slot0 = __ldg(p.slot_map + t0), back = slot0 >= 0 ? slot0 % kPageSize : 0;
  float top_before = -1.f;
  if (back > 0 && back <= t0 && __ldg(p.slot_map + t0 - back) == slot0 - back) {  // (uniform)
    int pos[4];
    const bool good = me.positions(p, t0 - back, pos);
    Row x;
    uint4 a, b;
    load(t0 - back, true, a, b);
    unpack(a, x.a);
    unpack(b, x.b);
    float cs[8], sn[8];
    if (!is_v) me.angles(p, pos, good, cs, sn);
    me.turn(p, x, weight != nullptr, weight, !is_v, cs, sn);
    const float top = largest(x);
    if (good) top_before = top;
  }
  Row x[kRows];
  float top[kRows];  // of a page's first row; -1 of others
  bool good[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int t = min(t0 + k * kSegs + seg, p.n_tokens - 1);
    int pos[4];
    good[k] = me.positions(p, t, pos);
    unpack(ra[k], x[k].a);
    unpack(rb[k], x[k].b);
    float cs[8], sn[8];
    if (!is_v) me.angles(p, pos, good[k], cs, sn);
    me.turn(p, x[k], weight != nullptr, weight, !is_v, cs, sn);
    top[k] = largest(x[k]);
    if (slot[k] < 0 || slot[k] % kPageSize != 0 || !good[k]) top[k] = -1.f;
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    // the token that opens this one's page, counted from t0
    const int in_page = slot[k] < 0 ? 0 : slot[k] % kPageSize, first = k * kSegs + seg - in_page;
    const int from = max(first, 0), source = from % kSegs * kLanes;
    float opener = -1.f;
    int opener_slot = -1;
#pragma unroll
    for (int m = 0; m < kRows; ++m) {
      const float v = __shfl_sync(0xffffffffu, top[m], source);
      const int sl = __shfl_sync(0xffffffffu, slot[m], source);
      if (from / kSegs == m) {
        opener = v;
        opener_slot = sl;
      }
    }
    if (first < 0) {
      opener = top_before;
      opener_slot = first == -back ? slot0 - back : -1;
    }
    const bool in_cache = slot[k] < static_cast<int64_t>(p.geom.num_pages) * kPageSize;
    if (slot[k] < 0 || !good[k] || !in_cache) continue;  // (reported with the token's queries)
    const int page = slot[k] / kPageSize;
    const int64_t at = static_cast<int64_t>(page) * Hkv + g;
    float scale;
    if (opener >= 0.f && opener_slot == slot[k] - in_page) {
      scale = opener > 0.f ? __fdiv_rn(opener * 2.f, 448.f) : 1.f;
      if (in_page == 0 && me.i == 0) scales[at] = scale;
    } else {
      scale = scales[at];
    }
    if (!me.mine) continue;
    uint2* dst = reinterpret_cast<uint2*>(static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache) + page * p.geom.page_stride +
                                          g * p.geom.head_stride + in_page * p.geom.slot_stride);
    dst[me.ca] = pack_e4m3(x[k].a, scale);
    dst[me.cb] = pack_e4m3(x[k].b, scale);
  }
}

template <int kLanes, bool kPairs, bool kFp8>
__global__ void __launch_bounds__(kRopeWarps * 32) rope_append_kernel(const __grid_constant__ RopeAppendParams p, int quantised) {
  const int lane = threadIdx.x & 31;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kRopeWarps + (threadIdx.x >> 5);
  if constexpr (kFp8) {  // (the longer items first)
    if (item < quantised) quantised_rows<kLanes, kPairs>(p, static_cast<int>(item), lane);
    else token_rows<kLanes, kPairs, false>(p, item - quantised, lane);
  } else {
    token_rows<kLanes, kPairs, true>(p, item, lane);
  }
}

template <int kLanes>
cudaError_t launch(const RopeAppendParams& p, bool interleaved, cudaStream_t stream) {
  constexpr int kStep = 32 / kLanes * kRows;
  const bool fp8 = p.geom.dtype == PDA_FP8_E4M3;
  const int Hkv = p.geom.num_kv_heads, heads = p.num_q_heads + (fp8 ? 0 : 2 * Hkv);
  const int64_t quantised = fp8 ? 2ll * Hkv * ((static_cast<int64_t>(p.n_tokens) + kStep - 1) / kStep) : 0;
  const int64_t items = quantised + static_cast<int64_t>(p.n_tokens) * ((heads + kStep - 1) / kStep);
  const unsigned blocks = static_cast<unsigned>((items + kRopeWarps - 1) / kRopeWarps);
  const auto kernel = interleaved ? (fp8 ? rope_append_kernel<kLanes, true, true> : rope_append_kernel<kLanes, true, false>)
                                  : (fp8 ? rope_append_kernel<kLanes, false, true> : rope_append_kernel<kLanes, false, false>);
  kernel<<<blocks, kRopeWarps * 32, 0, stream>>>(p, static_cast<int>(quantised));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_append(const RopeAppendParams& p, bool interleaved, cudaStream_t stream) {
  if (p.geom.head_dim <= 64) return launch<4>(p, interleaved, stream);
  if (p.geom.head_dim <= 128) return launch<8>(p, interleaved, stream);
  return launch<16>(p, interleaved, stream);
}

}  // namespace pda
