// rope_kv_append: norm of each query and key head, rotation by the token's position and the way into the paged cache, in
// one pass over the projection's output.
//
// A head's row lies across D / 16 lanes, each with two 16-byte vectors: for the rotation of halves the vectors i and
// i + rot/16, whose elements are each other's partners, so that it needs no exchange between lanes; the elements that are not
// rotated as neighbouring vectors. A warp takes kRows rows of one token at a time for each of its segments: the
// token's cosines and sines are read once for all of them, and the rows' loads are in flight together. The norm's sum goes
// over the segment by shuffles. All of it is held in 32 bits and rounded once.
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

template <int kLanes, bool kPairs, bool kFp8>
__global__ void __launch_bounds__(kRopeWarps * 32) rope_append_kernel(const __grid_constant__ RopeAppendParams p) {
  constexpr int kSegs = 32 / kLanes, kStep = kSegs * kRows;  // rows of a token that a warp takes
  const int lane = threadIdx.x & 31, seg = lane / kLanes, i = lane % kLanes;
  const int D = p.geom.head_dim, Hkv = p.geom.num_kv_heads, heads = p.num_q_heads + 2 * Hkv;
  const int steps = (heads + kStep - 1) / kStep;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kRopeWarps + (threadIdx.x >> 5);
  const int t = static_cast<int>(item / steps), row0 = static_cast<int>(item % steps) * kStep + seg;
  if (t >= p.n_tokens) return;
  const int slot = p.slot_map[t];
  if (slot < 0) return;  // a padding entry
  const int half = p.rot_dim / 2;
  const bool mine = 16 * i < D, rotated = 16 * i < p.rot_dim;  // (of the last lanes some have no elements)
  const int ca = rotated ? i : 2 * i, cb = rotated ? i + p.rot_dim / 16 : 2 * i + 1;  // this lane's vectors

  // A token's positions and, for this lane's elements, cosines and sines: of halves frequency 8 i + e, the same for both
  // vectors; of pairs 4 i + e for the first vector's and rot / 4 + 4 i + e for the second's. False: a position outside the table.
  auto angles = [&](int tok, float (&c)[8], float (&s)[8]) {
    bool good = true;
    int pos[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const bool used = (p.axes_used >> a) & 1;
      pos[a] = used ? p.positions[a * p.positions_stride + tok] : 0;
      good &= !used || (pos[a] >= 0 && pos[a] < p.table_len);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
    }
    if (!rotated || !good) return good;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int f = kPairs ? (v == 0 ? 4 * i : p.rot_dim / 4 + 4 * i) : 8 * i + 4 * v;
      if ((p.axes_used & (p.axes_used - 1)) == 0) {  // one axis (the others' positions are 0)
        const float* at = p.cos_sin + static_cast<int64_t>(pos[0] + pos[1] + pos[2] + pos[3]) * p.rot_dim;
        const float4 c4 = __ldg(reinterpret_cast<const float4*>(at + f)), s4 = __ldg(reinterpret_cast<const float4*>(at + half + f));
        c[4 * v] = c4.x, c[4 * v + 1] = c4.y, c[4 * v + 2] = c4.z, c[4 * v + 3] = c4.w;
        s[4 * v] = s4.x, s[4 * v + 1] = s4.y, s[4 * v + 2] = s4.z, s[4 * v + 3] = s4.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int ax = p.freq_axis[f + e];
          const float* at = p.cos_sin + static_cast<int64_t>(ax == 0 ? pos[0] : ax == 1 ? pos[1] : ax == 2 ? pos[2] : pos[3]) * p.rot_dim;
          c[4 * v + e] = __ldg(at + f + e);
          s[4 * v + e] = __ldg(at + half + f + e);
        }
      }
    }
    return good;
  };
  float cs[8], sn[8];
  const bool bad_pos = !angles(t, cs, sn);
  const bool in_cache = slot < static_cast<int64_t>(p.geom.num_pages) * kPageSize;
  if (lane == 0 && row0 == 0 && bad_pos) report(p.status, PDA_DEV_BAD_SEQ_LEN);
  if (lane == 0 && row0 == 0 && !in_cache) report(p.status, PDA_DEV_BAD_PAGE);
  const bool store_kv = in_cache && !bad_pos;

  auto source = [&](int tok, int row) {
    return row < p.num_q_heads ? p.q + tok * p.q_token_stride + row * p.q_head_stride
           : row < p.num_q_heads + Hkv ? p.k + tok * p.k_token_stride + (row - p.num_q_heads) * p.k_head_stride
                                       : p.v + tok * p.v_token_stride + (row - p.num_q_heads - Hkv) * p.v_head_stride;
  };
  // norm and rotation of one row (the whole segment takes part)
  auto turn = [&](Row& x, int row, const float (&c)[8], const float (&s)[8]) {
    const __nv_bfloat16* weight = row < p.num_q_heads ? p.q_norm : row < p.num_q_heads + Hkv ? p.k_norm : nullptr;
    if (p.q_norm != nullptr || p.k_norm != nullptr) {  // (uniform: the shuffles are reached by all lanes)
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(x.a[e], x.a[e], fmaf(x.b[e], x.b[e], ss));
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (weight != nullptr && mine) {
        const float inv = 1.f / sqrtf(ss / static_cast<float>(D) + p.eps);
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
    if (row < p.num_q_heads + Hkv && rotated) {
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
  };

  uint4 ra[kRows], rb[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int row = row0 + k * kSegs;
    ra[k] = rb[k] = make_uint4(0, 0, 0, 0);
    if (mine && row < heads) {
      const uint4* src = reinterpret_cast<const uint4*>(source(t, row));
      ra[k] = src[ca];
      rb[k] = src[cb];
    }
  }
  const int page = slot / kPageSize, in_page = slot % kPageSize;
  // e4m3: the token of this call that opens the page, where there is one. Its rows are taken again for their scale.
  bool opened = false;
  float cs0[8], sn0[8];
  if constexpr (kFp8) {
    if (in_page > 0 && in_page <= t && p.slot_map[t - in_page] == slot - in_page) opened = angles(t - in_page, cs0, sn0);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int row = row0 + k * kSegs;
    Row x;
    unpack(ra[k], x.a);
    unpack(rb[k], x.b);
    turn(x, row, cs, sn);
    float scale = 1.f;
    if constexpr (kFp8) {
      const int first = row0 - seg + k * kSegs;  // (of the warp's rows)
      if (first + kSegs > p.num_q_heads && first < heads && store_kv) {  // (uniform)
        const bool kv = row >= p.num_q_heads && row < heads, is_v = row >= p.num_q_heads + Hkv;
        const int64_t at = static_cast<int64_t>(page) * Hkv + (kv ? row - p.num_q_heads - (is_v ? Hkv : 0) : 0);
        if (in_page == 0 || opened) {
          Row o = x;
          if (opened) {
            uint4 oa = make_uint4(0, 0, 0, 0), ob = oa;
            if (mine && kv) {
              const uint4* src = reinterpret_cast<const uint4*>(source(t - in_page, row));
              oa = src[ca];
              ob = src[cb];
            }
            unpack(oa, o.a);
            unpack(ob, o.b);
            turn(o, row, cs0, sn0);
          }
          float top = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(fabsf(o.a[e]), fabsf(o.b[e])));
#pragma unroll
          for (int d = kLanes / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          scale = top > 0.f ? __fdiv_rn(top * 2.f, 448.f) : 1.f;
          if (in_page == 0 && kv && i == 0) (is_v ? p.v_scale : p.k_scale)[at] = scale;
        } else if (kv) {
          scale = (is_v ? p.v_scale : p.k_scale)[at];
        }
      }
    }
    if (!mine || row >= heads) continue;
    if (row < p.num_q_heads) {
      uint4* dst = reinterpret_cast<uint4*>(p.q_out + t * p.qo_token_stride + row * p.qo_head_stride);
      const uint4 zero = make_uint4(0, 0, 0, 0);
      dst[ca] = bad_pos ? zero : pack(x.a);
      dst[cb] = bad_pos ? zero : pack(x.b);
    } else if (store_kv) {
      const bool is_v = row >= p.num_q_heads + Hkv;
      const int g = row - p.num_q_heads - (is_v ? Hkv : 0);
      const int64_t at = page * p.geom.page_stride + g * p.geom.head_stride + in_page * p.geom.slot_stride;
      if constexpr (kFp8) {
        uint2* dst = reinterpret_cast<uint2*>(static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache) + at);
        dst[ca] = pack_e4m3(x.a, scale);
        dst[cb] = pack_e4m3(x.b, scale);
      } else {
        uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(is_v ? p.v_cache : p.k_cache) + at);
        dst[ca] = pack(x.a);
        dst[cb] = pack(x.b);
      }
    }
  }
}

template <int kLanes>
cudaError_t launch(const RopeAppendParams& p, bool interleaved, cudaStream_t stream) {
  const int heads = p.num_q_heads + 2 * p.geom.num_kv_heads, step = 32 / kLanes * kRows;
  const int64_t items = static_cast<int64_t>(p.n_tokens) * ((heads + step - 1) / step);
  const unsigned blocks = static_cast<unsigned>((items + kRopeWarps - 1) / kRopeWarps);
  const bool fp8 = p.geom.dtype == PDA_FP8_E4M3;
  const auto kernel = interleaved ? (fp8 ? rope_append_kernel<kLanes, true, true> : rope_append_kernel<kLanes, true, false>)
                                  : (fp8 ? rope_append_kernel<kLanes, false, true> : rope_append_kernel<kLanes, false, false>);
  kernel<<<blocks, kRopeWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_append(const RopeAppendParams& p, bool interleaved, cudaStream_t stream) {
  if (p.geom.head_dim <= 64) return launch<4>(p, interleaved, stream);
  if (p.geom.head_dim <= 128) return launch<8>(p, interleaved, stream);
  return launch<16>(p, interleaved, stream);
}

}  // namespace pda
