// rope_kv_append: norm of each query and key head, rotation by the token's position and the way into the paged cache, in
// one pass over the projection's output: bytes (16411 tokens of 32 + 16 heads: 391 MB).
//
// A head's row lies across D / 16 lanes, each with two 16-byte vectors: for the rotation of halves the vectors i and
// i + rot/16, whose elements are each other's partners, so that it needs no exchange between lanes; the elements that are not
// rotated as neighbouring vectors. A warp takes kRows rows of one token and one kind at a time for each of its segments
// (queries; or keys and the same heads' values, which are copied): the token's cosines and sines times the norm's weights are
// made once for all of them, and a row's address is one multiply-add. The rows are asked for first, before anything that they
// wait for is known (slot, position, then angles). All of it is held in 32 bits and rounded once.
// e4m3 caches: keys and values go another way, since a row's scale is that of its page's first row. A warp takes one head's
// keys, or values, of kRows tokens a segment one behind the other; of them the first rows of pages give the others their
// scale by shuffles, and only a page that begins before the warp's tokens has its first row read once more.
// Measured: 16411 tokens of 32 + 16 heads with norm 70 us, 5.6 TB/s (0.85 of the copy rate); 5000 tokens of 28 + 8 heads, three
// axes, e4m3 30 us; 64 tokens 4.3 us, which is the launch and the reads that wait for one another.
#include "shaped.cuh"
#include "tcgen05_ptx.cuh"
#include "tma_ptx.cuh"

namespace pda {

namespace {

constexpr int kRopeWarps = 4;
constexpr int kRows = 4;  // rows of each segment of a warp, even

// 16 elements of a row as pairs of floats: words 0 .. 3 of the lane's first vector, then those of the second.
struct Pairs {
  uint64_t x[8];
};
__device__ __forceinline__ Pairs unpack(const uint4& a, const uint4& b) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  Pairs r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.x[e] = f32x2(w[e] << 16, w[e] & 0xffff0000u);
  return r;
}
__device__ __forceinline__ uint64_t both(float v) { return f32x2(__float_as_uint(v), __float_as_uint(v)); }
__device__ __forceinline__ uint32_t to_bf16(uint64_t v) {
  float lo, hi;
  f32x2_split(v, lo, hi);
  return pack2<false>(lo, hi);
}
__device__ __forceinline__ uint2 to_e4m3(const uint64_t* v, float scale) {  // four pairs
  uint32_t h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float lo, hi;
    f32x2_split(v[e], lo, hi);
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(__fdiv_rn(hi, scale)), "f"(__fdiv_rn(lo, scale)));
    h[e] = r;
  }
  return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}

// What a lane has to do with a row: its two vectors, and what they are multiplied by.
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
  // Norm and rotation are y = (x A + x' B) / rms: x' the partner (of halves the other vector's element, of pairs the word's
  // other half), A = cos w, B = -+ sin w' with w, w' the weights of x and x'. They are the same for all of a token's rows of a kind.
  struct Factors {
    uint64_t a[8], b[8];
  };
  __device__ __forceinline__ Factors factors(const __nv_bfloat16* weight, const float (&c)[8], const float (&s)[8]) const {
    Pairs w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w.x[e] = both(1.f);
    if (weight != nullptr && mine)
      w = unpack(__ldg(reinterpret_cast<const uint4*>(weight) + ca), __ldg(reinterpret_cast<const uint4*>(weight) + cb));
    Factors f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (kPairs) {
        float w0, w1;
        f32x2_split(w.x[e], w0, w1);
        f.a[e] = mul_f32x2(w.x[e], both(c[e]));
        f.b[e] = f32x2(__float_as_uint(-s[e] * w1), __float_as_uint(s[e] * w0));
      } else {
        const int k = 2 * (e & 3);
        const uint64_t c2 = f32x2(__float_as_uint(c[k]), __float_as_uint(c[k + 1]));
        const uint64_t s2 = f32x2(__float_as_uint(s[k]), __float_as_uint(s[k + 1])), minus_s2 = f32x2(__float_as_uint(-s[k]), __float_as_uint(-s[k + 1]));
        f.a[e] = mul_f32x2(w.x[e], c2);
        f.b[e] = mul_f32x2(w.x[e ^ 4], e < 4 ? minus_s2 : s2);
      }
    }
    return f;
  }
  // A row by its whole segment (normed: the same in all lanes of the warp).
  __device__ __forceinline__ Pairs turn(const RopeAppendParams& p, const Pairs& x, bool normed, const Factors& f) const {
    float inv = 1.f;
    if (normed) {
      uint64_t s2[2] = {0ull, 0ull};
#pragma unroll
      for (int e = 0; e < 8; ++e) s2[e & 1] = fma_f32x2(x.x[e], x.x[e], s2[e & 1]);
      float s0, s1;
      f32x2_split(add_f32x2(s2[0], s2[1]), s0, s1);
      float ss = s0 + s1;
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      inv = rsqrtf(fmaf(ss, p.inv_dim, p.eps));
    }
    Pairs y;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint64_t partner = x.x[e ^ 4];
      if constexpr (kPairs) {
        float lo, hi;
        f32x2_split(x.x[e], lo, hi);
        partner = f32x2(__float_as_uint(hi), __float_as_uint(lo));
      }
      y.x[e] = mul_f32x2(x.x[e], f.a[e]);
      if (rotated) y.x[e] = fma_f32x2(partner, f.b[e], y.x[e]);
      if (normed) y.x[e] = mul_f32x2(y.x[e], both(inv));
    }
    return y;
  }
};

// A step of one token: kRows queries a segment, or (kKv, of a bf16 cache) the keys of half as many heads and their values.
template <int kLanes, bool kPairs, bool kKv>
__device__ __forceinline__ void token_rows(const RopeAppendParams& p, int t, int step, int lane) {
  constexpr int kSegs = 32 / kLanes, kTurned = kKv ? kRows / 2 : kRows;  // rows of a segment that are turned
  const Lane<kLanes, kPairs> me(p, lane);
  const int heads = kKv ? p.geom.num_kv_heads : p.num_q_heads, row0 = step * kSegs * kTurned + lane / kLanes;
  const __nv_bfloat16* from = kKv ? p.k + t * p.k_token_stride : p.q + t * p.q_token_stride;
  const __nv_bfloat16* from_v = p.v + t * p.v_token_stride;
  const int head_stride = static_cast<int>(kKv ? p.k_head_stride : p.q_head_stride);
  uint4 ra[kRows], rb[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const bool is_v = k >= kTurned;
    const int row = row0 + (is_v ? k - kTurned : k) * kSegs;
    ra[k] = rb[k] = make_uint4(0, 0, 0, 0);
    if (me.mine && row < heads) {
      const uint4* src = reinterpret_cast<const uint4*>(is_v ? from_v + static_cast<int64_t>(row) * static_cast<int>(p.v_head_stride)
                                                             : from + static_cast<int64_t>(row) * head_stride);
      ra[k] = src[me.ca];
      rb[k] = src[me.cb];
    }
  }
  const int slot = __ldg(p.slot_map + t);
  int pos[4];
  const bool good = me.positions(p, t, pos);
  if (slot < 0) return;  // a padding entry
  if (kKv) {
    if (!good) return;   // (reported with the token's queries)
    if (slot >= static_cast<int64_t>(p.geom.num_pages) * kPageSize) return;
  } else if (step == 0 && lane == 0) {
    if (!good) report(p.status, PDA_DEV_BAD_SEQ_LEN);
    if (slot >= static_cast<int64_t>(p.geom.num_pages) * kPageSize) report(p.status, PDA_DEV_BAD_PAGE);
  }
  float cs[8], sn[8];
  me.angles(p, pos, good, cs, sn);
  const __nv_bfloat16* weight = kKv ? p.k_norm : p.q_norm;
  const auto f = me.factors(weight, cs, sn);
  const int64_t cache_row = (slot / kPageSize) * p.geom.page_stride + (slot % kPageSize) * p.geom.slot_stride;
  __nv_bfloat16* to = kKv ? static_cast<__nv_bfloat16*>(p.k_cache) + cache_row : p.q_out + t * p.qo_token_stride;
  __nv_bfloat16* to_v = static_cast<__nv_bfloat16*>(p.v_cache) + cache_row;
  const int to_stride = static_cast<int>(kKv ? p.geom.head_stride : p.qo_head_stride);
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const bool is_v = k >= kTurned;
    const int row = row0 + (is_v ? k - kTurned : k) * kSegs;
    uint4 a = ra[k], b = rb[k];
    if (!is_v) {
      const Pairs y = me.turn(p, unpack(a, b), weight != nullptr, f);
      a = make_uint4(to_bf16(y.x[0]), to_bf16(y.x[1]), to_bf16(y.x[2]), to_bf16(y.x[3]));
      b = make_uint4(to_bf16(y.x[4]), to_bf16(y.x[5]), to_bf16(y.x[6]), to_bf16(y.x[7]));
      if (!kKv && !good) a = b = make_uint4(0, 0, 0, 0);
    }
    if (me.mine && row < heads) {
      uint4* dst = reinterpret_cast<uint4*>((is_v ? to_v : to) + static_cast<int64_t>(row) * to_stride);
      dst[me.ca] = a;
      dst[me.cb] = b;
    }
  }
}

// Keys, or values, of one head and kRows tokens a segment, into an e4m3 cache.
template <int kLanes, bool kPairs>
__device__ __forceinline__ void quantised_rows(const RopeAppendParams& p, uint32_t item, int lane) {
  constexpr int kSegs = 32 / kLanes, kTokens = kSegs * kRows;
  const Lane<kLanes, kPairs> me(p, lane);
  const int Hkv = p.geom.num_kv_heads, seg = lane / kLanes;
  const bool is_v = item & 1;
  const int g = static_cast<int>((item >> 1) % static_cast<uint32_t>(Hkv)), t0 = static_cast<int>((item >> 1) / static_cast<uint32_t>(Hkv)) * kTokens;
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
  // (values go through as they are)
  auto turned = [&](int t, const uint4& a, const uint4& b, bool& good) {
    int pos[4];
    good = me.positions(p, t, pos);
    const Pairs x = unpack(a, b);
    if (is_v) return x;
    float cs[8], sn[8];
    me.angles(p, pos, good, cs, sn);
    return me.turn(p, x, weight != nullptr, me.factors(weight, cs, sn));
  };
  auto largest = [&](const Pairs& x) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float lo, hi;
      f32x2_split(x.x[e], lo, hi);
      top = fmaxf(top, fmaxf(fabsf(lo), fabsf(hi)));
    }
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
    uint4 a, b;
    load(t0 - back, true, a, b);
    bool good;
    const float top = largest(turned(t0 - back, a, b, good));
    if (good) top_before = top;
  }
  Pairs x[kRows];
  float top[kRows];  // of a page's first row; -1 of others
  bool good[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    x[k] = turned(min(t0 + k * kSegs + seg, p.n_tokens - 1), ra[k], rb[k], good[k]);
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
    dst[me.ca] = to_e4m3(&x[k].x[0], scale);
    dst[me.cb] = to_e4m3(&x[k].x[4], scale);
  }
}

// quantised: items of e4m3 keys and values, before all others; q_steps, kv_steps: of a token.
template <int kLanes, bool kPairs, bool kFp8>
__global__ void __launch_bounds__(kRopeWarps * 32, 5) rope_append_kernel(const __grid_constant__ RopeAppendParams p, uint32_t quantised, uint32_t q_steps,
                                                                      uint32_t kv_steps) {
  const int lane = threadIdx.x & 31;
  uint32_t item = blockIdx.x * kRopeWarps + (threadIdx.x >> 5);  // (rows are fewer than 2^31)
  if constexpr (kFp8) {  // (the longer items first)
    if (item < quantised) {
      quantised_rows<kLanes, kPairs>(p, item, lane);
      return;
    }
    item -= quantised;
  }
  const uint32_t steps = q_steps + kv_steps, t = item / steps, step = item - t * steps;
  if (t >= static_cast<uint32_t>(p.n_tokens)) return;
  if (kFp8 || step < q_steps) token_rows<kLanes, kPairs, false>(p, static_cast<int>(t), static_cast<int>(step), lane);
  else token_rows<kLanes, kPairs, true>(p, static_cast<int>(t), static_cast<int>(step - q_steps), lane);
}

template <int kLanes>
cudaError_t launch(const RopeAppendParams& p, bool interleaved, cudaStream_t stream) {
  constexpr int kStep = 32 / kLanes * kRows;
  const bool fp8 = p.geom.dtype == PDA_FP8_E4M3;
  const int Hkv = p.geom.num_kv_heads;
  const uint32_t q_steps = static_cast<uint32_t>((p.num_q_heads + kStep - 1) / kStep), kv_steps = fp8 ? 0 : static_cast<uint32_t>((Hkv + kStep / 2 - 1) / (kStep / 2));
  const int64_t quantised = fp8 ? 2ll * Hkv * ((static_cast<int64_t>(p.n_tokens) + kStep - 1) / kStep) : 0;
  const int64_t items = quantised + static_cast<int64_t>(p.n_tokens) * (q_steps + kv_steps);
  const unsigned blocks = static_cast<unsigned>((items + kRopeWarps - 1) / kRopeWarps);
  const auto kernel = interleaved ? (fp8 ? rope_append_kernel<kLanes, true, true> : rope_append_kernel<kLanes, true, false>)
                                  : (fp8 ? rope_append_kernel<kLanes, false, true> : rope_append_kernel<kLanes, false, false>);
  kernel<<<blocks, kRopeWarps * 32, 0, stream>>>(p, static_cast<uint32_t>(quantised), q_steps, kv_steps);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_append(const RopeAppendParams& p, bool interleaved, cudaStream_t stream) {
  if (p.geom.head_dim <= 64) return launch<4>(p, interleaved, stream);
  if (p.geom.head_dim <= 128) return launch<8>(p, interleaved, stream);
  return launch<16>(p, interleaved, stream);
}

}  // namespace pda
