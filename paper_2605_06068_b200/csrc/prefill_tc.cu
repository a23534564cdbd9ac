// Launch of the tcgen05 prompt kernel over the paged cache (prefill_tc.cuh).
#include <cmath>
#include <cstring>

#include "prefill_tc.cuh"

namespace pda {

namespace {

// [tokens][heads][lines][64]: a copy takes one line of the group's heads of as many tokens as fill 128 rows
bool encode_q(CUtensorMap* map, const PrefillParams& p, int tile_rows) {
  EncodeFn enc = tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t dims[4] = {64, static_cast<cuuint64_t>(p.geom.head_dim / 64), static_cast<cuuint64_t>(p.num_q_heads), static_cast<cuuint64_t>(p.total_q)};
  // (a dimension of extent 1 is never stepped over)
  const cuuint64_t strides[3] = {128, p.num_q_heads == 1 ? 128 : static_cast<cuuint64_t>(p.q_head_stride) * 2,
                                 p.total_q == 1 ? 128 : static_cast<cuuint64_t>(p.q_token_stride) * 2};
  const cuuint32_t box[4] = {64, 1, static_cast<cuuint32_t>(p.group), static_cast<cuuint32_t>(tile_rows)};
  const cuuint32_t step[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16*>(p.q), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The polynomials of the cap in the product s: C tanh(u s), u = scale / softcap. Where u is so far from 1 that powers of u or
// of s could leave 32 bits' range, all go the other way.
void set_cap(const ScoreParams& score, int shape, PrefillPlan* plan) {
  // tanh(x) by odd polynomials whose largest error over the range is least (linear programming over 4000 points):
  // 5.3e-6 for |x| <= 1/2, 2.4e-6 for |x| <= 5/4
  static const double c5[3] = {0.9999248385429382, -0.33085504174232483, 0.11254137754440308};
  static const double c11[6] = {0.9999746680259705, -0.33283931016921997, 0.1305362582206726, -0.04692675918340683, 0.01253201998770237,
                                -0.0016820720629766583};
  // above kAbsoluteCap: see cap_score
  static const float relative[6] = PDA_TANH_COEFFICIENTS;
  const double u = static_cast<double>(score.mul) / score.cap;
  const auto twice = [](double v) {
    const float f = static_cast<float>(v);
    uint32_t bits;
    memcpy(&bits, &f, 4);
    return static_cast<uint64_t>(bits) << 32 | bits;
  };
  plan->relative = score.cap > kAbsoluteCap;
  plan->u = static_cast<float>(u);
  const bool usable = std::abs(u) >= 1.0 / 2048 && std::abs(u) <= 1024 && !plan->relative && score.cap >= 1.f / 4096;
  plan->limit[0] = usable ? static_cast<float>(0.5 / std::abs(u)) : -1.f;
  plan->limit[1] = usable ? static_cast<float>(1.25 / std::abs(u)) : -1.f;
  plan->ref = shape & kShapeBias ? 0.f : std::max(score.cap - kGFixedTop, 0.f);
  plan->ref_low = std::min(score.cap - kGFixedLow, plan->ref);
  plan->low_limit = static_cast<float>(std::max(static_cast<double>(kGFixedFloor) - plan->ref, 0.0) / std::abs(static_cast<double>(score.mul)));  // (weights below 2^-60)
  double power = score.mul;
  for (int i = 0; i < 6; ++i, power *= u * u) {
    if (i < 3) plan->poly5[i] = twice(usable ? c5[i] * power : 0.0);
    plan->poly11[i] = twice(plan->relative ? relative[i] * static_cast<double>(score.mul) : usable ? c11[i] * power : 0.0);
  }
}

template <int D, bool kFp8, int kShape>
cudaError_t launch(const PrefillParams& p, const PrefillMaps& maps, const PrefillPlan& plan, int pairs, cudaStream_t stream) {
  using C = GCfg<D, kFp8>;
  const auto kernel = prefill_tc_kernel<D, kShape, kFp8>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
  if (e != cudaSuccess) return e;
  kernel<<<static_cast<unsigned>(2 * pairs), C::kThreads, C::kSmemBytes, stream>>>(maps, p, plan);
  if ((e = cudaGetLastError()) != cudaSuccess || !plan.cut) return e;
  prefill_merge_kernel<D><<<dim3(static_cast<unsigned>(pairs), 8), 256, 0, stream>>>(p, plan, kShape == kShapeNone && !kFp8 ? plan.scale_log2 : 0.f,
                                                                                       (kShape & kShapeCap) && !(kShape & kShapeBias) ? 0.f : 5.4210109e-20f);
  return cudaGetLastError();
}

template <int D, bool kFp8>
cudaError_t launch_shape(const PrefillParams& p, const PrefillMaps& maps, const PrefillPlan& plan, int shape, int pairs, cudaStream_t stream) {
  if (shape == kShapeNone) return launch<D, kFp8, kShapeNone>(p, maps, plan, pairs, stream);
  if (shape == kShapeCap) return launch<D, kFp8, kShapeCap>(p, maps, plan, pairs, stream);
  if (shape == (kShapeCap | kShapeLow)) return launch<D, kFp8, kShapeCap | kShapeLow>(p, maps, plan, pairs, stream);
  if (shape == kShapeBias) return launch<D, kFp8, kShapeBias>(p, maps, plan, pairs, stream);
  return launch<D, kFp8, kShapeCap | kShapeBias>(p, maps, plan, pairs, stream);
}

// e4m3 pages, dims (byte of the line, slot, line, head, page), in lines of 64 bytes: not swizzled, as threads read them that convert
// them to lines of 64 bf16.
bool encode_bytes(CUtensorMap* map, const void* base, const CacheGeom& g) {
  EncodeFn enc = tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t line = 64, lines = static_cast<cuuint64_t>(g.head_dim) / line;
  const cuuint64_t dims[5] = {line, static_cast<cuuint64_t>(kPageSize), lines, static_cast<cuuint64_t>(g.num_kv_heads), static_cast<cuuint64_t>(g.num_pages)};
  const cuuint64_t strides[4] = {static_cast<cuuint64_t>(g.slot_stride), line, static_cast<cuuint64_t>(g.head_stride), static_cast<cuuint64_t>(g.page_stride)};
  const cuuint32_t box[5] = {static_cast<cuuint32_t>(line), kPageSize, 1, 1, 1};
  const cuuint32_t step[5] = {1, 1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 5, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool prefill_tc_supports(const PrefillParams& p) {
  if (p.geom.head_dim != 128 && (p.geom.head_dim != 64 || p.geom.dtype != PDA_BF16)) return false;
  if (p.group > 128 || p.geom.num_pages < 1 || p.geom.num_pages == INT32_MAX) return false;
  const auto fits = [](int64_t stride, int64_t extent) { return extent == 1 || (stride > 0 && stride < (1ll << 38)); };
  if (!fits(p.q_token_stride, p.total_q) || !fits(p.q_head_stride, p.num_q_heads)) return false;
  // (row numbers are counted in 32 bits, up to one block behind the last)
  if (p.total_q > INT32_MAX - 1024) return false;
  const int block_rows = 4 * (128 / p.group);
  return static_cast<int64_t>((p.max_q + block_rows - 1) / block_rows) * p.batch <= INT32_MAX;
}

int64_t prefill_workspace_bytes(int head_dim) {
  return head_dim == 64 || head_dim == 128 ? prefill_records_at(head_dim) + kPreMaxPairs * static_cast<int64_t>(sizeof(PrefillRecord)) : 256;
}

cudaError_t launch_prefill_tc(const PrefillParams& p, cudaStream_t stream) {
  const int tile_rows = 128 / p.group, block_rows = 4 * tile_rows, heads = p.geom.num_kv_heads;
  PrefillMaps maps{};
  const CacheGeom& g = p.geom;
  const bool fp8 = g.dtype == PDA_FP8_E4M3;
  const auto encode_cache = [&](CUtensorMap* map, const void* base) {
    return fp8 ? encode_bytes(map, base, g)
               : make_cache_tensor_map(map, base, g.page_stride, g.head_stride, g.slot_stride, g.num_pages, heads, g.head_dim, 2, 1);
  };
  if (!encode_q(&maps.q, p, tile_rows) || !encode_cache(&maps.k, p.k_cache) || !encode_cache(&maps.v, p.v_cache))
    return cudaErrorNotSupported;
  // One pair of CTAs per two SMs at most; the row blocks of all sequences are at most one a sequence and one for
  // every block_rows query tokens.
  int dev = 0, sms = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  const int all_pairs = std::max(sms / 2, 1);
  const int q_blocks = (p.max_q + block_rows - 1) / block_rows;
  const int64_t places = static_cast<int64_t>(p.batch) + p.total_q / block_rows;
  const int64_t most = std::min(places, static_cast<int64_t>(p.batch) * q_blocks);
  const int listed = most <= kGMaxList ? 1 : 0;
  int64_t pairs = std::min(most * heads, static_cast<int64_t>(all_pairs));
  // Blocks are cut along the keys where that gives each at least two pairs and the table has room for many keys: the merge is a
  // launch of its own.
  const int cut = listed && p.workspace != nullptr && 2 * most * heads <= std::min(all_pairs, kPreMaxPairs) &&
                          static_cast<int64_t>(p.block_table_stride) * kPageSize >= kPreCutKeys ? 1 : 0;
  if (cut) pairs = std::min(all_pairs, kPreMaxPairs);
  // Scores that are only capped have a fixed reference, if the cap allows it; otherwise the bias's form takes them, with slopes of
  // 0, and so it does scores that are not shaped if their factor is not above 0 (they are scaled behind the maximum).
  const float cap = p.score.cap;
  int shape = (cap > 0.f ? kShapeCap : 0) |
              (p.score.slopes != nullptr || cap > kGFixedCap || (cap == 0.f && !(p.score.mul > 0.f)) ? kShapeBias : 0);
  if (shape == kShapeCap && cap + std::max(cap - kGFixedTop, 0.f) > kGFixedFloor) shape |= kShapeLow;
  PrefillPlan plan{q_blocks, tile_rows, listed, listed ? 0 : places, cut, p.score.mul};
  if (cap > 0.f) set_cap(p.score, shape, &plan);
  const int n = static_cast<int>(pairs);
  if (fp8) return launch_shape<128, true>(p, maps, plan, shape, n, stream);
  if (g.head_dim == 128) return launch_shape<128, false>(p, maps, plan, shape, n, stream);
  return launch_shape<64, false>(p, maps, plan, shape, n, stream);
}

}  // namespace pda
