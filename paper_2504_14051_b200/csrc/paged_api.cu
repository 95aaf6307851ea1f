// C ABI of the paged cache and of packed prompts (include/caote_paged.h): argument validation, workspace carving, dispatch.
#include "../../include/caote_paged.h"

#include <type_traits>

#include "launch.cuh"
#include "paged_common.cuh"
#include "paged_decode.cuh"
#include "paged_evict.cuh"
#include "paged_generic.cuh"
#include "paged_tc.cuh"

namespace caote {
namespace paged {

// Slots of a sequence: numbers of slots a few blocks and rounds of CTAs behind the last one still fit 32 bits.
constexpr long long kMostSlots = (1LL << 31) - (1LL << 16);
static bool params_ok(const caote_paged_params_t* p, bool pages) {
  if (!p) return false;
  if (p->batch < 1 || p->n_kv_heads < 1 || p->n_q_heads < 1 || p->total_new < 1 || p->max_new < 1) return false;
  if (p->n_q_heads % p->n_kv_heads != 0 || p->n_q_heads / p->n_kv_heads > 16 || p->n_kv_heads > 65535) return false;
  if (p->max_new > p->total_new || p->flags != 0 || !(p->scale == p->scale)) return false;
  if ((long long)p->total_new * (p->n_q_heads / p->n_kv_heads) >= (1LL << 28)) return false;
  if (pages) {
    if (p->n_pages < 1 || p->max_pages < 1) return false;
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128 && p->page_size != 256) return false;
    if ((long long)p->n_pages * p->n_kv_heads * p->page_size >= (1LL << 31)) return false;
    if ((long long)p->max_pages * p->page_size > kMostSlots) return false;
  }
  return true;
}
static bool params_supported(const caote_paged_params_t* p) {
  return (p->dtype == CAOTE_BF16 || p->dtype == CAOTE_F32) && (p->head_dim == 64 || p->head_dim == 128);
}
// 0 = dense; else at least a dense row, a multiple of 16 bytes.
static bool stride_ok(const caote_paged_params_t* p, int64_t stride, int heads) {
  const int64_t row = (int64_t)heads * p->head_dim;
  return stride == 0 || (stride >= row && stride % (p->dtype == CAOTE_BF16 ? 8 : 4) == 0 && stride < (1LL << 31));
}

static PDims make_dims(const caote_paged_params_t* p, bool pages, int64_t q_stride, int64_t kv_stride) {
  PDims d;
  d.B = p->batch;
  d.Hq = p->n_q_heads;
  d.Hkv = p->n_kv_heads;
  d.G = d.Hq / d.Hkv;
  d.D = p->head_dim;
  d.page_shift = 0;
  d.n_pages = pages ? p->n_pages : 0;
  d.max_pages = pages ? p->max_pages : 0;
  if (pages)
    while ((1 << d.page_shift) < p->page_size) ++d.page_shift;
  d.T = p->total_new;
  d.max_new = p->max_new;
  d.scale = p->scale;
  d.q_stride = q_stride ? q_stride : (int64_t)d.Hq * d.D;
  d.kv_stride = kv_stride ? kv_stride : (int64_t)d.Hkv * d.D;
  return d;
}

// ---- workspace ------------------------------------------------------------------------------------
// One or the other, never both in one call:
struct Scratch {
  float* lse2;   // [Hkv, T, G] log2-domain log-sum-exp of every row
  float* lpart;  // [splits, T, Hq] and
  float* opart;  // [splits, T, Hq, D]: what the splits of the keys contribute
  float* mass_part;  // prompts: [kMostChunks, T, Hkv] the weights received from the chunks of a prompt's rows
  tcore::SplitNote* notes;  // [1 + SMs] which items' keys were split
  few::Records rec;
};
constexpr int kMostSplits = 16;
constexpr int kMostChunks = 8;    // of a prompt's rows, in the pass for the weights
constexpr int kItemCounter = 12;  // word of the workspace header
// fp32: splits are only made where the row blocks of a call leave room for two CTAs of 64 rows per SM, so splits x rows stays
// below what these hold; a bound that grows with T and does not depend on how the rows lie. bf16: 256 rows of the last round's
// items per SM.
static long long split_rows(const PDims& dm, int dtype) {
  const long long rows = (long long)dm.T * dm.Hq, most = 128LL * g_sm_count;
  if (dtype == CAOTE_BF16) return 256LL * g_sm_count;
  return rows * kMostSplits < most ? rows * kMostSplits : most;
}
// Calls with few rows per sequence over pages take the kernels of paged_decode.cuh: single tokens of groups up to 16, a few drafted
// tokens of small groups. With the weights wanted, up to 16 rows of a pair, since every row's logits are kept in the workspace
// (4 bytes per slot and row); without, up to 32.
constexpr int kFewRowsMass = 16, kFewRows = 32;
static bool few_rows(const PDims& dm, int dtype, bool mass) {
  const long long tiles = ((long long)dm.max_pages << dm.page_shift) / 16 * dm.B * dm.Hkv;  // (at most)
  return dtype == CAOTE_BF16 && dm.max_pages > 0 && dm.scale > 0.f && (long long)dm.max_new * dm.G <= (mass ? kFewRowsMass : kFewRows) &&
         tiles <= kMostSlots && dm.B * dm.Hkv <= 65535;
}
static int few_workers() { return g_sm_count * few::kWarps; }
static size_t carve(const PDims& dm, int dtype, char* base, Scratch* out) {
  size_t off = 0;
  auto take = [&](size_t floats) {
    float* p = reinterpret_cast<float*>(base + off);
    off = align_up(off + floats * sizeof(float), 256);
    return p;
  };
  Scratch s;
  s.lse2 = take((size_t)dm.T * dm.Hq);
  s.lpart = take((size_t)split_rows(dm, dtype));
  s.opart = take((size_t)split_rows(dm, dtype) * dm.D);
  s.notes = reinterpret_cast<tcore::SplitNote*>(take(4 * (size_t)(1 + g_sm_count)));
  s.mass_part = take(dtype == CAOTE_BF16 ? (size_t)kMostChunks * dm.T * dm.Hkv : 0);
  size_t most = off;
  if (dtype == CAOTE_BF16 && dm.max_pages > 0) {
    // (a workspace for more rows per sequence serves calls with fewer: sized for the most rows that come here)
    off = 0;
    const long long r = (long long)dm.max_new * dm.G;
    const size_t rows = r > kFewRows ? kFewRows : (size_t)(r + 7) / 8 * 8, pairs = (size_t)dm.B * dm.Hkv;
    s.rec.slots = dm.max_pages << dm.page_shift;
    s.rec.plan = reinterpret_cast<int*>(take((size_t)dm.B + 1));
    const size_t records = pairs + few_workers();
    s.rec.stat = take(records * rows);
    s.rec.o = take(records * rows * dm.D);
    s.rec.logits = take(pairs * s.rec.slots * (rows > kFewRowsMass ? kFewRowsMass : rows));
    if (off > most) most = off;
  }
  if (out) *out = s;
  return most;
}
static size_t workspace_bytes(const caote_paged_params_t* p) {
  refresh_sm_count();
  return kHeaderBytes + carve(make_dims(p, p->page_size > 0, 0, 0), p->dtype, nullptr, nullptr);
}
static bool workspace_ok(const void* workspace, size_t have, size_t need) { return workspace && have >= need && aligned(workspace, 256); }

// ---- the any-type path --------------------------------------------------------------------------------
template <typename T, int D, bool kPaged>
static int attend_generic(const PDims& dm, const Seqs& sq, const void* q, const void* K, const void* V, void* o, float* lse, float* mass,
                          char* ws, cudaStream_t st) {
  Scratch sc;
  carve(dm, std::is_same<T, float>::value ? CAOTE_F32 : CAOTE_BF16, ws + kHeaderBytes, &sc);
  int* status = reinterpret_cast<int*>(ws);
  const long long cap = (long long)dm.max_pages << dm.page_shift;
  auto row_blocks = [&](int rows) { return ((long long)dm.T * dm.G + dm.B * (rows - 1LL)) / rows; };  // (no way to lie makes more)
  auto key_blocks = [&](int keys) { return kPaged ? dm.B * ((cap + keys - 1) / keys) : ((long long)dm.T + dm.B * (keys - 1LL)) / keys; };
  if (key_blocks(16) > 0x7fffffffLL) return CAOTE_ERR_UNSUPPORTED;
  // Sixteen rows per CTA where sequences have no more, and 32 where 64 leave SMs idle (prompts of 243, 363 and 95 tokens, 4/2 heads,
  // 64 channels: 55 us with 64, 29 with 16, 26 with 32).
  auto attention = [&](auto rpt) -> int {
    constexpr int RPT = decltype(rpt)::value;
    const size_t smem = generic::attend_smem<D, RPT>();
    const long long blocks = row_blocks(generic::kRows<RPT>);
    long long splits = 2LL * g_sm_count / (blocks * dm.Hkv);
    const long long tiles = kPaged ? (cap + generic::kKeys - 1) / generic::kKeys : 0;
    if (splits > tiles / generic::kLeastTiles) splits = tiles / generic::kLeastTiles;
    if (splits > kMostSplits) splits = kMostSplits;
    if (splits < 1) splits = 1;
    int rc = allow_smem(generic::attend_kernel<T, D, RPT, kPaged>, smem);
    if (rc) return rc;
    CAOTE_LAUNCH("paged_attend_generic", st,
                 launch_pdl(generic::attend_kernel<T, D, RPT, kPaged>, dim3((unsigned)blocks, dm.Hkv, (unsigned)splits), dim3(generic::kThreads),
                            smem, st, dm, sq, (const T*)q, (const T*)K, (const T*)V, (T*)o, lse, sc.lse2, sc.opart, sc.lpart, status));
    if (splits > 1)
      CAOTE_LAUNCH("paged_combine", st,
                   launch_pdl(generic::combine_kernel<T, D>, dim3((unsigned)(((long long)dm.T * dm.Hq + 7) / 8)), dim3(256), 0, st, dm, sq,
                              (int)splits, generic::kKeys, generic::kLeastTiles, (const float*)sc.opart, (const float*)sc.lpart, (T*)o, lse,
                              sc.lse2));
    return CAOTE_OK;
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 4> four;
  const std::integral_constant<int, 2> two;
  int rc = dm.max_new * dm.G <= 24 ? attention(one) : row_blocks(64) * dm.Hkv < 2 * g_sm_count ? attention(two) : attention(four);
  if (rc || !mass) return rc;
  auto weights = [&](auto rpt, auto kpt) -> int {
    constexpr int RPT = decltype(rpt)::value, KPT = decltype(kpt)::value;
    const size_t smem = generic::mass_smem<D, RPT, KPT>();
    int rc = allow_smem(generic::mass_kernel<T, D, RPT, KPT, kPaged>, smem);
    if (rc) return rc;
    CAOTE_LAUNCH("paged_mass_generic", st,
                 launch_pdl(generic::mass_kernel<T, D, RPT, KPT, kPaged>, dim3((unsigned)key_blocks(16 * KPT), dm.Hkv), dim3(generic::kThreads), smem,
                            st, dm, sq, (const T*)q, (const T*)K, (const float*)sc.lse2, mass, status));
    return CAOTE_OK;
  };
  if (dm.max_new * dm.G <= 24) return weights(one, four);
  return key_blocks(64) * dm.Hkv < 2 * g_sm_count ? weights(four, one) : weights(four, four);
}

// ---- the tensor-core path -------------------------------------------------------------------------------
static int encode_failed(CUresult r) {
  snprintf(g_cuda_error, sizeof(g_cuda_error), "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
  return CAOTE_ERR_CUDA;
}
// q [T, Hq, d] as boxes of 64 channels x G heads x 128 / G tokens.
static int encode_q(const PDims& dm, const void* q, CUtensorMap* tm) {
  const cuuint64_t dim[3] = {(cuuint64_t)dm.D, (cuuint64_t)dm.Hq, (cuuint64_t)dm.T};
  const cuuint64_t stride[2] = {(cuuint64_t)dm.D * 2, (cuuint64_t)dm.q_stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)dm.G, (cuuint32_t)(tcore::kTile / dm.G)}, step[3] = {1, 1, 1};
  const CUresult r = tensor_map_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(q), dim, stride, box, step,
                                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? CAOTE_OK : encode_failed(r);
}
// K or V as boxes of 64 channels x `box` tokens: the pool's rows, or a prompt's rows with their heads side by side.
static int encode_keys(const PDims& dm, const void* x, bool pages, int box_tokens, CUtensorMap* tm) {
  const cuuint64_t dim[2] = {(cuuint64_t)dm.D * (pages ? 1 : dm.Hkv),
                             pages ? (cuuint64_t)dm.n_pages * dm.Hkv << dm.page_shift : (cuuint64_t)dm.T};
  const cuuint64_t stride[1] = {(cuuint64_t)(pages ? dm.D : dm.kv_stride) * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_tokens}, step[2] = {1, 1};
  const CUresult r = tensor_map_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(x), dim, stride, box, step,
                                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? CAOTE_OK : encode_failed(r);
}

template <int D, bool kPaged>
static int attend_tc(const PDims& dm, const Seqs& sq, const void* q, const void* K, const void* V, void* o, float* lse, float* mass, char* ws,
                     cudaStream_t st) {
  if (!tensor_map_encoder()) {
    snprintf(g_cuda_error, sizeof(g_cuda_error), "cuTensorMapEncodeTiled is not to be had");
    return CAOTE_ERR_CUDA;
  }
  Scratch sc;
  carve(dm, CAOTE_BF16, ws + kHeaderBytes, &sc);
  int* status = reinterpret_cast<int*>(ws);
  const int box = kPaged && dm.page_shift < 7 ? 1 << dm.page_shift : tcore::kTile;
  CUtensorMap tmQ, tmK, tmV;
  int rc = encode_q(dm, q, &tmQ);
  if (!rc) rc = encode_keys(dm, K, kPaged, box, &tmK);
  if (!rc) rc = encode_keys(dm, V, kPaged, box, &tmV);
  if (!rc) rc = allow_smem(tcore::attend_kernel<D, kPaged>, tcore::attend_smem<D>());
  if (!rc && mass) rc = allow_smem(tcore::mass_kernel<D, kPaged>, tcore::mass_smem<D>());
  if (rc) return rc;
  const int tok = tcore::kTile / dm.G;
  const long long items = (dm.T + dm.B * (2LL * tok - 1)) / (2 * tok) * dm.Hkv, cap = (long long)dm.max_pages << dm.page_shift;
  // Keys are split where a last round would leave SMs idle and there are keys to split. Prompts of many rounds end with short
  // items as it is.
  const long long tiles = ((kPaged ? cap : dm.max_new) + tcore::kTile - 1) / tcore::kTile;
  const int most_splits = tiles >= 2 * tcore::kLeastTiles && (kPaged || items < 2 * g_sm_count) ? kMostSplits : 1;
  // (items of the mass kernel are numbered in 32 bits)
  const long long key_blocks = (kPaged ? (cap + tcore::kKeys - 1) / tcore::kKeys * dm.B : ((long long)dm.T / tcore::kKeys + dm.B) * kMostChunks) * dm.Hkv;
  if (items > 0x7fff0000LL || key_blocks > 0x7fff0000LL) return CAOTE_ERR_UNSUPPORTED;
  CAOTE_LAUNCH("paged_attend_kernel", st,
               launch_pdl(tcore::attend_kernel<D, kPaged>, dim3((unsigned)(items + (most_splits > 1 ? g_sm_count : 0))),
                          dim3(tcore::kAttendThreads), tcore::attend_smem<D>(), st, tmQ, tmK, tmV, dm, sq, box, (__nv_bfloat16*)o, lse, sc.lse2,
                          sc.opart, sc.lpart, sc.notes, g_sm_count, most_splits, status + kItemCounter, status));
  if (most_splits > 1)
    CAOTE_LAUNCH("paged_combine", st,
                 launch_pdl(tcore::combine_kernel<D>, dim3((unsigned)(items < g_sm_count ? items : g_sm_count - 1), 8), dim3(256), 0, st, dm, sq, (__nv_bfloat16*)o, lse, sc.lse2,
                            (const float*)sc.opart, (const float*)sc.lpart, (const tcore::SplitNote*)sc.notes));
  if (mass) {
    // row blocks of the longest prompt, of an SM's share if the prompts are alike, and of a chunk
    const long long longest = (dm.max_new + tok - 1) / tok, share = (long long)dm.Hkv * dm.T / tcore::kKeys * (dm.T / dm.B / tok) / 2 / g_sm_count;
    long long chunk = longest;
    if (!kPaged) {
      chunk = share / 3 > 16 ? share / 3 : 16;
      if (chunk < (longest + kMostChunks - 1) / kMostChunks) chunk = (longest + kMostChunks - 1) / kMostChunks;
    }
    const int chunks = (int)((longest + chunk - 1) / chunk);
    CAOTE_LAUNCH("paged_mass_kernel", st,
                 launch_pdl(tcore::mass_kernel<D, kPaged>, dim3(g_sm_count), dim3(tcore::kMassThreads), tcore::mass_smem<D>(), st, tmQ, tmK, dm,
                            sq, box, (const float*)sc.lse2, chunks > 1 ? sc.mass_part : mass, chunks, (int)chunk, status + kItemCounter, status));
    if (chunks > 1)
      CAOTE_LAUNCH("paged_sum_kernel", st,
                   launch_pdl(tcore::sum_kernel, dim3((unsigned)(((long long)dm.T * dm.Hkv + 255) / 256)), dim3(256), 0, st, dm, sq,
                              (const float*)sc.mass_part, (int)chunk, mass));
  }
  return CAOTE_OK;
}

template <int D, int NT>
static int attend_few(const PDims& dm, const Seqs& sq, const void* q, const void* K, const void* V, void* o, float* lse, float* mass, char* ws,
                      cudaStream_t st) {
  if (!tensor_map_encoder()) {
    snprintf(g_cuda_error, sizeof(g_cuda_error), "cuTensorMapEncodeTiled is not to be had");
    return CAOTE_ERR_CUDA;
  }
  Scratch sc;
  carve(dm, CAOTE_BF16, ws + kHeaderBytes, &sc);
  if (!mass) sc.rec.logits = nullptr;
  int* status = reinterpret_cast<int*>(ws);
  CUtensorMap tmK, tmV;
  int rc = encode_keys(dm, K, true, 16, &tmK);
  if (!rc) rc = encode_keys(dm, V, true, 16, &tmV);
  if (!rc) rc = allow_smem(few::decode_kernel<D, NT>, few::decode_smem<D>());
  if (rc) return rc;
  CAOTE_LAUNCH("paged_decode_kernel", st,
               launch_pdl(few::decode_kernel<D, NT>, dim3(g_sm_count), dim3(few::kThreads), few::decode_smem<D>(), st, tmK, tmV, dm, sq,
                          (const __nv_bfloat16*)q, sc.rec, status));
  const int pieces = mass ? (sc.rec.slots + few::kChunk - 1) / few::kChunk : 0;
  CAOTE_LAUNCH("paged_finish_kernel", st,
               launch_pdl(few::finish_kernel<D, NT>, dim3(1 + pieces, dm.B * dm.Hkv), dim3(few::kFinishThreads), 0, st, dm, sq, sc.rec, few_workers(),
                          (__nv_bfloat16*)o, lse, mass,
                          status));
  return CAOTE_OK;
}

template <bool kPaged>
static int attend(const caote_paged_params_t* p, const PDims& dm, const Seqs& sq, const void* q, const void* K, const void* V, void* o,
                  float* lse, float* mass, char* ws, cudaStream_t st) {
  if (p->dtype == CAOTE_F32)
    return dm.D == 128 ? attend_generic<float, 128, kPaged>(dm, sq, q, K, V, o, lse, mass, ws, st)
                       : attend_generic<float, 64, kPaged>(dm, sq, q, K, V, o, lse, mass, ws, st);
  if constexpr (kPaged) {
    if (few_rows(dm, p->dtype, mass != nullptr)) {
      auto run = [&](auto d) -> int {
        constexpr int D = decltype(d)::value;
        switch ((dm.max_new * dm.G + 7) / 8) {
          case 1: return attend_few<D, 1>(dm, sq, q, K, V, o, lse, mass, ws, st);
          case 2: return attend_few<D, 2>(dm, sq, q, K, V, o, lse, mass, ws, st);
          case 3: return attend_few<D, 3>(dm, sq, q, K, V, o, lse, mass, ws, st);
          default: return attend_few<D, 4>(dm, sq, q, K, V, o, lse, mass, ws, st);
        }
      };
      return dm.D == 128 ? run(std::integral_constant<int, 128>{}) : run(std::integral_constant<int, 64>{});
    }
  }
  if (dm.scale > 0.f)  // (the tensor-core kernels take the largest product for the largest logit)
    return dm.D == 128 ? attend_tc<128, kPaged>(dm, sq, q, K, V, o, lse, mass, ws, st) : attend_tc<64, kPaged>(dm, sq, q, K, V, o, lse, mass, ws, st);
  return dm.D == 128 ? attend_generic<__nv_bfloat16, 128, kPaged>(dm, sq, q, K, V, o, lse, mass, ws, st)
                     : attend_generic<__nv_bfloat16, 64, kPaged>(dm, sq, q, K, V, o, lse, mass, ws, st);
}

}  // namespace paged
}  // namespace caote

using namespace caote;

extern "C" {

size_t caote_paged_workspace_bytes(const caote_paged_params_t* p) {
  if (!p || !paged::params_ok(p, p->page_size != 0) || !paged::params_supported(p)) return 0;
  return paged::workspace_bytes(p);
}

int caote_prompt_attend(const caote_paged_params_t* p, const void* q, int64_t q_stride, const void* k, const void* v, int64_t kv_stride,
                        const int32_t* cu, void* o, float* lse, float* mass, void* workspace, size_t workspace_bytes,
                        caote_stream_t stream) {
  if (!paged::params_ok(p, false) || !q || !k || !v || !cu || !o) return CAOTE_ERR_INVALID_ARG;
  if (!paged::params_supported(p)) return CAOTE_ERR_UNSUPPORTED;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16)) return CAOTE_ERR_INVALID_ARG;
  if (!paged::stride_ok(p, q_stride, p->n_q_heads) || !paged::stride_ok(p, kv_stride, p->n_kv_heads)) return CAOTE_ERR_INVALID_ARG;
  refresh_sm_count();
  const paged::PDims dm = paged::make_dims(p, false, q_stride, kv_stride);
  if (!paged::workspace_ok(workspace, workspace_bytes, kHeaderBytes + paged::carve(dm, p->dtype, nullptr, nullptr))) return CAOTE_ERR_INVALID_ARG;
  int rc = check_device();
  if (rc) return rc;
  return paged::attend<false>(p, dm, paged::Seqs{cu, nullptr, nullptr}, q, k, v, o, lse, mass, (char*)workspace, (cudaStream_t)stream);
}

int caote_paged_append(const caote_paged_params_t* p, void* K, void* V, float* mass, int32_t* pos, const int32_t* page_table,
                       int32_t* len, int32_t* n_seen, const void* k_new, const void* v_new, int64_t kv_stride,
                       const float* mass_new, const int32_t* cu, void* workspace, size_t workspace_bytes, caote_stream_t stream) {
  if (!paged::params_ok(p, true) || !K || !V || !page_table || !len || !k_new || !v_new || !cu) return CAOTE_ERR_INVALID_ARG;
  if (!paged::params_supported(p)) return CAOTE_ERR_UNSUPPORTED;
  if (!aligned(K, 16) || !aligned(V, 16) || !aligned(k_new, 16) || !aligned(v_new, 16)) return CAOTE_ERR_INVALID_ARG;
  if (!paged::stride_ok(p, kv_stride, p->n_kv_heads)) return CAOTE_ERR_INVALID_ARG;
  if (!paged::workspace_ok(workspace, workspace_bytes, kHeaderBytes)) return CAOTE_ERR_INVALID_ARG;
  int rc = check_device();
  if (rc) return rc;
  refresh_sm_count();
  const paged::PDims dm = paged::make_dims(p, true, 0, kv_stride);
  const int e = p->dtype == CAOTE_BF16 ? 2 : 4, row_bytes = dm.D * e;
  const long long pieces = (long long)dm.T * dm.Hkv * 2 * (row_bytes / 16);
  long long ctas = (pieces + paged::kAppendThreads - 1) / paged::kAppendThreads;
  if (ctas > (long long)paged::kAppendCtas * g_sm_count) ctas = (long long)paged::kAppendCtas * g_sm_count;
  CAOTE_LAUNCH("paged_append_kernel", (cudaStream_t)stream,
               launch_pdl(paged::append_kernel, dim3((unsigned)ctas), dim3(paged::kAppendThreads), 0, (cudaStream_t)stream, dm,
                          paged::Seqs{cu, len, page_table}, row_bytes, dm.kv_stride * e, (char*)K, (char*)V, mass, pos, len, n_seen,
                          (const char*)k_new, (const char*)v_new, mass_new, (int*)workspace, (int*)workspace + 4));
  return CAOTE_OK;
}

int caote_paged_attend(const caote_paged_params_t* p, const void* q, int64_t q_stride, const void* K, const void* V, float* mass,
                       const int32_t* page_table, const int32_t* len, const int32_t* cu, void* o, float* lse, void* workspace,
                       size_t workspace_bytes, caote_stream_t stream) {
  if (!paged::params_ok(p, true) || !q || !K || !V || !page_table || !len || !cu || !o) return CAOTE_ERR_INVALID_ARG;
  if (!paged::params_supported(p)) return CAOTE_ERR_UNSUPPORTED;
  if (!aligned(q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(o, 16)) return CAOTE_ERR_INVALID_ARG;
  if (!paged::stride_ok(p, q_stride, p->n_q_heads)) return CAOTE_ERR_INVALID_ARG;
  refresh_sm_count();
  const paged::PDims dm = paged::make_dims(p, true, q_stride, 0);
  if (!paged::workspace_ok(workspace, workspace_bytes, kHeaderBytes + paged::carve(dm, p->dtype, nullptr, nullptr))) return CAOTE_ERR_INVALID_ARG;
  int rc = check_device();
  if (rc) return rc;
  return paged::attend<true>(p, dm, paged::Seqs{cu, len, page_table}, q, K, V, o, lse, mass, (char*)workspace, (cudaStream_t)stream);
}

int caote_paged_evict(const caote_paged_params_t* p, void* K, void* V, float* mass, int32_t* pos, const int32_t* page_table,
                      int32_t* len, const int32_t* n_seen, const int32_t* budget, int32_t sinks, int32_t recent, int32_t* evict_idx,
                      int32_t max_evict, int32_t* n_evict, void* workspace, size_t workspace_bytes, caote_stream_t stream) {
  if (!paged::params_ok(p, true) || !K || !V || !mass || !pos || !page_table || !len || !n_seen || !budget || !evict_idx || !n_evict)
    return CAOTE_ERR_INVALID_ARG;
  if (!paged::params_supported(p)) return CAOTE_ERR_UNSUPPORTED;
  if (sinks < 0 || recent < 0 || max_evict < 1 || !aligned(K, 16) || !aligned(V, 16)) return CAOTE_ERR_INVALID_ARG;
  if ((long long)p->batch * p->n_kv_heads >= (1LL << 28)) return CAOTE_ERR_INVALID_ARG;
  if (!paged::workspace_ok(workspace, workspace_bytes, kHeaderBytes)) return CAOTE_ERR_INVALID_ARG;
  int rc = check_device();
  if (rc) return rc;
  const paged::PDims dm = paged::make_dims(p, true, 0, 0);
  const int row_bytes = dm.D * (p->dtype == CAOTE_BF16 ? 2 : 4);
  // One token per pair: a cluster per sequence, whose first CTA moves the length on. Several: up to four CTAs per pair while they
  // all run at once, for the rows that move (64 pairs, 512 rows each: 9 us of moves on single CTAs, half of it on two).
  const bool by_sequence = max_evict == 1 && dm.Hkv <= 8;
  int c = by_sequence ? dm.Hkv : 1;
  if (!by_sequence && max_evict >= 64) {
    refresh_sm_count();
    while (c < 4 && (long long)dm.B * dm.Hkv * 2 * c <= g_sm_count) c *= 2;
  }
  CAOTE_LAUNCH("paged_evict_kernel", (cudaStream_t)stream,
               launch_pdl_clusters(paged::evict_kernel, dim3((unsigned)(dm.B * dm.Hkv * (by_sequence ? 1 : c))), dim3(paged::kEvictThreads), 0, c,
                                   (cudaStream_t)stream, dm, paged::Seqs{nullptr, len, page_table}, paged::Pool{(char*)K, (char*)V, mass, pos},
                                   row_bytes, len, n_seen, budget, sinks, recent, evict_idx, max_evict, n_evict, by_sequence, (int*)workspace,
                                   (int*)workspace + 4));
  return CAOTE_OK;
}

}  // extern "C"
