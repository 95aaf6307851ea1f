// Attention of few rows per sequence over pages (single tokens, a few drafted ones), bf16: up to 8 NT rows r = i * G + g of a
// (sequence, KV head) pair. Every byte of K and V is used once, so the time is HBM's; the products are made to cost little beside
// it, not the other way round.
//
//   decode_kernel   Every warp is a worker of its own, with a ring of copied tiles that it fills itself, and waits for nobody. All
//                   pairs' tiles are numbered through; worker w takes tiles [w * per, (w + 1) * per), whatever pairs they belong
//                   to, so that ragged lengths leave no worker behind. Of every pair that it meets it leaves a record: the
//                   part's output, normalised, and its log2-sum. (SMs do not get equal shares of the memory, and are busy 83 % of
//                   the time; an eighth of the work drawn in pieces from a counter did not shorten the kernel, 109 us either way
//                   for 8 caches of 16 385 tokens, 64/8 heads, and left hundreds of records to the last pairs.)
//                   Tokens are on the M side of mma.sync (m16n8k16): S^T = K Q^T has a token per row and a query row per
//                   column, O^T += V^T P^T the channels per row; both products take K and V by ldmatrix straight from the
//                   swizzled tiles, and P^T goes from accumulator to operand layout by movmatrix. Maxima are compared with the
//                   reference where they are; only when a logit passes it by 2^8 do lanes exchange anything.
//   finish_kernel   log-sum-exp and output of a pair from its records; and, if wanted, the weight of every slot from the logits
//                   that the decode kernel left in the workspace (8 NT floats per slot beside the 4 D bytes read: reading K a
//                   second time would be 2 D).
//
// P is rounded to bf16 for its product, as in paged_tc.cuh; everything that is summed or carried is fp32. NaN and logits of +inf make
// a row, its statistic and its weights NaN, as there.
#pragma once

#include <cuda.h>

#include "paged_common.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace caote {
namespace paged {
namespace few {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
// Tokens per tile: two 16-token products side by side where a row of 64 channels alone is short work.
template <int D>
constexpr int kTok = D == 128 ? 16 : 32;
template <int D>
constexpr int kTileBytes = kTok<D> * D * 2;
constexpr int kStages = 3;
constexpr int kLeast = 2;  // tiles per worker: fewer only make more records
template <int D>
constexpr size_t decode_smem() { return 1024 + (size_t)kWarps * kStages * 2 * kTileBytes<D> + kWarps * kStages * 8; }
__host__ __device__ inline int tiles_per_worker(int tiles, int workers) {
  const int even = (tiles + workers - 1) / workers;
  return even < kLeast ? kLeast : even;
}

struct Records {
  float* o;       // [pairs + workers][8 NT][D]: worker w's part of pair p at p + w
  float* stat;    // [pairs + workers][8 NT] log2 of the sum of 2^logit
  float* logits;  // [pairs][slots][8 NT] log2 domain; null: no weights wanted
  int* plan;      // [B + 1]: the number of the first tile of every sequence, all tiles
  int slots;      // max_pages * page
};

template <int D>
__device__ __forceinline__ int tiles_of(const Seq& s) { return s.m > 0 ? (s.n + kTok<D> - 1) / kTok<D> : 0; }

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A place in the numbered tiles: a pair, and which of its tiles.
template <int D>
struct Cursor {
  int b, h, tile, tiles;
  Seq s;
  // the next sequence that has tiles (there is one: the caller counts)
  __device__ void enter(const PDims& dm, const Seqs& sq) {
    for (;; ++b) {
      s = sequence(dm, sq, b);
      tiles = tiles_of<D>(s);
      if (tiles > 0) return;
    }
  }
  // true: another pair begins
  __device__ bool advance(const PDims& dm, const Seqs& sq, bool more) {
    if (++tile < tiles) return false;
    tile = 0;
    if (++h == dm.Hkv) {
      h = 0;
      ++b;
      if (more) enter(dm, sq);
    }
    return true;
  }
};

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, 1)
decode_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, PDims dm, Seqs sq,
              const __nv_bfloat16* __restrict__ q, Records rec, int* status) {
  constexpr int kTB = kTileBytes<D>, kT = kTok<D>, kS = kStages, kBoxes = D / 64, kRows = 8 * NT, kSub = kT / 16;
  constexpr int kIds = 32 / kSub;  // tiles whose pages a warp holds
  if (threadIdx.x == 0) {
    ptx::prefetch_map(&tmK);
    ptx::prefetch_map(&tmV);
  }
  ptx::pdl_wait();
  ptx::pdl_trigger();
  extern __shared__ char smem_raw[];
  char* sm = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, lane = tid & 31, warp = ptx::warp_index();
  char* ring = sm + warp * kS * 2 * kTB;  // [stage][K, V]
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + kWarps * kS * 2 * kTB) + warp * kS;
  if (lane == 0) {
    for (int i = 0; i < kS; ++i) ptx::mbar_init(&full[i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  // all tiles, and (one warp of the launch) where the sequences begin
  const bool writes_plan = blockIdx.x == 0 && warp == 0;
  const int workers = gridDim.x * kWarps, w = warp * gridDim.x + blockIdx.x;
  auto what = [&](const Seq& s) { return tiles_of<D>(s) * dm.Hkv; };
  const Scan first = scan(dm, sq, 0, 1, what, writes_plan ? status : nullptr);
  if (writes_plan && lane < dm.B) rec.plan[lane] = first.incl - first.mine;
  int W = first.total;
  for (int b0 = 32; b0 < dm.B; b0 += 32) {
    const Scan c = scan(dm, sq, b0, 1, what, writes_plan ? status : nullptr);
    if (writes_plan && b0 + lane < dm.B) rec.plan[b0 + lane] = W + c.incl - c.mine;
    W += c.total;
  }
  if (writes_plan && lane == 0) rec.plan[dm.B] = W;
  const int per = tiles_per_worker(W, workers);
  const long long begin = (long long)w * per;
  if (begin >= W) return;
  const int count = min(per, W - (int)begin);
  Cursor<D> c;
  {
    Place p;
    find_block(dm, sq, 1, (int)begin, what, first, p);
    c.b = p.b;
    c.s = p.s;
    c.tiles = tiles_of<D>(p.s);
    c.h = p.block / c.tiles;
    c.tile = p.block % c.tiles;
  }
  // ---- copies, a few tiles ahead: lane l of `ids` holds the page of 16-token unit ids_from * kSub + l of the cursor's pair ----
  Cursor<D> p = c;
  int ids = 0, ids_from = -64, issued = 0;
  auto issue = [&]() {
    if (p.tile < ids_from || p.tile >= ids_from + kIds) {
      ids_from = p.tile;
      const int j = ids_from * kT + lane * 16;
      ids = 0;
      if (j < p.s.n) {
        ids = __ldg(sq.table + (size_t)p.b * dm.max_pages + (j >> dm.page_shift));
        if ((unsigned)ids >= (unsigned)dm.n_pages) {
          set_status(status, CAOTE_ERR_BAD_PAGE);
          ids = 0;
        }
      }
    }
    const int st = issued % kS;
    char* dst = ring + st * 2 * kTB;
    int row[kSub];
#pragma unroll
    for (int u = 0; u < kSub; ++u) {  // (behind the length: rows of page 0, masked like all of them)
      const int id = __shfl_sync(0xffffffffu, ids, (p.tile - ids_from) * kSub + u);
      row[u] = ((id * dm.Hkv + p.h) << dm.page_shift) + ((p.tile * kT + u * 16) & ((1 << dm.page_shift) - 1));
    }
    if (ptx::elect_one()) {
      ptx::mbar_expect_tx(&full[st], 2 * kTB);
#pragma unroll
      for (int x = 0; x < kBoxes; ++x)
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
          ptx::tma_load_2d(dst + (x * kT + u * 16) * 128, &tmK, 64 * x, row[u], &full[st]);
          ptx::tma_load_2d(dst + kTB + (x * kT + u * 16) * 128, &tmV, 64 * x, row[u], &full[st]);
        }
    }
    __syncwarp();
    ++issued;
    if (p.advance(dm, sq, issued < count)) ids_from = -64;
  };
  for (int i = 0; i < kS && issued < count; ++i) issue();

  const float scale2 = dm.scale * kLog2e;
  const int quad = lane & 3, oct = lane >> 2;
  uint32_t qf[NT][D / 16][2];
  float ref[NT][2], l[NT][2], acc[NT][D / 16][4];
  int vis[NT][2];  // slots that the lane's two rows of a group of eight see (0: no such row)
  auto begin_pair = [&]() {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int r = 8 * t + oct;
      const bool there = r < c.s.m * dm.G;
      const __nv_bfloat16* src = q + (size_t)(c.s.t0 + (there ? r / dm.G : 0)) * dm.q_stride + (size_t)(c.h * dm.G + (there ? r % dm.G : 0)) * D;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        qf[t][ks][0] = there ? *reinterpret_cast<const uint32_t*>(src + 16 * ks + 2 * quad) : 0u;
        qf[t][ks][1] = there ? *reinterpret_cast<const uint32_t*>(src + 16 * ks + 8 + 2 * quad) : 0u;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = 8 * t + 2 * quad + e;
        vis[t][e] = rr < c.s.m * dm.G ? c.s.n - c.s.m + rr / dm.G + 1 : 0;
        ref[t][e] = -INFINITY;
        l[t][e] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][i][e] = 0.f;
    }
  };
  auto end_pair = [&](int b, int h) {
    const size_t slot = (size_t)(b * dm.Hkv + h) + w;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float inv[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float sum = l[t][e];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        // (0: the row sees none of this part's tokens, or logits of -inf alone; NaN goes on)
        inv[e] = sum == 0.f ? 0.f : 1.f / sum;
        if (oct == 0) rec.stat[slot * kRows + 8 * t + 2 * quad + e] = sum == 0.f ? -INFINITY : ref[t][e] + __log2f(sum);
      }
      float* dst = rec.o + (slot * kRows + 8 * t + 2 * quad) * D + oct;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) dst[(e & 1) * D + 16 * i + 8 * (e >> 1)] = acc[t][i][e] * inv[e & 1];
    }
  };
  // ldmatrix addresses: lane l gives row (l & 15) of the tile, 16 bytes number (l >> 4) of a pair; K as it lies, V transposed:
  // there the matrices are (channels 0-7, tokens 0-7), (channels 8-15, tokens 0-7), (0-7, 8-15), (8-15, 8-15)
  const int krow = lane & 15, kchunk = lane >> 4;
  const int vrow = (lane & 7) + ((lane >> 4) << 3), vchunk = (lane >> 3) & 1;
  const uint32_t ring_a = ptx::smem_u32(ring);
  auto at = [&](int row, int chunk) { return (uint32_t)((chunk >> 3) * (kT * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)); };
  begin_pair();
  for (int i = 0; i < count; ++i) {
    const int st = i % kS;
    tc::mbar_wait(&full[st], (i / kS) & 1, status);
    const uint32_t ka = ring_a + st * 2 * kTB, va = ka + kTB;
    const int j0 = c.tile * kT;
    const int left = c.s.n - j0;
    if (left < kT) {
      // rows behind the length hold anything: zeros, so that 0 * NaN cannot reach O
      for (int x = lane; x < (kT - left) * (D / 8); x += 32) {
        const int row = left + x / (D / 8), chunk = x % (D / 8);
        *reinterpret_cast<uint4*>(ring + st * 2 * kTB + kTB + at(row, chunk)) = make_uint4(0u, 0u, 0u, 0u);
      }
      __syncwarp();
    }
    float sc[kSub][NT][4];
#pragma unroll
    for (int u = 0; u < kSub; ++u)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[u][t][e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        uint32_t a[4];
        ldsm4(ka + at(u * 16 + krow, 2 * ks + kchunk), a);
#pragma unroll
        for (int t = 0; t < NT; ++t) mma16816(sc[u][t], a, qf[t][ks][0], qf[t][ks][1]);
      }
    uint32_t pb[kSub][NT][2];
    // sc[u][t][e]: token 16 u + oct + 8 (e >> 1), row 8 t + 2 quad + (e & 1)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sc[u][t][e] *= scale2;
          if (j0 + u * 16 + oct + 8 * (e >> 1) >= vis[t][e & 1]) sc[u][t][e] = -INFINITY;
          top[e & 1] = fmaxf(top[e & 1], sc[u][t][e]);
        }
        if (rec.logits) {
          float* dst = rec.logits + ((size_t)(c.b * dm.Hkv + c.h) * rec.slots + j0 + u * 16 + oct) * kRows + 8 * t + 2 * quad;
          if (kSub == 1 || j0 + u * 16 < rec.slots) {
            *reinterpret_cast<float2*>(dst) = make_float2(sc[u][t][0], sc[u][t][1]);
            *reinterpret_cast<float2*>(dst + 8 * kRows) = make_float2(sc[u][t][2], sc[u][t][3]);
          }
        }
      }
      if (__any_sync(0xffffffffu, top[0] > ref[t][0] + 8.f || top[1] > ref[t][1] + 8.f)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], o));
          if (top[e] > ref[t][e] + 8.f) {
            const float corr = ptx::fast_exp2(ref[t][e] - top[e]);
            ref[t][e] = top[e];
            l[t][e] *= corr;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) {
              acc[t][x][e] *= corr;
              acc[t][x][e + 2] *= corr;
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        float pr[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) pr[e] = sc[u][t][e] == -INFINITY ? 0.f : ptx::fast_exp2(sc[u][t][e] - ref[t][e & 1]);
        l[t][0] += pr[0] + pr[2];
        l[t][1] += pr[1] + pr[3];
        pb[u][t][0] = transpose8x8(tc::pack_bf16(pr[0], pr[1]));
        pb[u][t][1] = transpose8x8(tc::pack_bf16(pr[2], pr[3]));
      }
    }
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        uint32_t a[4];
        ldsm4t(va + at(u * 16 + vrow, 2 * x + vchunk), a);
#pragma unroll
        for (int t = 0; t < NT; ++t) mma16816(acc[t][x], a, pb[u][t][0], pb[u][t][1]);
      }
    // the stage's reads are done in every lane before the copy that takes its place
    ptx::fence_async_smem();
    __syncwarp();
    if (issued < count) issue();
    const int b = c.b, h = c.h;
    const bool pair_ends = c.advance(dm, sq, i + 1 < count);
    if (pair_ends || i + 1 == count) end_pair(b, h);
    if (pair_ends && i + 1 < count) begin_pair();
  }
}

// grid = (1 + pieces of kChunk slots if the weights are wanted, pairs): CTA 0 of a pair merges its output, CTA 1 + i has the weights of
// slots [i * kChunk, (i + 1) * kChunk).
constexpr int kChunk = 4096, kFinishThreads = 512;
template <int D, int NT>
__global__ void __launch_bounds__(kFinishThreads)
finish_kernel(PDims dm, Seqs sq, Records rec, int workers, __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ mass,
              int* status) {
  constexpr int kRows = 8 * NT;
  ptx::pdl_wait();
  ptx::pdl_trigger();
  __shared__ float s_stat[kRows];
  __shared__ float4 s_part[kFinishThreads];
  const int tid = threadIdx.x, pair = blockIdx.y, b = pair / dm.Hkv, h = pair % dm.Hkv, j0 = ((int)blockIdx.x - 1) * kChunk;
  const Seq s = sequence(dm, sq, b);
  const int start0 = rec.plan[b], all = rec.plan[dm.B];
  if (s.m == 0 || j0 >= s.n) return;
  const int per = tiles_per_worker(all, workers), tiles = tiles_of<D>(s), start = start0 + h * tiles;
  const int first = start / per, n_rec = (start + tiles - 1) / per - first + 1, R = s.m * dm.G;
  const size_t slot = (size_t)pair + first;
  // log2-sums of the rows: 16 threads per row
  for (int r = tid >> 4; r < kRows; r += kFinishThreads / 16) {
    const int e = tid & 15;
    float mx = -INFINITY;
    for (int i = e; i < n_rec; i += 16) mx = fmaxf(mx, rec.stat[(slot + i) * kRows + r]);
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
    float sum = 0.f;  // (the maximum leaves NaN out, the sum does not)
    for (int i = e; i < n_rec; i += 16) {
      const float x = rec.stat[(slot + i) * kRows + r];
      sum += x == -INFINITY ? 0.f : ptx::fast_exp2(x - mx);
    }
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    if (e == 0) s_stat[r] = mx + __log2f(sum);
  }
  __syncthreads();
  if (blockIdx.x == 0) {
    if (lse && tid < R) lse[(size_t)(s.t0 + tid / dm.G) * dm.Hq + h * dm.G + tid % dm.G] = s_stat[tid] * kLn2;
    // four channels per thread; as many groups of threads as there is room for share the records
    const int pieces = R * (D / 4), groups = max(1, kFinishThreads / pieces), at_once = groups > 1 ? pieces : kFinishThreads;
    for (int x0 = 0; x0 < pieces; x0 += at_once) {
      const int grp = tid / at_once, x = x0 + tid % at_once, r = x / (D / 4), ch = x % (D / 4) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (grp < groups && x < pieces) {
#pragma unroll 8
        for (int i = grp; i < n_rec; i += groups) {
          const float wt = ptx::fast_exp2(rec.stat[(slot + i) * kRows + r] - s_stat[r]);
          const float4 y = *reinterpret_cast<const float4*>(rec.o + ((slot + i) * kRows + r) * D + ch);
          v.x = fmaf(wt, y.x, v.x);
          v.y = fmaf(wt, y.y, v.y);
          v.z = fmaf(wt, y.z, v.z);
          v.w = fmaf(wt, y.w, v.w);
        }
      }
      if (groups > 1) {
        s_part[tid] = v;
        __syncthreads();
        if (grp == 0)
          for (int g = 1; g < groups; ++g) {
            const float4 y = s_part[tid + g * at_once];
            v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
          }
        __syncthreads();
      }
      if (grp == 0 && x < pieces)
        *reinterpret_cast<uint2*>(o + ((size_t)(s.t0 + r / dm.G) * dm.Hq + h * dm.G + r % dm.G) * D + ch) =
            make_uint2(tc::pack_bf16(v.x, v.y), tc::pack_bf16(v.z, v.w));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kChunk / kFinishThreads; ++i) {
    const int j = j0 + i * kFinishThreads + tid;
    if (j >= s.n) break;
    float* out = pool_weight(dm, sq, b, h, j, mass, status);
    const float before = out ? *out : 0.f;
    const float4* src = reinterpret_cast<const float4*>(rec.logits + ((size_t)pair * rec.slots + j) * kRows);
    float sum = 0.f;
    if (j <= s.n - s.m) {
#pragma unroll
      for (int e = 0; e < kRows / 4; ++e) {
        if (4 * e >= R) break;
        const float4 x = src[e];
        sum += ptx::fast_exp2(x.x - s_stat[4 * e]);
        if (4 * e + 1 < R) sum += ptx::fast_exp2(x.y - s_stat[4 * e + 1]);
        if (4 * e + 2 < R) sum += ptx::fast_exp2(x.z - s_stat[4 * e + 2]);
        if (4 * e + 3 < R) sum += ptx::fast_exp2(x.w - s_stat[4 * e + 3]);
      }
    } else {  // (new tokens, but the first: the rows before them have nothing to say, even if they are NaN)
#pragma unroll 1
      for (int r = (j - (s.n - s.m)) * dm.G; r < R; ++r) sum += ptx::fast_exp2(reinterpret_cast<const float*>(src)[r] - s_stat[r]);
    }
    if (out) *out = before + sum;
  }
}

}  // namespace few
}  // namespace paged
}  // namespace caote
