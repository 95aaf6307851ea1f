// Attention of packed rows over prompts or pages in fp32 on the CUDA cores: every fp32 call, and the bf16 ones whose scale is
// not positive.
//
//   attend_kernel    kRows query rows of a (sequence, KV head) pair against its keys (or one of their splits), 64 keys at a
//                    time: logits, running maximum and sum per row, output. A thread has RPT rows x 4 keys of the logits
//                    and RPT rows x D / 16 channels of the output. Copies of K and V take turns with the arithmetic.
//   combine_kernel   o = sum_s o_s 2^(lse_s - lse) over the splits of a row.
//   mass_kernel      16 KPT keys against all rows that see them: the logits again, 2^(s - lse) summed over the rows. Every
//                    key's sum is formed by one CTA in a fixed order.
//
// What bounds them: shared-memory reads, 8 of 16 bytes for 64 multiply-adds in the logits (RPT 4).
#pragma once

#include "paged_common.cuh"
#include "ptx.cuh"

namespace caote {
namespace paged {
namespace generic {

constexpr int kThreads = 256, kKeys = 64, kLeastTiles = 4;
constexpr int kP = kKeys + 4;  // pitch of the weights
template <int D>
constexpr int kPitch = D + 4;  // pitch of q, K and V rows: 16 bytes further per row, so that 16 rows read without conflicts
template <int RPT>
constexpr int kRows = 16 * RPT;
template <int D, int RPT>
constexpr size_t attend_smem() { return sizeof(float) * (size_t)((kRows<RPT> + 2 * kKeys) * kPitch<D> + kRows<RPT> * kP) + 64; }
template <int D, int RPT, int KPT>
constexpr size_t mass_smem() { return sizeof(float) * (size_t)((2 * kRows<RPT> + 16 * KPT) * kPitch<D> + 16 * kP) + 64; }

// Four elements into shared memory as floats: fp32 by an asynchronous copy of the thread's own, bf16 through registers.
__device__ __forceinline__ void put4(float* dst, const float* src, bool there) { ptx::cp_async16(dst, src, there); }
__device__ __forceinline__ void put4(float* dst, const __nv_bfloat16* src, bool there) {
  *reinterpret_cast<float4*>(dst) = there ? load4(src) : make_float4(0.f, 0.f, 0.f, 0.f);
}
// Rows of q into shared memory, padded with zeros: row r0 + i of the pair. One group of copies.
template <typename T, int D, int RPT>
__device__ __forceinline__ void load_rows(const PDims& dm, const GroupDiv& by_g, const T* __restrict__ q, const Seq& s, int h, int r0, float* Qs) {
  const int R = s.m * dm.G;
  for (int i = threadIdx.x; i < kRows<RPT> * (D / 4); i += kThreads) {
    const int row = i / (D / 4), c = i % (D / 4), r = r0 + row;
    const bool there = r < R;
    const int t = by_g(r);
    put4(Qs + row * kPitch<D> + 4 * c, there ? q + (size_t)(s.t0 + t) * dm.q_stride + (size_t)(h * dm.G + r - t * dm.G) * D + 4 * c : q, there);
  }
  ptx::cp_async_commit();
}
// 16 KPT rows of K or V from slot j0 on; rows behind the length are zeros (whatever lies there does not reach a product). One group.
template <typename T, int D, int KPT, bool kPaged>
__device__ __forceinline__ void load_keys(const PDims& dm, const Seqs& sq, const T* __restrict__ X, const Seq& s, int b, int h, int j0,
                                          float* Xs, int* status) {
  for (int i = threadIdx.x; i < 16 * KPT * (D / 4); i += kThreads) {
    const int row = i / (D / 4), c = i % (D / 4), j = j0 + row;
    const bool there = j < s.n;
    size_t at = 0;
    if (there) at = (kPaged ? pool_row(dm, sq, b, h, j, status) * D : (size_t)(s.t0 + j) * dm.kv_stride + (size_t)h * D) + 4 * c;
    put4(Xs + row * kPitch<D> + 4 * c, X + at, there);
  }
  ptx::cp_async_commit();
}
// Logits in the log2 domain of rows ty * RPT + r and keys tx + 16 c.
template <int D, int RPT, int KPT>
__device__ __forceinline__ void logits(const float* Qs, const float* Ks, float scale2, float (&s)[RPT][KPT]) {
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int r = 0; r < RPT; ++r)
#pragma unroll
    for (int c = 0; c < KPT; ++c) s[r][c] = 0.f;
#pragma unroll 4
  for (int k = 0; k < D; k += 4) {
    float4 kv[KPT];
#pragma unroll
    for (int c = 0; c < KPT; ++c) kv[c] = *reinterpret_cast<const float4*>(Ks + (tx + 16 * c) * kPitch<D> + k);
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
      const float4 qv = *reinterpret_cast<const float4*>(Qs + (ty * RPT + r) * kPitch<D> + k);
#pragma unroll
      for (int c = 0; c < KPT; ++c)
        s[r][c] = fmaf(qv.w, kv[c].w, fmaf(qv.z, kv[c].z, fmaf(qv.y, kv[c].y, fmaf(qv.x, kv[c].x, s[r][c]))));
    }
  }
#pragma unroll
  for (int r = 0; r < RPT; ++r)
#pragma unroll
    for (int c = 0; c < KPT; ++c) s[r][c] *= scale2;
}

// grid = (row blocks of all sequences, Hkv, splits).
template <typename T, int D, int RPT, bool kPaged>
__global__ void __launch_bounds__(kThreads)
attend_kernel(PDims dm, Seqs sq, const T* __restrict__ q, const T* __restrict__ K, const T* __restrict__ V, T* __restrict__ o,
              float* __restrict__ lse, float* __restrict__ lse2, float* __restrict__ opart, float* __restrict__ lpart, int* status) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  extern __shared__ __align__(16) float smf[];
  float* Qs = smf;
  float* Ks = Qs + kRows<RPT> * kPitch<D>;
  float* Vs = Ks + kKeys * kPitch<D>;
  float* Ps = Vs + kKeys * kPitch<D>;
  int* where = reinterpret_cast<int*>(Ps + kRows<RPT> * kP);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, h = blockIdx.y, split = blockIdx.z;
  if (tid < 32) {
    auto what = [&](const Seq& x) { return x.m * dm.G; };
    Place p;
    Scan c = scan(dm, sq, 0, kRows<RPT>, what, nullptr);
    const bool there = find_block(dm, sq, kRows<RPT>, blockIdx.x, what, c, p);
    if (tid == 0) { where[0] = there ? p.b : -1; where[1] = p.block; }
    if (blockIdx.x == 0 && h == 0 && split == 0)
      for (int x = tid; x < dm.B; x += 32) sequence(dm, sq, x, status);
  }
  __syncthreads();
  const int b = where[0], r0 = where[1] * kRows<RPT>;
  if (b < 0) return;
  const Seq s = sequence(dm, sq, b);
  const GroupDiv by_g(dm.G);
  const int R = s.m * dm.G, first = s.n - s.m;  // row r sees slots up to first + r / G
  const int last_row = min(r0 + kRows<RPT>, R) - 1;
  int per, count;
  key_splits((s.n + kKeys - 1) / kKeys, gridDim.z, kLeastTiles, per, count);
  if (split >= count) return;
  const int tiles = (first + last_row / dm.G) / kKeys + 1;  // that any row of the block sees
  const int kt0 = split * per, kt1 = min(kt0 + per, tiles);
  // K of the next tile is on its way while V of this one is used, and the other way round
  if (kt0 < kt1) {
    load_rows<T, D, RPT>(dm, by_g, q, s, h, r0, Qs);
    load_keys<T, D, 4, kPaged>(dm, sq, K, s, b, h, kt0 * kKeys, Ks, status);
    load_keys<T, D, 4, kPaged>(dm, sq, V, s, b, h, kt0 * kKeys, Vs, status);
  }
  const float scale2 = dm.scale * kLog2e;
  float top[RPT], l[RPT], acc[RPT][D / 16];
  int sees[RPT];
#pragma unroll
  for (int r = 0; r < RPT; ++r) {
    const int row = r0 + ty * RPT + r;
    sees[r] = row < R ? first + by_g(row) : -1;
    top[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) acc[r][c] = 0.f;
  }
  for (int kt = kt0; kt < kt1; ++kt) {
    const int j0 = kt * kKeys;
    ptx::cp_async_wait<1>();
    __syncthreads();
    float x[RPT][4];
    logits<D, RPT, 4>(Qs, Ks, scale2, x);
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (j0 + tx + 16 * c > sees[r]) x[r][c] = -INFINITY;
        mx = fmaxf(mx, x[r][c]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float ref = fmaxf(top[r], mx);
      const float keep = ref == -INFINITY ? 1.f : ptx::fast_exp2(top[r] - ref);
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float p = x[r][c] == -INFINITY ? 0.f : ptx::fast_exp2(x[r][c] - ref);
        sum += p;
        Ps[(ty * RPT + r) * kP + tx + 16 * c] = p;
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
      l[r] = l[r] * keep + sum;
      top[r] = ref;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) acc[r][c] *= keep;
    }
    __syncthreads();
    if (kt + 1 < kt1) load_keys<T, D, 4, kPaged>(dm, sq, K, s, b, h, j0 + kKeys, Ks, status);
    else ptx::cp_async_commit();  // (an empty group in its place)
    ptx::cp_async_wait<1>();
    __syncthreads();
#pragma unroll 2
    for (int j = 0; j < kKeys; j += 4) {
      float4 pv[RPT];
#pragma unroll
      for (int r = 0; r < RPT; ++r) pv[r] = *reinterpret_cast<const float4*>(Ps + (ty * RPT + r) * kP + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float4 vv[D / 64];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) vv[c] = *reinterpret_cast<const float4*>(Vs + (j + e) * kPitch<D> + 64 * c + 4 * tx);
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
          const float p = e == 0 ? pv[r].x : (e == 1 ? pv[r].y : (e == 2 ? pv[r].z : pv[r].w));
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            acc[r][4 * c] = fmaf(p, vv[c].x, acc[r][4 * c]);
            acc[r][4 * c + 1] = fmaf(p, vv[c].y, acc[r][4 * c + 1]);
            acc[r][4 * c + 2] = fmaf(p, vv[c].z, acc[r][4 * c + 2]);
            acc[r][4 * c + 3] = fmaf(p, vv[c].w, acc[r][4 * c + 3]);
          }
        }
      }
    }
    __syncthreads();
    if (kt + 1 < kt1) load_keys<T, D, 4, kPaged>(dm, sq, V, s, b, h, j0 + kKeys, Vs, status);
    else ptx::cp_async_commit();
  }
#pragma unroll
  for (int r = 0; r < RPT; ++r) {
    const int row = r0 + ty * RPT + r;
    if (row >= R) continue;
    const size_t at = (size_t)(s.t0 + row / dm.G) * dm.Hq + h * dm.G + row % dm.G;  // the row's place in lse and o
    // (l is 0 where the row sees no key of this split, which the merge leaves out, or logits of -inf alone: no number)
    const float inv = 1.f / l[r], stat = top[r] + __log2f(l[r]);
    if (count == 1) {
      if (tx == 0) {
        lse2[stat_at(dm, s, h, row)] = stat;
        if (lse) lse[at] = stat * kLn2;
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[at * D + 64 * (c / 4) + 4 * tx + c % 4] = from_float<T>(acc[r][c] * inv);
    } else {
      const size_t slot = (size_t)split * dm.T * dm.Hq + at;
      if (tx == 0) lpart[slot] = stat;
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        *reinterpret_cast<float4*>(opart + slot * D + 64 * c + 4 * tx) =
            make_float4(acc[r][4 * c] * inv, acc[r][4 * c + 1] * inv, acc[r][4 * c + 2] * inv, acc[r][4 * c + 3] * inv);
    }
  }
}

// grid = ceil(T * Hq / 8) CTAs of 8 warps, a warp per row; splits: what the attend kernel was launched with.
template <typename T, int D>
__global__ void __launch_bounds__(256)
combine_kernel(PDims dm, Seqs sq, int splits, int keys_per_tile, int least_tiles, const float* __restrict__ opart,
               const float* __restrict__ lpart, T* __restrict__ o, float* __restrict__ lse, float* __restrict__ lse2) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  constexpr int CPL = D / 32;
  const int lane = threadIdx.x & 31;
  const long long at = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (at >= (long long)dm.T * dm.Hq) return;
  // the sequence of packed row t: the last one that begins at or before it
  const int t = (int)(at / dm.Hq);
  int lo = 0, hi = dm.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sq.cu[mid] <= t) lo = mid; else hi = mid;
  }
  const Seq s = sequence(dm, sq, lo);
  if (t < s.t0 || t >= s.t0 + s.m) return;
  int per, count;
  key_splits((s.n + keys_per_tile - 1) / keys_per_tile, splits, least_tiles, per, count);
  if (count == 1) return;
  float stat = -INFINITY;
  for (int i = 0; i < count; ++i) stat = fmaxf(stat, lpart[(size_t)i * dm.T * dm.Hq + at]);
  float sum = 0.f, x[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) x[c] = 0.f;
  for (int i = 0; i < count; ++i) {
    const size_t slot = (size_t)i * dm.T * dm.Hq + at;
    const float w = ptx::fast_exp2(lpart[slot] - stat);
    if (w == 0.f) continue;
    sum += w;
#pragma unroll
    for (int c = 0; c < CPL; ++c) x[c] = fmaf(w, opart[slot * D + c * 32 + lane], x[c]);
  }
#pragma unroll
  for (int c = 0; c < CPL; ++c) o[at * D + c * 32 + lane] = from_float<T>(x[c] / sum);
  if (lane == 0) {
    stat += __log2f(sum);
    const int hq = (int)(at % dm.Hq);
    lse2[stat_at(dm, s, hq / dm.G, (t - s.t0) * dm.G + hq % dm.G)] = stat;
    if (lse) lse[at] = stat * kLn2;
  }
}

// grid = (blocks of 16 KPT keys of all sequences, Hkv). Prompts: mass[t, h] = sum; pages: mass[page, h, row] += sum.
template <typename T, int D, int RPT, int KPT, bool kPaged>
__global__ void __launch_bounds__(kThreads)
mass_kernel(PDims dm, Seqs sq, const T* __restrict__ q, const T* __restrict__ K, const float* __restrict__ lse2,
            float* __restrict__ mass, int* status) {
  constexpr int kMine = 16 * KPT;
  ptx::pdl_wait();
  ptx::pdl_trigger();
  extern __shared__ __align__(16) float smf[];
  float* Qs = smf;  // [2] blocks of rows
  float* Ks = Qs + 2 * kRows<RPT> * kPitch<D>;
  float* sums = Ks + kMine * kPitch<D>;  // [16][kP]
  int* where = reinterpret_cast<int*>(sums + 16 * kP);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, h = blockIdx.y;
  if (tid < 32) {
    auto what = [&](const Seq& x) { return x.m > 0 ? x.n : 0; };
    Place p;
    Scan c = scan(dm, sq, 0, kMine, what, nullptr);
    const bool there = find_block(dm, sq, kMine, blockIdx.x, what, c, p);
    if (tid == 0) { where[0] = there ? p.b : -1; where[1] = p.block; }
  }
  __syncthreads();
  const int b = where[0], j0 = where[1] * kMine;
  if (b < 0) return;
  const Seq s = sequence(dm, sq, b);
  const GroupDiv by_g(dm.G);
  const int R = s.m * dm.G, first = s.n - s.m;
  const float scale2 = dm.scale * kLog2e;
  float sum[KPT];
#pragma unroll
  for (int c = 0; c < KPT; ++c) sum[c] = 0.f;
  // the first row that sees any of these keys
  int r0 = max(0, j0 - first) * dm.G;
  r0 -= r0 % kRows<RPT>;
  load_keys<T, D, KPT, kPaged>(dm, sq, K, s, b, h, j0, Ks, status);
  load_rows<T, D, RPT>(dm, by_g, q, s, h, r0, Qs);
  const float* stats = lse2 + stat_at(dm, s, h, 0);
  for (int buf = 0; r0 < R; r0 += kRows<RPT>, buf ^= 1) {
    float stat[RPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r) stat[r] = r0 + ty * RPT + r < R ? stats[r0 + ty * RPT + r] : 0.f;
    // the next block of rows goes where the one before this lay (the barrier at the end)
    if (r0 + kRows<RPT> < R) load_rows<T, D, RPT>(dm, by_g, q, s, h, r0 + kRows<RPT>, Qs + (buf ^ 1) * kRows<RPT> * kPitch<D>);
    else ptx::cp_async_commit();
    ptx::cp_async_wait<1>();
    __syncthreads();
    float x[RPT][KPT], part[KPT];
    logits<D, RPT, KPT>(Qs + buf * kRows<RPT> * kPitch<D>, Ks, scale2, x);
#pragma unroll
    for (int c = 0; c < KPT; ++c) part[c] = 0.f;
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
      const int row = r0 + ty * RPT + r;
      const int sees = row < R ? first + by_g(row) : -1;
#pragma unroll
      for (int c = 0; c < KPT; ++c)
        if (j0 + tx + 16 * c <= sees) part[c] += ptx::fast_exp2(x[r][c] - stat[r]);
    }
#pragma unroll
    for (int c = 0; c < KPT; ++c) sum[c] += part[c];
    __syncthreads();
  }
#pragma unroll
  for (int c = 0; c < KPT; ++c) sums[ty * kP + tx + 16 * c] = sum[c];
  __syncthreads();
  if (tid < kMine && j0 + tid < s.n) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += sums[i * kP + tid];
    if (kPaged) {
      if (float* out = pool_weight(dm, sq, b, h, j0 + tid, mass, status)) *out += v;
    } else {
      mass[(size_t)(s.t0 + j0 + tid) * dm.Hkv + h] = v;
    }
  }
}

}  // namespace generic
}  // namespace paged
}  // namespace caote
