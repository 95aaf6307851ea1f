// Append to and eviction from a cache in pages.
//
// Eviction by accumulated attention weight: of the n tokens of a (sequence, KV head) pair the k = n - budget first ones in the
// order (sheltered, weight bits, position) go; sheltered are the positions below `sinks` and the `recent` newest ones of the
// sequence. The survivors among the last k slots move into the holes below the new length, so that a pair's tokens stay in its
// first slots and whole pages come free behind them.
//
// What bounds them: chains of dependent reads (length, page table, weights, picks, rows), a CTA per pair; the traffic is 8 bytes
// per token and four rows per evicted one.
#pragma once

#include "paged_common.cuh"
#include "ptx.cuh"
#include "select.cuh"

namespace caote {
namespace paged {

constexpr int kEvictThreads = sel::kSelThreads;
constexpr unsigned kSheltered = 0xffffffffu;  // as the score bits of a sheltered token: behind every other

// Whether all pages of slots [from, to) lie in the pool; for a whole CTA, the same result in every thread.
__device__ __forceinline__ bool pages_ok(const PDims& dm, const int* __restrict__ table, int from, int to) {
  bool ok = true;
  for (int p = (from >> dm.page_shift) + threadIdx.x; p <= (to - 1) >> dm.page_shift; p += blockDim.x)
    ok = ok && (unsigned)__ldg(table + p) < (unsigned)dm.n_pages;
  return __syncthreads_and(ok) != 0;
}

// New rows into the pages: a thread per 16 bytes of a K or V row, grid-stride over (token, KV head, K or V, piece). The CTA that
// finishes last moves the lengths on; a sequence that does not fit, or one of whose pages is none, keeps its length.
__global__ void __launch_bounds__(256)
append_kernel(PDims dm, Seqs sq, int row_bytes, long long src_stride, char* __restrict__ K, char* __restrict__ V,
              float* __restrict__ mass, int* __restrict__ pos, int* __restrict__ len, int* __restrict__ n_seen,
              const char* __restrict__ k_new, const char* __restrict__ v_new, const float* __restrict__ mass_new, int* status,
              int* ticket) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  const int pieces = row_bytes / 16, per_token = dm.Hkv * 2 * pieces;
  const long long total = (long long)dm.T * per_token;
  const long long cap = (long long)dm.max_pages << dm.page_shift;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
    const int t = (int)(i / per_token), rest = (int)(i % per_token);
    const int h = rest / (2 * pieces), which = rest / pieces & 1, c = rest % pieces;
    int lo = 0, hi = dm.B;  // the sequence of token t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(sq.cu + mid) <= t) lo = mid; else hi = mid;
    }
    const int t0 = __ldg(sq.cu + lo), t1 = __ldg(sq.cu + lo + 1), n = len[lo];
    if (t < t0 || t >= t1 || t1 > dm.T || t0 < 0 || t1 - t0 > dm.max_new || n < 0 || n + (long long)(t1 - t0) > cap) continue;
    const int j = n + t - t0;
    const int page = __ldg(sq.table + (size_t)lo * dm.max_pages + (j >> dm.page_shift));
    if ((unsigned)page >= (unsigned)dm.n_pages) continue;
    const size_t at = (((size_t)page * dm.Hkv + h) << dm.page_shift) + (j & ((1 << dm.page_shift) - 1));
    const char* src = (which ? v_new : k_new) + (size_t)t * src_stride + (size_t)h * row_bytes + c * 16;
    *reinterpret_cast<uint4*>((which ? V : K) + at * row_bytes + c * 16) = *reinterpret_cast<const uint4*>(src);
    if (which == 0 && c == 0) {
      if (mass) mass[at] = mass_new ? mass_new[(size_t)t * dm.Hkv + h] : 0.f;
      if (pos) pos[at] = (n_seen ? n_seen[lo] : n) + t - t0;
    }
  }
  __shared__ int s_last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = atomicAdd(ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  for (int b = threadIdx.x; b < dm.B; b += blockDim.x) {
    const int t0 = sq.cu[b], t1 = sq.cu[b + 1], m = t1 - t0, n = len[b];
    if (t0 < 0 || t1 < t0 || t1 > dm.T || m > dm.max_new || n < 0) {
      set_status(status, CAOTE_ERR_BAD_LENGTH);
    } else if (n + (long long)m > cap) {
      set_status(status, CAOTE_ERR_OVERFLOW);
    } else if (m > 0) {
      bool ok = true;
      for (int p = n >> dm.page_shift; p <= (n + m - 1) >> dm.page_shift; ++p)
        ok = ok && (unsigned)__ldg(sq.table + (size_t)b * dm.max_pages + p) < (unsigned)dm.n_pages;
      if (!ok) {
        set_status(status, CAOTE_ERR_BAD_PAGE);
      } else {
        len[b] = n + m;
        if (n_seen) n_seen[b] += m;
      }
    }
  }
  if (threadIdx.x == 0) *ticket = 0;
}

struct Pool {
  char *K, *V;
  float* mass;
  int* pos;
};

// One CTA per (sequence, KV head) pair: selection, compaction; the CTA that finishes last moves the lengths.
__global__ void __launch_bounds__(kEvictThreads)
evict_kernel(PDims dm, Seqs sq, Pool pool, int row_bytes, int* __restrict__ len, const int* __restrict__ n_seen,
             const int* __restrict__ budget, int sinks, int recent, int* __restrict__ evict_idx, int max_evict,
             int* __restrict__ n_evict, int* status, int* ticket) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  __shared__ int s_picks[sel::kMaxSharedPicks];
  __shared__ unsigned long long s_key[kEvictThreads / 32];
  __shared__ int s_slot[kEvictThreads / 32];
  const int b = blockIdx.x / dm.Hkv, h = blockIdx.x % dm.Hkv;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int* table = sq.table + (size_t)b * dm.max_pages;
  const int n = len[b], seen = n_seen[b];
  int k = n - max(budget[b], 1);
  if (k < 0) k = 0;
  if (n > (long long)dm.max_pages << dm.page_shift || n < 0) {
    if (tid == 0) set_status(status, CAOTE_ERR_BAD_LENGTH);
    k = 0;
  }
  if (k > max_evict) {
    if (tid == 0) set_status(status, CAOTE_ERR_OVERFLOW);
    k = 0;
  }
  if (k > 0 && !pages_ok(dm, table, 0, n)) {  // (every pair of the sequence comes to the same answer)
    if (tid == 0) set_status(status, CAOTE_ERR_BAD_PAGE);
    k = 0;
  }
  if (h == 0 && tid == 0) n_evict[b] = k;
  if (k > 0) {
    const int shift = dm.page_shift, low = (1 << shift) - 1, Hkv = dm.Hkv;
    auto row = [=](int j) { return (((size_t)__ldg(table + (j >> shift)) * Hkv + h) << shift) + (j & low); };
    const float* mass = pool.mass;
    const int* pos = pool.pos;
    const long long newest = (long long)seen - recent;
    auto position = [=](int j) { return (unsigned)pos[row(j)]; };
    auto score = [=](int j) {
      const size_t at = row(j);
      const unsigned w = __float_as_uint(mass[at]);
      const int p = pos[at];
      return p < sinks || p >= newest ? kSheltered : min(w, kSheltered - 1u);
    };
    int* out = evict_idx + (size_t)blockIdx.x * max_evict;
    const int left = n - k;
    const int* E;
    if (k == 1) {
      unsigned long long best = ~0ull;
      int best_slot = n;
      for (int j = tid; j < n; j += kEvictThreads) {
        const size_t at = row(j);
        const unsigned w = __float_as_uint(mass[at]);
        const int p = pos[at];
        const unsigned long long key = sel::make_key(p < sinks || p >= newest ? kSheltered : min(w, kSheltered - 1u), (unsigned)p);
        if (key < best || best_slot == n) { best = key; best_slot = j; }
      }
      auto reduce = [&]() {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const unsigned long long ok = __shfl_xor_sync(0xffffffffu, best, o);
          const int os = __shfl_xor_sync(0xffffffffu, best_slot, o);
          if (ok < best || (ok == best && os < best_slot)) { best = ok; best_slot = os; }
        }
      };
      reduce();
      if (lane == 0) { s_key[warp] = best; s_slot[warp] = best_slot; }
      __syncthreads();
      best = s_key[lane];
      best_slot = s_slot[lane];
      reduce();
      if (tid == 0) { s_picks[0] = best_slot; out[0] = best_slot; }
      E = s_picks;
    } else {
      int* picks = k <= sel::kMaxSharedPicks ? s_picks : nullptr;
      if (n <= 8 * kEvictThreads) sel::select_cached<8>(n, k, score, position, out, picks);
      else if (n <= sel::kMaxCached * kEvictThreads) sel::select_cached<sel::kMaxCached>(n, k, score, position, out, picks);
      else sel::select_long(n, k, score, position, out, picks);
      E = picks ? s_picks : out;
    }
    __syncthreads();
    // the i-th survivor among slots [left, n) moves into the i-th hole below `left`: half a warp per row of up to 256 bytes
    const int holes = sel::lower_bound(E, k, left);
    const int glanes = row_bytes <= 256 ? 16 : 32, gl = lane & (glanes - 1);
    const int group = warp * (32 / glanes) + lane / glanes, groups = (kEvictThreads / 32) * (32 / glanes);
    for (int t = group; t < k; t += groups) {
      const int src = left + t, lb = holes + sel::lower_bound(E + holes, k - holes, src);
      if (lb < k && E[lb] == src) continue;  // goes itself
      const int dst = E[t - (lb - holes)];
      const size_t so = row(src), to = row(dst);
      if (gl * 16 < row_bytes) {
        const uint4 kr = *reinterpret_cast<const uint4*>(pool.K + so * row_bytes + gl * 16);
        const uint4 vr = *reinterpret_cast<const uint4*>(pool.V + so * row_bytes + gl * 16);
        *reinterpret_cast<uint4*>(pool.K + to * row_bytes + gl * 16) = kr;
        *reinterpret_cast<uint4*>(pool.V + to * row_bytes + gl * 16) = vr;
      }
      if (gl == 0) {
        pool.mass[to] = pool.mass[so];
        pool.pos[to] = pool.pos[so];
      }
    }
  }
  sel::finish_lengths(dm.B, len, n_evict, ticket);
}

}  // namespace paged
}  // namespace caote
