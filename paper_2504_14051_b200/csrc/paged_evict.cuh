// Append to and eviction from a cache in pages.
//
// Eviction by accumulated attention weight: of the n tokens of a (sequence, KV head) pair the k = n - budget first ones in the
// order (sheltered, weight bits, position) go; sheltered are the positions below `sinks` and the `recent` newest ones of the
// sequence. The survivors among the last k slots move into the holes below the new length, so that a pair's tokens stay in its
// first slots and whole pages come free behind them.
//
// What bounds them: chains of dependent reads (length, page table, weights, picks, rows); the traffic is 8 bytes per token and four
// rows per evicted one.
#pragma once

#include "paged_common.cuh"
#include "ptx.cuh"
#include "select.cuh"

namespace caote {
namespace paged {

constexpr int kEvictThreads = sel::kSelThreads;
constexpr unsigned kSheltered = 0xffffffffu;  // as the score bits of a sheltered token: behind every other

// New rows into the pages: a thread per 16 bytes of a K or V row, the pieces of a token side by side. The CTA that finishes last moves
// the lengths on; a sequence that does not fit, or one of whose pages is none, keeps its length, and all do where cu does not ascend (the
// search for a row's sequence means nothing then). Up to as many CTAs as are resident at
// once: more would wait for their turn (8 sequences of 512 tokens, 8 KV heads, 16.8 MB, cold: 20.5 us with five per SM, 19 with six, 20
// with eight, whose 32 registers do not suffice; two and four tokens on their way per thread: 1 and 5 us longer).
constexpr int kAppendThreads = 256, kAppendCtas = 6, kSharedStarts = 1024;
__global__ void __launch_bounds__(kAppendThreads, kAppendCtas)
append_kernel(PDims dm, Seqs sq, int row_bytes, long long src_stride, char* __restrict__ K, char* __restrict__ V,
              float* __restrict__ mass, int* __restrict__ pos, int* __restrict__ len, int* __restrict__ n_seen,
              const char* __restrict__ k_new, const char* __restrict__ v_new, const float* __restrict__ mass_new, int* status,
              int* ticket) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  __shared__ int s_cu[kSharedStarts + 1];
  const int tid = threadIdx.x;
  // (a search of dependent reads: from shared memory where the starts fit)
  const bool in_smem = dm.B <= kSharedStarts;
  if (in_smem) {
    for (int b = tid; b <= dm.B; b += kAppendThreads) s_cu[b] = sq.cu[b];
    __syncthreads();
  }
  auto start = [&](int b) { return in_smem ? s_cu[b] : __ldg(sq.cu + b); };
  const int pieces = row_bytes / 16, per_token = dm.Hkv * 2 * pieces;
  const int at_once = per_token < kAppendThreads ? kAppendThreads / per_token : 1;  // tokens
  const long long cap = (long long)dm.max_pages << dm.page_shift;
  const int sub = per_token < kAppendThreads ? tid / per_token : 0, rest0 = tid - sub * per_token;
  const int h0 = rest0 / (2 * pieces), which0 = rest0 / pieces & 1, c0 = rest0 % pieces;
  for (int t = blockIdx.x * at_once + sub; t < dm.T && sub < at_once; t += gridDim.x * at_once) {
    auto source = [&](int h, int which, int c) {
      return *reinterpret_cast<const uint4*>((which ? v_new : k_new) + (size_t)t * src_stride + (size_t)h * row_bytes + c * 16);
    };
    int h = h0, which = which0, c = c0;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);  // (on its way while the token's place is looked up)
    if (rest0 < per_token) x = source(h, which, c);
    int lo = 0, hi = dm.B;  // the sequence of token t: the last one that begins at or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start(mid) <= t) lo = mid; else hi = mid;
    }
    const int t0 = start(lo), t1 = start(lo + 1), n = len[lo], seen = n_seen ? n_seen[lo] : n;
    if (t < t0 || t >= t1 || t1 > dm.T || t0 < 0 || t1 - t0 > dm.max_new || n < 0 || n + (long long)(t1 - t0) > cap) continue;
    const int j = n + t - t0;
    const int page = __ldg(sq.table + (size_t)lo * dm.max_pages + (j >> dm.page_shift));
    if ((unsigned)page >= (unsigned)dm.n_pages) continue;
    const size_t row0 = ((size_t)page * dm.Hkv << dm.page_shift) + (j & ((1 << dm.page_shift) - 1));  // of head 0
    for (int rest = rest0; rest < per_token;) {
      const size_t at = row0 + ((size_t)h << dm.page_shift);
      *reinterpret_cast<uint4*>((which ? V : K) + at * row_bytes + c * 16) = x;
      if (which == 0 && c == 0) {
        if (mass) mass[at] = mass_new ? mass_new[(size_t)t * dm.Hkv + h] : 0.f;
        if (pos) pos[at] = seen + t - t0;
      }
      rest += kAppendThreads;
      if (rest < per_token) {
        h = rest / (2 * pieces);
        which = rest / pieces & 1;
        c = rest % pieces;
        x = source(h, which, c);
      }
    }
  }
  __shared__ int s_last;
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    s_last = atomicAdd(ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  bool descends = false;
  for (int b = tid; b < dm.B; b += kAppendThreads) descends |= start(b + 1) < start(b);
  descends = __syncthreads_or(descends) != 0;
  // (a power of two of lanes per sequence, so that one round of the CTA does where it can: they share the look at its pages)
  int lanes = 32;
  while (lanes > 1 && (long long)lanes * dm.B > kAppendThreads) lanes >>= 1;
  const int lane = tid & 31, in = lane & (lanes - 1);
  for (int b0 = 0; b0 < dm.B; b0 += kAppendThreads / lanes) {
    const int b = b0 + tid / lanes;
    const bool there = b < dm.B;
    const int t0 = there ? start(b) : 0, t1 = there ? start(b + 1) : 0, m = t1 - t0, n = there ? len[b] : 0;
    const bool sound = !descends && t0 >= 0 && t1 <= dm.T && m <= dm.max_new && n >= 0, fits = sound && n + (long long)m <= cap;
    bool ok = true;
    if (fits && m > 0) {
#pragma unroll 4
      for (int p = (n >> dm.page_shift) + in; p <= (n + m - 1) >> dm.page_shift; p += lanes)
        ok &= (unsigned)__ldg(sq.table + (size_t)b * dm.max_pages + p) < (unsigned)dm.n_pages;
    }
    const unsigned wrong = __ballot_sync(0xffffffffu, !ok) >> (lane - in) & (unsigned)((1ull << lanes) - 1ull);
    if (!there || in != 0) continue;
    if (!sound) {
      set_status(status, CAOTE_ERR_BAD_LENGTH);
    } else if (!fits) {
      set_status(status, CAOTE_ERR_OVERFLOW);
    } else if (wrong != 0u) {
      set_status(status, CAOTE_ERR_BAD_PAGE);
    } else if (m > 0) {
      len[b] = n + m;
      if (n_seen) n_seen[b] += m;
    }
  }
  if (tid == 0) *ticket = 0;
}

constexpr int kMoves = 512;   // rows whose moves are worked out at a time
struct Pool {
  char *K, *V;
  float* mass;
  int* pos;
};

// The position of slot j of a pair.
struct Positions {
  const int *table, *pos;
  int Hkv, h, shift, n_pages;
  __device__ __noinline__ unsigned operator()(int j) const {
    const int page = __ldg(table + (j >> shift));
    return (unsigned)page < (unsigned)n_pages ? (unsigned)pos[(((size_t)page * Hkv + h) << shift) + (j & ((1 << shift) - 1))] : 0u;
  }
};

// Selection and compaction. grid = (sequence, KV head) pairs x C in clusters:
//   by_sequence (one token goes per pair at most): a cluster is a sequence, a CTA a pair; rank 0 moves the length on.
//   else: a cluster is a pair. Rank 0 selects, all of its CTAs move rows; the CTA that finishes last moves the lengths on.
__global__ void __launch_bounds__(kEvictThreads)
evict_kernel(PDims dm, Seqs sq, Pool pool, int row_bytes, int* __restrict__ len, const int* __restrict__ n_seen,
             const int* __restrict__ budget, int sinks, int recent, int* __restrict__ evict_idx, int max_evict,
             int* __restrict__ n_evict, bool by_sequence, int* status, int* ticket) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  __shared__ int s_picks[sel::kMaxSharedPicks];
  __shared__ unsigned s_min[3][kEvictThreads / 32];
  __shared__ int2 s_moves[kMoves];
  const int C = by_sequence ? 1 : (int)ptx::cluster_nctarank(), rank = by_sequence ? 0 : (int)ptx::cluster_ctarank();
  const int pair = blockIdx.x / C, b = pair / dm.Hkv, h = pair % dm.Hkv;
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
  const int shift = dm.page_shift, low = (1 << shift) - 1, Hkv = dm.Hkv, n_pages = dm.n_pages;
  // (a page outside the pool is read as page 0 and remembered: nothing is written then)
  bool bad = false;
  auto row = [&](int j) {
    int page = __ldg(table + (j >> shift));
    if ((unsigned)page >= (unsigned)n_pages) {
      bad = true;
      page = 0;
    }
    return (((size_t)page * Hkv + h) << shift) + (j & low);
  };
  const float* mass = pool.mass;
  const int* pos = pool.pos;
  const long long newest = (long long)seen - recent;
  auto bits = [&](unsigned w, int p) { return p < sinks || p >= newest ? kSheltered : min(w, kSheltered - 1u); };
  int* out = evict_idx + (size_t)pair * max_evict;
  const int left = n - k;
  if (k == 1) {
    if (rank == 0) {
      // the last row, which fills the hole, is on its way while the hole is looked for: warp 0 has K, warp 1 V
      const bool mover = warp < 2 && lane * 16 < row_bytes;
      char* rows = warp == 0 ? pool.K : pool.V;
      const size_t last = warp < 3 ? row(left) : 0;
      uint4 moved = make_uint4(0u, 0u, 0u, 0u);
      if (mover) moved = *reinterpret_cast<const uint4*>(rows + last * row_bytes + lane * 16);
      float last_mass = 0.f;
      int last_pos = 0;
      if (warp == 2 && lane == 0) {
        last_mass = mass[last];
        last_pos = pos[last];
      }
      unsigned bw = ~0u, bp = ~0u, bs = ~0u;  // the first token so far: score bits, position, slot
      constexpr int kAtOnce = 8;
      for (int j0 = tid; j0 < n; j0 += kAtOnce * kEvictThreads) {
        unsigned w[kAtOnce];
        int p[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
          const int j = j0 + e * kEvictThreads;
          w[e] = 0u;
          p[e] = 0;
          if (j < n) {
            const size_t at = row(j);
            w[e] = __float_as_uint(mass[at]);
            p[e] = pos[at];
          }
        }
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
          const int j = j0 + e * kEvictThreads;
          const unsigned x = bits(w[e], p[e]);
          if (j < n && (bs == ~0u || x < bw || (x == bw && (unsigned)p[e] < bp))) { bw = x; bp = (unsigned)p[e]; bs = (unsigned)j; }
        }
      }
      // the smallest bits, of these the smallest position, of these the smallest slot
      auto reduce = [&]() {
        const unsigned mw = __reduce_min_sync(0xffffffffu, bs == ~0u ? ~0u : bw);
        const unsigned mp = __reduce_min_sync(0xffffffffu, bs != ~0u && bw == mw ? bp : ~0u);
        const unsigned ms = __reduce_min_sync(0xffffffffu, bs != ~0u && bw == mw && bp == mp ? bs : ~0u);
        bw = mw; bp = mp; bs = ms;
      };
      reduce();
      if (lane == 0) { s_min[0][warp] = bw; s_min[1][warp] = bp; s_min[2][warp] = bs; }
      if (__syncthreads_or(bad)) {
        if (tid == 0) set_status(status, CAOTE_ERR_BAD_PAGE);
        k = 0;
      } else if (warp < 3) {
        bw = s_min[0][lane];
        bp = s_min[1][lane];
        bs = s_min[2][lane];
        reduce();
        const size_t hole = row((int)bs);
        if ((int)bs != left) {
          if (mover) *reinterpret_cast<uint4*>(rows + hole * row_bytes + lane * 16) = moved;
          if (warp == 2 && lane == 0) {
            pool.mass[hole] = last_mass;
            pool.pos[hole] = last_pos;
          }
        }
        if (tid == 0) out[0] = (int)bs;
      }
    }
    if (!by_sequence) ptx::cluster_sync_all();
  } else if (k > 0) {
    if (rank == 0) {
      // (asked for where weights tie only: kept out of the way of the code that always runs)
      const Positions position{table, pos, Hkv, h, shift, n_pages};
      // eight or nine tokens' pages, then all of their weights and positions, are on their way at a time
      auto scores = [&](int first, int count, auto& v) {
        constexpr int kC = (int)(sizeof(v) / sizeof(v[0])), kAtOnce = kC % 9 == 0 ? 9 : 8;
        static_assert(kC % kAtOnce == 0, "");
#pragma unroll
        for (int i0 = 0; i0 < kC; i0 += kAtOnce) {
          unsigned at[kAtOnce];  // (pools have less than 2^31 rows)
          int p[kAtOnce];
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) {
            const int j = first + (i0 + e) * kEvictThreads;
            at[e] = (unsigned)row(j < count ? j : 0);
          }
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) {
            v[i0 + e] = __float_as_uint(mass[at[e]]);
            p[e] = pos[at[e]];
          }
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) v[i0 + e] = bits(v[i0 + e], p[e]);
        }
      };
      int* picks = k <= sel::kMaxSharedPicks ? s_picks : nullptr;
      if (n <= 8 * kEvictThreads) sel::select_cached<8, true>(n, k, scores, position, out, picks);
      else if (n <= 18 * kEvictThreads) sel::select_cached<18, true>(n, k, scores, position, out, picks);
      else if (n <= sel::kMaxCached * kEvictThreads) sel::select_cached<sel::kMaxCached, true>(n, k, scores, position, out, picks);
      else {
        // (by value, not by reference: that would put what the lambdas above refer to on the stack for good)
        for (int q = tid; q <= (n - 1) >> shift; q += kEvictThreads) bad = bad || (unsigned)__ldg(table + q) >= (unsigned)n_pages;
        const size_t rows = ((size_t)n_pages * Hkv) << shift;
        auto row_v = [=](int j) {
          const size_t at = (((size_t)(unsigned)__ldg(table + (j >> shift)) * Hkv + h) << shift) + (j & low);
          return at < rows ? at : 0;
        };
        auto position_v = [=](int j) { return (unsigned)pos[row_v(j)]; };
        auto score_v = [=](int j) {
          const size_t at = row_v(j);
          const int q = pos[at];
          return q < sinks || q >= newest ? kSheltered : min(__float_as_uint(mass[at]), kSheltered - 1u);
        };
        sel::select_long(n, k, score_v, position_v, out, picks);
      }
    } else {
      for (int q = tid; q <= (n - 1) >> shift; q += kEvictThreads) bad = bad || (unsigned)__ldg(table + q) >= (unsigned)n_pages;
    }
    // (every CTA of the sequence comes to the same answer: each has looked at all of its pages)
    const bool skip = __syncthreads_or(bad) != 0;
    if (C > 1) ptx::cluster_sync_all();  // rank 0's picks are written
    if (skip) {
      if (tid == 0) set_status(status, CAOTE_ERR_BAD_PAGE);
      k = 0;
    } else {
      const int* E = k <= sel::kMaxSharedPicks ? s_picks : out;
      if (rank > 0 && k <= sel::kMaxSharedPicks) {
        for (int i = tid; i < k; i += kEvictThreads) s_picks[i] = out[i];
        __syncthreads();
      }
      // The i-th survivor among slots [left, n) moves into the i-th hole below `left`. First where from and where to, a thread per
      // slot; then half a warp per row of up to 256 bytes, several rows on their way at once.
      const int holes = sel::lower_bound(E, k, left);
      const int glanes = row_bytes <= 256 ? 16 : 32, gl = lane & (glanes - 1);
      const int group = warp * (32 / glanes) + lane / glanes, groups = (kEvictThreads / 32) * (32 / glanes);
      const int share = (k + C - 1) / C, from = rank * share, to = min(k, from + share);
      for (int t0 = from; t0 < to; t0 += kMoves) {
        if (t0 > from) __syncthreads();
        const int moves = min(kMoves, to - t0);
        for (int t = tid; t < moves; t += kEvictThreads) {
          const int src = left + t0 + t, lb = holes + sel::lower_bound(E + holes, k - holes, src);
          int2 mv = make_int2(-1, -1);
          if (!(lb < k && E[lb] == src)) mv = make_int2((int)row(src), (int)row(E[t0 + t - (lb - holes)]));
          s_moves[t] = mv;
        }
        __syncthreads();
        constexpr int kAtOnce = 4;
        for (int g0 = group; g0 < moves; g0 += kAtOnce * groups) {
          uint4 kr[kAtOnce], vr[kAtOnce];
          int2 mv[kAtOnce];
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) {
            const int g = g0 + e * groups;
            mv[e] = g < moves ? s_moves[g] : make_int2(-1, -1);
            if (mv[e].x >= 0 && gl * 16 < row_bytes) {
              kr[e] = *reinterpret_cast<const uint4*>(pool.K + (size_t)mv[e].x * row_bytes + gl * 16);
              vr[e] = *reinterpret_cast<const uint4*>(pool.V + (size_t)mv[e].x * row_bytes + gl * 16);
            }
          }
#pragma unroll
          for (int e = 0; e < kAtOnce; ++e) {
            if (mv[e].x < 0) continue;
            if (gl * 16 < row_bytes) {
              *reinterpret_cast<uint4*>(pool.K + (size_t)mv[e].y * row_bytes + gl * 16) = kr[e];
              *reinterpret_cast<uint4*>(pool.V + (size_t)mv[e].y * row_bytes + gl * 16) = vr[e];
            }
            if (gl == 0) {
              pool.mass[mv[e].y] = pool.mass[mv[e].x];
              pool.pos[mv[e].y] = pool.pos[mv[e].x];
            }
          }
        }
      }
    }
  }
  if (h == 0 && rank == 0 && tid == 0) n_evict[b] = k;
  if (by_sequence) {
    ptx::cluster_sync_all();  // every pair has read the length
    if (h == 0 && tid == 0) len[b] = n - k;
  } else {
    sel::finish_lengths(dm.B, len, n_evict, ticket);
  }
}

}  // namespace paged
}  // namespace caote
