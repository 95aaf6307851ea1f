// The k smallest (score bits, position) pairs of a unit by one CTA, wherever the scores lie, and the small parts that
// selection, compaction and append share between the dense and the paged cache.
#pragma once

#include "common.cuh"

namespace caote {
namespace sel {

constexpr int kSelThreads = 1024;
constexpr int kMaxSharedPicks = 2048;
constexpr int kMaxCached = 24;  // scores per thread that a selection can keep in registers

// 64-bit sort key: score bits in the high word (scores are >= +0, so the unsigned order of the bit
// patterns is the numeric order; +inf sorts last), original position in the low word.
__device__ __forceinline__ unsigned long long make_key(unsigned score_bits, unsigned pos) {
  return ((unsigned long long)score_bits << 32) | pos;
}
__device__ __forceinline__ unsigned long long make_key(float score, int pos) { return make_key(__float_as_uint(score), (unsigned)pos); }

// The k smallest of n keys, 1 < k < n, by the CTA: the slots in ascending order to out (and picks, if not null). Up to kC
// scores per thread stay in registers. The bits above the highest one in which any two scores differ are skipped (the scores
// of one unit share their leading bits); below it, 11 bits are decided per pass of a histogram (1.1 us, of the latency of its
// barriers and atomics), until a whole bucket is taken or no more than kRank tokens are left in it: these are then ranked
// against one another by (score bits, position), a thread per token. Mostly that is one pass. Where more tokens than that
// have the score at the threshold, the search goes on over their positions. (Up to eight passes of 8 bits over 64-bit keys:
// 8 units, n 4224, k 128: 17.5 -> 15.2 us between events; n 16 896, k 512, scores read again in every pass: 53 -> 36 us.)
// score(first, n, v): the score bits of tokens first + i * kSelThreads < n, of whatever the cache looks like; position(j): a token's
// position. kLast: tokens with all bits set are
// left out of the search where there are k others (many of them would share one counter, and widen the range of bits).
template <int kC, bool kLast = false, typename Score, typename Position>
__device__ __forceinline__ void select_cached(int n, int k, Score score, Position position, int* out, int* picks) {
  constexpr int kW = kSelThreads / 32;
  constexpr unsigned kRank = 128u;
  __shared__ __align__(16) unsigned hist[2048];
  __shared__ unsigned s_lo[kW], s_hi[kW], s_tot[kW];
  __shared__ unsigned s_digit, s_below, s_count, s_list;
  __shared__ unsigned long long s_kth;
  __shared__ int s_cnt[kC * kW];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  unsigned v[kC], live = 0u;  // score bits, and which of them are there; later the positions of the tokens at the threshold
  score(tid, n, v);
#pragma unroll
  for (int i = 0; i < kC; ++i) live |= (tid + i * kSelThreads < n ? 1u : 0u) << i;
  hist[tid] = 0u;
  hist[tid + kSelThreads] = 0u;
  if (tid == 0) s_list = 0u;
  unsigned left = (unsigned)n;
  if constexpr (kLast) {
    unsigned others = live;
#pragma unroll
    for (int i = 0; i < kC; ++i)
      if (v[i] == 0xffffffffu) others &= ~(1u << i);
    const unsigned mine = __reduce_add_sync(0xffffffffu, (unsigned)__popc(others));
    if (lane == 0) s_tot[warp] = mine;
    __syncthreads();
    const unsigned all = __reduce_add_sync(0xffffffffu, s_tot[lane]);
    if (all >= (unsigned)k) {
      live = others;
      left = all;
    }
    __syncthreads();  // (s_tot is written again below)
  }
  // thr: the threshold so far as it is known (prefix, then zeros); bits [0, top) of it are still to be decided;
  // want: how many to take of the `left` tokens with this prefix
  unsigned thr, want = (unsigned)k, taken = 0u;
  int top;  // 0 .. 32 (a caller's own scores may have any bits)
  auto above = [](unsigned x, int t) { return __funnelshift_rc(x, 0u, t); };  // x >> t, also for t = 32
  auto alive = [&](int i) { return (live >> i & 1u) != 0u; };
  auto prefix_of_all = [&]() {
    unsigned lo = 0xffffffffu, hi = 0u;
#pragma unroll
    for (int i = 0; i < kC; ++i) {
      lo = min(lo, alive(i) ? v[i] : 0xffffffffu);
      hi = max(hi, alive(i) ? v[i] : 0u);
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) { s_lo[warp] = lo; s_hi[warp] = hi; }
    __syncthreads();
    lo = __reduce_min_sync(0xffffffffu, s_lo[lane]);
    hi = __reduce_max_sync(0xffffffffu, s_hi[lane]);
    top = 32 - __clz(lo ^ hi);
    thr = lo & ~((1ull << top) - 1ull);
  };
  prefix_of_all();
  for (bool by_position = false;;) {
    while (top > 0 && left != want && left > kRank) {
      const int width = min(11, top), shift = top - width;
#pragma unroll
      for (int i = 0; i < kC; ++i)
        if (alive(i) && above(v[i] ^ thr, top) == 0u) atomicAdd(&hist[(v[i] >> shift) & ((1u << width) - 1u)], 1u);
      __syncthreads();
      const unsigned c0 = hist[2 * tid], c1 = hist[2 * tid + 1];
      unsigned incl = c0 + c1;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
      }
      if (lane == 31) s_tot[warp] = incl;
      __syncthreads();
      hist[2 * tid] = 0u;  // (for the next pass)
      hist[2 * tid + 1] = 0u;
      const unsigned before = __reduce_add_sync(0xffffffffu, lane < warp ? s_tot[lane] : 0u) + incl - c0 - c1;
      if (before < want && want <= before + c0 + c1) {  // one thread
        const bool second = want > before + c0;
        s_digit = 2u * tid + (second ? 1u : 0u);
        s_below = before + (second ? c0 : 0u);
        s_count = second ? c1 : c0;
      }
      __syncthreads();
      want -= s_below;
      left = s_count;
      thr |= s_digit << shift;
      top = shift;
    }
    if (by_position || left == want || left <= kRank) break;
    by_position = true;  // top == 0: the scores at the threshold are equal to the last bit
#pragma unroll
    for (int i = 0; i < kC; ++i) {
      taken |= (alive(i) && v[i] < thr ? 1u : 0u) << i;
      if (v[i] != thr) live &= ~(1u << i);
      if (alive(i)) v[i] = position(tid + i * kSelThreads);
    }
    __syncthreads();
    prefix_of_all();
  }
  // the largest (v, position) that is taken
  unsigned kv = thr | (unsigned)((1ull << top) - 1ull), kp = 0xffffffffu;
  if (left != want && left <= kRank) {
    unsigned long long* list = reinterpret_cast<unsigned long long*>(hist);
#pragma unroll
    for (int i = 0; i < kC; ++i)
      if (alive(i) && above(v[i] ^ thr, top) == 0u)  // (the order of the list does not matter)
        list[atomicAdd(&s_list, 1u)] = ((unsigned long long)v[i] << 32) | position(tid + i * kSelThreads);
    if (tid == 0 && (left & 1u)) list[left] = ~0ull;
    __syncthreads();
    if (tid < (int)left) {
      const unsigned long long mine = list[tid];
      unsigned below = 0u, same = 0u;
#pragma unroll 4
      for (unsigned q = 0; q < left; q += 2) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(list + q);
        below += (o.x < mine) + (o.y < mine);
        same += (o.x == mine) + (o.y == mine);
      }
      if (below < want && want <= below + same) s_kth = mine;
    }
    __syncthreads();
    kv = (unsigned)(s_kth >> 32);
    kp = (unsigned)s_kth;
  }
  // one scan over the (round, warp) counts, which is the ascending order of the slots tid + round * kSelThreads
  unsigned ballots[kC];
#pragma unroll
  for (int i = 0; i < kC; ++i) {
    bool in = (taken >> i & 1u) != 0u;
    if (alive(i)) in = v[i] < kv || (v[i] == kv && (kp == 0xffffffffu || position(tid + i * kSelThreads) <= kp));
    ballots[i] = __ballot_sync(0xffffffffu, in);
    if (lane == 0) s_cnt[i * kW + warp] = __popc(ballots[i]);
  }
  __syncthreads();
  if (warp == 0) {
    int c[kC], sum = 0;
#pragma unroll
    for (int q = 0; q < kC; ++q) { c[q] = s_cnt[kC * lane + q]; sum += c[q]; }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += t;
    }
    int run = incl - sum;
#pragma unroll
    for (int q = 0; q < kC; ++q) { s_cnt[kC * lane + q] = run; run += c[q]; }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kC; ++i) {
    if (ballots[i] >> lane & 1u) {
      const int idx = s_cnt[i * kW + warp] + __popc(ballots[i] & ((1u << lane) - 1u));
      if (idx < k) {
        out[idx] = tid + i * kSelThreads;
        if (picks) picks[idx] = tid + i * kSelThreads;
      }
    }
  }
}

// The same for a unit of any length, on 64-bit keys read again in every pass: 8 passes of an 8-bit radix histogram at most,
// then an ordered compaction of 1024 slots at a time.
template <typename Score, typename Position>
__device__ __noinline__ void select_long(int n, int k, Score score, Position position, int* out, int* picks) {
  __shared__ unsigned int hist[256];
  __shared__ unsigned long long s_prefix;
  __shared__ int s_remaining, s_running, s_done;
  __shared__ int s_warp_tot[kSelThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) { s_prefix = 0ull; s_remaining = k; s_done = 0; }
  unsigned long long kth = ~0ull;
  for (int pass = 0; pass < 8; ++pass) {
    const int shift = 56 - 8 * pass;
    if (tid < 256) hist[tid] = 0u;
    __syncthreads();
    const unsigned long long prefix = s_prefix;
    const unsigned long long mask = (pass == 0) ? 0ull : (~0ull << (shift + 8));
    for (int j = tid; j < n; j += kSelThreads) {
      const unsigned long long key = make_key(score(j), position(j));
      if ((key & mask) == prefix) atomicAdd(&hist[(unsigned int)(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (warp == 0) {
      // the first digit whose cumulative count reaches the number still wanted: 8 bins per lane
      unsigned int c[8], sum = 0u;
#pragma unroll
      for (int q = 0; q < 8; ++q) { c[q] = hist[8 * lane + q]; sum += c[q]; }
      unsigned int incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned int t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
      }
      const unsigned int rem = (unsigned int)s_remaining;
      const unsigned int reach = __ballot_sync(0xffffffffu, rem <= incl);
      const int f = reach ? __ffs((int)reach) - 1 : 31;
      if (lane == f) {
        unsigned int r = rem - (incl - sum);
        int q = 0;
        for (; q < 7; ++q) {
          if (r <= c[q]) break;
          r -= c[q];
        }
        s_remaining = (int)r;
        s_prefix = prefix | ((unsigned long long)(8 * lane + q) << shift);
        s_done = (r == c[q]) ? 1 : 0;
      }
    }
    __syncthreads();
    if (s_done || pass == 7) {
      kth = s_prefix | (shift ? ((1ull << shift) - 1ull) : 0ull);  // the largest key that is taken
      break;
    }
  }
  if (tid == 0) s_running = 0;
  __syncthreads();
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    const unsigned long long key = (j < n) ? make_key(score(j), position(j)) : ~0ull;
    const int flag = (j < n) && (key <= kth);
    const unsigned int ballot = __ballot_sync(0xffffffffu, flag);
    const int in_warp = __popc(ballot & ((1u << lane) - 1u));
    if (lane == 0) s_warp_tot[warp] = __popc(ballot);
    __syncthreads();
    int before = s_running;
    for (int w = 0; w < warp; ++w) before += s_warp_tot[w];
    const int idx = before + in_warp;
    if (flag && idx < k) {
      out[idx] = j;
      if (picks) picks[idx] = j;
    }
    __syncthreads();
    if (tid == 0) {
      int tot = s_running;
      for (int w = 0; w < kSelThreads / 32; ++w) tot += s_warp_tot[w];
      s_running = tot;
    }
    __syncthreads();
  }
}

// Copy one row of `bytes` bytes (a multiple of 16, 16-byte aligned on both sides) with one warp.
__device__ __forceinline__ void warp_copy_row(char* dst, const char* src, int bytes, int lane) {
  for (int o = lane * 16; o < bytes; o += 32 * 16)
    *reinterpret_cast<uint4*>(dst + o) = *reinterpret_cast<const uint4*>(src + o);
}

// First index in sorted a[0..n) whose value is >= x.
__device__ __forceinline__ int lower_bound(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] < x) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// Every CTA's last step: whichever CTA of the launch finishes last (a ticket counter in the workspace header, which that CTA
// also resets) moves the lengths on, so that no other CTA still needs the old ones.
__device__ __forceinline__ void finish_lengths(int B, int* __restrict__ len, const int* __restrict__ n_evict, int* ticket) {
  __shared__ int s_last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = (atomicAdd(ticket, 1) == (int)(gridDim.x * gridDim.y) - 1);
  }
  __syncthreads();
  if (s_last) {
    __threadfence();
    for (int b = threadIdx.x; b < B; b += blockDim.x) len[b] -= __ldcg(&n_evict[b]);
    if (threadIdx.x == 0) *ticket = 0;
  }
}

}  // namespace sel
}  // namespace caote
