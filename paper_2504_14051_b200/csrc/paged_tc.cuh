// Attention of packed rows over prompts or pages on the tensor cores (tcgen05 + TMEM): bf16, head_dim 64 or 128.
//
//   attend_kernel   rows x keys. A CTA owns two blocks of up to 128 query rows of a (sequence, KV head) pair (a block: 128 / G
//                   tokens with all G heads) and walks the keys that they see in tiles of 128, K and V of a tile read once for
//                   both blocks. S = Q K^T into TMEM; a thread per row takes its logits out of TMEM, keeps a reference and the
//                   sum, and writes its numerators P as bf16 over the S it came from, 64 keys at a time; O += P V with P as
//                   the TMEM-side A operand. The two blocks take turns: while one's logits are being exponentiated, the
//                   other's products run.
//   mass_kernel     keys x rows. A CTA owns 256 keys of a pair and walks the rows that see them: S^T = K Q^T into TMEM, one key
//                   per lane, so that a thread sums 2^(s - lse) over the rows of its own key without any exchange.
//   combine_kernel  adds up what the splits of a row's keys left, sum_kernel what the chunks of a key's rows left.
//
// Roundings: P is rounded to bf16 once (2^-8 of each weight at most, of random sign), since the product takes bf16 on both sides; o,
// of which it is a weighted sum, is rounded to bf16 itself, so o's error against 64 bits is sqrt(2) of what the output's type costs at
// most (measured: 1.04 to 1.11 of it).
// Maximum, sum, O, lse and mass are fp32; the sum takes the numerators before they are rounded.
//
// A row that sees a NaN or a logit of +inf is NaN, and so are its statistic and the weights that it gives; a masked weight is
// exactly 0. Where a row sees none of a split's keys, its statistic there is -inf, and the merge leaves the split out.
//
// Operands come by TMA as boxes of 64 channels with the 128-byte swizzle: of q a box of all heads of the group x 128 / G tokens,
// of K and V a box per page (pages of 16 tokens: eight per tile), by the lanes of a warp side by side. Every mbarrier wait is
// bounded; one that runs out records CAOTE_ERR_TIMEOUT and the thread carries on in bounds, or, where it waited for its next item,
// comes to its end.
#pragma once

#include <cuda.h>

#include "paged_common.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace caote {
namespace paged {
namespace tcore {

using namespace caote::tc;
using ptx::tma_load_3d;

constexpr int kLeastTiles = 4;  // key tiles per split
constexpr int kPolyOf = 4;      // of so many pairs of exponentials one goes to the FMA pipe (none: 260, one of four: 242 us, 12 001 prompt tokens)
template <int D>
constexpr int kKStages = D == 128 ? 2 : 4;
template <int D>
constexpr int kVStages = D == 128 ? 3 : 4;
constexpr int kRowThreads = 512;                  // two threads per row of two blocks
constexpr int kAttendThreads = kRowThreads + 96;  // and warps for products, Q and K copies, V copies
template <int D>
constexpr size_t attend_smem() { return 1024 + (size_t)(2 + kKStages<D> + kVStages<D>) * kTileBytesOf<D> + 2 * kTile * sizeof(float) + 512; }

// Tiles of 128 keys come as boxes of `box` tokens: min(page, 128), prompts 128. Lane l of a warp copies box l of a tile.
// The page of this lane's box of the tile at slot j0 (of no meaning behind the length).
template <bool kPaged>
__device__ __forceinline__ int page_of(const PDims& dm, const Seqs& sq, int b, int n, int j0, int box, int* status) {
  if (!kPaged) return 0;
  const int lane = threadIdx.x & 31, j = j0 + lane * box;
  if (lane * box >= kTile || j >= n) return 0;
  int id = __ldg(sq.table + (size_t)b * dm.max_pages + (j >> dm.page_shift));
  if ((unsigned)id >= (unsigned)dm.n_pages) {
    set_status(status, CAOTE_ERR_BAD_PAGE);
    id = 0;
  }
  return id;
}
template <bool kPaged>
__device__ __forceinline__ int boxes_of(const Seq& s, int j0, int box) { return kPaged ? (min(kTile, s.n - j0) + box - 1) / box : 1; }
// Copies a tile of K or V into a stage, bytes announced by the caller; the whole warp.
template <int D, bool kPaged>
__device__ __forceinline__ void copy_keys(const PDims& dm, const CUtensorMap* tm, const Seq& s, int h, int j0, int box, int id, char* dst,
                                          uint64_t* bar) {
  const int lane = threadIdx.x & 31;
  if (lane < boxes_of<kPaged>(s, j0, box)) {
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {
      if (kPaged)
        tma_load_2d(dst + x * kHalfBytes + lane * box * 128, tm, 64 * x,
                    ((id * dm.Hkv + h) << dm.page_shift) + ((j0 + lane * box) & ((1 << dm.page_shift) - 1)), bar);
      else
        tma_load_2d(dst + x * kHalfBytes, tm, h * D + 64 * x, s.t0 + j0, bar);
    }
  }
  __syncwarp();
}

// Work is numbered in items: a pair of row blocks of one KV head, the heads in turn, a sequence's longest first. Whole rounds of
// items, one per SM, are taken as they are; the keys of the last items, fewer than SMs, are split among the SMs (most_splits > 1).
struct Schedule {
  int items, whole, splits;  // items [whole, items) are cut into `splits`
};
__device__ __forceinline__ Schedule schedule(const PDims& dm, int per_head, int sms, int most_splits) {
  Schedule c;
  c.items = (int)min((long long)per_head * dm.Hkv, (long long)kMostBlocks);
  c.whole = c.items / sms * sms;
  c.splits = c.items > c.whole ? min(most_splits, sms / (c.items - c.whole)) : 1;
  return c;
}
// What a CTA works on.
struct Where {
  int b, i0, h;           // sequence (-1: nothing), first token, KV head
  int split, splits, x;   // split of the keys of how many, place behind the whole items
  Seq s;
};
// What combine_kernel needs to know, left by attend_kernel: [0] = (split items, splits), [1 + i] = (sequence, first token, KV head,
// splits in use) of split item i.
typedef int4 SplitNote;

// grid: CTA x takes item x, or behind the whole ones split (x - whole) % splits of item whole + (x - whole) / splits. lse2: the
// rows' statistics for the mass (stat_at); a split leaves its rows' normalised outputs and statistics at opart, lpart
// [x - whole][256 rows].
template <int D, bool kPaged>
__global__ void __launch_bounds__(kAttendThreads, 1)
attend_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
              PDims dm, Seqs sq, int box, __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ lse2,
              float* __restrict__ opart, float* __restrict__ lpart, SplitNote* __restrict__ notes, int sms, int most_splits, int* next_item, int* status) {
  constexpr int kTB = kTileBytesOf<D>, kBoxes = D / 64, kSteps = D / 16, kKS = kKStages<D>, kVS = kVStages<D>;
  if (threadIdx.x == 0) {
    ptx::prefetch_map(&tmQ);
    ptx::prefetch_map(&tmK);
    ptx::prefetch_map(&tmV);
  }
  ptx::pdl_wait();
  ptx::pdl_trigger();
  extern __shared__ char smem_raw[];
  // (aligned by an offset into the array: the pointer keeps its address space)
  char* sm = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  char* Qs = sm;                  // [2]
  char* Ks = Qs + 2 * kTB;        // [kKS]
  char* Vs = Ks + kKS * kTB;      // [kVS]
  float* xch = reinterpret_cast<float*>(Vs + kVS * kTB);  // [2][kTile] a row's maximum on its way between its two threads
  uint64_t* bars = reinterpret_cast<uint64_t*>(xch + 2 * kTile);
  uint64_t *q_bar = &bars[0], *k_bar = &bars[1], *v_bar = k_bar + kKS, *k_free = v_bar + kVS, *v_free = k_free + kKS,
           *s_bar = v_free + kVS, *h_bar = s_bar + 2, *o_bar = h_bar + 2, *p_bar = o_bar + 2;  // p_bar: [block][part]
  constexpr int kBars1 = 1 + 2 * (kKS + kVS) + 6;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kBars1 + 4);
  Where* where = reinterpret_cast<Where*>(tmem_slot + 1);

  const int tid = threadIdx.x, lane = tid & 31, warp = ptx::warp_index();
  const int tok = kTile / dm.G;  // tokens per row block
  // three warps set up side by side: which item, barriers, TMEM
  if (warp == 0) {
    auto what = [](const Seq& x) { return x.m; };
    Scan first;
    const Schedule c = schedule(dm, count_blocks(dm, sq, 2 * tok, what, blockIdx.x == 0 ? status : nullptr, first), sms, most_splits);
    const int x = blockIdx.x - c.whole, item = x < 0 ? blockIdx.x : c.whole + x / c.splits;
    Place p;
    const bool there = item < c.items && find_block(dm, sq, 2 * tok, item / dm.Hkv, what, first, p);
    if (lane == 0) {
      *where = Where{there ? p.b : -1, (p.blocks - 1 - p.block) * 2 * tok, item % dm.Hkv, x < 0 ? 0 : x % c.splits, x < 0 ? 1 : c.splits, x, p.s};
      if (blockIdx.x == 0) {
        *next_item = sms;  // (for the mass kernel, whose CTAs begin with items of their own number)
        notes[0] = make_int4(c.splits > 1 ? c.items - c.whole : 0, c.splits, 0, 0);
      }
    }
  } else if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
  } else if (tid == 64) {
    for (int i = 0; i < kBars1; ++i) mbar_init(&bars[i], 1);
    for (int i = 0; i < 4; ++i) mbar_init(&p_bar[i], 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // columns: S (and P) of block i at 128 i, O at 256 + 128 i
  const uint32_t tmem = *tmem_slot;
  const int b = where->b, i0 = where->i0, h = where->h, split = where->split;
  const Seq s = where->s;
  const int first = s.n - s.m;  // token i sees slots up to first + i
  int per = 1, count = 0;
  if (b >= 0) key_splits((s.n + kTile - 1) / kTile, where->splits, kLeastTiles, per, count);
  if (split == 0 && where->splits > 1 && b >= 0 && tid == 0) notes[1 + where->x / where->splits] = make_int4(b, i0, h, count);
  if (split >= count) {
    if (warp == 1) tmem_dealloc(tmem, 512);
    return;
  }
  // this CTA's tiles [kt0, kt0 + c) for either block
  const int kt0 = split * per;
  const int c0 = min(per, (first + min(i0 + tok, s.m) - 1) / kTile + 1 - kt0);
  const int c1 = i0 + tok < s.m ? min(per, (first + min(i0 + 2 * tok, s.m) - 1) / kTile + 1 - kt0) : 0;
  const int tiles = max(max(c0, c1), 0);

  if (warp >= 17) {
    // =============================== copies: warp 17 Q and K, warp 18 V ===============================
    const bool is_v = warp == 18;
    const CUtensorMap* tm = is_v ? &tmV : &tmK;
    char* ring = is_v ? Vs : Ks;
    uint64_t *full = is_v ? v_bar : k_bar, *free = is_v ? v_free : k_free;
    const int stages = is_v ? kVS : kKS;
    if (!is_v && lane == 0 && tiles > 0) {
      const int blocks = c1 > 0 ? 2 : 1;
      mbar_expect_tx(q_bar, blocks * kBoxes * tok * dm.G * 128);
      for (int i = 0; i < blocks; ++i)
#pragma unroll
        for (int x = 0; x < kBoxes; ++x)
          tma_load_3d(Qs + i * kTB + x * kHalfBytes, &tmQ, 64 * x, h * dm.G, s.t0 + i0 + i * tok, q_bar);
    }
    int st = 0, round = 0;
    int id = page_of<kPaged>(dm, sq, b, s.n, kt0 * kTile, box, status);
    for (int kt = 0; kt < tiles; ++kt) {
      const int j0 = (kt0 + kt) * kTile;
      const int next = page_of<kPaged>(dm, sq, b, s.n, j0 + kTile, box, status);
      if (round > 0) mbar_wait_idle(&free[st], (round - 1) & 1, status);
      if (lane == 0) mbar_expect_tx(&full[st], boxes_of<kPaged>(s, j0, box) * box * D * 2);
      __syncwarp();
      copy_keys<D, kPaged>(dm, tm, s, h, j0, box, id, ring + st * kTB, &full[st]);
      id = next;
      if (++st == stages) { st = 0; ++round; }
    }
  } else if (warp == 16) {
    // =============================== products (one lane) ===============================
    if (ptx::elect_one() && tiles > 0) {
      constexpr uint32_t kIdescS = instr_desc_n(false, kTile), kIdescO = instr_desc_n(true, D);
      const uint64_t qdesc0 = smem_desc(smem_u32(Qs), 16, 1024), kdesc0 = smem_desc(smem_u32(Ks), 16, 1024),
                     vdesc0 = smem_desc(smem_u32(Vs), kHalfBytes, 1024);
      auto issue_s = [&](int i, int kt) {  // S of block i and tile kt
        const int st = kt % kKS;
        mbar_wait(&k_bar[st], (kt / kKS) & 1, status);
        tc_fence_after();
        const uint64_t qd = qdesc0 + (uint64_t)((i * kTB) >> 4), kd = kdesc0 + (uint64_t)((st * kTB) >> 4);
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) umma(tmem + i * 128, qd + k_major_step(ks), kd + k_major_step(ks), kIdescS, ks > 0);
        // (the last block that reads this K hands its stage back, if anyone waits for it)
        if (kt + kKS < tiles && (i == 1 || kt >= c1)) umma_commit(&k_free[st]);
        umma_commit(&s_bar[i]);
      };
      mbar_wait(q_bar, 0, status);
      if (c0 > 0) issue_s(0, 0);
      if (c1 > 0) issue_s(1, 0);
      for (int kt = 0; kt < tiles; ++kt) {
        const int st = kt % kVS;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int c = i ? c1 : c0;
          if (kt >= c) continue;
          mbar_wait(&v_bar[st], (kt / kVS) & 1, status);
          const uint64_t vd = vdesc0 + (uint64_t)((st * kTB) >> 4);
#pragma unroll
          for (int part = 0; part < 2; ++part) {  // 32 keys of either half, as the rows hand them over
            mbar_wait(&p_bar[2 * i + part], kt & 1, status);
            tc_fence_after();
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int ks = (x >> 1) * 4 + 2 * part + (x & 1);
              umma_ts(tmem + 256 + i * 128, tmem + i * 128 + (ks >> 2) * 64 + (ks & 3) * 8, vd + mn_major_step(ks), kIdescO, kt > 0 || ks > 0);
            }
            if (part == 0) umma_commit(&h_bar[i]);
          }
          if (kt + kVS < tiles && (i == 1 || kt >= c1)) umma_commit(&v_free[st]);
          umma_commit(&o_bar[i]);
          // (in the order of issue: the product above has read P before this one overwrites it)
          if (kt + 1 < c) issue_s(i, kt + 1);
        }
      }
    }
  } else {
    // =============================== two threads per query row ===============================
    // Threads t and t + 128 of a block's 256 share row t: each has 64 of a tile's keys and half of the channels when O is touched.
    // (A thread per row: a warp alone on its scheduler takes 4 cycles per instruction and twice what the exponentials take.)
    const int i = warp >> 3, hf = (warp >> 2) & 1, row = tid & 127, c = i ? c1 : c0;
    const int pair_bar = 1 + i * 4 + (warp & 3);  // the two warps that share 32 rows
    const int tkn = i0 + i * tok + row / dm.G;
    const bool valid = row < tok * dm.G && tkn < s.m;
    const int vis = valid ? first + tkn + 1 : s.n;       // keys this row sees
    const int plain = first + i0 + i * tok + 1;          // ... and every row of the block
    const float scale2 = dm.scale * kLog2e;
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16) + i * 128;
    const uint32_t t_s = t_lane + hf * 64, t_o = t_lane + 256 + hf * (D / 2);
    // the larger of a value of this thread and one of the row's other thread
    auto row_max = [&](float x) {
      float* at = xch + i * kTile + row;
      if (hf == 1) *at = x;
      asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
      if (hf == 0) *at = x = fmaxf(x, *at);
      asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
      if (hf == 1) x = *at;
      return x;
    };
    // whether any thread of the two warps says so
    auto any_of_pair = [&](bool x) {
      uint32_t r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.u32 q, %1, 0;\n\t"
          "bar.red.or.pred p, %2, 64, q;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(r) : "r"((uint32_t)x), "r"(pair_bar) : "memory");
      return r != 0;
    };
    // Numerators are 2^(logit - m_ref) for a reference that is left alone until a logit passes it by 20: nothing is lost meanwhile
    // (P, l and O are floats, their ratios do not depend on it), and no maximum stands between a logit and its exponential. The
    // 32 keys of a part are exponentiated and their maximum is formed at the same time; only where it has passed the mark is the
    // part done again, with a new reference. (O holds up to 2^20 n times the values: with a mark of 60 those beyond 2^67 / n overflowed.)
    constexpr float kMark = 20.f;
    float m_ref = -INFINITY, l = 0.f;
    const float2 scale22 = make_float2(scale2, scale2);
    for (int kt = 0; kt < c; ++kt) {
      const int j0 = (kt0 + kt) * kTile;
      const bool masked = j0 + kTile > plain;
      const int lim = vis - j0 - hf * 64;
      mbar_wait(&s_bar[i], kt & 1, status);
      tc_fence_after();
      if (kt == 0) {  // the first reference: the largest of the first 32 logits of either half
        float mx = -INFINITY;
#pragma unroll 1
        for (int e0 = 0; e0 < 32; e0 += 16) {
          uint32_t v[16];
          tmem_ld16_issue(t_s + e0, v);
          tmem_ld16_wait(v);
#pragma unroll
          for (int e = 0; e < 16; ++e) mx = fmaxf(mx, e0 + e < lim ? __uint_as_float(v[e]) : -INFINITY);
        }
        m_ref = row_max(mx * scale2);
      }
      const int n_valid = s.n - j0;
      if (n_valid < kTile) {
        // V rows behind the length hold anything: they become zeros, so that 0 * NaN cannot reach O. (Both blocks' rows write
        // the same zeros, each before its own products.)
        mbar_wait(&v_bar[kt % kVS], (kt / kVS) & 1, status);
        if (row >= n_valid) {
          char* vt = Vs + (kt % kVS) * kTB;
#pragma unroll
          for (int x = hf * (D / 16); x < (hf + 1) * (D / 16); ++x)
            *reinterpret_cast<uint4*>(vt + (x >> 3) * kHalfBytes + row * 128 + (((x & 7) ^ (row & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
        }
        ptx::fence_async_smem();
      }
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        uint32_t pk[16];
        float2 sum;
        for (;;) {
          uint32_t v[32];
          tmem_ld32_issue(t_s + 32 * part, v);
          tmem_ld32_wait(v);
          const float neg = m_ref == -INFINITY ? 0.f : -m_ref;
          const float2 neg2 = make_float2(neg, neg);
          if (masked) {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 32 * part + e < lim ? v[e] : 0xff800000u;
          }
          float2 ls[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), scale22, neg2);
            const float2 p = e % kPolyOf == kPolyOf - 1 ? poly_exp2x2(x, -127.f) : make_float2(ptx::fast_exp2(x.x), ptx::fast_exp2(x.y));
            ls[e & 1] = __fadd2_rn(ls[e & 1], p);
            pk[e] = pack_bf16(p.x, p.y);
          }
          float pm[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 32; e += 8)
#pragma unroll
            for (int f = 0; f < 4; ++f) pm[f] = ptx::max3_nan(pm[f], __uint_as_float(v[e + f]), __uint_as_float(v[e + f + 4]));
          const float mx = ptx::max3_nan(ptx::max3_nan(pm[0], pm[1], pm[2]), pm[3], pm[3]) * scale2;
          sum = __fadd2_rn(ls[0], ls[1]);
          // (a NaN or +inf among the keys whose exponentials are polynomials, which do not hand it on)
          if (!(mx < INFINITY)) sum.x = NAN;
          if (!any_of_pair(mx > m_ref + kMark)) break;
          const float both = row_max(mx);
          float corr = 1.f;
          if (both > m_ref + kMark) {
            corr = ptx::fast_exp2(m_ref - both);
            m_ref = both;
            l *= corr;
          }
          // O holds all tiles before this one (S of this tile was formed behind their products), and behind the first part
          // that too
          if (part == 1) {
            mbar_wait(&h_bar[i], kt & 1, status);
            tc_fence_after();
          }
          if (kt > 0 || part == 1) {
#pragma unroll 1
            for (int cc = 0; cc < D / 32; ++cc) {
              uint32_t w[16];
              tmem_ld16_issue(t_o + cc * 16, w);
              tmem_ld16_wait(w);
#pragma unroll
              for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * corr);
              tmem_st16u(t_o + cc * 16, w);
            }
          }
        }
        l += sum.x + sum.y;
        tmem_st16u(t_s + 16 * part, pk);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_bar[2 * i + part]);
      }
    }
    if (c > 0) {
      mbar_wait(&o_bar[i], (c - 1) & 1, status);
      tc_fence_after();
    }
    // ---- the row's output and statistic; rows go out by way of the block's Q tile, which its products are done with, 16 bytes
    // number c of a row at place c ^ (row & 7) (a thread's own row straight to memory: 32 lines per store) ----
    {
      // the sums of the row's two threads
      float* at = xch + i * kTile + row;
      if (hf == 1) *at = l;
      asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
      if (hf == 0) *at = l += *at;
      asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
      if (hf == 1) l = *at;
    }
    // (l is 0 where the row sees nothing but logits of -inf: none of this split's keys, or a softmax that is no number; NaN goes on)
    const float inv = 1.f / l, stat = m_ref + __log2f(l);
    char* mine = Qs + i * kTB + (warp & 3) * (kTB / 4);  // the pair's 32 rows
    auto place = [&](int r, int piece) { return mine + r * (kTB / 128) + ((piece ^ (r & 7)) << 4); };
    if (count == 1) {
      if (valid && hf == 0) {
        lse2[stat_at(dm, s, h, (i0 + i * tok) * dm.G + row)] = stat;
        if (lse) lse[(size_t)(s.t0 + tkn) * dm.Hq + h * dm.G + row % dm.G] = stat * kLn2;
      }
      if (c > 0) {
#pragma unroll
        for (int cc = 0; cc < D / 64; ++cc) {
          float v[32];
          tmem_ld32(t_o + cc * 32, v);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(place(lane, hf * (D / 16) + cc * 4 + e)) =
                make_uint4(pack_bf16(v[8 * e] * inv, v[8 * e + 1] * inv), pack_bf16(v[8 * e + 2] * inv, v[8 * e + 3] * inv),
                           pack_bf16(v[8 * e + 4] * inv, v[8 * e + 5] * inv), pack_bf16(v[8 * e + 6] * inv, v[8 * e + 7] * inv));
        }
        asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
        constexpr int kPieces = D / 8, kAtOnce = 32 / kPieces;
#pragma unroll 4
        for (int r0 = hf * 16; r0 < hf * 16 + 16; r0 += kAtOnce) {
          const int r = r0 + lane / kPieces, br = (warp & 3) * 32 + r, t = i0 + i * tok + br / dm.G;
          if (br < tok * dm.G && t < s.m)
            *reinterpret_cast<uint4*>(o + ((size_t)(s.t0 + t) * dm.Hq + h * dm.G + br % dm.G) * D + lane % kPieces * 8) =
                *reinterpret_cast<const uint4*>(place(r, lane % kPieces));
        }
      }
    } else {
      // [x][block][quarter of the channels][row], pieces as they lie in shared memory: a warp has 32 rows x two quarters
      const size_t slot = (size_t)where->x * (2 * kTile) + i * kTile;
      if (valid && hf == 0) lpart[slot + row] = stat;
      if (c > 0) {
        constexpr int kQ = D / 4, kPieces = kQ / 4;
        char* quarter = mine + hf * (kTB / 8);
#pragma unroll
        for (int e0 = 0; e0 < 2; ++e0) {
          if (e0 == 1) {
            if (lane == 0) ptx::bulk_wait_read();
            __syncwarp();
          }
#pragma unroll
          for (int cc = 0; cc < kQ / 16; ++cc) {
            uint32_t v[16];
            tmem_ld16_issue(t_o + e0 * kQ + cc * 16, v);
            tmem_ld16_wait(v);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<float4*>(quarter + lane * (kQ * 4) + (((cc * 4 + e) ^ (lane & (kPieces - 1))) << 4)) =
                  make_float4(__uint_as_float(v[4 * e]) * inv, __uint_as_float(v[4 * e + 1]) * inv, __uint_as_float(v[4 * e + 2]) * inv,
                              __uint_as_float(v[4 * e + 3]) * inv);
          }
          ptx::fence_async_smem();
          __syncwarp();
          if (lane == 0) {
            ptx::bulk_store(opart + (slot * 4 + (hf * 2 + e0) * kTile + (warp & 3) * 32) * kQ, quarter, 32 * kQ * 4);
            ptx::bulk_commit();
          }
        }
        if (lane == 0) ptx::bulk_wait();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// o = sum_s o_s 2^(lse_s - lse) over the splits of the rows of split items. grid = (most split items, 8): a CTA has 32 rows of an item,
// four per warp; a lane has 16 bytes of a row's partial output (head_dim 64: of every other split's).
template <int D>
__global__ void __launch_bounds__(256)
combine_kernel(PDims dm, Seqs sq, __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ lse2,
               const float* __restrict__ opart, const float* __restrict__ lpart, const SplitNote* __restrict__ notes) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  constexpr int kR = 4, kLanes = D / 4, kStep = 32 / kLanes, kQ = D / 4, kPieces = kQ / 4;
  const int tok = kTile / dm.G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const SplitNote all = notes[0], it = notes[1 + blockIdx.x];
  if ((int)blockIdx.x >= all.x || it.w == 1) return;
  const int t0 = sq.cu[it.x], m = sq.cu[it.x + 1] - t0, i0 = it.y, h = it.z, count = it.w;
  const int local0 = blockIdx.y * 32 + warp * kR, i = local0 / kTile, row0 = local0 % kTile;
  const size_t base = (size_t)blockIdx.x * all.y * (2 * kTile) + i * kTile;  // of split 0
  // this lane's four channels, and where they lie for row r: in quarter `qu`, piece `piece` of the row
  const int ch = lane % kLanes * 4, qu = ch / kQ, piece = ch % kQ / 4, sp0 = lane / kLanes;
  float mine[kR];
#pragma unroll
  for (int e = 0; e < kR; ++e) {
    const bool there = row0 + e < tok * dm.G && i0 + i * tok + (row0 + e) / dm.G < m;
    mine[e] = there && lane < count ? lpart[base + (size_t)lane * (2 * kTile) + row0 + e] : -INFINITY;
  }
  float stat[kR];
  float4 v[kR];
#pragma unroll
  for (int e = 0; e < kR; ++e) {
    // (the maximum leaves NaN out, the sum does not; nothing but -inf: 0 / 0)
    const float top = warp_max(mine[e]);
    mine[e] = mine[e] == -INFINITY ? 0.f : ptx::fast_exp2(mine[e] - top);
    const float sum = warp_sum(mine[e]);
    stat[e] = top + __log2f(sum);
    mine[e] = mine[e] / sum;
    v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll 4
  for (int s0 = 0; s0 < count; s0 += kStep) {
    const int sp = s0 + sp0;
#pragma unroll
    for (int e = 0; e < kR; ++e) {
      const float w = __shfl_sync(0xffffffffu, mine[e], min(sp, 31));
      if (w != 0.f && sp < count) {  // (a split in which the row sees no key has written no output)
        const int row = row0 + e;
        const float4 x = *reinterpret_cast<const float4*>(
            opart + ((base + (size_t)sp * (2 * kTile)) * 4 + qu * kTile + row) * kQ + ((piece ^ (row & (kPieces - 1))) << 2));
        v[e].x = fmaf(w, x.x, v[e].x);
        v[e].y = fmaf(w, x.y, v[e].y);
        v[e].z = fmaf(w, x.z, v[e].z);
        v[e].w = fmaf(w, x.w, v[e].w);
      }
    }
  }
  Seq s;
  s.t0 = t0;
#pragma unroll
  for (int e = 0; e < kR; ++e) {
    if (kStep == 2) {
      v[e].x += __shfl_xor_sync(0xffffffffu, v[e].x, 16);
      v[e].y += __shfl_xor_sync(0xffffffffu, v[e].y, 16);
      v[e].z += __shfl_xor_sync(0xffffffffu, v[e].z, 16);
      v[e].w += __shfl_xor_sync(0xffffffffu, v[e].w, 16);
    }
    const int tkn = i0 + i * tok + (row0 + e) / dm.G;
    if (row0 + e >= tok * dm.G || tkn >= m) continue;
    const size_t at = (size_t)(t0 + tkn) * dm.Hq + h * dm.G + (row0 + e) % dm.G;
    if (lane < kLanes) *reinterpret_cast<uint2*>(o + at * D + ch) = make_uint2(pack_bf16(v[e].x, v[e].y), pack_bf16(v[e].z, v[e].w));
    if (lane == 0) {
      lse2[stat_at(dm, s, h, (i0 + i * tok) * dm.G + row0 + e)] = stat[e];
      if (lse) lse[at] = stat[e] * kLn2;
    }
  }
}

// ---- the weight that every key received ------------------------------------------------------------------
// Persistent: a CTA takes items of 256 keys from a counter, the next item's K on its way while this one's rows go by. The warps
// that copy and issue run ahead of the key threads across items; rows, statistics and S buffers are counted through.
// Of a prompt the first keys are seen by all rows: where that is more than a third of an SM's share, the rows are cut into chunks
// that are items of their own and leave partial sums, which sum_kernel adds up in order (whole calls, one prompt of 6 000 tokens, 64/8
// heads: 1 025 - 1 050 us in one chunk, 870 - 970 in five; of 4 000, 32/2 heads: 692 and 304 - 331).
constexpr int kKeys = 2 * kTile;                       // keys per item
constexpr int kKeyThreads = 2 * kKeys;                 // two threads per key: 64 rows of a row block each
constexpr int kMassThreads = kKeyThreads + 128;        // + products, items and K, Q, statistics
constexpr int kStatStages = 4;
template <int D>
constexpr int kQStages = D == 128 ? 2 : 4;
template <int D>
constexpr size_t mass_smem() { return 1024 + (size_t)(4 + kQStages<D>) * kTileBytesOf<D> + (kStatStages * kTile + 2 * kKeys) * sizeof(float) + 512; }

// Adds the weights 2^(s * scale2 + stat) of a key in 16 rows to acc; two of eight exponentials on the FMA pipe. kMasked: only rows
// [lo, hi) of them count (the others' products may be anything).
template <bool kMasked>
__device__ __forceinline__ void add_weights(const uint32_t (&v)[16], const float4 (&st)[4], float scale2, int lo, int hi, float2 (&acc)[2]) {
  const float2 scale22 = make_float2(scale2, scale2);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float2 a = __ffma2_rn(make_float2(__uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1])), scale22, make_float2(st[k].x, st[k].y));
    float2 b = __ffma2_rn(make_float2(__uint_as_float(v[4 * k + 2]), __uint_as_float(v[4 * k + 3])), scale22, make_float2(st[k].z, st[k].w));
    if (kMasked) {
      if (4 * k < lo || 4 * k >= hi) a.x = -INFINITY;
      if (4 * k + 1 < lo || 4 * k + 1 >= hi) a.y = -INFINITY;
      if (4 * k + 2 < lo || 4 * k + 2 >= hi) b.x = -INFINITY;
      if (4 * k + 3 < lo || 4 * k + 3 >= hi) b.y = -INFINITY;
    }
    acc[0] = __fadd2_rn(acc[0], make_float2(ptx::fast_exp2(a.x), ptx::fast_exp2(a.y)));
    if (k & 1) b = poly_exp2x2<true>(b, -127.f);
    else b = make_float2(ptx::fast_exp2(b.x), ptx::fast_exp2(b.y));
    acc[1] = __fadd2_rn(acc[1], b);
  }
}

struct Item {
  int b, h, j0, rb0, blocks;  // b < 0: no more; row blocks (of 128 / G tokens) [rb0, rb0 + blocks) of the chunk that see any of the keys
  int chunk;
  Seq s;
};

// grid: one CTA per SM. chunks > 1 (prompts): rows in chunks of chunk_blocks blocks, mass [chunks, T, Hkv] their sums. next_item:
// the grid's size at the start (the attention pass leaves it so).
template <int D, bool kPaged>
__global__ void __launch_bounds__(kMassThreads, 1)
mass_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, PDims dm, Seqs sq, int box,
            const float* __restrict__ lse2, float* __restrict__ mass, int chunks, int chunk_blocks, int* next_item, int* status) {
  constexpr int kTB = kTileBytesOf<D>, kBoxes = D / 64, kSteps = D / 16, kQS = kQStages<D>;
  if (threadIdx.x == 0) {
    ptx::prefetch_map(&tmQ);
    ptx::prefetch_map(&tmK);
  }
  ptx::pdl_wait();
  ptx::pdl_trigger();
  extern __shared__ char smem_raw[];
  char* sm = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  char* Ks = sm;                                              // [2][2] tiles of an item
  char* Qs = Ks + 4 * kTB;                                    // [kQS]
  float* Ss = reinterpret_cast<float*>(Qs + kQS * kTB);       // [kStatStages][kTile] minus the rows' lse2
  float* half = Ss + kStatStages * kTile;                     // [2][kKeys] the upper halves' sums
  uint64_t* bars = reinterpret_cast<uint64_t*>(half + 2 * kKeys);
  uint64_t *k_bar = &bars[0], *q_bar = k_bar + 2, *q_free = q_bar + kQS, *s_bar = q_free + kQS, *st_bar = s_bar + 2,
           *s_free = st_bar + kStatStages, *st_free = s_free + 2, *item_free = st_free + kStatStages;
  constexpr int kBars1 = 2 + 2 * kQS + 2 + kStatStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(item_free + 2);
  __shared__ Item items[2];

  const int tid = threadIdx.x, lane = tid & 31, warp = ptx::warp_index();
  const int tok = kTile / dm.G;
  // the item of number `it`, its K tiles' pages (this lane's) and boxes, false if no row of it sees a key; the warp of the items
  auto what = [](const Seq& x) { return x.m > 0 ? x.n : 0; };
  struct Next { Item x; int id[2], boxes[2]; } nx;
  Scan seqs;
  auto find = [&](int it) {
    // A prompt's first keys are seen by most rows: the heads take turns, so that what comes last is short. (Head by head the
    // last head's first keys come late: 2.84 instead of 1.4 ms, 64/8 heads, prompts of 7 428 and 8 956 tokens.)
    Place p;
    nx.id[0] = nx.id[1] = nx.boxes[0] = nx.boxes[1] = 0;
    const int at = it / dm.Hkv;
    if (!find_block(dm, sq, kKeys, at / chunks, what, seqs, p)) {
      nx.x.b = -1;
      return true;
    }
    nx.x.b = p.b;
    nx.x.h = it % dm.Hkv;
    nx.x.s = p.s;
    nx.x.j0 = p.block * kKeys;
    nx.x.chunk = at % chunks;
    nx.x.rb0 = max(max(0, nx.x.j0 - (p.s.n - p.s.m)) / tok, nx.x.chunk * chunk_blocks);
    nx.x.blocks = (int)min((long long)((p.s.m + tok - 1) / tok), (nx.x.chunk + 1LL) * chunk_blocks) - nx.x.rb0;
    if (nx.x.blocks <= 0) return false;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
      if (nx.x.j0 + kk * kTile < p.s.n) {
        nx.id[kk] = page_of<kPaged>(dm, sq, p.b, p.s.n, nx.x.j0 + kk * kTile, box, status);
        nx.boxes[kk] = boxes_of<kPaged>(p.s, nx.x.j0 + kk * kTile, box);
      }
    return true;
  };
  // ... the next one that has rows, from item `it` on
  auto draw = [&]() {
    int it = 0;
    if ((threadIdx.x & 31) == 0) it = atomicAdd(next_item, 1);
    return __shfl_sync(0xffffffffu, it, 0);
  };
  auto find_next = [&](int it) {
    while (!find(it)) it = draw();
  };
  // the set-up's parts side by side
  if (warp == 17) {
    seqs = scan(dm, sq, 0, kKeys, what, nullptr);
    find_next(blockIdx.x);
  } else if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
  } else if (tid == 0) {
    for (int i = 0; i < kBars1; ++i) mbar_init(&bars[i], 1);
    for (int i = 0; i < 2 + kStatStages; ++i) mbar_init(&s_free[i], kKeyThreads / 32);
    // an item's place comes free when the key warps, the Q copies, the statistics and the products are done with it
    for (int i = 0; i < 2; ++i) mbar_init(&item_free[i], kKeyThreads / 32 + 3);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;  // S^T of key tile kk, buffer buf: columns [kk * 256 + buf * 128, + 128)

  if (warp == 17) {
    // =============================== items and their K (the warp) ===============================
    for (int c = 0;; ++c) {
      const int buf = c & 1;
      if (c > 0) find_next(draw());
      const Item& x = nx.x;
      if (c >= 2 && !__all_sync(0xffffffffu, mbar_wait_idle(&item_free[buf], ((c >> 1) - 1) & 1, status))) break;
      if (lane == 0) {
        items[buf] = x;
        if (x.b >= 0) mbar_expect_tx(&k_bar[buf], (nx.boxes[0] + nx.boxes[1]) * box * D * 2);  // (also says that the item is there)
        else mbar_arrive(&k_bar[buf]);
      }
      __syncwarp();
      if (x.b < 0) break;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        if (nx.boxes[kk] > 0) copy_keys<D, kPaged>(dm, &tmK, x.s, x.h, x.j0 + kk * kTile, box, nx.id[kk], Ks + (2 * buf + kk) * kTB, &k_bar[buf]);
    }
  } else if (warp == 18) {
    // =============================== copies of the Q blocks (one lane) ===============================
    if (ptx::elect_one()) {
      int qb = 0;
      for (int c = 0;; ++c) {
        if (!mbar_wait_idle(&k_bar[c & 1], (c >> 1) & 1, status)) break;
        const Item x = items[c & 1];
        if (x.b < 0) break;
        for (int rb = 0; rb < x.blocks; ++rb, ++qb) {
          const int st = qb % kQS;
          if (qb >= kQS) mbar_wait_idle(&q_free[st], (qb / kQS - 1) & 1, status);
          mbar_expect_tx(&q_bar[st], kBoxes * tok * dm.G * 128);
#pragma unroll
          for (int e = 0; e < kBoxes; ++e) tma_load_3d(Qs + st * kTB + e * kHalfBytes, &tmQ, 64 * e, x.h * dm.G, x.s.t0 + (x.rb0 + rb) * tok, &q_bar[st]);
        }
        mbar_arrive(&item_free[c & 1]);
      }
    }
  } else if (warp == 19) {
    // =============================== the rows' statistics (the warp) ===============================
    int qb = 0;
    for (int c = 0;; ++c) {
      if (!__all_sync(0xffffffffu, mbar_wait_idle(&k_bar[c & 1], (c >> 1) & 1, status))) break;
      const Item x = items[c & 1];
      if (x.b < 0) break;
      const float* src = lse2 + stat_at(dm, x.s, x.h, x.rb0 * tok * dm.G);
      const int rows = tok * dm.G;
      int left = (x.s.m - x.rb0 * tok) * dm.G;  // rows of the pair from this block on
      // (the next block's statistics are on their way while this one's wait for their place: fetched only then, a block took 3 200
      // cycles, twice what its exponentials take)
      float v[4], w[4];
      auto fetch = [&](float (&to)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = lane + 32 * e;
          to[e] = r < rows && r < left ? -src[r] : -INFINITY;
        }
        src += rows;
        left -= rows;
      };
      fetch(v);
      for (int rb = 0; rb < x.blocks; ++rb, ++qb) {
        const int ss = qb % kStatStages;
        if (rb + 1 < x.blocks) fetch(w);
        if (qb >= kStatStages) mbar_wait_idle(&st_free[ss], (qb / kStatStages - 1) & 1, status);
#pragma unroll
        for (int e = 0; e < 4; ++e) Ss[ss * kTile + lane + 32 * e] = v[e];
        __syncwarp();
        if (lane == 0) mbar_arrive(&st_bar[ss]);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = w[e];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_free[c & 1]);
    }
  } else if (warp == 16) {
    // =============================== products (one lane) ===============================
    if (ptx::elect_one()) {
      constexpr uint32_t kIdesc = instr_desc_n(false, kTile);
      int qb = 0;
      for (int c = 0;; ++c) {
        if (!mbar_wait_idle(&k_bar[c & 1], (c >> 1) & 1, status)) break;
        const int b = items[c & 1].b, blocks = items[c & 1].blocks;
        if (b < 0) break;
        const int tiles = items[c & 1].j0 + kTile < items[c & 1].s.n ? 2 : 1;
        const uint64_t kd0 = smem_desc(smem_u32(Ks + 2 * (c & 1) * kTB), 16, 1024);
        for (int rb = 0; rb < blocks; ++rb, ++qb) {
          const int buf = qb & 1, st = qb % kQS;
          mbar_wait_idle(&q_bar[st], (qb / kQS) & 1, status);
          if (qb >= 2) mbar_wait_idle(&s_free[buf], ((qb - 2) >> 1) & 1, status);
          tc_fence_after();
          const uint64_t qd0 = smem_desc(smem_u32(Qs + st * kTB), 16, 1024);
          for (int kk = 0; kk < tiles; ++kk) {
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks)
              umma(tmem + kk * 256 + buf * 128, kd0 + (uint64_t)((kk * kTB) >> 4) + k_major_step(ks), qd0 + k_major_step(ks), kIdesc, ks > 0);
          }
          umma_commit(&q_free[st]);
          if (rb + 1 == blocks) umma_commit(&item_free[c & 1]);
          umma_commit(&s_bar[buf]);
        }
      }
      // (no arrival may still be on its way to this CTA's barriers when the CTA ends)
      if (qb > 0) mbar_wait_idle(&q_free[(qb - 1) % kQS], ((qb - 1) / kQS) & 1, status);
    }
  } else {
    // =============================== two threads per key ===============================
    const float scale2 = dm.scale * kLog2e;
    const int kk = (warp >> 2) & 1, rh = warp >> 3, key = tid & (kKeys - 1);
    const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16) + kk * 256 + rh * 64;
    auto all_of_pair = [&](bool x) {
      uint32_t r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.u32 q, %1, 0;\n\t"
          "bar.red.and.pred p, %2, 64, q;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(r) : "r"((uint32_t)x), "r"(1 + (warp & 7)) : "memory");
      return r != 0;
    };
    int qb = 0;
    for (int c = 0;; ++c) {
      // (the two warps that share 32 keys, which meet below, go on together or not at all)
      if (!all_of_pair(mbar_wait(&k_bar[c & 1], (c >> 1) & 1, status))) break;
      const Item x = items[c & 1];
      if (x.b < 0) break;
      const int j = x.j0 + key, first = x.s.n - x.s.m;
      const int need = max(j - first, 0) * dm.G;  // the first of the pair's rows that sees the key (of older keys far less than 0 otherwise)
      // where the sum goes, and what is there already: fetched now, used at the end
      float* out = nullptr;
      float total = 0.f, low = 0.f;  // the sum over row blocks, and what its additions lost
      float before = 0.f;
      if (rh == 0 && j < x.s.n) {
        if (kPaged) {
          out = pool_weight(dm, sq, x.b, x.h, j, mass, status);
          if (out) before = *out;
        } else {
          out = mass + ((size_t)x.chunk * dm.T + x.s.t0 + j) * dm.Hkv + x.h;
        }
      }
      for (int rb = 0; rb < x.blocks; ++rb, ++qb) {
        const int buf = qb & 1, ss = qb % kStatStages, i0 = (x.rb0 + rb) * tok;
        // rows of the half block that see the key; masked: not all 64 of them for all keys of the item
        const int lo = need - i0 * dm.G - rh * 64, hi = min(tok, x.s.m - i0) * dm.G - rh * 64;
        const bool masked = i0 < x.j0 + kKeys - 1 - first || hi < 64;
        mbar_wait(&s_bar[buf], (qb >> 1) & 1, status);
        mbar_wait(&st_bar[ss], (qb / kStatStages) & 1, status);
        tc_fence_after();
        float2 acc[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        uint32_t va[16], vb[16];
        float4 sa[4], sb[4];
        const float* stat = Ss + ss * kTile + rh * 64;
        const uint32_t t_s = t_lane + buf * 128;
        if (!masked) {
          // two register sets take turns: the next 16 rows' logits and statistics are on their way while these are summed
          tmem_ld16_issue(t_s, va);
          lds16_issue(stat, sa);
          tmem_ld16_wait(va);
          tmem_ld16_issue(t_s + 16, vb);
          lds16_issue(stat + 16, sb);
          add_weights<false>(va, sa, scale2, 0, 0, acc);
          tmem_ld16_wait(vb);
          tmem_ld16_issue(t_s + 32, va);
          lds16_issue(stat + 32, sa);
          add_weights<false>(vb, sb, scale2, 0, 0, acc);
          tmem_ld16_wait(va);
          tmem_ld16_issue(t_s + 48, vb);
          lds16_issue(stat + 48, sb);
          add_weights<false>(va, sa, scale2, 0, 0, acc);
          tmem_ld16_wait(vb);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s_free[buf]);
          add_weights<false>(vb, sb, scale2, 0, 0, acc);
        } else {
#pragma unroll 1
          for (int e = 0; e < 64 && e < hi; e += 16) {  // (a block of few rows is mostly padding)
            tmem_ld16_issue(t_s + e, va);
            lds16_issue(stat + e, sa);
            tmem_ld16_wait(va);
            add_weights<true>(va, sa, scale2, lo - e, hi - e, acc);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&s_free[buf]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&st_free[ss]);
        const float y = ((acc[0].x + acc[0].y) + (acc[1].x + acc[1].y)) - low;
        const float t = total + y;
        low = (t - total) - y;
        total = t;
      }
      // the two warps that share 32 keys meet (two places in turn: a warp is at most one item ahead of its partner)
      if (rh == 1) half[(c & 1) * kKeys + key] = total;
      asm volatile("bar.sync %0, 64;" ::"r"(1 + (warp & 7)) : "memory");
      if (out) *out = before + (total + half[(c & 1) * kKeys + key]);
      if (lane == 0) mbar_arrive(&item_free[c & 1]);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// Prompts: mass = the sum over the chunks whose rows see the token. grid = ceil(T * Hkv / 256).
__global__ void __launch_bounds__(256)
sum_kernel(PDims dm, Seqs sq, const float* __restrict__ part, int chunk_blocks, float* __restrict__ mass) {
  ptx::pdl_wait();
  ptx::pdl_trigger();
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= (long long)dm.T * dm.Hkv) return;
  const int t = (int)(i / dm.Hkv), tok = kTile / dm.G;
  int lo = 0, hi = dm.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(sq.cu + mid) <= t) lo = mid; else hi = mid;
  }
  const Seq s = sequence(dm, sq, lo);
  if (t < s.t0 || t >= s.t0 + s.m) return;
  const int first = (t - s.t0) / kKeys * kKeys / tok / chunk_blocks, last = ((s.m + tok - 1) / tok - 1) / chunk_blocks;
  float sum = 0.f;
#pragma unroll 4
  for (int c = first; c <= last; ++c) sum += part[(size_t)c * dm.T * dm.Hkv + i];
  mass[i] = sum;
}

}  // namespace tcore
}  // namespace paged
}  // namespace caote
