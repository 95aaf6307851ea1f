// What the kernels of the paged cache and of packed prompts share: where a sequence's rows and tokens lie.
//
// New tokens are packed: those of sequence b are rows cu[b] .. cu[b + 1] of q, k_new, v_new, o and lse. Query rows of a
// (sequence, KV head) pair are numbered r = i * G + g (token i, head g of the group), so that a block of rows is a block of
// tokens with all heads of the group and every key tile is read once for all of them.
//
// A cached token, slot j of sequence b, lies in page table[b, j / page] at row j % page. Pools are [pages, Hkv, page, d] (K,
// V) and [pages, Hkv, page] (mass, pos): the tokens of a page and a head lie side by side.
#pragma once

#include "common.cuh"

namespace caote {
namespace paged {

struct PDims {
  int B, Hq, Hkv, G, D;
  int page_shift, n_pages, max_pages;  // pages of 2^page_shift tokens; prompts: no pages (max_pages 0)
  int T, max_new;                      // new tokens of all sequences, most of one sequence
  float scale;
  long long q_stride, kv_stride;  // elements from one packed token to the next
};

// Row numbers of a pair divided by G, by a multiplication: exact below 2^28, as many as a call may have.
struct GroupDiv {
  unsigned magic;
  int g;
  __device__ explicit GroupDiv(int g_) : magic(0xffffffffu / (unsigned)g_ + 1u), g(g_) {}
  __device__ __forceinline__ int operator()(int r) const { return g == 1 ? r : (int)__umulhi((unsigned)r, magic); }
};

// Where the sequences begin, how long they are.
struct Seqs {
  const int* cu;
  const int* len;    // null: prompts, as long as they have new tokens
  const int* table;  // null: prompts
};

struct Seq {
  int t0, m, n;  // first packed row, new tokens, all tokens; m = 0: nothing to do for this sequence
};

// A sequence whose numbers do not fit together is left alone (m = 0); `status` (one caller per sequence) gets the code.
__device__ __forceinline__ Seq sequence(const PDims& dm, const Seqs& sq, int b, int* status = nullptr) {
  Seq s;
  const int t1 = sq.cu[b + 1];
  s.t0 = sq.cu[b];
  s.m = t1 - s.t0;
  s.n = sq.len ? sq.len[b] : s.m;
  if (s.t0 < 0 || t1 < s.t0 || t1 > dm.T || s.m > dm.max_new ||
      (s.m > 0 && sq.len && (s.n < s.m || s.n > (long long)dm.max_pages << dm.page_shift))) {
    if (status) set_status(status, CAOTE_ERR_BAD_LENGTH);
    s.m = 0;
  }
  return s;
}

// Where the statistic of query row r of a pair lies in the workspace: [Hkv][T][G], so that a block of rows is contiguous.
__device__ __forceinline__ size_t stat_at(const PDims& dm, const Seq& s, int h, int r) { return ((size_t)h * dm.T + s.t0) * dm.G + r; }

// Work is numbered over all sequences: a sequence has ceil(what / per) blocks of it, what = its new tokens or its keys. A scan holds
// one sequence per lane (32 at a time); for one whole warp. Sums stop at kMostBlocks: sequences that overlap (cu does not ascend) may have
// any number of blocks together, those of a sound call have less. Which block of its sequence an index is stays in range all the same.
constexpr unsigned kMostBlocks = 0x7fff0000u;
__device__ __forceinline__ int add_blocks(int a, int b) { return (int)min((unsigned)a + (unsigned)b, kMostBlocks); }
struct Scan {
  Seq s;           // this lane's sequence
  int mine, incl;  // its blocks, and those of all lanes up to it
  int total;       // blocks of these 32 sequences
};
template <typename What>
__device__ __forceinline__ Scan scan(const PDims& dm, const Seqs& sq, int b0, int per, What what, int* status) {
  const int lane = threadIdx.x & 31;
  Scan c;
  c.s.t0 = c.s.m = c.s.n = 0;
  if (b0 + lane < dm.B) c.s = sequence(dm, sq, b0 + lane, status);
  c.mine = (what(c.s) + per - 1) / per;
  c.incl = c.mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, c.incl, o);
    if (lane >= o) c.incl = add_blocks(c.incl, t);
  }
  c.total = __shfl_sync(0xffffffffu, c.incl, 31);
  return c;
}
// All blocks; `c` holds the first 32 sequences' scan afterwards.
template <typename What>
__device__ __forceinline__ int count_blocks(const PDims& dm, const Seqs& sq, int per, What what, int* status, Scan& c) {
  c = scan(dm, sq, 0, per, what, status);
  int total = c.total;
  for (int b0 = 32; b0 < dm.B; b0 += 32) total = add_blocks(total, scan(dm, sq, b0, per, what, status).total);
  return total;
}
// The sequence that block `index` belongs to, and its number in there, from the first scan on; false: no such block. The same
// result in all lanes.
struct Place {
  int b, block, blocks;  // blocks: of the sequence
  Seq s;
};
template <typename What>
__device__ __forceinline__ bool find_block(const PDims& dm, const Seqs& sq, int per, int index, What what, Scan c, Place& p) {
  for (int b0 = 0;;) {
    const unsigned reach = __ballot_sync(0xffffffffu, index < c.incl);
    if (reach) {
      const int f = __ffs((int)reach) - 1;
      p.b = b0 + f;
      p.blocks = __shfl_sync(0xffffffffu, c.mine, f);
      p.block = index - (__shfl_sync(0xffffffffu, c.incl, f) - p.blocks);
      p.s.t0 = __shfl_sync(0xffffffffu, c.s.t0, f);
      p.s.m = __shfl_sync(0xffffffffu, c.s.m, f);
      p.s.n = __shfl_sync(0xffffffffu, c.s.n, f);
      return true;
    }
    index -= c.total;
    b0 += 32;
    if (b0 >= dm.B) return false;
    c = scan(dm, sq, b0, per, what, nullptr);
  }
}

// Row of the pools' [pages * Hkv * page] rows that holds slot j of sequence b for KV head h. A page outside the pool is
// recorded and read as page 0: its sequence's results mean nothing then, but nothing is read out of bounds.
__device__ __forceinline__ size_t pool_row(const PDims& dm, const Seqs& sq, int b, int h, int j, int* status) {
  int page = __ldg(sq.table + (size_t)b * dm.max_pages + (j >> dm.page_shift));
  if ((unsigned)page >= (unsigned)dm.n_pages) {
    set_status(status, CAOTE_ERR_BAD_PAGE);
    page = 0;
  }
  return (((size_t)page * dm.Hkv + h) << dm.page_shift) + (j & ((1 << dm.page_shift) - 1));
}

// Where the weight of that token is kept, to be written: null where the page lies outside the pool (page 0 is another sequence's).
__device__ __forceinline__ float* pool_weight(const PDims& dm, const Seqs& sq, int b, int h, int j, float* mass, int* status) {
  const int page = __ldg(sq.table + (size_t)b * dm.max_pages + (j >> dm.page_shift));
  if ((unsigned)page >= (unsigned)dm.n_pages) {
    set_status(status, CAOTE_ERR_BAD_PAGE);
    return nullptr;
  }
  return mass + ((((size_t)page * dm.Hkv + h) << dm.page_shift) + (j & ((1 << dm.page_shift) - 1)));
}

// Splits of a sequence's key tiles (device and combine kernel agree on it): `per` tiles each, `count` of them.
__device__ __forceinline__ void key_splits(int tiles, int most, int least_tiles, int& per, int& count) {
  int ns = tiles / least_tiles;
  ns = ns < 1 ? 1 : (ns > most ? most : ns);
  per = (tiles + ns - 1) / ns;
  count = (tiles + per - 1) / per;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

}  // namespace paged
}  // namespace caote
