// Attention over the paged 8-bit K/V cache for groups of requests whose sequences begin
// with the same pages (daf_cache_attn_shared).
//
// exp(s - m) sums over disjoint sets of keys join by their maxima, so a row's keys fall in
// two: the pages that are its group's, which every row of the group takes together from one
// copy of them in LDS, and the rest of its own sequence. One launch has both kinds of work:
//  * of a group's pages: row blocks of all its requests' (row, head) pairs by the kernel for
//    many rows of daf_cache_attn, split over the pages;
//  * of the rest: the line of daf_cache_attn's few rows, from the first page that is not
//    the group's on.
// A second launch joins a row's partial results. Weights have the bits that daf_cache_attn
// gives them: where it takes its few rows' kernel the groups' pages have two bf16 terms too (32
// decode rows over 32768 shared keys 42.5 us a call, with one fp16 term 36.1), else one fp16
// term (8 requests' 301 question rows 167 us, with two bf16 terms 219; daf_cache_attn 188).
//
// Question rows are bound by the issue of the many rows' kernel (its comment): 301 of 28 heads on
// 4 of 128 over 32768 shared keys 157 + 13.4 us (141 GFLOP, 0.90 PFLOP/s; by daf_cache_attn 188;
// fp32 473, by daf_cache_attn 412). Decode rows fill no device by themselves: 32 over 32768 shared
// keys and up to 700 of their own 39.4 + 6.2 us (one copy of the pages, 33.5 MB, is 7 us of HBM;
// by daf_cache_attn, a copy for each from the caches, 111; fp32 73 and 132), in 256 workgroups of
// 16 pages and a wave per SIMD, whose matrix and vector instructions take 75% of its cycles: the
// rest is waiting, for its own chain and at barriers. A page takes such a workgroup 2.0 us, with
// one fp16 term 1.5, one of two on a CU 2.5; ahead of its pages are 6 us of launch, page ids, scales
// and first copies. (Row blocks of 256 pairs, 64 rows a wave, 502 registers, one workgroup per CU,
// at their best splits, all with one fp16 term: 48 us for 36 and 254 for 167.)
#include <algorithm>

#include "cache_attn.h"

namespace daf {
namespace {

// The rows of a group over its first pages. A row's limit follows from its own sequence's
// length; rows at the end of sequences past those pages, as a decode step has them, see all.
template <int MT>
struct GroupRows {
  static constexpr bool kKnown = true;
  const SharedLaunch &p;
  Request &r;     // of all the group's rows
  int b0, n_req;  // the group's requests
  int pages;      // its pages
  int *cu, *len;  // LDS, for requests of different rows: first rows from the group's on and tokens
  int mine[4];    // else tokens of its requests: of lane, 64 + lane, ..; or of thread
  __device__ __forceinline__ int sequence(int i) const { return p.seq ? p.seq[b0 + i] : b0 + i; }
  __device__ __forceinline__ int tokens_of(int seq) const {
    return min(seq_len(p.c.len, p.c.n_seqs, p.c.max_seq_pages, seq), p.max_len);
  }
  __device__ __forceinline__ int tokens(int i) const { return tokens_of(sequence(i)); }
  // The group's pages are in the tables of its sequences that reach their end. At first they
  // are taken from the first sequence that is in range (batches are padded), which needs no
  // length; where that one is shorter (as a freed slot of the batch), from the first that is not, or
  // the longest.
  __device__ __forceinline__ void take_pages(int seq) {
    r.pages = p.c.table + (int64_t)seq * p.c.max_seq_pages;
    r.L = tokens_of(seq);
  }
  __device__ __forceinline__ bool other_pages() {
    if (r.L >= pages * kPage || n_req == 1) return false;
    const int lane = threadIdx.x & 63;
    int longest = -1, at = 0;
    for (int i = 0; i < n_req && longest < pages * kPage; i += 64) {
      const int seq = sequence(min(i + lane, n_req - 1)), n = min(tokens_of(seq), pages * kPage);
      int top = n;
#pragma unroll
      for (int m = 32; m; m >>= 1) top = max(top, __shfl_xor(top, m));
      if (top > longest) {
        longest = __builtin_amdgcn_readfirstlane(top);
        at = __builtin_amdgcn_readlane(seq, __builtin_ctzll(__ballot(n == top)));
      }
    }
    if (longest <= r.L) return false;  // the first is the longest
    take_pages(at);
    return true;
  }
  // loads, and what waits for them
  __device__ __forceinline__ void start() {
    if (!p.per_req) {
      mine[0] = (int)threadIdx.x < n_req ? tokens(threadIdx.x) : 0;
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j * 64 < n_req) mine[j] = tokens(min(j * 64 + (int)(threadIdx.x & 63), n_req - 1));
  }
  __device__ __forceinline__ void prepare() {
    if (p.per_req) return;
    const int i = threadIdx.x;
    if (i < n_req) cu[i] = p.cu[b0 + i] - r.row0, len[i] = mine[0];
    if (i == 0) cu[n_req] = p.cu[b0 + n_req] - r.row0;
    __syncthreads();
  }
  __device__ __forceinline__ bool exact() const { return p.exact; }
  __device__ __forceinline__ bool empty() const { return false; }
  __device__ __forceinline__ int seen() const { return pages; }
  __device__ __forceinline__ int limit(int row) const {
    int L, next;  // tokens of the row's sequence, and the row after its request's last
    if (p.per_req) {
      const int b = row / p.per_req;
      next = (b + 1) * p.per_req;
      L = __shfl(mine[0], b & 63);
#pragma unroll
      for (int j = 1; j < 4; ++j)
        if (j * 64 < n_req) {
          const int y = __shfl(mine[j], b & 63);
          L = b >> 6 == j ? y : L;
        }
    } else {
      int b = 0;
      for (int step = kMaxCacheReqs / 2; step; step >>= 1)
        if (b + step < n_req && cu[b + step] <= row) b += step;
      L = len[b];
      next = cu[b + 1];
    }
    const int at = p.pos ? min(p.pos[r.row0 + row], L - 1) : L - next + row;
    return max(-1, min(at, pages * kPage - 1));
  }
};

// A group, its requests and its first workgroup
struct Group {
  int b0, b1, wg0;
};
// The last group whose `from` is at most x, one x for each STEP lanes. All that is asked of the
// groups comes in one trip to the arguments, 64 groups at a time.
template <int STEP, typename F>
__device__ __forceinline__ Group find_group(const SharedLaunch &p, int x, F from) {
  Group gr{0, p.n_req, 0};
  const int lane = threadIdx.x & 63;
  for (int i = 0; i < p.n_groups; i += 64) {
    const int g = min(i + lane, p.n_groups - 1);
    const int b0 = p.first[g], b1 = g + 1 < p.n_groups ? p.first[g + 1] : p.n_req, wg0 = p.wg0[g];
    const int at = from(b0, wg0);
    int n = 0;  // groups of these that begin by x
#pragma unroll
    for (int k = 0; k < 64; k += STEP) {
      const int y = __builtin_popcountll(__ballot(i + lane < p.n_groups && at <= __builtin_amdgcn_readlane(x, k)));
      if (lane / STEP == k / STEP) n = y;
    }
    const Group y{__shfl(b0, max(n - 1, 0)), __shfl(b1, max(n - 1, 0)), __shfl(wg0, max(n - 1, 0))};
    if (n > 0) gr = y;
  }
  return gr;
}

// The workgroups of a group's units, (split, head) pairs, and of their row blocks. The row
// blocks of a unit read the same pages: neighbours on one XCD, the units on the XCDs in
// turn; the last units, fewer than XCDs, on all of them.
struct UnitBlock {
  int unit, block;
};
__device__ __forceinline__ UnitBlock unit_block(int wg, int units, int blocks) {
  const int even = units / kXcdCount * kXcdCount, at = wg / kXcdCount;
  if (wg < even * blocks) return {at / blocks * kXcdCount + wg % kXcdCount, at % blocks};
  return {wg / blocks, wg % blocks};
}
__device__ __forceinline__ int workgroup_of(UnitBlock u, int units, int blocks) {
  const int even = units / kXcdCount * kXcdCount;
  if (u.unit < even) return (u.unit / kXcdCount * blocks + u.block) * kXcdCount + u.unit % kXcdCount;
  return u.unit * blocks + u.block;
}

template <bool BF16, int D, int MT>
union SharedMemory {
  struct {
    unsigned char lds[kStages * Wide<BF16, D, MT>::PAGE_BYTES];
    int cu[kMaxCacheReqs + 1], len[kMaxCacheReqs];
  } wide;
  FewShared<D> few;
};

template <bool BF16, int D, int MT>
__device__ __forceinline__ void group_job(const SharedLaunch &p, SharedMemory<BF16, D, MT> &sh) {
  using W = Wide<BF16, D, MT>;
  constexpr int PAIRS = kWaves * 16 * MT;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n16 = lane & 15, quad = lane >> 4;
  Group gr{0, p.n_req, 0};
  if (p.n_groups > 1) {
    gr = find_group<64>(p, blockIdx.x, [](int, int wg0) { return wg0; });
    gr = {__builtin_amdgcn_readfirstlane(gr.b0), __builtin_amdgcn_readfirstlane(gr.b1),
          __builtin_amdgcn_readfirstlane(gr.wg0)};
  }
  Request r;
  r.b = gr.b0;
  r.row0 = p.row_of(gr.b0);
  r.n = p.row_of(gr.b1) - r.row0;
  const int total = r.n * p.group, blocks = (total + PAIRS - 1) / PAIRS, pages = p.first_page(gr.b0);
  const UnitBlock ub = unit_block(blockIdx.x - gr.wg0, (pages + p.split_pages - 1) / p.split_pages * p.c.hkv, blocks);
  const int h = ub.unit % p.c.hkv, pg0 = ub.unit / p.c.hkv * p.split_pages;
  r.block = ub.block;
  int seq = 0;  // the first one in range
  bool there = false;
  for (int b = gr.b0; b < gr.b1 && !there; b += 64) {
    const int at = min(b + lane, gr.b1 - 1), mine = p.seq ? p.seq[at] : at;
    const unsigned long long in = __ballot((unsigned)mine < (unsigned)p.c.n_seqs);
    there = in != 0;
    if (there) seq = __builtin_amdgcn_readlane(mine, __builtin_ctzll(in));
  }
  GroupRows<MT> rows{p, r, gr.b0, gr.b1 - gr.b0, there ? pages : 0, sh.wide.cu, sh.wide.len, {}};
  rows.take_pages(seq);
  rows.start();
  W w;
  float unit;
  wide_rows<BF16, D, MT>(p, sh.wide.lds, r, h, pg0, min(p.split_pages, pages - pg0), rows, w, unit);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float l = row_sum(w.l[mt]), inv = over(l);
    const float lse = l == 0.f ? -INFINITY : (w.m[mt] + log2f(l)) * kLn2;
    const size_t place = (size_t)blockIdx.x * PAIRS + (wave * MT + mt) * 16 + n16;
    if (quad == 0) p.part_lse[place] = lse;
#pragma unroll
    for (int db = 0; db < W::DB; ++db)
      *reinterpret_cast<f32x4 *>(p.part_o + place * D + db * 16 + quad * 4) = w.o[mt][db] * inv * unit;
  }
}

template <bool BF16, int D, int MT>
__global__ __launch_bounds__(kThreads, (BF16 || D == 64 ? 2 : 1)) void cache_shared_kernel(const SharedLaunch p) {
  __shared__ __align__(16) SharedMemory<BF16, D, MT> sh;
  if ((int)blockIdx.x < p.first_wgs) {
    group_job<BF16, D, MT>(p, sh);
  } else {
    const int job = blockIdx.x - p.first_wgs;
    line_job<BF16, D>(p, sh.few, job % p.c.hkv, job / p.c.hkv);
  }
}

// Join a (row, head)'s partial results, o = sum_s e^(lse_s - lse) o_s: those of its group's
// pages, then those of the line. A workgroup's groups of D / 4 lanes take a pair each, or
// TEAM of them one: its results in turn, FLIGHT at a time, their sums joined through LDS.
template <bool BF16, int D, int TEAM>
__global__ __launch_bounds__(kThreads) void cache_shared_join_kernel(const SharedLaunch p) {
  constexpr int LP = D / 4, GROUPS = kThreads / LP, FLIGHT = 4;
  __shared__ f32x4 sh_o[GROUPS][LP];
  __shared__ float sh_m[GROUPS], sh_l[GROUPS];
  const int t = threadIdx.x, lanes = t / LP, g = lanes % TEAM, c = t % LP, lane = t & 63;
  const int64_t job = (int64_t)blockIdx.x * (GROUPS / TEAM) + lanes / TEAM;
  const bool mine = job < (int64_t)p.rows * p.hq;
  const int row = mine ? (int)(job / p.hq) : p.rows - 1, head = mine ? (int)(job % p.hq) : 0;
  // the wave's pairs one after the other: searches by all lanes
  int b = p.per_req ? row / p.per_req : 0;
  constexpr int STEP = TEAM == GROUPS ? 64 : LP;  // lanes of one pair
  if (!p.per_req) {
#pragma unroll
    for (int k = 0; k < 64; k += STEP) {
      const int at = find_in(p.cu, p.n_req, __builtin_amdgcn_readlane(row, k));
      if (lane / STEP == k / STEP) b = at;
    }
  }
  Group gr{0, p.n_req, 0};
  if (p.n_groups > 1) gr = find_group<STEP>(p, b, [](int b0, int) { return b0; });
  const int h = head / p.group, in_head = head % p.group;
  // the line: piece s of n_line, the first one's place is its workgroup's second
  const int pair = (row - p.row_of(b)) * p.group + in_head;
  int k0 = 0, n_line = 1;
  if (!p.whole) {
    const int piece = p.line[2 * kMaxCacheReqs], units = p.line[kMaxCacheReqs + b];
    const int from = p.line[b] + pair / kRows * units;
    k0 = from / piece;
    n_line = (from + units - 1) / piece - k0 + 1;
  }
  // the group's pages
  const int row0 = p.row_of(gr.b0);
  const int in_group = (row - row0) * p.group + in_head;
  const int blocks = ((p.row_of(gr.b1) - row0) * p.group + p.block_rows - 1) / p.block_rows;
  const int n_first = (p.first_page(gr.b0) + p.split_pages - 1) / p.split_pages, n = n_first + n_line;
  auto at = [&](int s) {
    if (s < n_first) {
      const int wg = gr.wg0 + workgroup_of({s * p.c.hkv + h, in_group / p.block_rows}, n_first * p.c.hkv, blocks);
      return wg * p.block_rows + in_group % p.block_rows;
    }
    s -= n_first;
    return n_line == 1 ? p.whole_pair(h) + row * p.group + in_head : p.edge_place(h, k0 + s, s == 0) + pair % kRows;
  };
  float m = -INFINITY, l = 0.f;
  f32x4 x = {};
  for (int s0 = g; s0 < n; s0 += FLIGHT * TEAM) {
    float lse[FLIGHT];
    f32x4 y[FLIGHT];
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) {
      const int s = s0 + j * TEAM;
      const size_t place = at(min(s, n - 1));
      lse[j] = s < n ? p.part_lse[place] : -INFINITY;
      y[j] = s < n ? *reinterpret_cast<const f32x4 *>(p.part_o + place * D + c * 4) : f32x4{};
    }
    float to = m;
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) to = fmaxf(to, lse[j]);
    const float ref = to == -INFINITY ? 0.f : to;  // a row that sees no key there, or NaN
    const float a = __expf(m - ref);
    m = to;
    l *= a;
    x *= a;
#pragma unroll
    for (int j = 0; j < FLIGHT; ++j) {
      const float w = __expf(lse[j] - ref);
      l += w;
      x += w * y[j];
    }
  }
  if constexpr (TEAM > 1) {
    sh_o[lanes][c] = x;
    if (c == 0) sh_m[lanes] = m, sh_l[lanes] = l;
    __syncthreads();
    if (g) return;
    for (int k = 1; k < TEAM; ++k) m = fmaxf(m, sh_m[lanes + k]);
    const float ref = m == -INFINITY ? 0.f : m;
    l = 0.f;
    x = f32x4{};
    for (int k = 0; k < TEAM; ++k) {
      const float w = __expf(sh_m[lanes + k] - ref);
      l += w * sh_l[lanes + k];
      x += w * sh_o[lanes + k][c];
    }
  }
  if (!mine) return;
  const float inv = over(l);
  const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
  store_out<BF16>(p, row, head, c * 4, y, D);
  if (c == 0 && p.lse) p.lse[(size_t)head * p.lse_stride + row] = l == 0.f ? -INFINITY : m + __logf(l);
}

// A join of few pairs gives each a workgroup; one of many, which fill the device by
// themselves, helps a group of lanes where it would have more than 8 results to take (301
// question rows of 28 heads of 128, 12 results each, us of the join: teams of 2 13.9, of 8 19.0;
// 4 rows, 7 each: of 1 4.5, of 8 4.0).
constexpr int kJoinTurns = 8, kJoinPairs = 4096;

template <bool BF16, int D, int MT>
hipError_t launch(const SharedLaunch &p, hipStream_t st) {
  cache_shared_kernel<BF16, D, MT><<<p.first_wgs + p.n_splits * p.c.hkv, kThreads, 0, st>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  int most = 1;  // partial results of a row
  for (int g = 0; g < p.n_groups; ++g) most = std::max(most, (p.pages[p.first[g]] + p.split_pages - 1) / p.split_pages + 1);
  if (!p.whole) most += p.n_splits / 4;  // of the line's workgroups few have a part of one row
  const int64_t pairs = (int64_t)p.rows * p.hq;
  auto join = [&](auto kern, int team) {
    const int per_wg = kThreads / (D / 4) / team;
    kern<<<(unsigned)((pairs + per_wg - 1) / per_wg), kThreads, 0, st>>>(p);
  };
  constexpr int ALL = kThreads / (D / 4);
  if (pairs < kJoinPairs || most > 4 * kJoinTurns) join(cache_shared_join_kernel<BF16, D, ALL>, ALL);
  else if (most > 2 * kJoinTurns) join(cache_shared_join_kernel<BF16, D, 4>, 4);
  else if (most > kJoinTurns) join(cache_shared_join_kernel<BF16, D, 2>, 2);
  else join(cache_shared_join_kernel<BF16, D, 1>, 1);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_shared(bool bf16, const SharedLaunch &p, hipStream_t st) {
  const bool two = p.block_rows == 128;
  if (p.c.d == 128)
    return !bf16 ? launch<false, 128, 1>(p, st) : two ? launch<true, 128, 2>(p, st) : launch<true, 128, 1>(p, st);
  return !bf16 ? launch<false, 64, 1>(p, st) : two ? launch<true, 64, 2>(p, st) : launch<true, 64, 1>(p, st);
}

}  // namespace daf
