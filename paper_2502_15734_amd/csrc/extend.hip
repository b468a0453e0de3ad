// cc_extend_segments: segment table, page table and the rows' positions and slots of tokens that come behind what the pages hold.
//
// Per segment old tokens are held and add come behind them; pages(x) = ceil(x / 16).  A request's need is
// sum(pages(old + add) - pages(old)) pages and sum(add) rows.  Who is served is decided by one exclusive scan of the needs in
// request order; the places of what is served (rows, pages of the free list, token offsets) come from a second one.
//
// Bound by latency: a step of some hundred answers reads and writes some ten kilobytes, and a launch costs more than that.  So batches
// whose tables fit a workgroup's LDS are one launch of one workgroup (extend_small_kernel); others are a launch for the needs, one that
// places the segments (every workgroup scans all needs again, which is cheaper than a launch between) and one for the rows.
// 32 requests of one row each (5 to 10 segments) 7.7 us, where a launch alone takes 2.4; 250 requests, some with a question, 13.9; the tables of 500 whole
// prompts, 2.8 million rows, 22 us (1.6 TB/s, of which a third is the chain through the two kernels in front).
#include <algorithm>

#include "device_util.h"

namespace cc {

namespace {

struct ExtendArgs {
  const cc_segment* segs_in;
  const int32_t *n_new, *tab_cap, *req_seg_off, *free_blocks;
  int32_t* block_tab;
  int n_segs, n_requests, n_free, n_tab, n_blocks, max_rows;
  cc_segment* segs;
  int32_t *cu_q, *q_pos, *slot_map, *row_req, *last_row, *status, *counts;
  bool aligned_rows;        // q_pos, slot_map and row_req at addresses of 16 bytes
};

struct Need {             // of a request; status: one of CC_EXTEND_*
  int pages, rows, status, old_tokens;
};
struct Place {            // where a request's share begins
  int page, row, token, served;
};

__device__ __forceinline__ int pages_of(unsigned tokens) { return static_cast<int>((tokens + (kBlock - 1)) / kBlock); }
// (lengths are not negative here; the sum of two may be beyond int, and is then refused)
__device__ __forceinline__ int new_pages(int old, int add) { return pages_of(static_cast<unsigned>(old) + static_cast<unsigned>(add)) - pages_of(old); }

// sums over the lanes of a group of 16
__device__ __forceinline__ long long sum16(long long v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o, 16);
  return v;
}
__device__ __forceinline__ int before16(int v) {          // sum of the lanes in front
  const int lane = threadIdx.x & 15;
  int in = v;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    const int up = __shfl_up(in, o, 16);
    if (lane >= o) in += up;
  }
  return in - v;
}

__device__ __forceinline__ bool segment_full(const ExtendArgs& a, int old, int add, int off, int cap) {
  const long long after = (static_cast<long long>(old) + add + kBlock - 1) / kBlock;
  return add > 0 && (off < 0 || after > cap || off + after > a.n_tab);
}

// A request's need, by 16 lanes with a segment each.
__global__ __launch_bounds__(256) void extend_need_kernel(ExtendArgs a, Need* __restrict__ need) {
  const int r = blockIdx.x * 16 + (threadIdx.x >> 4), lane = threadIdx.x & 15;
  if (r >= a.n_requests) return;
  const int s0 = max(a.req_seg_off[r], 0), s1 = min(a.req_seg_off[r + 1], a.n_segs);
  long long rows = 0, pages = 0, tokens = 0;
  int first_grown = 0x7fffffff, last_held = -1;
  bool full = false;
  for (int s = s0 + lane; s < s1; s += 16) {
    const int old = max(a.segs_in[s].n_tokens, 0), add = max(a.n_new[s], 0);
    full |= segment_full(a, old, add, a.segs_in[s].tab_off, a.tab_cap[s]);
    if (add > 0) first_grown = min(first_grown, s);
    if (old > 0) last_held = s;
    pages += (static_cast<long long>(old) + add + kBlock - 1) / kBlock - pages_of(old);
    rows += add;
    tokens += old;
  }
  rows = sum16(rows);
  pages = sum16(pages);
  tokens = sum16(tokens);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    first_grown = min(first_grown, __shfl_xor(first_grown, o, 16));
    last_held = max(last_held, __shfl_xor(last_held, o, 16));
    full |= __shfl_xor(static_cast<int>(full), o, 16) != 0;
  }
  if (lane != 0) return;
  int status = first_grown < last_held ? CC_EXTEND_ORDER : CC_EXTEND_OK;
  if (full || rows + tokens > 0x7fffffffll) status = CC_EXTEND_TABLE_FULL;
  if (status != CC_EXTEND_OK) rows = pages = 0;
  need[r] = Need{static_cast<int>(pages), static_cast<int>(rows), status, static_cast<int>(tokens)};
}

// Sums of what is wanted stop at 2^32 - 1 (beyond any limit).
__device__ __forceinline__ unsigned add_up(unsigned x, unsigned y) { return __builtin_elementwise_add_sat(x, y); }

// Inclusive scan over the workgroup's 64 W threads, of N sums at once.  STOP: sums stop at 2^32 - 1, otherwise they are mod 2^32.
template <bool STOP, int N, int W>
__device__ __forceinline__ void block_scan(unsigned (&v)[N], unsigned (*part)[N], unsigned (&all)[N]) {      // all: the totals
  auto add = [](unsigned x, unsigned y) { return STOP ? add_up(x, y) : x + y; };
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned up = __shfl_up(v[i], o, 64);
      if (lane >= o) v[i] = add(v[i], up);
    }
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < N; ++i) part[wave][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {                        // (lane w of each wavefront takes the sum of wavefront w)
    unsigned sum = lane < W ? part[lane][i] : 0u;
#pragma unroll
    for (int o = 1; o < W; o <<= 1) {
      const unsigned up = __shfl_up(sum, o, 64);
      if (lane >= o) sum = add(sum, up);
    }
    all[i] = __builtin_amdgcn_readlane(sum, W - 1);
    if (wave > 0) v[i] = add(v[i], __builtin_amdgcn_readlane(sum, max(wave - 1, 0)));
  }
}

// Sums over the requests in front: their wishes, and what they get.
struct Running {
  unsigned pages_wanted, rows_wanted, pages, rows, tokens, refused;
};

// Decides the requests of one round (one per thread; need: this thread's, nothing where there is none) and places them behind `run`, which moves on.
template <int W>
__device__ __forceinline__ Place place_round(const ExtendArgs& a, Need n, bool here, Running& run, Need* decided) {
  __shared__ unsigned part2[W][2], part4[W][4];
  unsigned w[2] = {static_cast<unsigned>(n.pages), static_cast<unsigned>(n.rows)};
  unsigned all_w[2], all_g[4];
  block_scan<true, 2, W>(w, part2, all_w);
  if (n.rows > 0 && add_up(run.rows_wanted, w[1]) > static_cast<unsigned>(a.max_rows)) n.status = CC_EXTEND_NO_ROWS;
  if (n.pages > 0 && add_up(run.pages_wanted, w[0]) > static_cast<unsigned>(a.n_free)) n.status = CC_EXTEND_NO_PAGES;
  const bool ok = n.status == CC_EXTEND_OK;
  if (!ok) n.pages = n.rows = 0;
  unsigned g[4] = {static_cast<unsigned>(n.pages), static_cast<unsigned>(n.rows), static_cast<unsigned>(n.old_tokens) + n.rows, here && !ok};
  block_scan<false, 4, W>(g, part4, all_g);
  const Place p{static_cast<int>(run.pages + g[0]) - n.pages, static_cast<int>(run.rows + g[1]) - n.rows,
                static_cast<int>(run.tokens + g[2]) - n.old_tokens - n.rows, ok};
  run.pages_wanted = add_up(run.pages_wanted, all_w[0]);
  run.rows_wanted = add_up(run.rows_wanted, all_w[1]);
  run.pages += all_g[0];
  run.rows += all_g[1];
  run.tokens += all_g[2];
  run.refused += all_g[3];
  __syncthreads();
  *decided = n;
  return p;
}

__device__ __forceinline__ void write_request(const ExtendArgs& a, int r, const Need& n, const Place& p) {
  a.cu_q[r + 1] = p.row + n.rows;
  a.last_row[r] = n.rows > 0 ? p.row + n.rows - 1 : -1;
  a.status[r] = n.status;
}
__device__ __forceinline__ void write_counts(const ExtendArgs& a, const Running& run) {
  a.cu_q[0] = 0;
  a.counts[0] = static_cast<int>(run.rows);
  a.counts[1] = static_cast<int>(run.pages);
  a.counts[2] = static_cast<int>(run.refused);
  a.counts[3] = static_cast<int>(run.tokens);
}

// Places 16 requests per workgroup: all needs are scanned (256 at a time) up to the workgroup's own, by the last one to the end; then 16
// lanes write a request's segments.
__global__ __launch_bounds__(256) void extend_segments_kernel(ExtendArgs a, const Need* __restrict__ need, int32_t* __restrict__ page0) {
  __shared__ Place mine[16];
  const int r_first = blockIdx.x * 16, tid = threadIdx.x, lane = tid & 15;
  const bool to_end = blockIdx.x == gridDim.x - 1;
  const int end = to_end ? a.n_requests : min(a.n_requests, r_first + 16);
  Running run{0, 0, 0, 0, 0, 0};
  Need next = tid < a.n_requests ? need[tid] : Need{0, 0, CC_EXTEND_OK, 0};
  for (int r0 = 0; r0 < end; r0 += 256) {
    const int r = r0 + tid;
    const Need n = next;
    next = r + 256 < a.n_requests ? need[r + 256] : Need{0, 0, CC_EXTEND_OK, 0};
    Need decided;
    const Place p = place_round<4>(a, n, r < a.n_requests, run, &decided);
    if (r >= r_first && r < r_first + 16 && r < a.n_requests) {
      mine[r - r_first] = p;
      write_request(a, r, decided, p);
    }
  }
  if (to_end && tid == 0) write_counts(a, run);
  __syncthreads();
  const int r = r_first + (tid >> 4);
  if (r >= a.n_requests) return;
  Place p = mine[tid >> 4];
  const int s0 = max(a.req_seg_off[r], 0), s1 = min(a.req_seg_off[r + 1], a.n_segs);
  int start = 0;
  for (int s = s0 + lane; s - lane < s1; s += 16) {
    cc_segment sg{};
    int old = 0, add = 0;
    if (s < s1) {
      sg = a.segs_in[s];
      old = max(sg.n_tokens, 0);
      add = p.served ? max(a.n_new[s], 0) : 0;
    }
    const int pages = new_pages(old, add), tokens0 = before16(old + add), rows0 = before16(add), pages0 = before16(pages);
    if (s < s1) {
      sg.req = r;
      sg.logical_start = start + tokens0;
      sg.n_tokens = old + add;
      sg.n_select = add;
      sg.tok_off = p.token + tokens0;
      sg.sel_off = p.row + rows0;
      a.segs[s] = sg;
      page0[s] = p.page + pages0;
    }
    const int tokens = __shfl(tokens0 + old + add, 15, 16);
    start += tokens;
    p.token += tokens;
    p.row += __shfl(rows0 + add, 15, 16);
    p.page += __shfl(pages0 + pages, 15, 16);
  }
}

struct RowSegment {                   // what a row has to know of its segment
  int row0, old, start, tab_off, page0, req;
};
struct RowOut {
  int pos, slot, req, entry, page;    // entry: of the page table, to hold the page (-1: none)
};
// Row j: token t of its segment, in a page of the table, or, where the segment had none, of the free list (whose first token writes the table).
__device__ __forceinline__ RowOut row_of(const ExtendArgs& a, const RowSegment& sg, int j) {
  const int t = sg.old + j - sg.row0, nth = t / kBlock - pages_of(sg.old);
  int page;
  page = nth >= 0 ? a.free_blocks[sg.page0 + nth] : a.block_tab[sg.tab_off + t / kBlock];
  const int entry = nth >= 0 && t % kBlock == 0 ? sg.tab_off + t / kBlock : -1;
  return RowOut{sg.start + t, page >= 0 && page < a.n_blocks ? page * kBlock + t % kBlock : -1, sg.req, entry, page};
}

// kRowsPer consecutive rows per thread.  The segments of a workgroup's rows are found by two searches of a wavefront each (64 places at a
// time); a thread's by bisection between them, moved on when its rows pass the segment's end.  A segment is the last one that begins at or
// before the row: those without rows begin where the next one does.
constexpr int kRowsPer = 4;
__global__ __launch_bounds__(256) void extend_rows_kernel(ExtendArgs a, const int32_t* __restrict__ page0) {
  __shared__ int range[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, j0 = blockIdx.x * 256 * kRowsPer, n_rows = a.cu_q[a.n_requests];
  if (wave < 2 && j0 < n_rows) {
    const int j = wave == 0 ? j0 : min(j0 + 256 * kRowsPer, n_rows) - 1;
    int lo = 0, hi = a.n_segs;                                        // sel_off[lo] <= j, sel_off[hi] > j
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, at = lo + lane * step;
      const bool not_behind = at < hi && a.segs[at].sel_off <= j;      // (lane 0's: true)
      const int n = __popcll(__ballot(not_behind));
      hi = min(hi, lo + n * step);
      lo += (n - 1) * step;
    }
    if (lane == 0) range[wave] = lo;
  }
  __syncthreads();
  const int j = j0 + tid * kRowsPer;
  if (j >= a.max_rows) return;
  RowOut out[kRowsPer];
  RowSegment sg{0, 0, 0, 0, 0, 0};
  int end = -1;                                                       // of the segment's rows
#pragma unroll
  for (int i = 0; i < kRowsPer; ++i) {
    out[i] = RowOut{0, -1, -1, -1, 0};
    if (j + i < n_rows) {
      if (j + i >= end) {
        int lo = range[0], hi = range[1] + 1;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (a.segs[mid].sel_off <= j + i) lo = mid; else hi = mid;
        }
        const cc_segment s = a.segs[lo];
        sg = RowSegment{s.sel_off, s.n_tokens - s.n_select, s.logical_start, s.tab_off, page0[lo], s.req};
        end = s.sel_off + s.n_select;
      }
      out[i] = row_of(a, sg, j + i);
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsPer; ++i)
    if (out[i].entry >= 0) a.block_tab[out[i].entry] = out[i].page;
  if (j + kRowsPer <= a.max_rows && a.aligned_rows) {
    *reinterpret_cast<int4*>(a.q_pos + j) = make_int4(out[0].pos, out[1].pos, out[2].pos, out[3].pos);
    *reinterpret_cast<int4*>(a.slot_map + j) = make_int4(out[0].slot, out[1].slot, out[2].slot, out[3].slot);
    *reinterpret_cast<int4*>(a.row_req + j) = make_int4(out[0].req, out[1].req, out[2].req, out[3].req);
  } else {
#pragma unroll
    for (int i = 0; i < kRowsPer; ++i)
      if (j + i < a.max_rows) { a.q_pos[j + i] = out[i].pos; a.slot_map[j + i] = out[i].slot; a.row_req[j + i] = out[i].req; }
  }
}

// All of it by one workgroup, whose LDS holds the tables.
// (W wavefronts: 128 W segments, 64 W requests, 512 W rows)
constexpr int kOwn = 2, kOwnRows = 8;
template <int W> struct SmallShared {
  static constexpr int kSmallSegs = 64 * W * kOwn, kSmallRequests = 64 * W, kSmallRows = 64 * W * kOwnRows;
  unsigned add[kSmallSegs + 1], pages[kSmallSegs + 1], held[kSmallSegs + 1];       // sums over the segments in front (mod 2^32: differences count)
  int start[kSmallSegs], tab_off[kSmallSegs];
  unsigned long long tokens[kSmallRequests];
  int off[kSmallRequests + 1], flags[kSmallRequests];
  Place place[kSmallRequests];
  unsigned short row_seg[kSmallRows];                                              // 1 + the segment that begins at the row
  unsigned short seg_req[kSmallSegs];
};

template <int W>
__global__ __launch_bounds__(64 * W) void extend_small_kernel(ExtendArgs a) {
  constexpr int kThreads = 64 * W, kSmallSegs = SmallShared<W>::kSmallSegs, kSmallRows = SmallShared<W>::kSmallRows;
  __shared__ SmallShared<W> sh;
  __shared__ unsigned wave_sum[W][3];
  __shared__ int wave_last[W];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // ---- the segments (kOwn consecutive ones per thread), sums in front of them
  cc_segment sg[kOwn];
  int old[kOwn], add[kOwn], cap[kOwn];
  unsigned v[3] = {0, 0, 0}, in[3];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int s = tid * kOwn + i;
    old[i] = add[i] = cap[i] = 0;
    if (s < a.n_segs) {
      sg[i] = a.segs_in[s];
      old[i] = max(sg[i].n_tokens, 0);
      add[i] = max(a.n_new[s], 0);
      cap[i] = a.tab_cap[s];
    }
    v[0] += add[i];
    v[1] += new_pages(old[i], add[i]);
    v[2] += old[i];
  }
  for (int r = tid; r <= a.n_requests; r += kThreads) {
    sh.off[r] = max(min(a.req_seg_off[r], a.n_segs), 0);
    if (r < a.n_requests) { sh.flags[r] = 0; sh.tokens[r] = 0; }
  }
  for (int j = tid; j < kSmallRows / 2; j += kThreads) reinterpret_cast<unsigned*>(sh.row_seg)[j] = 0;
  unsigned all[3];
  for (int i = 0; i < 3; ++i) in[i] = v[i];
  block_scan<false, 3, W>(in, wave_sum, all);
  for (int i = 0; i < 3; ++i) in[i] -= v[i];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int s = tid * kOwn + i;
    sh.add[s] = in[0]; sh.pages[s] = in[1]; sh.held[s] = in[2];
    in[0] += add[i];
    in[1] += new_pages(old[i], add[i]);
    in[2] += old[i];
  }
  if (tid == kThreads - 1) { sh.add[kSmallSegs] = in[0]; sh.pages[kSmallSegs] = in[1]; sh.held[kSmallSegs] = in[2]; }
  __syncthreads();
  // ---- which request, and what it cannot have
  int req[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int s = tid * kOwn + i;
    req[i] = -1;
    if (s >= a.n_segs) continue;
    int lo = 0, hi = a.n_requests;                                   // the last request that begins at or before s
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (sh.off[mid] <= s) lo = mid; else hi = mid;
    }
    if (sh.off[lo] > s || sh.off[lo + 1] <= s) continue;              // (of no request)
    req[i] = lo;
    atomicAdd(&sh.tokens[lo], static_cast<unsigned long long>(old[i]) + add[i]);
    int flags = segment_full(a, old[i], add[i], sg[i].tab_off, cap[i]) ? 1 : 0;
    if (add[i] > 0 && sh.held[sh.off[lo + 1]] != sh.held[s + 1]) flags |= 2;
    if (flags) atomicOr(&sh.flags[lo], flags);
  }
  __syncthreads();
  // ---- the requests
  Running run{0, 0, 0, 0, 0, 0};
  {
    const int r = tid;
    Need n{0, 0, CC_EXTEND_OK, 0}, decided;
    if (r < a.n_requests) {
      const int s0 = sh.off[r], s1 = max(sh.off[r + 1], s0);
      n.status = (sh.flags[r] & 1) != 0 || sh.tokens[r] > 0x7fffffffull ? CC_EXTEND_TABLE_FULL : (sh.flags[r] & 2) != 0 ? CC_EXTEND_ORDER : CC_EXTEND_OK;
      n.old_tokens = static_cast<int>(sh.held[s1] - sh.held[s0]);
      if (n.status == CC_EXTEND_OK) {
        n.pages = static_cast<int>(sh.pages[s1] - sh.pages[s0]);
        n.rows = static_cast<int>(sh.add[s1] - sh.add[s0]);
      }
    }
    const Place p = place_round<W>(a, n, r < a.n_requests, run, &decided);
    if (r < a.n_requests) {
      sh.place[r] = p;
      write_request(a, r, decided, p);
    }
    if (tid == 0) write_counts(a, run);
  }
  __syncthreads();
  // ---- the segments' places; the offsets in LDS become those of what is served
  unsigned row0[kOwn], page0[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int s = tid * kOwn + i;
    if (req[i] < 0) continue;
    const Place p = sh.place[req[i]];
    const int s0 = sh.off[req[i]];
    const unsigned rows = p.served ? sh.add[s] - sh.add[s0] : 0, held = sh.held[s] - sh.held[s0];
    if (!p.served) add[i] = 0;
    row0[i] = p.row + rows;
    page0[i] = p.page + (p.served ? sh.pages[s] - sh.pages[s0] : 0);
    sg[i].req = req[i];
    sg[i].logical_start = static_cast<int>(held + rows);
    sg[i].n_tokens = old[i] + add[i];
    sg[i].n_select = add[i];
    sg[i].tok_off = p.token + sg[i].logical_start;
    sg[i].sel_off = static_cast<int>(row0[i]);
    a.segs[s] = sg[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int s = tid * kOwn + i;
    if (req[i] < 0 || add[i] == 0) continue;
    sh.add[s] = row0[i];
    sh.pages[s] = page0[i];
    sh.held[s] = old[i];
    sh.start[s] = sg[i].logical_start;
    sh.tab_off[s] = sg[i].tab_off;
    sh.row_seg[row0[i]] = static_cast<unsigned short>(s + 1);
    sh.seg_req[s] = static_cast<unsigned short>(req[i]);
  }
  __syncthreads();
  // ---- the rows: the segment that began last (they begin in the rows' order)
  unsigned short* mine = sh.row_seg + tid * kOwnRows;
  int last = 0, upto;
#pragma unroll
  for (int i = 0; i < kOwnRows; ++i) last = max(last, static_cast<int>(mine[i]));
  upto = last;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o, 64);
    if (lane >= o) upto = max(upto, up);
  }
  if (lane == 63) wave_last[wave] = upto;
  int seg = __shfl_up(upto, 1, 64);
  if (lane == 0) seg = 0;
  __syncthreads();
  for (int w = 0; w < wave; ++w) seg = max(seg, wave_last[w]);
#pragma unroll
  for (int i = 0; i < kOwnRows; ++i) {
    seg = max(seg, static_cast<int>(mine[i]));
    mine[i] = static_cast<unsigned short>(seg);
  }
  __syncthreads();
  const int n_rows = static_cast<int>(run.rows);
  RowOut out[kOwnRows];
#pragma unroll
  for (int i = 0; i < kOwnRows; ++i) {                               // (the rows' loads are all under way before the first is used)
    const int j = tid + i * kThreads;
    if (j >= n_rows) break;
    const int s = sh.row_seg[j] - 1;
    out[i] = row_of(a, RowSegment{static_cast<int>(sh.add[s]), static_cast<int>(sh.held[s]), sh.start[s], sh.tab_off[s], static_cast<int>(sh.pages[s]), sh.seg_req[s]}, j);
  }
#pragma unroll
  for (int i = 0; i < kOwnRows; ++i) {
    const int j = tid + i * kThreads;
    if (j >= a.max_rows) break;
    if (j >= n_rows) out[i] = RowOut{0, -1, -1, -1, 0};
    if (out[i].entry >= 0) a.block_tab[out[i].entry] = out[i].page;
    a.q_pos[j] = out[i].pos;
    a.slot_map[j] = out[i].slot;
    a.row_req[j] = out[i].req;
  }
}

// Wavefronts of the workgroup that does it alone; 0: the tables are too large for one.  (32 requests: 4 wavefronts 7.5 us, 16 9.7, three launches 14.9; 250
// requests with 1600 segments: 16 wavefronts 13.8, three launches 18.1)
int small_waves(int n_segs, int n_requests, int max_rows) {
  for (int w : {4, 16})
    if (n_segs <= 64 * w * kOwn && n_requests <= 64 * w && max_rows <= 64 * w * kOwnRows) return w;
  return 0;
}

}  // namespace

size_t extend_bytes(int n_segs, int n_requests) {
  return static_cast<size_t>(n_requests) * sizeof(Need) + static_cast<size_t>(n_segs) * sizeof(int32_t);
}

void launch_extend_segments(const cc_segment* segs_in, const int32_t* n_new, const int32_t* tab_cap, int n_segs,
                            const int32_t* req_seg_off, int n_requests, const int32_t* free_blocks, int n_free, int32_t* block_tab,
                            int n_tab, int n_blocks, cc_segment* segs, int32_t* cu_q, int32_t* q_pos, int32_t* slot_map, int32_t* row_req,
                            int max_rows, int32_t* last_row, int32_t* status, int32_t* counts, void* workspace, hipStream_t stream) {
  const ExtendArgs a{segs_in, n_new, tab_cap, req_seg_off, free_blocks, block_tab, n_segs, n_requests, n_free, n_tab, n_blocks, max_rows,
                     segs, cu_q, q_pos, slot_map, row_req, last_row, status, counts, aligned16(q_pos) && aligned16(slot_map) && aligned16(row_req)};
  const int waves = n_requests > 0 ? small_waves(n_segs, n_requests, max_rows) : 0;
  if (waves == 4) hipLaunchKernelGGL(extend_small_kernel<4>, dim3(1), dim3(256), 0, stream, a);
  if (waves == 16) hipLaunchKernelGGL(extend_small_kernel<16>, dim3(1), dim3(1024), 0, stream, a);
  if (waves != 0) return;
  Need* need = static_cast<Need*>(workspace);
  int32_t* page0 = reinterpret_cast<int32_t*>(need + n_requests);
  const dim3 per_request(std::max(1, (n_requests + 15) / 16));        // (no request: the totals, and rows of nothing)
  if (n_requests > 0) hipLaunchKernelGGL(extend_need_kernel, per_request, dim3(256), 0, stream, a, need);
  hipLaunchKernelGGL(extend_segments_kernel, per_request, dim3(256), 0, stream, a, need, page0);
  if (max_rows > 0) hipLaunchKernelGGL(extend_rows_kernel, dim3((max_rows + 256 * kRowsPer - 1) / (256 * kRowsPer)), dim3(256), 0, stream, a, page0);
}

}  // namespace cc
