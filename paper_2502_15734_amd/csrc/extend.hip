// cc_extend_segments: segment table, page table and the rows' positions and slots of tokens that come behind what the pages hold.
//
// Per segment old tokens are held and add come behind them; pages(x) = ceil(x / 16).  A request's need is
// sum(pages(old + add) - pages(old)) pages and sum(add) rows.  Who is served is decided by one exclusive scan of the needs in
// request order; the places of what is served (rows, pages of the free list, token offsets) come from a second one.
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
};

struct Need {             // of a request; status: one of CC_EXTEND_*
  int pages, rows, status, old_tokens;
};
struct Place {            // where a request's share begins
  int page, row, token, served;
};

__device__ __forceinline__ int pages_of(int tokens) { return static_cast<int>((static_cast<unsigned>(tokens) + (kBlock - 1)) / kBlock); }

__device__ __forceinline__ Need need_of(const ExtendArgs& a, int r) {
  const int s0 = max(a.req_seg_off[r], 0), s1 = min(a.req_seg_off[r + 1], a.n_segs);
  long long rows = 0, pages = 0, old_tokens = 0;
  bool grown = false, full = false, order = false;
  for (int s = s0; s < s1; ++s) {
    const int old = max(a.segs_in[s].n_tokens, 0), add = max(a.n_new[s], 0), off = a.segs_in[s].tab_off;
    order |= grown && old > 0;
    if (add > 0) {
      const long long after = (static_cast<long long>(old) + add + kBlock - 1) / kBlock;
      grown = true;
      full |= off < 0 || after > a.tab_cap[s] || off + after > a.n_tab;
      pages += after - pages_of(old);
    }
    rows += add;
    old_tokens += old;
  }
  int status = order ? CC_EXTEND_ORDER : CC_EXTEND_OK;
  if (full || rows + old_tokens > 0x7fffffffll) status = CC_EXTEND_TABLE_FULL;
  if (status != CC_EXTEND_OK) rows = pages = 0;
  return Need{static_cast<int>(pages), static_cast<int>(rows), status, static_cast<int>(old_tokens)};
}

__global__ __launch_bounds__(256) void extend_need_kernel(ExtendArgs a, Need* __restrict__ need) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < a.n_requests) need[r] = need_of(a, r);
}

// inclusive scan over the workgroup's 1024 threads, of N sums at once
template <int N>
__device__ __forceinline__ void block_scan(long long (&v)[N], long long (*part)[N]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const long long up = __shfl_up(v[i], o, 64);
      if (lane >= o) v[i] += up;
    }
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < N; ++i) part[wave][i] = v[i];
  __syncthreads();
  for (int w = 0; w < wave; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += part[w][i];
  __syncthreads();
}

__global__ __launch_bounds__(1024) void extend_scan_kernel(ExtendArgs a, const Need* __restrict__ need, Place* __restrict__ place) {
  __shared__ long long part[16][3];
  __shared__ long long last[6];
  long long wanted[2] = {0, 0}, given[3] = {0, 0, 0}, refused = 0;        // sums over the requests before this round's
  for (int r0 = 0; r0 < a.n_requests; r0 += 1024) {
    const int r = r0 + threadIdx.x;
    Need n{0, 0, CC_EXTEND_OK, 0};
    if (r < a.n_requests) n = need[r];
    long long w[3] = {n.pages, n.rows, 0};
    block_scan<3>(w, part);
    if (n.rows > 0 && wanted[1] + w[1] > a.max_rows) n.status = CC_EXTEND_NO_ROWS;
    if (n.pages > 0 && wanted[0] + w[0] > a.n_free) n.status = CC_EXTEND_NO_PAGES;
    const bool ok = n.status == CC_EXTEND_OK;
    if (!ok) n.pages = n.rows = 0;
    long long g[3] = {n.pages, n.rows, static_cast<long long>(n.old_tokens) + n.rows};
    block_scan<3>(g, part);
    const int n_bad = __syncthreads_count(r < a.n_requests && !ok);
    if (r < a.n_requests) {
      const int row1 = static_cast<int>(given[1] + g[1]);
      place[r] = Place{static_cast<int>(given[0] + g[0]) - n.pages, row1 - n.rows, static_cast<int>(given[2] + g[2] - n.old_tokens - n.rows), ok};
      a.cu_q[r + 1] = row1;
      a.last_row[r] = n.rows > 0 ? row1 - 1 : -1;
      a.status[r] = n.status;
    }
    if (threadIdx.x == 1023) {
      for (int i = 0; i < 2; ++i) last[i] = w[i];
      for (int i = 0; i < 3; ++i) last[2 + i] = g[i];
    }
    __syncthreads();
    for (int i = 0; i < 2; ++i) wanted[i] += last[i];
    for (int i = 0; i < 3; ++i) given[i] += last[2 + i];
    refused += n_bad;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    a.cu_q[0] = 0;
    a.counts[0] = static_cast<int>(given[1]);
    a.counts[1] = static_cast<int>(given[0]);
    a.counts[2] = static_cast<int>(refused);
    a.counts[3] = static_cast<int>(given[2]);
  }
}

__global__ __launch_bounds__(256) void extend_segments_kernel(ExtendArgs a, const Place* __restrict__ place, int32_t* __restrict__ page0) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= a.n_requests) return;
  Place p = place[r];
  const int s0 = max(a.req_seg_off[r], 0), s1 = min(a.req_seg_off[r + 1], a.n_segs);
  int start = 0;
  for (int s = s0; s < s1; ++s) {
    cc_segment sg = a.segs_in[s];
    const int old = max(sg.n_tokens, 0), add = p.served ? max(a.n_new[s], 0) : 0;
    sg.req = r;
    sg.logical_start = start;
    sg.n_tokens = old + add;
    sg.n_select = add;
    sg.tok_off = p.token;
    sg.sel_off = p.row;
    a.segs[s] = sg;
    page0[s] = p.page;
    start += old + add;
    p.token += old + add;
    p.row += add;
    p.page += pages_of(old + add) - pages_of(old);
  }
}

// One row of the list: its segment by bisection of the row offsets (the last one that begins at or before the row: those without
// rows begin where the next one does), then its token, its page (from the free list where the row's segment had none) and slot.
__global__ __launch_bounds__(256) void extend_rows_kernel(ExtendArgs a, const int32_t* __restrict__ page0) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= a.max_rows) return;
  if (j >= a.cu_q[a.n_requests]) {
    a.q_pos[j] = 0;
    a.slot_map[j] = -1;
    a.row_req[j] = -1;
    return;
  }
  int lo = 0, hi = a.n_segs;                   // sel_off[lo] <= j, sel_off[hi] > j
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.segs[mid].sel_off <= j) lo = mid; else hi = mid;
  }
  const cc_segment sg = a.segs[lo];
  const int old = sg.n_tokens - sg.n_select, t = old + j - sg.sel_off, nth = t / kBlock - pages_of(old);
  int page;
  if (nth >= 0) {
    page = a.free_blocks[page0[lo] + nth];
    if (t % kBlock == 0) a.block_tab[sg.tab_off + t / kBlock] = page;
  } else {
    page = sg.tab_off >= 0 ? a.block_tab[sg.tab_off + t / kBlock] : -1;
  }
  a.q_pos[j] = sg.logical_start + t;
  a.slot_map[j] = page >= 0 && page < a.n_blocks ? page * kBlock + t % kBlock : -1;
  a.row_req[j] = sg.req;
}

}  // namespace

size_t extend_bytes(int n_segs, int n_requests) {
  return static_cast<size_t>(n_requests) * (sizeof(Need) + sizeof(Place)) + static_cast<size_t>(n_segs) * sizeof(int32_t);
}

void launch_extend_segments(const cc_segment* segs_in, const int32_t* n_new, const int32_t* tab_cap, int n_segs,
                            const int32_t* req_seg_off, int n_requests, const int32_t* free_blocks, int n_free, int32_t* block_tab,
                            int n_tab, int n_blocks, cc_segment* segs, int32_t* cu_q, int32_t* q_pos, int32_t* slot_map, int32_t* row_req,
                            int max_rows, int32_t* last_row, int32_t* status, int32_t* counts, void* workspace, hipStream_t stream) {
  const ExtendArgs a{segs_in, n_new, tab_cap, req_seg_off, free_blocks, block_tab, n_segs, n_requests, n_free, n_tab, n_blocks, max_rows,
                     segs, cu_q, q_pos, slot_map, row_req, last_row, status, counts};
  Need* need = static_cast<Need*>(workspace);
  Place* place = reinterpret_cast<Place*>(need + n_requests);
  int32_t* page0 = reinterpret_cast<int32_t*>(place + n_requests);
  const dim3 per_request((n_requests + 255) / 256);
  hipLaunchKernelGGL(extend_need_kernel, per_request, dim3(256), 0, stream, a, need);
  hipLaunchKernelGGL(extend_scan_kernel, dim3(1), dim3(1024), 0, stream, a, need, place);
  hipLaunchKernelGGL(extend_segments_kernel, per_request, dim3(256), 0, stream, a, place, page0);
  if (max_rows > 0) hipLaunchKernelGGL(extend_rows_kernel, dim3((max_rows + 255) / 256), dim3(256), 0, stream, a, page0);
}

}  // namespace cc
