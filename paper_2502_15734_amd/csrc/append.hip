// cc_append_attention: causal attention of the last rows of each request over its whole paged context, a few rows or one at a time.
//
// Bound by the bytes of the keys and values: a page of 16 tokens is read once for all rows and all heads of its group, and a row brings
// 2 G multiply-adds per element read (G query heads on a KV head), far below what the matrix cores take.  So the rows and heads
// of a group are the 16 columns of a matrix instruction (most of them empty when one token is written: they cost nothing), and the keys
// are divided: a workgroup takes one (request, KV head, 16 NC columns, range of pages), its four wavefronts every fourth tile of
// the range, and merge at the end; a second kernel joins the ranges of a row.
//
// Layout: S^T = K Q^T and O^T = V^T P^T with lane = (n = lane % 16, g = lane / 16), column n.  No operand passes through LDS: the
// contraction order of either product is free as long as both operands agree.  bf16, a tile of two pages: of the first product's two
// 16-key blocks block t takes, as row 4 g' + j, token 8 (g' % 2) + 4 t + j of page g' / 2, so that lane (n, g) ends up with the
// logits of tokens 8 (g % 2) .. + 7 of page g / 2: as the second product's 32-token operand they meet a 16-byte piece of a
// dimension-major V row.  fp32, a tile of one page: steps of four tokens, as in qk_f32.hip.
//
// The softmax reference of a column is shared by the four lane groups and moves only when a logit is more than kSlack above it.
#include <algorithm>

#include "device_util.h"

namespace cc {

namespace {

constexpr float kSlack = 8.f;         // in powers of two
constexpr int kWindow = 256;          // pages listed in LDS at a time
constexpr float kLog2e = 1.4426950408889634f;

struct AppendArgs {
  const void* q;
  const int32_t *src_rows, *q_pos, *cu_q;
  const void *k_pool, *v_pool;
  const int32_t* block_tab;
  const cc_segment* segs;
  const int32_t* req_seg_off;
  void* out;
  float* lse;
  ValueSource vs;
  int n_requests, n_blocks, hq, hkv;
  // division of the keys
  int n_splits, split_pages;
  float *part_o, *part_ml;            // [row][head][split][D], [row][head][split][2]
  int32_t* row_splits;                // [row] ranges its request has (1: the output is written)
};

struct Page {
  int blk, pos0, n_valid, value;      // value: block of the own pool, or -1 - block of the shared one
};

__device__ __forceinline__ int pages_of(int tokens) { return (max(tokens, 0) + kBlock - 1) / kBlock; }

// Pages [first, first + kWindow) of a request into list[] (thread i: page first + i), those behind its last one with n_valid 0;
// returns the number of pages the request has.  Thread i also takes segment i of 256 at a time, whose page counts are scanned.
__device__ __forceinline__ int list_pages(const AppendArgs& a, int s_begin, int s_end, int first, int p_max, Page* list, int4* segs, int* seg_end,
                                          int* wave_pages) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, want = first + tid;
  Page page{0, 0, 0, 0};
  int total = 0;
  for (int s0 = s_begin; s0 < s_end; s0 += 256) {
    const int s = s0 + tid;
    int4 mine{0, 0, 0, 0};
    if (s < s_end) mine = *reinterpret_cast<const int4*>(&a.segs[s].logical_start);     // start, tokens, table offset, (rows)
    const int n = pages_of(mine.y);
    int end = n;
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(end, o, 64);
      if (lane >= o) end += up;
    }
    if (lane == 63) wave_pages[wave] = end;
    __syncthreads();
    int before = total;
    for (int w = 0; w < 4; ++w) {
      if (w < wave) before += wave_pages[w];
      total += wave_pages[w];
    }
    seg_end[tid] = before + end;
    segs[tid] = mine;
    __syncthreads();
    const int base = total - (wave_pages[0] + wave_pages[1] + wave_pages[2] + wave_pages[3]);
    if (want >= base && want < total) {
      int lo = 0, hi = 255;                                       // the first segment whose end lies behind the page
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (seg_end[mid] > want) hi = mid; else lo = mid + 1;
      }
      const int4 sg = segs[lo];
      const int nth = want - (seg_end[lo] - pages_of(sg.y)), blk = a.block_tab[sg.z + nth];
      page.pos0 = sg.x + nth * kBlock;
      if (blk >= 0 && blk < a.n_blocks && page.pos0 <= p_max) {
        page.blk = page.value = blk;
        page.n_valid = min(sg.y - nth * kBlock, kBlock);
        if (a.vs.v_map != nullptr) {
          const int m = a.vs.v_map[blk];
          if (m >= 0 && m < a.vs.n_shared_blocks) page.value = -1 - m;
        }
      }
    }
    __syncthreads();
  }
  list[tid] = page;
  __syncthreads();
  return total;
}

template <typename T, int D> struct Tile;           // operands of one tile of keys

template <int D> struct Tile<bf16_t, D> {
  static constexpr int kPages = 2, kTok = 8;        // pages of a tile; tokens of it that a lane holds
  typedef bf16x8 Piece;
  Piece k[2][D / 32], v[D / 16];
  static __device__ __forceinline__ int page_of(int lane) { return lane >> 5; }                // of the tokens the lane holds
  static __device__ __forceinline__ int token_of(int lane) { return ((lane >> 4) & 1) * 8; }
  __device__ __forceinline__ void load(const bf16_t* k_pool, const bf16_t* v_pool, const bf16_t* v_shared, const Page* pages, size_t block_elems,
                                       size_t head_off, int lane) {
    const int n = lane & 15, g = lane >> 4;
    const bf16_t* kp = k_pool + pages[n >> 3].blk * block_elems + head_off + (((n >> 2) & 1) * 8 + (n & 3)) * D + 8 * g;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) k[t][i] = *reinterpret_cast<const Piece*>(kp + t * 4 * D + 32 * i);
    const int value = pages[g >> 1].value;
    const bf16_t* vp = (value >= 0 ? v_pool + value * block_elems : v_shared + (-1 - value) * block_elems) + head_off + n * kBlock + (g & 1) * 8;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) v[i] = *reinterpret_cast<const Piece*>(vp + i * 16 * kBlock);
  }
  __device__ __forceinline__ void logits(const Piece (&q)[D / 32], float (&s)[kTok]) const {
    f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][i], q[i], acc[t], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < kTok; ++e) s[e] = acc[e >> 2][e & 3];
  }
  static __device__ __forceinline__ f32x4 add_values(const Piece& v, const Piece& p, f32x4 o) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o, 0, 0, 0);
  }
  // (queries and weights: their one rounding, as the matrix instruction takes bf16)
  static __device__ __forceinline__ Piece piece(const float (&x)[8]) {
    Piece w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = static_cast<bf16_t>(x[e]);
    return w;
  }
};

template <int D> struct Tile<float, D> {
  static constexpr int kPages = 1, kTok = 4;
  typedef f32x4 Piece;
  Piece k[1][D / 16], v[D / 16];
  static __device__ __forceinline__ int page_of(int) { return 0; }
  static __device__ __forceinline__ int token_of(int lane) { return (lane >> 4) * 4; }
  __device__ __forceinline__ void load(const float* k_pool, const float* v_pool, const float* v_shared, const Page* pages, size_t block_elems,
                                       size_t head_off, int lane) {
    const int n = lane & 15, g = lane >> 4;
    const float* kp = k_pool + pages[0].blk * block_elems + head_off + n * D + 4 * g;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) k[0][i] = *reinterpret_cast<const Piece*>(kp + 16 * i);
    const int value = pages[0].value;
    const float* vp = (value >= 0 ? v_pool + value * block_elems : v_shared + (-1 - value) * block_elems) + head_off + n * kBlock + 4 * g;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) v[i] = *reinterpret_cast<const Piece*>(vp + i * 16 * kBlock);
  }
  // (four chains of additions: one of D would lose two bits)
  __device__ __forceinline__ void logits(const Piece (&q)[D / 16], float (&s)[kTok]) const {
    f32x4 acc[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0][i][e], q[i][e], acc[e], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < kTok; ++e) s[e] = (acc[0][e] + acc[1][e]) + (acc[2][e] + acc[3][e]);
  }
  static __device__ __forceinline__ f32x4 add_values(const Piece& v, const Piece& p, f32x4 o) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], p[e], o, 0, 0, 0);
    return o;
  }
  static __device__ __forceinline__ Piece piece(const float (&x)[4]) { return Piece{x[0], x[1], x[2], x[3]}; }
};

// One (range of pages, KV head and 16 NC columns, request).  Column c is head c % G of the request's row c / G.
template <typename T, int D, int NC>
__global__ __launch_bounds__(256, NC == 4 ? 1 : 2) void append_split_kernel(AppendArgs a, InvFreq inv_freq) {
  typedef Tile<T, D> Keys;
  typedef typename Keys::Piece Piece;
  constexpr int kTok = Keys::kTok, kPer = 16 / sizeof(T), kQ = D / 4 / kPer;      // elements of a piece; pieces of a query a lane holds
  constexpr int kRow = D + 4;                                                    // (a column of the outputs in LDS: banks apart)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const int r = blockIdx.z, kvh = blockIdx.y, split = blockIdx.x % a.n_splits, group = a.hq / a.hkv;
  const int col0 = blockIdx.x / a.n_splits * 16 * NC, row0 = a.cu_q[r], n_cols = (a.cu_q[r + 1] - row0) * group;
  if (col0 >= n_cols) return;
  const int s_begin = a.req_seg_off[r], s_end = a.req_seg_off[r + 1];

  union Shared {
    struct { Page list[kWindow]; int4 segs[256]; int seg_end[256]; int wave_pages[4]; } in;
    struct { float o[4][16][kRow]; float m[4][16], l[4][16]; } out;
  };
  __shared__ Shared sh;

  // ---- positions of the columns, and the rows themselves (loads first, turned later)
  int pos[NC], p_min = 0x7fffffff, p_max = -1;
  Piece q[NC][kQ];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = col0 + 16 * c + n, row = row0 + min(col, n_cols - 1) / group;
    pos[c] = a.q_pos[row];
    if (col < n_cols) { p_min = min(p_min, pos[c]); p_max = max(p_max, pos[c]); }
    const int src = a.src_rows != nullptr ? a.src_rows[row] : row;
    const T* qp = static_cast<const T*>(a.q) + (static_cast<size_t>(src) * a.hq + kvh * group + min(col, n_cols - 1) % group) * D + kPer * g;
#pragma unroll
    for (int i = 0; i < kQ; ++i) q[c][i] = *reinterpret_cast<const Piece*>(qp + 4 * kPer * i);
  }
  p_min = wave_min_i(p_min);
  p_max = wave_max_i(p_max);

  const size_t block_elems = static_cast<size_t>(a.hkv) * kBlock * D, head_off = static_cast<size_t>(kvh) * kBlock * D;
  const T *k_pool = static_cast<const T*>(a.k_pool), *v_pool = static_cast<const T*>(a.v_pool), *v_shared = static_cast<const T*>(a.vs.v_shared);
  float m[NC], l[NC];
  f32x4 o[NC][D / 16];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    m[c] = -3.4028235e38f;
    l[c] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[c][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int first_page = split * a.split_pages;
  int n_pages = list_pages(a, s_begin, s_end, first_page, p_max, sh.in.list, sh.in.segs, sh.in.seg_end, sh.in.wave_pages);
  if (first_page >= max(n_pages, 1)) return;                                        // (the same in all wavefronts)
  const int n_splits = min((max(n_pages, 1) + a.split_pages - 1) / a.split_pages, a.n_splits);
  const int end_page = split == a.n_splits - 1 ? n_pages : min(n_pages, first_page + a.split_pages);

  // ---- the queries at their positions, in units of the logits' powers of two
  const float scale = rsqrtf(static_cast<float>(D)) * kLog2e;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < kQ / 2; ++i) {
      float x[kPer], y[kPer];
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        float cs, sn;
        const double freq = inv_freq.f[4 * kPer * i + kPer * g + e];
        if (sizeof(T) == 2) rot_cos_sin_fast(pos[c], freq, &cs, &sn);          // (the result is rounded to bf16)
        else rot_cos_sin(pos[c], freq, &cs, &sn);
        const float u = to_float(q[c][i][e]), w = to_float(q[c][i + kQ / 2][e]);
        x[e] = (u * cs - w * sn) * scale;
        y[e] = (w * cs + u * sn) * scale;
      }
      q[c][i] = Keys::piece(x);
      q[c][i + kQ / 2] = Keys::piece(y);
    }

  auto take = [&](Keys& t, const Page& held) __attribute__((always_inline)) {
    const int tok0 = Keys::token_of(lane), first = held.pos0 + tok0;       // of this lane's tokens
    const bool whole = __all(held.n_valid == kBlock && held.pos0 + kBlock - 1 <= p_min);
    bool apart = false;                                                    // some value that only some columns see is not finite
    if (!whole) {
      const int seen = min(held.n_valid - tok0, p_max - first + 1);        // of the lane's tokens: any column sees the first `seen`,
      const int by_all = min(seen, p_min - first + 1);                     // every column the first `by_all`
      bool odd = false;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < kTok; ++e) {
          if (e >= seen) t.v[i][e] = static_cast<T>(0.f);
          odd |= e >= by_all && !(fabsf(to_float(t.v[i][e])) < INFINITY);
        }
      apart = __any(odd);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float s[kTok];
      t.logits(q[c], s);
      if (!whole) {
        const int seen = min(held.n_valid - tok0, pos[c] - first + 1);
#pragma unroll
        for (int e = 0; e < kTok; ++e) s[e] = e < seen ? s[e] : -INFINITY;
      }
      float top = s[0];
#pragma unroll
      for (int e = 1; e < kTok; ++e) top = fmaxf(top, s[e]);
      if (__any(top > m[c] + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m[c], top), f = exp2f(m[c] - m_new);
        m[c] = m_new;
        l[c] *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[c][i] *= f;
      }
      float p[kTok], sum = 0.f;
#pragma unroll
      for (int e = 0; e < kTok; ++e) { p[e] = __builtin_amdgcn_exp2f(s[e] - m[c]); sum += p[e]; }
      l[c] += sum;
      if (!apart) {
        const Piece w = Keys::piece(p);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[c][i] = Keys::add_values(t.v[i], w, o[c][i]);
      } else {
        // 0 x value would reach the columns that do not see it: one column at a time
#pragma unroll 1
        for (int k = 0; k < 16; ++k) {
          const int seen = __shfl(pos[c], k, 16) - first + 1;
          float only[kTok];
#pragma unroll
          for (int e = 0; e < kTok; ++e) only[e] = n == k ? p[e] : 0.f;
          const Piece w = Keys::piece(only);
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            Piece v = t.v[i];
#pragma unroll
            for (int e = 0; e < kTok; ++e)
              if (e >= seen) v[e] = static_cast<T>(0.f);
            const f32x4 add = Keys::add_values(v, w, f32x4{0.f, 0.f, 0.f, 0.f});
            if (n == k) o[c][i] += add;
          }
        }
      }
    }
  };

  // ---- the keys: every fourth tile of the window is this wavefront's
  for (int at = first_page;;) {
    const int here = min(end_page - at, kWindow);
    for (int i = wave * Keys::kPages; i < here; i += 4 * Keys::kPages) {
      Keys t;
      t.load(k_pool, v_pool, v_shared, sh.in.list + i, block_elems, head_off, lane);
      Page held = sh.in.list[i + Keys::page_of(lane)];
      if (i + Keys::page_of(lane) >= here) held.n_valid = 0;               // (the next range's)
      take(t, held);
    }
    at += kWindow;
    __syncthreads();
    if (at >= end_page) break;
    list_pages(a, s_begin, s_end, at, p_max, sh.in.list, sh.in.segs, sh.in.seg_end, sh.in.wave_pages);
  }

  // ---- the four wavefronts' sums, and the result of this range
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    l[c] += __shfl_xor(l[c], 16, 64);
    l[c] += __shfl_xor(l[c], 32, 64);
    if (g == 0) { sh.out.m[wave][n] = m[c]; sh.out.l[wave][n] = l[c]; }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(&sh.out.o[wave][n][16 * i + 4 * g]) = o[c][i];
    __syncthreads();
    for (int i = tid; i < 16 * (D / 4); i += 256) {
      const int k = i / (D / 4), d = i % (D / 4) * 4, col = col0 + 16 * c + k;
      if (col < n_cols) {
        float top = sh.out.m[0][k];
        for (int w = 1; w < 4; ++w) top = fmaxf(top, sh.out.m[w][k]);
        float sum = 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < 4; ++w) {
          const float f = exp2f(sh.out.m[w][k] - top);
          sum += f * sh.out.l[w][k];
          v += *reinterpret_cast<const f32x4*>(&sh.out.o[w][k][d]) * f;
        }
        const int row = row0 + col / group;
        const size_t at = static_cast<size_t>(row) * a.hq + kvh * group + col % group;
        if (n_splits == 1) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;           // (no key: zeros, and -inf for the logarithm)
          T* op = static_cast<T*>(a.out) + at * D + d;
#pragma unroll
          for (int e = 0; e < 4; ++e) op[e] = from_float<T>(v[e] * inv);
          if (d == 0 && a.lse != nullptr) a.lse[at] = sum == 0.f ? -INFINITY : top / kLog2e + logf(sum);
        } else {
          *reinterpret_cast<f32x4*>(a.part_o + (at * a.n_splits + split) * D + d) = v;
          if (d == 0) {
            float* ml = a.part_ml + (at * a.n_splits + split) * 2;
            ml[0] = top;
            ml[1] = sum;
          }
        }
        if (split == 0 && d == 0 && kvh == 0 && col % group == 0) a.row_splits[row] = n_splits;
      }
    }
    __syncthreads();
  }
}

// Joins the ranges of one row and head: sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  The threads of a group of D / 4 take four dims
// each, the groups every so-manieth range.
template <typename T, int D>
__global__ __launch_bounds__(256) void append_join_kernel(AppendArgs a) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ float top_of[4], sum_of[kGroups];
  __shared__ f32x4 part[kGroups][kLanes];
  const int row = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, lane = tid % kLanes, grp = tid / kLanes;
  if (row >= a.cu_q[a.n_requests]) return;
  const int ns = a.row_splits[row];
  if (ns <= 1) return;
  const size_t at = static_cast<size_t>(row) * a.hq + h;
  const float* ml = a.part_ml + at * a.n_splits * 2;
  float top = -INFINITY;
  for (int s = tid; s < ns; s += 256) top = fmaxf(top, ml[2 * s]);
  top = wave_max(top);
  if ((tid & 63) == 0) top_of[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(top_of[0], top_of[1]), fmaxf(top_of[2], top_of[3]));
  float sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s = grp; s < ns; s += kGroups) {
    const float f = exp2f(ml[2 * s] - top);
    sum += f * ml[2 * s + 1];
    v += *reinterpret_cast<const f32x4*>(a.part_o + (at * a.n_splits + s) * D + 4 * lane) * f;
  }
  part[grp][lane] = v;
  if (lane == 0) sum_of[grp] = sum;
  __syncthreads();
  if (grp != 0) return;
  for (int k = 1; k < kGroups; ++k) { v += part[k][lane]; sum += sum_of[k]; }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* op = static_cast<T*>(a.out) + at * D + 4 * lane;
#pragma unroll
  for (int e = 0; e < 4; ++e) op[e] = from_float<T>(v[e] * inv);
  if (lane == 0 && a.lse != nullptr) a.lse[at] = sum == 0.f ? -INFINITY : top / kLog2e + logf(sum);
}

// How the work of a call is divided: from host scalars alone.
struct AppendPlan {
  int nc, col_groups, n_splits, split_pages;
};
AppendPlan plan_append(const cc_ctx* ctx, int max_q_per_req, int n_requests, int max_ctx_tokens, int max_segs_per_req) {
  const long long cols = static_cast<long long>(max_q_per_req) * (ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads);
  AppendPlan p;
  p.nc = cols <= 16 ? 1 : cols <= 32 ? 2 : 4;
  p.col_groups = static_cast<int>((cols + 16 * p.nc - 1) / (16 * p.nc));
  const long long pages = max_ctx_tokens / kBlock + static_cast<long long>(max_segs_per_req), units = static_cast<long long>(p.col_groups) * ctx->cfg.n_kv_heads * n_requests;
  const long long splits = std::max(1ll, std::min(2048 / std::max(1ll, units), (pages + 7) / 8));
  p.split_pages = static_cast<int>((pages + splits - 1) / splits + 1) & ~1;
  p.n_splits = static_cast<int>((pages + p.split_pages - 1) / p.split_pages);
  return p;
}

}  // namespace

// Plain form (CC_IMPL_SCALAR): one wavefront per (row, query head), one key at a time with the running maximum and sum of the softmax.
template <typename T, int D>
__global__ __launch_bounds__(64) void append_scalar_kernel(
    const T* __restrict__ q, const int32_t* __restrict__ src_rows, const int32_t* __restrict__ q_pos, const int32_t* __restrict__ cu_q,
    int n_requests, const T* __restrict__ k_pool, const T* __restrict__ v_pool, int n_blocks, const int32_t* __restrict__ block_tab,
    const cc_segment* __restrict__ segs, const int32_t* __restrict__ req_seg_off, int hq, int hkv, InvFreq inv_freq,
    T* __restrict__ out, float* __restrict__ lse, ValueSource vs) {
  const int j = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  if (j >= cu_q[n_requests]) return;                  // (the list may be shorter than its capacity)
  int lo = 0, hi = n_requests;                        // cu_q[lo] <= j < cu_q[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu_q[mid] <= j) lo = mid; else hi = mid;
  }
  const int r = lo, p = q_pos[j], kvh = h / (hq / hkv);
  const bool own = lane < D / 2;
  float qx = 0.f, qy = 0.f;
  if (own) {
    const T* qp = q + (static_cast<size_t>(src_rows != nullptr ? src_rows[j] : j) * hq + h) * D;
    const float x = to_float(qp[lane]), y = to_float(qp[lane + D / 2]);
    float c, s;
    rot_cos_sin(p, inv_freq.f[lane], &c, &s);
    qx = x * c - y * s;
    qy = y * c + x * s;
  }
  const float scale = rsqrtf(static_cast<float>(D));
  float m = -INFINITY, z = 0.f, ox = 0.f, oy = 0.f;
  for (int s = req_seg_off[r]; s < req_seg_off[r + 1]; ++s) {
    const cc_segment ks = segs[s];
    const int n_vis = min(ks.n_tokens, p - ks.logical_start + 1);
    for (int t = 0; t < n_vis; ++t) {
      const int blk = block_tab[ks.tab_off + t / kBlock];
      if (blk < 0 || blk >= n_blocks) continue;
      const T* kp = k_pool + ((static_cast<size_t>(blk) * hkv + kvh) * kBlock + t % kBlock) * D;
      const float logit = wave_sum(own ? qx * to_float(kp[lane]) + qy * to_float(kp[lane + D / 2]) : 0.f) * scale;
      if (logit > m) {                                // (the same in all lanes)
        const float a = expf(m - logit);
        z *= a; ox *= a; oy *= a;
        m = logit;
      }
      const float e = logit == -INFINITY ? 0.f : expf(logit - m);
      z += e;
      if (own) {
        const T* vp = value_block<T>(v_pool, static_cast<const T*>(vs.v_shared), vs.n_shared_blocks, vs.v_map, blk,
                                     static_cast<size_t>(hkv) * D * kBlock) + static_cast<size_t>(kvh) * D * kBlock + t % kBlock;
        ox += e * to_float(vp[static_cast<size_t>(lane) * kBlock]);
        oy += e * to_float(vp[static_cast<size_t>(lane + D / 2) * kBlock]);
      }
    }
  }
  const float inv = z == 0.f ? 0.f : 1.f / z;         // (a row without keys: zeros, and -inf for the logarithm)
  if (own) {
    T* op = out + (static_cast<size_t>(j) * hq + h) * D;
    op[lane] = from_float<T>(ox * inv);
    op[lane + D / 2] = from_float<T>(oy * inv);
  }
  if (lse != nullptr && lane == 0) lse[static_cast<size_t>(j) * hq + h] = z == 0.f ? -INFINITY : m + logf(z);
}

size_t append_bytes(const cc_ctx* ctx, int n_q_tot, int max_q_per_req, int n_requests, int max_ctx_tokens, int max_segs_per_req) {
  if (ctx->impl == CC_IMPL_SCALAR || n_q_tot == 0) return 0;
  const AppendPlan p = plan_append(ctx, max_q_per_req, n_requests, max_ctx_tokens, max_segs_per_req);
  return (static_cast<size_t>(n_q_tot) * ctx->cfg.n_q_heads * p.n_splits * (ctx->cfg.head_dim + 2) + n_q_tot) * sizeof(float);
}

template <typename T, int D>
static void launch_append_t(const cc_ctx* ctx, const AppendArgs& a, const AppendPlan& p, int n_q_tot, hipStream_t stream) {
  const dim3 grid(p.n_splits * p.col_groups, a.hkv, a.n_requests);
  if (p.nc == 1) hipLaunchKernelGGL((append_split_kernel<T, D, 1>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
  else if (p.nc == 2) hipLaunchKernelGGL((append_split_kernel<T, D, 2>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
  else hipLaunchKernelGGL((append_split_kernel<T, D, 4>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
  if (p.n_splits > 1) hipLaunchKernelGGL((append_join_kernel<T, D>), dim3(n_q_tot, a.hq), dim3(256), 0, stream, a);
}

void launch_append_attention(const cc_ctx* ctx, const void* q, const int32_t* src_rows, const int32_t* q_pos, const int32_t* cu_q, int n_q_tot,
                             int max_q_per_req, const void* k_pool, const void* v_pool, int n_blocks, const int32_t* block_tab,
                             const cc_segment* segs, const int32_t* req_seg_off, int n_requests, int max_ctx_tokens, int max_segs_per_req,
                             void* out, float* lse, void* workspace, hipStream_t stream, const ValueSource& vs) {
  const bool bf = ctx->cfg.dtype == CC_BF16;
  const int d = ctx->cfg.head_dim, hq = ctx->cfg.n_q_heads, hkv = ctx->cfg.n_kv_heads;
  if (ctx->impl == CC_IMPL_SCALAR) {
#define CC_LAUNCH(T, D)                                                                                                          \
  hipLaunchKernelGGL((append_scalar_kernel<T, D>), dim3(n_q_tot, hq), dim3(64), 0, stream, static_cast<const T*>(q), src_rows, q_pos, \
                     cu_q, n_requests, static_cast<const T*>(k_pool), static_cast<const T*>(v_pool), n_blocks, block_tab, segs,      \
                     req_seg_off, hq, hkv, ctx->inv_freq, static_cast<T*>(out), lse, vs)
    if (bf && d == 128) CC_LAUNCH(bf16_t, 128);
    else if (bf) CC_LAUNCH(bf16_t, 64);
    else if (d == 128) CC_LAUNCH(float, 128);
    else CC_LAUNCH(float, 64);
#undef CC_LAUNCH
    return;
  }
  const AppendPlan p = plan_append(ctx, max_q_per_req, n_requests, max_ctx_tokens, max_segs_per_req);
  float* part_o = static_cast<float*>(workspace);
  float* part_ml = part_o + static_cast<size_t>(n_q_tot) * hq * p.n_splits * d;
  const AppendArgs a{q, src_rows, q_pos, cu_q, k_pool, v_pool, block_tab, segs, req_seg_off, out, lse, vs, n_requests, n_blocks, hq, hkv,
                     p.n_splits, p.split_pages, part_o, part_ml, reinterpret_cast<int32_t*>(part_ml + static_cast<size_t>(n_q_tot) * hq * p.n_splits * 2)};
  if (bf && d == 128) launch_append_t<bf16_t, 128>(ctx, a, p, n_q_tot, stream);
  else if (bf) launch_append_t<bf16_t, 64>(ctx, a, p, n_q_tot, stream);
  else if (d == 128) launch_append_t<float, 128>(ctx, a, p, n_q_tot, stream);
  else launch_append_t<float, 64>(ctx, a, p, n_q_tot, stream);
}

}  // namespace cc
