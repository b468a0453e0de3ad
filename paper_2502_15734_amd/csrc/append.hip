// cc_append_attention: causal attention of the last rows of each request over its whole paged context, a few rows or one at a time.
//
// Bound by the bytes of the keys and values: a page of 16 tokens is read once for all rows and all heads of its group, and a row brings
// 2 G multiply-adds per element read (G query heads on a KV head), far below what the matrix cores take.  So the rows and heads
// of a group are the 16 columns of a matrix instruction (most of them empty when one token is written: they cost nothing), and the keys
// are divided: a workgroup takes one (request, KV head, 16 columns, range of pages), its four wavefronts every fourth tile of
// the range, and merge at the end; a second kernel joins the ranges of a row.
//
// Layout: S^T = K Q^T and O^T = V^T P^T with lane = (n = lane % 16, g = lane / 16), column n.  No operand passes through LDS: the
// contraction order of either product is free as long as both operands agree.  bf16, a tile of two pages: of the first product's two
// 16-key blocks block t takes, as row 4 g' + j, token 8 (g' % 2) + 4 t + j of page g' / 2, so that lane (n, g) ends up with the
// logits of tokens 8 (g % 2) .. + 7 of page g / 2: as the second product's 32-token operand they meet a 16-byte piece of a
// dimension-major V row.  fp32, a tile of one page: steps of four tokens, as in qk_f32.hip.
//
// One pass: o = sum_t 2^(s_t - m) v_t and l = sum_t 2^(s_t - m), where the reference m of a column is shared by its lane groups and moves (o and l times
// 2^(old - new)) only when a logit is more than kSlack above it.  m, l and o are fp32.  Queries, once they are turned to their position, and weights are what
// the matrix instructions take: bf16 as the sum of two, so that the output's own rounding is the only one to 8 bits and a row's error does not depend on how many
// rows its request brings (rms against 64 bits 0.0017 of the output, 0.0029 with one each).  Where the bytes of the keys are the bound that is next to free (one row
// over 700 tokens 12.3 -> 12.7 us, 32 requests 115.2 -> 115.6, 16 x 5 rows of 64 heads 79.6 -> 82.6); where the products are, there are twice as many of them (500
// rows over 16 000 tokens 158 -> 247; with two of the queries alone 197, of the weights alone 207, and 0.0024 either way).
//
// 32 heads on 8 of 128, bf16: 32 requests of one row over 1500 to 6700 tokens 115 us (4.5 TB/s of keys and values; a copy of 4 GiB moves 4.7), one
// row over 130 000 tokens 105 us (5.1 TB/s), one over 700 tokens 12.7 us, of which two launches take 5 and the chain of dependent loads (segments, page
// table, page, parts) most of the rest.
#include <algorithm>
#include <cstddef>
#include <type_traits>

#include "device_util.h"
#include "scatter.h"

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
  // division of the work
  int n_splits, split_pages, col_groups;
  float *part_o, *part_ml;            // [row][head][split][D], [row][head][split][2]
  // rows to write in front of the attention (k_new null: they are written already)
  const void *k_new, *v_new;
  const int32_t* slot_map;
  int32_t* row_splits;                // [row] ranges its request has (1: the output is written)
};

constexpr int kNowhere = -(1 << 30);  // position of an entry that is no page
struct Page {
  int blk, pos0, n_valid, value;      // value: block of the own pool, or -1 - block of the shared one
};

__device__ __forceinline__ int pages_of(int tokens) { return (max(tokens, 0) + kBlock - 1) / kBlock; }

// Pages [first, first + kWindow) of a request into list[] (thread i: page first + i), those behind its last one with n_valid 0;
// returns the number of pages the request has; *end_pos: the position behind its last token.  Thread i also takes segment i of 256 at a time, whose page counts are scanned.
__device__ __forceinline__ int list_pages(const AppendArgs& a, int s_begin, int s_end, int first, Page* list, int4* segs, int* seg_end,
                                          int* wave_pages, int* end_pos) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, want = first + tid;
  Page page{0, kNowhere, 0, 0};
  int total = 0;
  for (int s0 = s_begin; s0 < s_end; s0 += 256) {
    const int s = s0 + tid;
    int4 mine{0, 0, 0, 0};
    if (s < s_end) {                                              // start, tokens; table offset, (rows)
      static_assert(offsetof(cc_segment, logical_start) % alignof(int2) == 0 && sizeof(cc_segment) % alignof(int2) == 0, "these pieces are aligned");
      const int2* at = reinterpret_cast<const int2*>(&a.segs[s].logical_start);
      const int2 head = at[0], tail = at[1];
      mine = make_int4(head.x, head.y, tail.x, tail.y);
    }
    const int n = pages_of(mine.y);
    if (s == s_end - 1) *end_pos = mine.x + max(mine.y, 0);
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
      if (blk >= 0 && blk < a.n_blocks) {
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

// The request's new rows (up to kWriteRows) whose tokens lie in the `here` listed pages go into their slots: keys turned to their positions, values into
// their column of the page.  The keys are divided by position, so one workgroup of each KV head writes a row, the one that goes on to read it (a
// token's position may also fall behind the end of the segment in front, on the same page entry: then two write the same).  others: also
// those whose position no segment holds.
constexpr int kWriteRows = 16;
template <typename T, int D>
__device__ __forceinline__ void write_rows(const AppendArgs& a, const InvFreq& inv_freq, const Page* list, int here, bool others, int end_pos, int row0, int n_rows,
                                           int kvh) {
  __shared__ int owned[kWriteRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid < kWriteRows) owned[tid] = 0;
  __syncthreads();
  const int pos0 = tid < here ? list[tid].pos0 : kNowhere;
  for (int i = 0; i < n_rows; ++i) {
    const int p = a.q_pos[row0 + i];
    if ((p >= pos0 && p - pos0 < kBlock) || (others && tid == 0 && (p < 0 || p >= end_pos))) owned[i] = 1;
  }
  __syncthreads();
  for (int i = wave; i < n_rows; i += 4) {
    if (owned[i] == 0) continue;
    const int row = row0 + i, p = a.q_pos[row], slot = a.slot_map[row], src = a.src_rows != nullptr ? a.src_rows[row] : row;
    if (slot < 0 || slot >= a.n_blocks * kBlock || lane >= D / 2) continue;
    const size_t from = (static_cast<size_t>(src) * a.hkv + kvh) * D, head = (static_cast<size_t>(slot / kBlock) * a.hkv + kvh) * (kBlock * D);
    const T *kn = static_cast<const T*>(a.k_new) + from, *vn = static_cast<const T*>(a.v_new) + from;
    const float x = to_float(kn[lane]), y = to_float(kn[lane + D / 2]);
    float c, s;
    if (sizeof(T) == 2) rot_cos_sin_fast(p, inv_freq.f[lane], &c, &s);           // (the result is rounded to bf16)
    else rot_cos_sin(p, inv_freq.f[lane], &c, &s);
    T* ko = const_cast<T*>(static_cast<const T*>(a.k_pool)) + head + slot % kBlock * D;
    T* vo = const_cast<T*>(static_cast<const T*>(a.v_pool)) + head + slot % kBlock;
    ko[lane] = from_float<T>(x * c - y * s);
    ko[lane + D / 2] = from_float<T>(y * c + x * s);
    vo[lane * kBlock] = vn[lane];
    vo[(lane + D / 2) * kBlock] = vn[lane + D / 2];
  }
  __syncthreads();                                     // (the workgroup's loads behind it see the rows)
}

// x as the sum of two bf16.  Part 0: the upper 16 bits of the number in front of x (towards 0), x becomes the rest, whose nearest bf16 is part 1.  So neither
// part of a number is 0 - a product with an infinite factor is one infinity and not a difference of two or 0 x infinity - and both parts of 0 are: a masked
// key's weight takes nothing of its value, however large.  POSITIVE: x has no sign (NaN may).
template <bool POSITIVE = false>
__device__ __forceinline__ bf16_t take_part(float& x, int part) {
  if (part == 1) return static_cast<bf16_t>(x);
  const uint32_t sign = POSITIVE ? 0u : __float_as_uint(x) & 0x80000000u;
  const float up = __uint_as_float((__builtin_elementwise_sub_sat(__float_as_uint(x) ^ sign, 1u) & 0xffff0000u) | sign);
  x -= up;
  return static_cast<bf16_t>(up);
}

template <typename T, int D> struct Tile;           // operands of one tile of keys

template <int D> struct Tile<bf16_t, D> {
  static constexpr int kPages = 2, kTok = 8;        // pages of a tile; tokens of it that a lane holds
  static constexpr int kParts = 2;                  // of queries and weights, whose sum has 16 bits of them: the bytes of the keys bound this kernel, not its products
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
  __device__ __forceinline__ void logits(const Piece (&q)[kParts][D / 32], float (&s)[kTok]) const {
    f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int x = 0; x < kParts; ++x)
#pragma unroll
        for (int t = 0; t < 2; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][i], q[x][i], acc[t], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < kTok; ++e) s[e] = acc[e >> 2][e & 3];
  }
  static __device__ __forceinline__ f32x4 add_values(const Piece& v, const Piece& p, f32x4 o) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o, 0, 0, 0);
  }
  template <bool POSITIVE>
  static __device__ __forceinline__ Piece piece(float (&x)[8], int part) {
    Piece w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = take_part<POSITIVE>(x[e], part);
    return w;
  }
};

template <int D> struct Tile<float, D> {
  static constexpr int kPages = 1, kTok = 4, kParts = 1;
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
  __device__ __forceinline__ void logits(const Piece (&q)[kParts][D / 16], float (&s)[kTok]) const {
    f32x4 acc[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0][i][e], q[0][i][e], acc[e], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < kTok; ++e) s[e] = (acc[0][e] + acc[1][e]) + (acc[2][e] + acc[3][e]);
  }
  static __device__ __forceinline__ f32x4 add_values(const Piece& v, const Piece& p, f32x4 o) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], p[e], o, 0, 0, 0);
    return o;
  }
  template <bool>
  static __device__ __forceinline__ Piece piece(const float (&x)[4], int) { return Piece{x[0], x[1], x[2], x[3]}; }
};

// What a workgroup does.  Workgroups go to the eight XCDs in turn; the column groups of one range of keys, which read the same pages, follow
// each other on one XCD, whose L2 then has them.
struct Unit {
  int split, kvh, req, col_group;     // req: n_requests and more: nothing
};
__device__ __forceinline__ Unit unit_of(const AppendArgs& a) {
  const unsigned at = blockIdx.x / 8, u = blockIdx.x % 8 + 8 * (at / a.col_groups), rest = u / a.n_splits;
  return Unit{static_cast<int>(u % a.n_splits), static_cast<int>(rest % a.hkv), static_cast<int>(rest / a.hkv), static_cast<int>(at % a.col_groups)};
}
// where the result of a range goes: the parts, or the output if the request has no other
template <typename T, int D>
__device__ __forceinline__ void store_result(const AppendArgs& a, size_t at, int split, int n_splits, int d, const f32x4& v, float top, float sum) {
  if (n_splits == 1) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;                 // (no key: zeros, and -inf for the logarithm)
    T o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = from_float<T>(v[e] * inv);
    T* op = static_cast<T*>(a.out) + at * D + d;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(op) = *reinterpret_cast<const uint2*>(o);
    else *reinterpret_cast<uint4*>(op) = *reinterpret_cast<const uint4*>(o);
    if (d == 0 && a.lse != nullptr) a.lse[at] = sum == 0.f ? -INFINITY : top / kLog2e + logf(sum);
  } else {
    *reinterpret_cast<f32x4*>(a.part_o + (at * a.n_splits + split) * D + d) = v;
    if (d == 0) *reinterpret_cast<float2*>(a.part_ml + (at * a.n_splits + split) * 2) = make_float2(top, sum);
  }
}

// One (range of pages, KV head and 16 columns, request).  Column c is head c % G of the request's row c / G.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void append_split_kernel(AppendArgs a, InvFreq inv_freq) {
  typedef Tile<T, D> Keys;
  typedef typename Keys::Piece Piece;
  constexpr int kTok = Keys::kTok, kPer = 16 / sizeof(T), kQ = D / 4 / kPer;      // elements of a piece; pieces of a query a lane holds
  constexpr int kRow = D + 4;                                                    // (a column of the outputs in LDS: banks apart)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const Unit unit = unit_of(a);
  const int r = unit.req, kvh = unit.kvh, split = unit.split, group = a.hq / a.hkv;
  if (r >= a.n_requests) return;
  const int col0 = unit.col_group * 16, row0 = a.cu_q[r], n_cols = (a.cu_q[r + 1] - row0) * group;
  if (col0 >= n_cols) return;
  const int s_begin = a.req_seg_off[r], s_end = a.req_seg_off[r + 1];

  union Shared {
    struct { Page list[kWindow]; int4 segs[256]; int seg_end[256]; int wave_pages[4]; int end_pos; } in;
    struct { float o[4][16][kRow]; float m[4][16], l[4][16]; } out;
  };
  __shared__ Shared sh;

  // ---- positions of the columns, and the rows themselves (loads first, turned later)
  // (columns behind the last repeat its row)
  Piece q[Keys::kParts][kQ];
  const int my_col = min(col0 + n, n_cols - 1), pos = a.q_pos[row0 + my_col / group];
  {
    const int row = row0 + my_col / group;
    const int src = a.src_rows != nullptr ? a.src_rows[row] : row;
    const T* qp = static_cast<const T*>(a.q) + (static_cast<size_t>(src) * a.hq + kvh * group + my_col % group) * D + kPer * g;
#pragma unroll
    for (int i = 0; i < kQ; ++i) q[0][i] = *reinterpret_cast<const Piece*>(qp + 4 * kPer * i);
  }
  const size_t block_elems = static_cast<size_t>(a.hkv) * kBlock * D, head_off = static_cast<size_t>(kvh) * kBlock * D;
  const T *k_pool = static_cast<const T*>(a.k_pool), *v_pool = static_cast<const T*>(a.v_pool), *v_shared = static_cast<const T*>(a.vs.v_shared);
  float m = -3.4028235e38f, l = 0.f;
  f32x4 o[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int first_page = split * a.split_pages;
  int n_pages = list_pages(a, s_begin, s_end, first_page, sh.in.list, sh.in.segs, sh.in.seg_end, sh.in.wave_pages, &sh.in.end_pos);
  if (first_page >= max(n_pages, 1)) return;                                        // (the same in all wavefronts)
  const int n_splits = min((max(n_pages, 1) + a.split_pages - 1) / a.split_pages, a.n_splits);
  const int end_page = split == a.n_splits - 1 ? n_pages : min(n_pages, first_page + a.split_pages);

  const int p_min = wave_min_i(pos), p_max = wave_max_i(pos);             // (waited for behind the list's loads)

  // ---- the queries at their positions, in units of the logits' powers of two
  const float scale = rsqrtf(static_cast<float>(D)) * kLog2e;
#pragma unroll
  for (int i = 0; i < kQ / 2; ++i) {
    float x[kPer], y[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      float cs, sn;
      const double freq = inv_freq.f[4 * kPer * i + kPer * g + e];
      if (sizeof(T) == 2) rot_cos_sin_fast(pos, freq, &cs, &sn);          // (16 bits of the result are kept)
      else rot_cos_sin(pos, freq, &cs, &sn);
      const float u = to_float(q[0][i][e]), w = to_float(q[0][i + kQ / 2][e]);
      x[e] = (u * cs - w * sn) * scale;
      y[e] = (w * cs + u * sn) * scale;
    }
#pragma unroll
    for (int part = 0; part < Keys::kParts; ++part) {
      q[part][i] = Keys::template piece<false>(x, part);
      q[part][i + kQ / 2] = Keys::template piece<false>(y, part);
    }
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
    float s[kTok];
    t.logits(q, s);
    if (!whole) {
      const int seen = min(held.n_valid - tok0, pos - first + 1);
#pragma unroll
      for (int e = 0; e < kTok; ++e) s[e] = e < seen ? s[e] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int e = 1; e < kTok; ++e) top = fmaxf(top, s[e]);
    if (__any(top > m + kSlack)) {
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float m_new = fmaxf(m, top), f = exp2f(m - m_new);
      m = m_new;
      l *= f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[i] *= f;
    }
    float p[kTok], sum = 0.f;
#pragma unroll
    for (int e = 0; e < kTok; ++e) { p[e] = __builtin_amdgcn_exp2f(s[e] - m); sum += p[e]; }
    l += sum;
    if (!apart) {
#pragma unroll
      for (int part = 0; part < Keys::kParts; ++part) {
        const Piece w = Keys::template piece<true>(p, part);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] = Keys::add_values(t.v[i], w, o[i]);
      }
    } else {
      // 0 x value would reach the columns that do not see it: one column at a time
#pragma unroll 1
      for (int k = 0; k < 16; ++k) {
        const int seen = __shfl(pos, k, 16) - first + 1;
        float only[kTok];
#pragma unroll
        for (int e = 0; e < kTok; ++e) only[e] = n == k ? p[e] : 0.f;
        Piece w[Keys::kParts];
#pragma unroll
        for (int part = 0; part < Keys::kParts; ++part) w[part] = Keys::template piece<true>(only, part);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          Piece v = t.v[i];
#pragma unroll
          for (int e = 0; e < kTok; ++e)
            if (e >= seen) v[e] = static_cast<T>(0.f);
          f32x4 add = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int part = 0; part < Keys::kParts; ++part) add = Keys::add_values(v, w[part], add);
          if (n == k) o[i] += add;
        }
      }
    }
  };

  // ---- the keys: every fourth tile of the window is this wavefront's
  for (int at = first_page;;) {
    const int here = min(end_page - at, kWindow);
    if (a.k_new != nullptr) write_rows<T, D>(a, inv_freq, sh.in.list, here, split == 0 && at == first_page, s_end > s_begin ? sh.in.end_pos : 0, row0, n_cols / group, kvh);
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
    list_pages(a, s_begin, s_end, at, sh.in.list, sh.in.segs, sh.in.seg_end, sh.in.wave_pages, &sh.in.end_pos);
  }

  // ---- the four wavefronts' sums, and the result of this range
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (g == 0) { sh.out.m[wave][n] = m; sh.out.l[wave][n] = l; }
#pragma unroll
  for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(&sh.out.o[wave][n][16 * i + 4 * g]) = o[i];
  __syncthreads();
  for (int i = tid; i < 16 * (D / 4); i += 256) {
    const int k = i / (D / 4), d = i % (D / 4) * 4, col = col0 + k;
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
      store_result<T, D>(a, at, split, n_splits, d, v, top, sum);
      if (split == 0 && d == 0 && kvh == 0 && col % group == 0) a.row_splits[row] = n_splits;
    }
  }
  __syncthreads();
}

// ---- many columns -------------------------------------------------------------------------------
// A draft to check or a further question: 17 columns and more (rows times heads of a group) share the keys.  Workgroup = 32 CW columns x a range
// of pages; tiles of 64 keys go through LDS (two images, loads that write LDS while the other is multiplied, one barrier per tile), so that a page is read
// once for all its columns.  CW = 4: each wavefront multiplies its 32 columns with all 64 keys; CW = 2: two wavefronts per 32 columns take 32
// keys each and meet at the end.  Few columns are bound by the bytes (16 requests of 5 rows over 1000 to 8000 tokens, 64 heads on 8: 82 us, 3.6 TB/s), from some
// hundred on by the matrix instructions: 500 rows of 32 heads over 16 000 tokens take 247 us, of them about 230 in this kernel (264 GFLOP in two parts, 1.15 PF),
// with the matrix cores busy for 72 % of its cycles, and the rest in what lies between two products of a tile (maximum, mask, barrier) that the
// other workgroup of the compute unit does not cover.
//
// v_mfma_f32_32x32x16_bf16, S^T = K Q^T and O^T = V^T P^T with lane = (n = lane % 32, h = lane / 32), column n.  As above the key rows are
// ordered so that a lane's logits are the tokens 8 h .. 8 h + 7 of each page: row 8 a + 4 b + c of a 32-key block is token
// 8 b + 4 (a % 2) + c of page a / 2.  Image (16-byte pieces):
//   K  token t of the tile, piece ch of its row:        t * D / 8 + (ch ^ f(t)),  f(t) = t % 16, or t / 2 % 8 if D is 64
//   V  page, dim d, half h of its row of 16 tokens:     8 D + page * 2 D + h * D + (d ^ 4 h)
// (sixteen lanes of a read meet the sixteen 16-byte columns of the banks)
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
constexpr int kTileKeys = 64, kTilePages = kTileKeys / kBlock;

// 64 lanes x 16 bytes from memory straight into LDS: what lane L reads at from + at lands at `to` + 16 L.  The compiler does not know what
// it writes (it would wait for it in front of every read of LDS); vmcnt counts it.
__device__ __forceinline__ void load_to_lds(uint32_t at, const bf16_t* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(at), "s"(from), "s"(to) : "memory", "m0");
}

// (SHARED: values may lie in a second pool)
template <int D, int CW, bool SHARED>
__global__ __launch_bounds__(256, 2) void append_tile_kernel(AppendArgs a, InvFreq inv_freq) {
  constexpr int KS = 4 / CW, kStage = D / 32, kImage = 16 * D;          // pieces a thread stages of K (and of V); pieces of an image
  constexpr int kBlocks = 2 / KS;                                      // 32-key blocks of a tile that are this wavefront's
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
  const int cw = wave % CW, ks = wave / CW;
  const Unit unit = unit_of(a);
  const int r = unit.req, kvh = unit.kvh, split = unit.split, group = a.hq / a.hkv;
  if (r >= a.n_requests) return;
  const int row0 = a.cu_q[r], n_cols = (a.cu_q[r + 1] - row0) * group, wg_col = unit.col_group * 32 * CW;
  if (wg_col >= n_cols) return;
  const int s_begin = a.req_seg_off[r], s_end = a.req_seg_off[r + 1];

  __shared__ u32x4 image[2 * kImage];
  __shared__ Page list[kWindow];
  __shared__ int odd[kWindow / kTilePages];
  __shared__ int2 edge_pos[4];
  struct Scratch { int4 segs[256]; int seg_end[256]; int wave_pages[4]; };
  __shared__ int end_pos;
  Scratch& scratch = *reinterpret_cast<Scratch*>(image);               // (while a list is made no image is in use)

  const int col = wg_col + 32 * cw + n, my_col = min(col, n_cols - 1), row = row0 + my_col / group, pos = a.q_pos[row];
  u32x4 raw[D / 16];
  {
    const int src = a.src_rows != nullptr ? a.src_rows[row] : row;
    const bf16_t* qp = static_cast<const bf16_t*>(a.q) + (static_cast<size_t>(src) * a.hq + kvh * group + my_col % group) * D + 8 * h;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) raw[i] = *reinterpret_cast<const u32x4*>(qp + 16 * i);
  }
  const int first_page = split * a.split_pages;
  const int n_pages = list_pages(a, s_begin, s_end, first_page, list, scratch.segs, scratch.seg_end, scratch.wave_pages, &end_pos);
  if (first_page >= max(n_pages, 1)) return;
  const int n_splits = min((max(n_pages, 1) + a.split_pages - 1) / a.split_pages, a.n_splits);
  const int end_page = split == a.n_splits - 1 ? n_pages : min(n_pages, first_page + a.split_pages);
  // positions of the wavefront's columns and of the workgroup's (columns behind the last repeat its row)
  const int p_min = wave_min_i(pos), p_max = wave_max_i(pos);
  if (lane == 0) edge_pos[wave] = make_int2(p_min, p_max);
  __syncthreads();
  const int p_first = min(min(edge_pos[0].x, edge_pos[1].x), min(edge_pos[2].x, edge_pos[3].x));
  const int p_last = max(max(edge_pos[0].y, edge_pos[1].y), max(edge_pos[2].y, edge_pos[3].y));

  const size_t block_elems = static_cast<size_t>(a.hkv) * kBlock * D, head_off = static_cast<size_t>(kvh) * kBlock * D;
  const bf16_t *k_pool = static_cast<const bf16_t*>(a.k_pool) + head_off, *v_pool = static_cast<const bf16_t*>(a.v_pool) + head_off;
  const bf16_t* v_shared = static_cast<const bf16_t*>(a.vs.v_shared) + head_off;
  // A wavefront fetches the same 64 pieces of every 256 / (2 D)-th page straight into LDS, where lane L's piece lands 16 L behind a common address: the
  // image's order is made by what a lane reads, and page numbers are a wavefront's.
  constexpr int kApart = 128 / D;                                     // pages between a thread's
  const int pg0 = wave * 64 / (2 * D), place = tid % (2 * D), half = place / D;          // (place: of the thread's piece in its page's image; half: of the tokens of a V piece)
  const int token = place / (D / 8);
  auto turn = [](int t) { return D == 128 ? t & 15 : (t >> 1) & 7; };
  const uint32_t get_k = (token * (D / 8) + (place % (D / 8) ^ turn(token))) * 16, get_v = (2 * (place % D ^ (4 * half)) + half) * 16;
  typedef __attribute__((address_space(3))) u32x4 lds_piece;
  const uint32_t put = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_piece*)image)) + wave * 1024);
  // What the loop needs of the window's tiles, lane t of tile t: where its pages are, and
  //   flag 1: slots of it hold no key of this range,  flag 2: some column of the workgroup does not see all of it
  int w_blk[kTilePages], w_value[SHARED ? kTilePages : 1], w_flags;
  auto note_window = [&](int here) __attribute__((always_inline)) {
    w_flags = 0;
#pragma unroll
    for (int j = 0; j < kTilePages; ++j) {
      const int at = kTilePages * lane + j;
      const Page p = list[at];
      w_blk[j] = p.blk;
      if (SHARED) w_value[j] = p.value;
      w_flags |= at >= here || p.n_valid < kBlock ? 1 : 0;
      w_flags |= at < here && p.pos0 + kBlock - 1 > p_first ? 2 : 0;
    }
  };
  auto of_page = [&](const int* w, int j, int t) __attribute__((always_inline)) {       // entry of this wavefront's j-th page of tile t
    return __builtin_amdgcn_readlane(kApart == 1 || pg0 == 0 ? w[kApart * j] : w[kApart * j + kApart - 1], t);
  };
  // tile t into image `buf`
  auto fetch = [&](int buf, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kStage; ++j) {
      const int blk = of_page(w_blk, j, t), value = SHARED ? of_page(w_value, j, t) : blk;
      const bf16_t* from = !SHARED || value >= 0 ? v_pool + value * block_elems : v_shared + (-1 - value) * block_elems;
      const uint32_t to = put + buf * (kImage * 16) + j * kApart * 32 * D;
      load_to_lds(get_k, k_pool + blk * block_elems, to);
      load_to_lds(get_v, from, to + 128 * D);
    }
  };
  // ... until it is there.  Values in slots without a key become zeros (0 x what lies there would be a product).  A tile with values that are not finite
  // and that only some columns see is set aside (odd): 0 x such a value would reach the others.
  auto arrive = [&](int buf, int t, int flags, int here) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (flags != 0) {
      bool any = false;
#pragma unroll
      for (int j = 0; j < kStage; ++j) {
        const int at = kTilePages * t + pg0 + j * kApart, left = (at < here ? list[at].n_valid : 0) - 8 * half;     // of this thread's eight tokens
        auto keep = [&](int e) { return (e < left ? 0xffffu : 0u) | (e + 1 < left ? 0xffff0000u : 0u); };
        auto bad = [](uint32_t v) { return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u; };
        u32x4& v = image[buf * kImage + 8 * D + wave * 64 + lane + j * kApart * 2 * D];
        v &= u32x4{keep(0), keep(2), keep(4), keep(6)};
        any |= bad(v[0]) || bad(v[1]) || bad(v[2]) || bad(v[3]);
      }
      if ((flags & 2) && __any(any) && lane == 0) odd[t] = 1;
    }
  };

  // ---- the queries at their positions, in units of the logits' powers of two
  const float scale = rsqrtf(static_cast<float>(D)) * kLog2e;
  bf16x8 q[2][D / 16];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const bf16x8 x = __builtin_bit_cast(bf16x8, raw[i]), y = __builtin_bit_cast(bf16x8, raw[i + D / 32]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float cs, sn;
      rot_cos_sin_fast(pos, inv_freq.f[16 * i + 8 * h + e], &cs, &sn);
      const float u = to_float(x[e]), w = to_float(y[e]);
      float first = (u * cs - w * sn) * scale, second = (w * cs + u * sn) * scale;
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        q[part][i][e] = take_part(first, part);
        q[part][i + D / 32][e] = take_part(second, part);
      }
    }
  }
  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = 0.f, l = 0.f;
  float limit = -INFINITY;                                            // how far a logit may be above m: kSlack once the column has seen a key and m is a reference of its own
  // byte of this lane's key operand in an image: row of the block as token of its two pages; piece 2 kk + h is this one's, bits of kk flipped
  const int k_row = (n >> 4) * kBlock + ((n >> 2) & 1) * 8 + ((n >> 3) & 1) * 4 + (n & 3);
  const int k_byte = ((ks * kBlocks * 32 + k_row) * (D / 8) + (h ^ turn(k_row))) * 16, v_byte = (8 * D + ks * kBlocks * 4 * D + h * D + (n ^ (4 * h))) * 16;

  // One tile.  ODD: one that was set aside.  i: its first entry of the list, of which `here` count.
  // In the order  S(0), S(1) with the exponentials of block 0 under its products, P V(0) with those of block 1, P V(1), four operands read ahead; the
  // steps are fenced, because the compiler by itself reads every operand right in front of its product and takes the exponentials together.
  auto compute = [&](auto set_aside, const u32x4* img, int i, int here, int flags) __attribute__((always_inline)) {
    constexpr bool ODD = decltype(set_aside)::value;
    constexpr int kSteps = D / 16, kAhead = 2;   // pairs of products of a block; operands in flight
    const int b0 = ks * kBlocks;                                       // this wavefront's first 32-key block
    // (the operands' addresses are made here again: kept over the loop they would cost a register each)
    const char* bytes = reinterpret_cast<const char*>(img);
    int k_at = k_byte;
    asm volatile("" : "+v"(k_at));
    auto key = [&](int b, int kk) __attribute__((always_inline)) { return *reinterpret_cast<const bf16x8*>(bytes + (k_at ^ (32 * kk)) + b * 64 * D); };
    auto value = [&](int b, int g, int j) __attribute__((always_inline)) { return *reinterpret_cast<const bf16x8*>(bytes + v_byte + (2 * b + g) * 32 * D + j * 512); };
    bf16x8 ahead[kAhead];                                              // operands of the next products, also over the masks and maxima between two blocks
    f32x16 s[kBlocks];
    bf16x8 w[kBlocks][2], rest[kBlocks][2];                            // the weights' parts
    // the logits less the reference of the column, which enters as the products' first summand
    auto fence = []() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
    auto first_summand = [&]() __attribute__((always_inline)) {          // (there are no registers to hold it)
      f32x16 x;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = -m;
      return x;
    };
    // weights of the two logits 2 x, 2 x + 1 of a block
    auto weigh = [&](int b, int x) __attribute__((always_inline)) {
      float x0 = __builtin_amdgcn_exp2f(s[b][2 * x]), x1 = __builtin_amdgcn_exp2f(s[b][2 * x + 1]);
      l += x0;
      l += x1;
      w[b][x / 4][2 * x % 8] = take_part<true>(x0, 0);
      w[b][x / 4][2 * x % 8 + 1] = take_part<true>(x1, 0);
      rest[b][x / 4][2 * x % 8] = take_part<true>(x0, 1);
      rest[b][x / 4][2 * x % 8 + 1] = take_part<true>(x1, 1);
    };
    // S(b); under it the weights of block `under` (-1: none)
    auto products = [&](int b, auto under) __attribute__((always_inline)) {
      if (ODD || b == 0)
#pragma unroll
        for (int kk = 0; kk < kAhead; ++kk) ahead[kk] = key(b, kk);
      fence();
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk) {
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[kk % kAhead], q[0][kk], kk == 0 ? first_summand() : s[b], 0, 0, 0);
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[kk % kAhead], q[1][kk], s[b], 0, 0, 0);
        if (kk + kAhead < kSteps) ahead[kk % kAhead] = key(b, kk + kAhead);
        else if (!ODD && b + 1 < kBlocks) ahead[kk % kAhead] = key(b + 1, kk + kAhead - kSteps);
        else if (!ODD) ahead[kk % kAhead] = value(0, (kk + kAhead - kSteps) / (D / 32), (kk + kAhead - kSteps) % (D / 32));
        if constexpr (decltype(under)::value >= 0)
#pragma unroll
          for (int x = 0; x < 8 / kSteps; ++x) weigh(decltype(under)::value, kk * (8 / kSteps) + x);
        fence();
      }
      if constexpr (decltype(under)::value >= 0)
#pragma unroll
        for (int g = 0; g < 2; ++g) {                                  // (the weights are made here, not behind the next branch)
          u32x4 bits = __builtin_bit_cast(u32x4, w[decltype(under)::value][g]), low = __builtin_bit_cast(u32x4, rest[decltype(under)::value][g]);
          asm volatile("" : "+v"(bits), "+v"(low));
          w[decltype(under)::value][g] = __builtin_bit_cast(bf16x8, bits);
          rest[decltype(under)::value][g] = __builtin_bit_cast(bf16x8, low);
        }
    };
    // masks, and the reference where a logit lies too far above it; done: blocks whose weights are made but not multiplied yet
    auto settle = [&](int b, int done) __attribute__((always_inline)) {
      if (flags != 0) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const int at = i + (b0 + b) * 2 + g;
          const Page p = list[at];
          const int seen = min((at < here ? p.n_valid : 0) - 8 * h, pos - (p.pos0 + 8 * h) + 1);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[b][8 * g + e] = e < seen ? s[b][8 * g + e] : -INFINITY;
        }
      }
      float top = s[b][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[b][e]);
      if (__ballot(top > limit) != 0) {
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const bool first = limit < 0.f && top > -INFINITY;
        top = first ? top : fmaxf(top, 0.f);                           // how far the reference moves
        limit = first ? kSlack : limit;
        const float f = first ? 0.f : exp2f(-top);
        m += top;
        l *= f;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) o[j] *= f;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[b][e] -= top;
#pragma unroll
        for (int d = 0; d < done; ++d)
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float x = (to_float(w[d][g][e]) + to_float(rest[d][g][e])) * f;
              w[d][g][e] = take_part<true>(x, 0);
              rest[d][g][e] = take_part<true>(x, 1);
            }
      }
    };
    // o += V P(b); under it the weights of block `under`
    auto add_values = [&](int b, auto under) __attribute__((always_inline)) {
      if constexpr (!ODD) {
        constexpr int kV = D / 16;                                     // products: two pages of D / 32 groups of dims
        fence();
#pragma unroll
        for (int x = 0; x < kV; ++x) {
          const int j = x % (D / 32);
          o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[x % kAhead], w[b][x / (D / 32)], o[j], 0, 0, 0);
          o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[x % kAhead], rest[b][x / (D / 32)], o[j], 0, 0, 0);
          if (x + kAhead < kV) ahead[x % kAhead] = value(b, (x + kAhead) / (D / 32), (x + kAhead) % (D / 32));
          else if (b + 1 < kBlocks) ahead[x % kAhead] = value(b + 1, (x + kAhead - kV) / (D / 32), (x + kAhead - kV) % (D / 32));
          if constexpr (decltype(under)::value >= 0)
#pragma unroll
            for (int y = 0; y < 8 / kV; ++y) weigh(decltype(under)::value, x * (8 / kV) + y);
          fence();
        }
      } else {
        // the values that are not finite leave the product and are added to the columns that see them
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            bf16x8 v = value(b, g, j);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fabsf(to_float(v[e])) < INFINITY ? v[e] : static_cast<bf16_t>(0.f);
            o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[b][g], o[j], 0, 0, 0);
            o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, rest[b][g], o[j], 0, 0, 0);
          }
          const int pg = (b0 + b) * 2 + g, first = list[i + pg].pos0;
          const bf16_t* values = reinterpret_cast<const bf16_t*>(img + 8 * D + pg * 2 * D);
#pragma unroll 1
          for (int t = 0; t < kBlock; ++t) {
            int dim0 = 4 * h;
            asm volatile("" : "+v"(dim0));
            float weight = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) weight = t % 8 == e ? to_float(w[b][g][e]) + to_float(rest[b][g][e]) : weight;
            weight = __shfl(weight, n + 32 * (t >> 3), 64);
            const bool sees = first + t <= pos;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const int d = 32 * j + 8 * (e >> 2) + dim0 + (e & 3);
                const float v = to_float(values[((t >> 3) * D + (d ^ (4 * (t >> 3)))) * 8 + (t & 7)]);
                if (sees && !(fabsf(v) < INFINITY)) o[j][e] += weight * v;
                asm volatile("" ::: "memory");                        // (one value in flight: this is rare, and registers are not)
              }
          }
        }
      }
    };
    constexpr std::integral_constant<int, -1> none;
    constexpr std::integral_constant<int, 0> first_block;
    constexpr std::integral_constant<int, 1> second_block;
    products(0, none);
    settle(0, 0);
    if constexpr (kBlocks == 2 && !ODD) {
      // (ahead of the compute unit's other workgroup while exponentials and products go together, behind it where there are products alone: 500 rows
      // over 16 000 tokens 252 -> 247)
      __builtin_amdgcn_s_setprio(1);
      products(1, first_block);
      settle(1, 1);
      add_values(0, second_block);
      __builtin_amdgcn_s_setprio(0);
      add_values(1, none);
    } else {
#pragma unroll
      for (int x = 0; x < 8; ++x) weigh(0, x);
      add_values(0, none);
      if constexpr (kBlocks == 2) {
        products(1, none);
        settle(1, 0);
#pragma unroll
        for (int x = 0; x < 8; ++x) weigh(1, x);
        add_values(1, none);
      }
    }
  };

  // ---- the keys, until no column of the workgroup sees them
  for (int at = first_page; at == first_page || at < end_page; at += kWindow) {
    if (at > first_page) list_pages(a, s_begin, s_end, at, list, scratch.segs, scratch.seg_end, scratch.wave_pages, &end_pos);
    if (tid < kWindow / kTilePages) odd[tid] = 0;
    const int in_range = min(end_page - at, kWindow);
    if (a.k_new != nullptr) write_rows<bf16_t, D>(a, inv_freq, list, in_range, split == 0 && at == first_page, s_end > s_begin ? end_pos : 0, row0, n_cols / group, kvh);
    // (pages are in the order of their positions; one that does not exist has no keys)
    const int here = __syncthreads_count(tid < in_range && (list[tid].pos0 <= p_last || list[tid].n_valid == 0)), tiles = (here + kTilePages - 1) / kTilePages;
    note_window(here);
    auto flags_of = [&](int t) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(w_flags, t); };
    if (tiles > 0) {
      fetch(0, 0);
      arrive(0, 0, flags_of(0), here);
    }
    __syncthreads();
    bool aside = false;                                               // (of this window some tile)
    for (int t = 0; t < tiles; ++t) {
      if (t + 1 < tiles) fetch((t + 1) & 1, t + 1);
      const int flags = flags_of(t);
      const bool skip = (flags & 2) != 0 && __builtin_amdgcn_readfirstlane(odd[t]) != 0;
      aside |= skip;
      if (!skip) compute(std::false_type(), image + (t & 1) * kImage, t * kTilePages, here, flags);
      if (t + 1 < tiles) arrive((t + 1) & 1, t + 1, flags_of(t + 1), here);
      __syncthreads();
    }
    if (aside)
      for (int t = 0; t < tiles; ++t)
        if (odd[t] != 0) {
          fetch(0, t);
          arrive(0, t, flags_of(t), here);
          __syncthreads();
          compute(std::true_type(), image, t * kTilePages, here, flags_of(t));
          __syncthreads();
        }
  }

  // ---- results
  l += __shfl_xor(l, 32, 64);
  m = limit < 0.f ? -3.4028235e38f : m;
  float* mine = reinterpret_cast<float*>(image);
  if constexpr (KS == 2) {
    // the second stream's sums go through LDS to the first one's lanes: [value][lane]
    __syncthreads();
    if (ks == 1) {
      float* to = mine + cw * (D / 2 + 2) * 64 + lane;
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) to[(16 * j + e) * 64] = o[j][e];
      to[(D / 2) * 64] = m;
      to[(D / 2 + 1) * 64] = l;
    }
    __syncthreads();
    if (ks == 1) return;
    const float* from = mine + cw * (D / 2 + 2) * 64 + lane;
    const float m1 = from[(D / 2) * 64], top = fmaxf(m, m1), f0 = exp2f(m - top), f1 = exp2f(m1 - top);
    l = l * f0 + from[(D / 2 + 1) * 64] * f1;
    m = top;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][e] = o[j][e] * f0 + from[(16 * j + e) * 64] * f1;
  }
  if (col >= n_cols) return;
  const size_t at = static_cast<size_t>(row) * a.hq + kvh * group + my_col % group;
#pragma unroll
  for (int j = 0; j < D / 32; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      store_result<bf16_t, D>(a, at, split, n_splits, 32 * j + 8 * e + 4 * h, f32x4{o[j][4 * e], o[j][4 * e + 1], o[j][4 * e + 2], o[j][4 * e + 3]}, m, l);
  if (split == 0 && kvh == 0 && my_col % group == 0 && h == 0) a.row_splits[row] = n_splits;
}

// Joins the ranges of a row and head: sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  D / 4 threads take four dims each; where there are many
// ranges (WIDE) the groups of such threads of a workgroup share one row and head, every so-manieth range each, otherwise they take one each.
// Bound by the parts it reads: 500 rows of 32 heads in 4 ranges, 33 MB, 8 us; 16 x 5 rows of 64 heads in 4, 10 MB, 5 us; a few rows take a launch and two
// trips to memory, 2.5 to 4 us.  (8 rows over 8000 tokens, 63 ranges: WIDE 22.8 us of the whole call, otherwise 25.1; up to 8 ranges there is no difference.)
template <typename T, int D, bool WIDE>
__global__ __launch_bounds__(256) void append_join_kernel(AppendArgs a, int n_items) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ f32x4 part[WIDE ? kGroups : 1][kLanes];
  __shared__ float2 sum_of[WIDE ? kGroups : 1];
  const int tid = threadIdx.x, lane = tid % kLanes, grp = tid / kLanes;
  const int at = WIDE ? blockIdx.x : blockIdx.x * kGroups + grp;             // row and head
  if (at >= n_items) return;
  const int row = at / a.hq;
  if (row >= a.cu_q[a.n_requests]) return;
  const int ns = a.row_splits[row], step = WIDE ? kGroups : 1;
  if (ns <= 1) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part_ml) + static_cast<size_t>(at) * a.n_splits;
  const float* po = a.part_o + static_cast<size_t>(at) * a.n_splits * D + 4 * lane;
  float top = -INFINITY, sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  constexpr int kAhead = 4;                                                 // ranges whose loads are under way together
  for (int s0 = WIDE ? grp : 0; s0 < ns; s0 += kAhead * step) {
    float2 x[kAhead];
    f32x4 y[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = min(s0 + i * step, ns - 1);
      x[i] = ml[s];
      y[i] = *reinterpret_cast<const f32x4*>(po + static_cast<size_t>(s) * D);
    }
    float t = top;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (s0 + i * step < ns) t = fmaxf(t, x[i].x);
    const float f = exp2f(top - t);
    top = t;
    sum *= f;
    v *= f;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float w = s0 + i * step < ns ? exp2f(x[i].x - t) : 0.f;
      sum += w * x[i].y;
      v += y[i] * w;
    }
  }
  if constexpr (WIDE) {
    part[grp][lane] = v;
    if (lane == 0) sum_of[grp] = make_float2(top, sum);
    __syncthreads();
    if (grp != 0) return;
    float t = top;
#pragma unroll
    for (int k = 1; k < kGroups; ++k) t = fmaxf(t, sum_of[k].x);
    const float f = exp2f(top - t);
    sum *= f;
    v *= f;
#pragma unroll
    for (int k = 1; k < kGroups; ++k) {
      const float w = exp2f(sum_of[k].x - t);
      sum += w * sum_of[k].y;
      v += part[k][lane] * w;
    }
    top = t;
  }
  store_result<T, D>(a, at, 0, 1, 4 * lane, v, top, sum);
}

// How the work of a call is divided: from host scalars alone.  What either side of a choice takes (16 requests of 1000 to 8000 tokens, 64 heads on 8, if
// nothing else is said):
//   columns of a workgroup   up to 16: append_split_kernel; 32 columns as two groups of it 112 us, as one of 64 columns of append_tile_kernel 78.
//                            up to 64, then 128: 72 columns as two groups of 64 135 us, as one of 128 116
//   ranges                   about 512 workgroups, two on a compute unit: the tile kernel with 256 97 us, with 512 76, with 1024 92; the split kernel 70, 73, 82
//                            (and 32 requests of one row 118, 115, 125).  The split kernel's number is the nearest, the tile kernel's rounded down: 24
//                            requests with 1.3 workgroups a unit 83 us, with 2 70; 40 requests of 8 rows with 1.25 145 us, with 2.5 164
//   pages of a range         at least 8 (16 for a tile): 8 rows over 8000 tokens with 4 26 us, with 8 23, with 16 24.4
struct AppendPlan {
  int cols;                           // columns of a workgroup: 16 (append_split_kernel); 64, 128 (append_tile_kernel)
  int col_groups, n_splits, split_pages;
  long long groups;                   // workgroups
};
AppendPlan plan_append(const cc_ctx* ctx, int max_q_per_req, int n_requests, int max_ctx_tokens, int max_segs_per_req) {
  const long long cols = static_cast<long long>(max_q_per_req) * (ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads);
  AppendPlan p;
  p.cols = cols <= 16 || ctx->cfg.dtype != CC_BF16 ? 16 : cols <= 64 ? 64 : 128;
  p.col_groups = static_cast<int>((cols + p.cols - 1) / p.cols);
  const long long pages = max_ctx_tokens / kBlock + static_cast<long long>(max_segs_per_req), units = static_cast<long long>(ctx->cfg.n_kv_heads) * n_requests;
  const long long target = 512, least = p.cols == 16 ? 8 : 16, all = std::max(1ll, units * p.col_groups);
  const long long splits = std::max(1ll, std::min((p.cols == 16 ? target + all / 2 : target) / all, (pages + least - 1) / least));
  p.split_pages = static_cast<int>(((pages + splits - 1) / splits + 3) & ~3ll);
  p.n_splits = static_cast<int>((pages + p.split_pages - 1) / p.split_pages);
  p.groups = (units * p.n_splits + 7) / 8 * 8 * p.col_groups;
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

// The join: a workgroup for 1024 / D rows and heads, or, where there are more than eight ranges, for each (see append_join_kernel).
static bool join_is_wide(const AppendPlan& p) { return p.n_splits > 8; }
static long long join_groups(const AppendPlan& p, long long n_items, int d) {
  const int per = join_is_wide(p) ? 1 : 1024 / d;
  return p.n_splits > 1 ? (n_items + per - 1) / per : 0;
}

long long append_groups(const cc_ctx* ctx, int n_q_tot, int max_q_per_req, int n_requests, int max_ctx_tokens, int max_segs_per_req) {
  const long long rows = n_q_tot < 1 << 30 ? scatter_groups(n_q_tot) : n_q_tot;
  if (ctx->impl == CC_IMPL_SCALAR) return std::max(rows, (n_q_tot + 3ll) / 4);          // (workgroups of a quarter of the threads)
  const AppendPlan p = plan_append(ctx, max_q_per_req, n_requests, max_ctx_tokens, max_segs_per_req);
  return std::max({rows, p.groups, join_groups(p, static_cast<long long>(n_q_tot) * ctx->cfg.n_q_heads, ctx->cfg.head_dim)});
}

size_t append_bytes(const cc_ctx* ctx, int n_q_tot, int max_q_per_req, int n_requests, int max_ctx_tokens, int max_segs_per_req) {
  if (ctx->impl == CC_IMPL_SCALAR || n_q_tot == 0) return 0;
  const AppendPlan p = plan_append(ctx, max_q_per_req, n_requests, max_ctx_tokens, max_segs_per_req);
  return (static_cast<size_t>(n_q_tot) * ctx->cfg.n_q_heads * p.n_splits * (ctx->cfg.head_dim + 2) + n_q_tot) * sizeof(float);
}

template <typename T, int D>
static void launch_append_t(const cc_ctx* ctx, const AppendArgs& a, const AppendPlan& p, int n_q_tot, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.groups));
  if (p.cols == 16) hipLaunchKernelGGL((append_split_kernel<T, D>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
  if constexpr (sizeof(T) == 2) {
    const bool shared = a.vs.v_map != nullptr;
    if (p.cols == 64 && !shared) hipLaunchKernelGGL((append_tile_kernel<D, 2, false>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
    if (p.cols == 64 && shared) hipLaunchKernelGGL((append_tile_kernel<D, 2, true>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
    if (p.cols == 128 && !shared) hipLaunchKernelGGL((append_tile_kernel<D, 4, false>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
    if (p.cols == 128 && shared) hipLaunchKernelGGL((append_tile_kernel<D, 4, true>), grid, dim3(256), 0, stream, a, ctx->inv_freq);
  }
  const int n_items = n_q_tot * a.hq;
  const dim3 join(static_cast<unsigned>(join_groups(p, n_items, D)));
  if (p.n_splits > 1 && join_is_wide(p)) hipLaunchKernelGGL((append_join_kernel<T, D, true>), join, dim3(256), 0, stream, a, n_items);
  else if (p.n_splits > 1) hipLaunchKernelGGL((append_join_kernel<T, D, false>), join, dim3(256), 0, stream, a, n_items);
}

void launch_append_attention(const cc_ctx* ctx, const void* q, const int32_t* src_rows, const int32_t* q_pos, const int32_t* cu_q, int n_q_tot,
                             int max_q_per_req, const void* k_pool, const void* v_pool, int n_blocks, const int32_t* block_tab,
                             const cc_segment* segs, const int32_t* req_seg_off, int n_requests, int max_ctx_tokens, int max_segs_per_req,
                             void* out, float* lse, void* workspace, hipStream_t stream, const ScatterJob& scatter) {
  const ValueSource& vs = scatter.vs;
  const bool bf = ctx->cfg.dtype == CC_BF16;
  const int d = ctx->cfg.head_dim, hq = ctx->cfg.n_q_heads, hkv = ctx->cfg.n_kv_heads;
  if (ctx->impl == CC_IMPL_SCALAR) {
    launch_rope_scatter(ctx, scatter, stream);
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
  // Few rows are written by the workgroups that read them, which saves a launch (one row over 700 tokens 13.3 us instead of 18.6, 32 requests 116 instead of 122).  Not
  // with a value map: a page whose values are still in the chunk store is copied whole, for all KV heads at once, and whether a row lies in such a page
  // only the device knows.
  const bool write = p.col_groups == 1 && max_q_per_req <= kWriteRows && vs.v_map == nullptr;
  if (!write) launch_rope_scatter(ctx, scatter, stream);
  float* part_o = static_cast<float*>(workspace);
  float* part_ml = part_o + static_cast<size_t>(n_q_tot) * hq * p.n_splits * d;
  const AppendArgs a{q, src_rows, q_pos, cu_q, k_pool, v_pool, block_tab, segs, req_seg_off, out, lse, vs, n_requests, n_blocks, hq, hkv,
                     p.n_splits, p.split_pages, p.col_groups, part_o, part_ml, write ? scatter.k_new : nullptr, scatter.v_new, scatter.slot_map,
                     reinterpret_cast<int32_t*>(part_ml + static_cast<size_t>(n_q_tot) * hq * p.n_splits * 2)};
  if (bf && d == 128) launch_append_t<bf16_t, 128>(ctx, a, p, n_q_tot, stream);
  else if (bf) launch_append_t<bf16_t, 64>(ctx, a, p, n_q_tot, stream);
  else if (d == 128) launch_append_t<float, 128>(ctx, a, p, n_q_tot, stream);
  else launch_append_t<float, 64>(ctx, a, p, n_q_tot, stream);
}

}  // namespace cc
