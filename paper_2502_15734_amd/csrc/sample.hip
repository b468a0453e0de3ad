// cc_sample: one token per row of logits.
//
// With x_i = (z_i - max z) / T the weights are w_i = exp(x_i), taken in 64 bits and held as whole multiples of 2^-shift
// (shift = min(50, 62 - ceil(log2 vocab)): a row's sum stays below 2^62).  Sums of whole numbers come out the same in every order, so the
// drawn token does not depend on how a row is divided, and an error of 2^-46 per weight does not move a border that a float would.
// The kept tokens are the first ranks of the order (logit descending, index ascending), so every cut is one (logit, index).
//
// A row is read by several workgroups (sample_plan): three passes over parts of the row, of which the second and third find it in
// the caches, and a last kernel with a workgroup per row.
//   sample_max_kernel    largest and smallest logit of each part
//   sample_hist_kernel   rows with top-k or top-p: counts and weights per bin of equal width between the largest logit and the smallest
//                        (or the one whose weight is 2^-66, where that is larger)
//   sample_tiles_kernel  finds the bin a cut falls into; sums the weights of the bins in front of it per tile of the row, and lists the
//                        logits of that bin, the candidates
//   sample_draw_kernel   sorts the candidates, finds the cut among them, the tile the drawn number falls into and the token in it
// Rows with more candidates than the list holds (thousands of equal logits) are done by the last kernel alone, with radix descents
// over the whole row (32000 equal ones 0.4 ms, 128256 1.25 ms).  Rows of up to 12 Ki logits are the last kernel's alone: it holds them in LDS and takes the
// same steps there.
//
// Few rows are bound by latency: four launches, each with a chain of two or three loads, scans and barriers (1 x 32000 fp32 with top-p 23.3 us, of
// which the last kernel takes 7; 32 x 128256 bf16 35 to 39 us).  Many rows are bound by the three reads and the arithmetic in 64 bits beside the second and third:
// 256 x 128001 fp32 (131 MB) with all kinds of settings 104 to 111 us: 26 for the first pass (5 TB/s), 27, 37 and 10 to 23 for the last kernel, the
// longest where a row has many candidates to sort.
#include <algorithm>

#include "device_util.h"

namespace cc {

namespace {

constexpr uint32_t kKeyNone = 0x007fffffu;            // ordered key of -inf: never kept (a NaN counts as one)

constexpr uint32_t kKeyInf = 0xff800000u;             // of +inf: beside one, everything finite has weight 0

// monotone float -> uint; -0 and +0 are one value
__device__ __forceinline__ uint32_t logit_key(float v) {
  if (v != v) return kKeyNone;
  const uint32_t u = __float_as_uint(v + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key); }

struct SampleArgs {
  const void* logits;
  int n_rows, vocab;
  long long stride;
  const float *temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *u;
  int32_t* token;
  float* logprob;
  int32_t* n_kept;
  int shift;
};

struct RowSettings {
  double inv_t, top_p, min_p, u;
  int top_k;
  bool greedy;
};

__device__ __forceinline__ RowSettings settings_of(const SampleArgs& a, int row) {
  RowSettings s;
  const float t = a.temperature != nullptr ? a.temperature[row] : 1.f;
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  const float p = a.top_p != nullptr ? a.top_p[row] : 1.f, m = a.min_p != nullptr ? a.min_p[row] : 0.f, u = a.u[row];
  s.greedy = !(t > 0.f) || k == 1 || m > 1.f || p <= 0.f;                        // (the largest logit alone)
  s.inv_t = s.greedy ? 1.0 : 1.0 / static_cast<double>(t);
  s.top_k = (k <= 0 || k > a.vocab) ? a.vocab : k;
  s.top_p = p < 1.f ? static_cast<double>(p) : 1.0;                             // (a NaN: off)
  s.min_p = m > 0.f ? static_cast<double>(m) : 0.0;
  s.u = u > 0.f ? fmin(static_cast<double>(u), 1.0 - 0x1p-24) : 0.0;
  return s;
}

// exp of x <= 0: x = n ln 2 + r, |r| <= ln 2 / 2, the series of exp(r) to r^13 (the rest is below 2^-57)
__device__ __forceinline__ double exp_of(double x) {
  x = fmax(x, -800.0);                                 // (0 in 64 bits)
  const double n = rint(x * 1.4426950408889634074);
  const double r = fma(n, 0x1.8432a1b0e2634p-43, fma(n, -0x1.62e42fefa4000p-1, x));       // (ln 2 in two parts: its first 40 bits, so that their product is exact, and the rest)
  double p = 1.0 / 6227020800.0;
  p = fma(p, r, 1.0 / 479001600.0);
  p = fma(p, r, 1.0 / 39916800.0);
  p = fma(p, r, 1.0 / 3628800.0);
  p = fma(p, r, 1.0 / 362880.0);
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return ldexp(p, static_cast<int>(n));
}

// weight of a logit against the row's largest one
__device__ __forceinline__ double weight_of(uint32_t key, uint32_t top, double inv_t) {
  if (key == top) return 1.0;
  if (key <= kKeyNone || top == kKeyInf) return 0.0;
  return exp_of((static_cast<double>(logit_of(key)) - static_cast<double>(logit_of(top))) * inv_t);
}
// the nearest multiple of 2^-shift (shift <= 50, w <= 1: the sum with 2^52 has it in its last bits)
__device__ __forceinline__ unsigned long long fixed_of(double w, int shift) {
  return static_cast<unsigned long long>(__double_as_longlong(ldexp(w, shift) + 0x1p52) - __double_as_longlong(0x1p52));
}

template <typename T>
__device__ __forceinline__ uint32_t key_at(const SampleArgs& a, int row, int i) {
  return logit_key(to_float(static_cast<const T*>(a.logits)[static_cast<size_t>(row) * a.stride + i]));
}

// The row as pieces of 16 bytes at aligned addresses: element e of them is logit e - shift.
template <typename T>
struct RowReader {
  static constexpr int kPer = 16 / sizeof(T);
  const T* row;
  int shift, vocab;
  __device__ __forceinline__ RowReader(const SampleArgs& a, int r) {
    row = static_cast<const T*>(a.logits) + static_cast<size_t>(r) * a.stride;
    shift = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    vocab = a.vocab;
  }
  typedef __attribute__((__vector_size__(16))) T Piece;
  // f(logit, index) for the row's elements e0 .. e0 + kPer, e0 + step .., up to e1 (multiples of kPer), in the order of the indexes; kAhead pieces are
  // loaded before the first is used.  Only the row's own logits are read; -inf and NaN are passed over, and pieces with nothing from `least` up.
  template <typename F>
  __device__ __forceinline__ void each(int e0, int e1, int step, float least, F&& f) const {
    constexpr int kAhead = 4;
    for (int e = e0; e < e1; e += kAhead * step) {
      Piece v[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const int i = e + a * step - shift;
        if (i >= 0 && i + kPer <= vocab && e + a * step < e1) v[a] = *reinterpret_cast<const Piece*>(row + i);
      }
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const int i = e + a * step - shift;
        if (e + a * step >= e1) break;
        const bool whole = i >= 0 && i + kPer <= vocab;
        if (whole) {
          float most = to_float(v[a][0]);
#pragma unroll
          for (int j = 1; j < kPer; ++j) most = fmaxf(most, to_float(v[a][j]));
          if (most < least) continue;
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          if (!whole && (i + j < 0 || i + j >= vocab)) continue;
          const float z = to_float(whole ? v[a][j] : row[i + j]);
          if (z > -INFINITY) f(z, i + j);
        }
      }
    }
  }
};

struct Cut {              // the ranks above it: logits above key, and the first `ties` (by index) of those equal to it
  uint32_t key;
  unsigned ties;
};

template <int W>
struct RowShared {
  unsigned count[256];
  unsigned long long mass[256];
  unsigned wave_ties[W], wave_kept[W];
  unsigned long long wave_mass[W];
  unsigned found_digit, found_count;
  unsigned long long found_mass;
};

// The whole row by one workgroup, whatever its logits.  top: its largest one.
template <typename T, int W>
__device__ __forceinline__ void sample_row(const SampleArgs& a, int row, const RowSettings& s, uint32_t top, RowShared<W>& sh) {
  unsigned *count = sh.count, *wave_ties = sh.wave_ties, *wave_kept = sh.wave_kept;
  unsigned long long *mass = sh.mass, *wave_mass = sh.wave_mass;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = a.vocab;
  const RowReader<T> in(a, row);
  constexpr int kPer = RowReader<T>::kPer;

  // ---- radix descent: the cut behind the rank at which the count reaches `want` or the weights in front reach `target`
  unsigned long long set_mass = 0;                     // weights above the cut, its kept ties included
  auto descend = [&](bool by_mass, unsigned want, double target) {
    uint32_t prefix = 0;
    unsigned above = 0;
    unsigned long long above_mass = 0;
    for (int digit = 3; digit >= 0; --digit) {
      if (tid < 256) { count[tid] = 0; mass[tid] = 0; }
      __syncthreads();
      in.each(tid * kPer, n + in.shift, 64 * W * kPer, -INFINITY, [&](float z, int) __attribute__((always_inline)) {
        const uint32_t k = logit_key(z);
        if (digit < 3 && (k >> (8 * digit + 8)) != prefix) return;
        // (lanes with one logit add it together: such rows are why this is called, and 64 sums of one place would follow each other)
        const unsigned long long here = __ballot(true);
        const bool one = __ballot(k == static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(k)))) == here;
        if (one && lane != __builtin_ctzll(here)) return;
        const unsigned n_same = one ? __popcll(here) : 1u;
        atomicAdd(&count[(k >> (8 * digit)) & 255], n_same);
        atomicAdd(&mass[(k >> (8 * digit)) & 255], n_same * fixed_of(weight_of(k, top, s.inv_t), a.shift));
      });
      __syncthreads();
      if (tid == 0) {
        unsigned c = above;
        unsigned long long m = above_mass;
        int at = 255, last = -1;
        for (; at >= 0; --at) {
          if (count[at] == 0) continue;
          last = at;
          if (by_mass ? static_cast<double>(m + mass[at]) >= target : c + count[at] >= want) break;
          c += count[at];
          m += mass[at];
        }
        if (at < 0) { at = last; c -= count[at]; m -= mass[at]; }          // (fewer than wanted: all of them)
        sh.found_digit = at; sh.found_count = c; sh.found_mass = m;
      }
      __syncthreads();
      prefix = (prefix << 8) | sh.found_digit;
      above = sh.found_count;
      above_mass = sh.found_mass;
      __syncthreads();
    }
    const unsigned equal = count[prefix & 255];
    const unsigned long long each = fixed_of(weight_of(prefix, top, s.inv_t), a.shift);
    unsigned ties = equal;
    if (!by_mass) ties = min(equal, want - above);
    else if (each > 0) {                               // ranks whose weights in front stay below the target
      const double more = ceil((target - static_cast<double>(above_mass)) / static_cast<double>(each));
      ties = more >= equal ? equal : more < 1.0 ? (above == 0 ? 1u : 0u) : static_cast<unsigned>(more);
    }
    set_mass = above_mass + each * ties;
    __syncthreads();
    return Cut{prefix, ties};
  };
  Cut cut{0, 0xffffffffu};
  if (s.top_k < n || s.top_p < 1.0) cut = descend(false, s.top_k, 0.0);
  if (s.top_p < 1.0) {
    const Cut c = descend(true, 0, s.top_p * static_cast<double>(set_mass));
    if (c.key > cut.key || (c.key == cut.key && c.ties < cut.ties)) cut = c;
  }

  // ---- the draw, in the order of the indexes: a wavefront owns a contiguous share
  const int share = (n + in.shift + W * kPer - 1) / (W * kPer) * kPer, e0 = wave * share, e1 = min(n + in.shift, e0 + share), i0 = max(e0 - in.shift, 0), i1 = e1 - in.shift;
  auto weight = [&](uint32_t k) {
    const double w = k > kKeyNone ? weight_of(k, top, s.inv_t) : 0.0;
    return w >= s.min_p || k == top ? w : 0.0;
  };
  const bool tie_in = cut.key > kKeyNone && (weight(cut.key) > 0.0 || s.min_p == 0.0);
  const unsigned long long each = tie_in ? fixed_of(weight(cut.key), a.shift) : 0;
  unsigned kept = 0, ties = 0;
  unsigned long long sum = 0;
  in.each(e0 + lane * kPer, e1, 64 * kPer, -INFINITY, [&](float z, int) __attribute__((always_inline)) {
    const uint32_t k = logit_key(z);
    if (k == cut.key) ++ties;
    else if (k > cut.key) {
      const double w = weight_of(k, top, s.inv_t);
      if (w >= s.min_p || k == top) { ++kept; sum += fixed_of(w, a.shift); }
    }
  });
  for (int o = 32; o > 0; o >>= 1) { kept += __shfl_xor(kept, o, 64); ties += __shfl_xor(ties, o, 64); sum += __shfl_xor(sum, o, 64); }
  if (lane == 0) { wave_ties[wave] = ties; wave_kept[wave] = kept; wave_mass[wave] = sum; }
  __syncthreads();
  unsigned ties_before = 0, n_kept = 0, first_ties = 0;
  unsigned long long total = 0;
  for (int w = 0; w < W; ++w) {
    const unsigned left = cut.ties > ties_before ? cut.ties - ties_before : 0, t = tie_in ? min(left, wave_ties[w]) : 0;
    if (w == wave) first_ties = ties_before;
    n_kept += wave_kept[w] + t;
    total += wave_mass[w] + each * t;
    ties_before += wave_ties[w];
  }
  const double target = s.u * static_cast<double>(total);
  unsigned long long before = 0;
  unsigned tb = 0;
  int mine = -1;
  for (int w = 0; w < W; ++w) {
    const unsigned left = cut.ties > tb ? cut.ties - tb : 0, t = tie_in ? min(left, wave_ties[w]) : 0;
    const unsigned long long m = wave_mass[w] + each * t;
    tb += wave_ties[w];
    if (static_cast<double>(before + m) > target) { mine = w; break; }
    before += m;
  }
  if (wave != mine) return;
  unsigned seen = first_ties;
  constexpr int kNext = 4;                             // (logits that are read ahead)
  uint32_t next[kNext];
  for (int base = i0, turn = 0; base < i1; base += 64, turn = (turn + 1) % kNext) {
    const int i = base + lane;
    if (turn == 0)
#pragma unroll
      for (int j = 0; j < kNext; ++j) next[j] = i + 64 * j < i1 ? key_at<T>(a, row, i + 64 * j) : 0;
    const uint32_t k = turn == 0 ? next[0] : turn == 1 ? next[1] : turn == 2 ? next[2] : next[3];
    const bool tie = k > kKeyNone && k == cut.key;
    const unsigned long long tied = __ballot(tie);
    const unsigned rank = seen + __popcll(tied & ((1ull << lane) - 1));
    unsigned long long w = 0;
    if (k > kKeyNone && (k > cut.key || (tie && rank < cut.ties))) w = fixed_of(weight(k), a.shift);
    unsigned long long sums = w;
    for (int o = 1; o < 64; o <<= 1) {
      const unsigned long long up = __shfl_up(sums, o, 64);
      if (lane >= o) sums += up;
    }
    const unsigned long long hit = __ballot(static_cast<double>(before + sums) > target);
    if (hit != 0) {
      if (lane == __builtin_ctzll(hit)) {
        a.token[row] = i;
        if (a.logprob != nullptr) a.logprob[row] = static_cast<float>(log(weight(k) / ldexp(static_cast<double>(total), -a.shift)));
        if (a.n_kept != nullptr) a.n_kept[row] = static_cast<int>(n_kept);
      }
      return;
    }
    before += __shfl(sums, 63, 64);
    seen += __popcll(tied);
  }
}

// The weights of a row in parts: 2^(y / 256) with y = (z - max z) 256 / (T ln 2), as a table of 2^(j / 256) and the series of 2^(f / 256), |f| <= 1/2,
// to f^4 (the rest is below 2^-54), times 2^shift.  The passes over a large vocabulary are bound by these steps in 64 bits, so the
// nearest whole number is the last bits of a sum and the exponent is added to the table's entry as an integer.
constexpr int kTable = 256;
struct Weights {
  double top, per, least;             // least: min_p in the same units
  const double* table;
  int shift;
  // table: [kTable] in LDS, filled here by the workgroup (a barrier has to follow)
  __device__ __forceinline__ Weights(float top_logit, const RowSettings& s, int shift_, double* table_)
      : top(top_logit), per(s.inv_t * 369.3299304675746), least(ldexp(s.min_p, shift_)), table(table_), shift(shift_) {       // 256 / ln 2
    static_assert(kTable <= 256, "one entry a thread");
    if (threadIdx.x < kTable) table_[threadIdx.x] = exp_of(threadIdx.x * 0.0027076061740622863);       // ln 2 / 256
  }
  // w 2^shift; exactly 2^shift for the largest logit
  __device__ __forceinline__ double scaled(float z) const {
    const double y = fmax((static_cast<double>(z) - top) * per, -256.0 * 900.0), t = y + 0x1.8p52, f = y - (t - 0x1.8p52);       // (t: its low word is the nearest whole number)
    const int n = static_cast<int>(__double_as_longlong(t));
    double p = 2.239395190875157e-12;                                      // (ln 2 / 256)^4 / 4! and so on down
    p = fma(p, f, 3.3083026805413713e-09);
    p = fma(p, f, 3.6655655969101062e-06);
    p = fma(p, f, 0.0027076061740622863);
    p = fma(p, f, 1.0);
    // (2^-900 2^shift and more: the exponent stays that of a normal number)
    const double e = table[n & (kTable - 1)];
    return __hiloint2double(__double2hiint(e) + (((n >> 8) + shift) << 20), __double2loint(e)) * p;
  }
  // ... to the nearest whole number (shift <= 50: the sum with 2^52 has it in its last bits)
  static __device__ __forceinline__ unsigned long long whole(double w) {
    return static_cast<unsigned long long>(__double_as_longlong(w + 0x1p52) - __double_as_longlong(0x1p52));
  }
};

// ---- a row in parts ------------------------------------------------------------------------------
constexpr int kBins = 1024, kMaxParts = 64, kList = 4096, kLocal = 512;     // (kLocal: candidates of a part that are gathered in LDS)

struct SamplePlan {
  int parts, part_len;                // a part is read by a workgroup, a quarter of it by a wavefront; parts 0: the last kernel alone
  int wave_tiles, tile_len;           // a wavefront's quarter has 1, 2 or 4 tiles, whose sums are kept
};
constexpr int kTiles = 256;           // of a row
struct Part {
  float top, low;                     // largest and smallest logit (top -inf: none)
  int top_idx, unused;
};
struct Cuts {
  int p_lo, p_hi, k_bin;              // candidates: bins p_lo .. p_hi, and k_bin; bins in front of p_lo are kept whole
  unsigned count_lo, count_hi;        // tokens in front of p_lo, behind p_hi
  unsigned count_k;                   // tokens in front of k_bin
  unsigned listed;                    // candidates
  unsigned unlisted;                  // tokens of the last bin that pass top-k and have no weight: they count as kept, which of them does not matter
  unsigned long long mass_lo, mass_k, mass_all;      // weights in front of p_lo, of k_bin, of all bins
};

struct RowScratch {
  Part part[kMaxParts];
  unsigned long long mass[kBins];
  unsigned long long tile_mass[kTiles];
  uint2 list[kList];                  // key, index
  unsigned count[kBins];
  unsigned tile_kept[kTiles];
  unsigned n_list, unused[3];
  Cuts cuts;                          // (of a row that needs a cut and has bins)
};

// The row's extremes from its parts: every wavefront for itself.
__device__ __forceinline__ bool ahead(float z, int i, float than, int than_i) { return z > than || (z == than && i < than_i); }
__device__ __forceinline__ Part row_extremes(const RowScratch& ws, int parts) {
  const int lane = threadIdx.x & 63;
  Part p{-INFINITY, INFINITY, 0x7fffffff, 0};
  if (lane < parts) p = ws.part[lane];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float top = __shfl_xor(p.top, o, 64), low = __shfl_xor(p.low, o, 64);
    const int idx = __shfl_xor(p.top_idx, o, 64);
    if (ahead(top, idx, p.top, p.top_idx)) { p.top = top; p.top_idx = idx; }
    p.low = fminf(p.low, low);
  }
  return p;
}

// Bins of equal width from the largest logit (bin 0) down.  Rounded subtractions and products keep the order of the logits, so
// the bins are in that order and equal logits share one.
struct Bins {
  float top, per;
  bool usable, far;                   // far: the last bin holds nothing else than weights below 2^-66, zeros of the sums
  __device__ __forceinline__ Bins(float top_, float low, double inv_t) : top(top_) {
    const float most = static_cast<float>(46.0 / inv_t), span = fminf(top - low, most);
    far = most < top - low;
    per = span > 0.f ? kBins / span : 0.f;
    usable = span < INFINITY && per < INFINITY;
  }
  __device__ __forceinline__ int of(float z) const { return static_cast<int>(fminf((top - z) * per, static_cast<float>(kBins - 1))); }
};

// Where the cuts fall, from the histogram.  With both top-k and top-p the weight that top-p refers to is known to the bin that top-k's cut
// falls into, so top-p's has a first and a last possible bin.
template <int N>
__device__ __forceinline__ Cuts find_cuts(const unsigned* counts, const unsigned long long* masses, const RowSettings& s, bool far) {
  constexpr int kOwn = kBins / N;     // bins of a thread
  __shared__ unsigned long long wave_mass[N / 64];
  __shared__ unsigned wave_count[N / 64];
  __shared__ Cuts cuts;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  unsigned c[kOwn], count = 0;
  unsigned long long m[kOwn], mass = 0;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    c[i] = counts[tid * kOwn + i];
    m[i] = masses[tid * kOwn + i];
    count += c[i];
    mass += m[i];
  }
  unsigned count_in = count;
  unsigned long long mass_in = mass;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned cu = __shfl_up(count_in, o, 64);
    const unsigned long long mu = __shfl_up(mass_in, o, 64);
    if (lane >= o) { count_in += cu; mass_in += mu; }
  }
  if (lane == 63) { wave_count[wave] = count_in; wave_mass[wave] = mass_in; }
  __syncthreads();
  unsigned count_all = 0, count0 = count_in - count;
  unsigned long long mass_all = 0, mass0 = mass_in - mass;
  for (int w = 0; w < N / 64; ++w) {
    if (w < wave) { count0 += wave_count[w]; mass0 += wave_mass[w]; }
    count_all += wave_count[w];
    mass_all += wave_mass[w];
  }
  const bool by_k = static_cast<unsigned>(s.top_k) < count_all, by_p = s.top_p < 1.0;
  if (tid == 0) cuts = Cuts{kBins, kBins, kBins, count_all, count_all, count_all, 0, 0, mass_all, mass_all, mass_all};
  __syncthreads();
  // (f(bin, tokens in front, weights in front, with the bin's own) for this thread's bins)
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    unsigned cb = count0;
    unsigned long long mb = mass0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      f(tid * kOwn + i, cb, mb, cb + c[i], mb + m[i]);
      cb += c[i];
      mb += m[i];
    }
  };
  __shared__ unsigned long long mass_with_k;
  __shared__ unsigned count_with_k;
  if (tid == 0) { mass_with_k = mass_all; count_with_k = count_all; }
  __syncthreads();
  if (by_k)
    each([&](int b, unsigned cb, unsigned long long mb, unsigned ce, unsigned long long me) {
      if (cb < static_cast<unsigned>(s.top_k) && static_cast<unsigned>(s.top_k) <= ce) {
        cuts.k_bin = b; cuts.count_k = cb; cuts.mass_k = mb;
        mass_with_k = me; count_with_k = ce;
        if (!by_p) { cuts.p_lo = cuts.p_hi = b; cuts.count_lo = cb; cuts.count_hi = ce; cuts.mass_lo = mb; }
      }
    });
  __syncthreads();
  if (by_p) {
    const double lo = s.top_p * static_cast<double>(cuts.mass_k), hi = s.top_p * static_cast<double>(mass_with_k);
    each([&](int b, unsigned cb, unsigned long long mb, unsigned ce, unsigned long long me) {
      if (static_cast<double>(me) >= lo && (b == 0 || static_cast<double>(mb) < lo)) { cuts.p_lo = b; cuts.count_lo = cb; cuts.mass_lo = mb; }
      if (static_cast<double>(me) >= hi && (b == 0 || static_cast<double>(mb) < hi)) { cuts.p_hi = b; cuts.count_hi = ce; }
    });
  }
  __syncthreads();
  Cuts out = cuts;
  // top-k reaches into logits that were masked by a low number: no list of thousands of equal ones for that
  if (far && out.k_bin == kBins - 1 && !(s.min_p > 0.0 && s.min_p < 0x1p-60)) {
    if (!by_p) {
      out.unlisted = s.min_p > 0.0 ? 0u : static_cast<unsigned>(s.top_k) - out.count_k;
      out.p_lo = kBins - 1;
      out.p_hi = kBins - 2;
      out.count_hi = out.count_lo;
    }
    if (!by_p || out.p_hi < kBins - 1) out.k_bin = kBins;
  }
  out.listed = out.count_hi - out.count_lo + (out.k_bin < kBins && out.k_bin > out.p_hi ? count_with_k - out.count_k : 0u);
  return out;
}

__device__ __forceinline__ bool needs_cut(const SampleArgs& a, const RowSettings& s) { return s.top_k < a.vocab || s.top_p < 1.0; }

template <typename T>
__global__ __launch_bounds__(256) void sample_max_kernel(SampleArgs a, SamplePlan plan, RowScratch* __restrict__ scratch) {
  constexpr int kPer = RowReader<T>::kPer;
  __shared__ Part wave_part[4];
  const int part = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  RowScratch& ws = scratch[row];
  const RowReader<T> in(a, row);
  for (int b = part * 256 + tid; b < kBins; b += plan.parts * 256) { ws.count[b] = 0; ws.mass[b] = 0; }
  if (part == 0 && tid == 0) ws.n_list = 0;
  float top = -INFINITY, low = INFINITY;
  int at = 0x7fffffff;
  const int e1 = min((part + 1) * plan.part_len, a.vocab + in.shift);
  in.each(part * plan.part_len + tid * kPer, e1, 256 * kPer, -INFINITY, [&](float z, int i) __attribute__((always_inline)) {
    if (z > top) { top = z; at = i; }
    low = fminf(low, z);
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float t = __shfl_xor(top, o, 64);
    const int i = __shfl_xor(at, o, 64);
    if (ahead(t, i, top, at)) { top = t; at = i; }
    low = fminf(low, __shfl_xor(low, o, 64));
  }
  if (lane == 0) wave_part[wave] = Part{top, low, at, 0};
  __syncthreads();
  if (tid == 0) {
    Part p = wave_part[0];
    for (int w = 1; w < 4; ++w) {
      const Part o = wave_part[w];
      if (ahead(o.top, o.top_idx, p.top, p.top_idx)) { p.top = o.top; p.top_idx = o.top_idx; }
      p.low = fminf(p.low, o.low);
    }
    ws.part[part] = p;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void sample_hist_kernel(SampleArgs a, SamplePlan plan, RowScratch* __restrict__ scratch) {
  constexpr int kPer = RowReader<T>::kPer;
  __shared__ unsigned count[kBins];
  __shared__ unsigned long long mass[kBins];
  __shared__ double table[kTable];
  const int part = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
  RowScratch& ws = scratch[row];
  const RowSettings s = settings_of(a, row);
  if (s.greedy || !needs_cut(a, s)) return;
  const Part x = row_extremes(ws, plan.parts);
  const Bins bins(x.top, x.low, s.inv_t);
  if (!(fabsf(x.top) < INFINITY) || !bins.usable) return;
  const Weights weights(x.top, s, a.shift, table);
  for (int b = tid; b < kBins; b += 256) { count[b] = 0; mass[b] = 0; }
  __syncthreads();
  const RowReader<T> in(a, row);
  const bool weigh = s.top_p < 1.0;
  const int e1 = min((part + 1) * plan.part_len, a.vocab + in.shift);
  in.each(part * plan.part_len + tid * kPer, e1, 256 * kPer, -INFINITY, [&](float z, int) __attribute__((always_inline)) {
    const int b = bins.of(z);
    atomicAdd(&count[b], 1u);
    if (weigh) atomicAdd(&mass[b], Weights::whole(weights.scaled(z)));
  });
  __syncthreads();
  for (int b = tid; b < kBins; b += 256)
    if (count[b] != 0) {
      atomicAdd(&ws.count[b], count[b]);
      if (mass[b] != 0) atomicAdd(&ws.mass[b], mass[b]);
    }
}

// What becomes of a logit once the cuts are known.
struct Sieve {
  const Weights& weights;
  const Bins& bins;
  bool cut;
  int p_lo, p_hi, k_bin;
  float least_z, floor;               // logits below least_z are below min-p for certain, and those below floor are neither kept nor candidates: 2^-20 and a bin for the roundings
  __device__ __forceinline__ Sieve(const RowSettings& s, const Weights& w, const Bins& b, const Cuts& c, bool cut_) : weights(w), bins(b), cut(cut_) {
    p_lo = cut ? c.p_lo : kBins;
    p_hi = cut ? c.p_hi : kBins;
    k_bin = cut ? c.k_bin : kBins;
    const double reach = log(s.min_p) / s.inv_t;         // (-inf without min-p; a NaN: no such logit)
    least_z = static_cast<float>(w.top + reach - 0x1p-20 * (fabs(w.top) - reach));
    const int last_bin = k_bin < kBins ? max(p_hi, k_bin) : p_hi;
    floor = !cut ? least_z : last_bin < kBins - 2 ? b.top - (last_bin + 2) / b.per : -INFINITY;
  }
  template <typename F>
  __device__ __forceinline__ void take(float z, unsigned& kept, unsigned long long& sum, F&& candidate) const {
    const int b = cut ? bins.of(z) : -1;
    if (b < p_lo) {
      if (z < least_z) return;
      const double w = weights.scaled(z);
      if (w >= weights.least) { ++kept; sum += Weights::whole(w); }
    } else if (b <= p_hi || b == k_bin) {
      candidate();
    }
  }
};

template <typename T>
__global__ __launch_bounds__(256) void sample_tiles_kernel(SampleArgs a, SamplePlan plan, RowScratch* __restrict__ scratch) {
  constexpr int kPer = RowReader<T>::kPer;
  __shared__ double table[kTable];
  __shared__ uint2 list[kLocal];                       // the part's candidates: a place in the row's list for each would be a trip to memory in the loop
  __shared__ unsigned n_list, first;
  const int part = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  RowScratch& ws = scratch[row];
  const RowSettings s = settings_of(a, row);
  if (s.greedy) return;
  if (tid == 0) n_list = 0;
  const Part x = row_extremes(ws, plan.parts);
  const Bins bins(x.top, x.low, s.inv_t);
  const bool cut = needs_cut(a, s);
  if (!(fabsf(x.top) < INFINITY) || (cut && !bins.usable)) return;
  const Weights weights(x.top, s, a.shift, table);
  __syncthreads();
  Cuts c{};
  if (cut) {
    c = find_cuts<256>(ws.count, ws.mass, s, bins.far);
    if (part == 0 && tid == 0) ws.cuts = c;
    if (c.listed > kList) return;                      // (the last kernel does the row alone)
  }
  const Sieve sieve(s, weights, bins, c, cut);
  const RowReader<T> in(a, row);
  const int tile0 = (part * 4 + wave) * plan.wave_tiles;
  unsigned kept[4] = {0, 0, 0, 0};
  unsigned long long sum[4] = {0, 0, 0, 0};
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (t < plan.wave_tiles) {
      const int e0 = (tile0 + t) * plan.tile_len;
      in.each(e0 + lane * kPer, min(e0 + plan.tile_len, a.vocab + in.shift), 64 * kPer, sieve.floor, [&](float z, int i) __attribute__((always_inline)) {
        sieve.take(z, kept[t], sum[t], [&]() __attribute__((always_inline)) {
          const unsigned at = atomicAdd(&n_list, 1u);
          if (at < kLocal) {
            list[at] = make_uint2(logit_key(z), i);
          } else {
            const unsigned to = atomicAdd(&ws.n_list, 1u);
            if (to < kList) ws.list[to] = make_uint2(logit_key(z), i);
          }
        });
      });
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t < plan.wave_tiles) { kept[t] += __shfl_xor(kept[t], o, 64); sum[t] += __shfl_xor(sum[t], o, 64); }
  if (lane == 0)
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t < plan.wave_tiles) { ws.tile_kept[tile0 + t] = kept[t]; ws.tile_mass[tile0 + t] = sum[t]; }
  __syncthreads();
  const unsigned n = min(n_list, static_cast<unsigned>(kLocal));
  if (n == 0) return;
  if (tid == 0) first = atomicAdd(&ws.n_list, n);
  __syncthreads();
  for (unsigned i = tid; i < n; i += 256)
    if (first + i < kList) ws.list[first + i] = list[i];
}

template <int N, typename V>
__device__ __forceinline__ V block_sum(V v, V* part) {               // over the workgroup's 64 N threads
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  V all = 0;
  for (int w = 0; w < N; ++w) all += part[w];
  return all;
}
template <int N>
__device__ __forceinline__ unsigned long long block_before(unsigned long long v, unsigned long long* part) {     // sum of the threads in front
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned long long in = v;
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long up = __shfl_up(in, o, 64);
    if (lane >= o) in += up;
  }
  __syncthreads();
  if (lane == 63) part[wave] = in;
  __syncthreads();
  for (int w = 0; w < wave; ++w) in += part[w];
  return in - v;
}

// n_pow (a power of two, E N or at most N) places of LDS by N threads, the largest in front: bitonic, with place e N + t in thread t's register e.
// Exchanges over less than 64 places go through the wavefront's lanes, over N and more between a thread's registers, and only those
// between through LDS: of a list of 512 by 256 threads 5 steps of 45.
template <int E, int N>
__device__ __forceinline__ void sort_down(unsigned long long* order, int n_pow) {
  const int tid = threadIdx.x;
  const bool on = E > 1 || tid < n_pow;
  unsigned long long v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = on ? order[e * N + tid] : 0ull;
  // (place, distance, length: whether the place takes the larger one)
  auto larger = [](int at, int half, int len) { return ((at & half) == 0) == ((at & len) == 0); };
  for (int len = 2; len <= n_pow; len <<= 1)
    for (int half = len >> 1; half > 0; half >>= 1) {
      if (half >= N) {
#pragma unroll
        for (int step = 1; step < E; step <<= 1)
          if (half == step * N)
#pragma unroll
            for (int e = 0; e < E; ++e)
              if ((e & step) == 0) {
                const unsigned long long a = v[e], b = v[e | step];
                const bool up = larger(e * N + tid, half, len) == (a > b);
                v[e] = up ? a : b;
                v[e | step] = up ? b : a;
              }
        continue;
      }
      unsigned long long u[E];
      if (half < 64) {
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = __shfl_xor(v[e], half, 64);
      } else {
        __syncthreads();
        if (on)
#pragma unroll
          for (int e = 0; e < E; ++e) order[e * N + tid] = v[e];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = on ? order[(e * N + tid) ^ half] : 0ull;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = larger(e * N + tid, half, len) == (v[e] > u[e]) ? v[e] : u[e];
    }
  __syncthreads();
  if (on)
#pragma unroll
    for (int e = 0; e < E; ++e) order[e * N + tid] = v[e];
  __syncthreads();
}

// W wavefronts.  ROW: bytes of LDS that hold the row, of which this is then the only kernel; 0: it comes behind the others.
template <typename T, int W, int ROW>
__global__ __launch_bounds__(64 * W) void sample_draw_kernel(SampleArgs a, SamplePlan plan, RowScratch* __restrict__ scratch) {
  constexpr bool kParts = ROW == 0;
  constexpr int kThreads = 64 * W, kCap = kParts ? kList : 1024, kPer = RowReader<T>::kPer, kBinsHere = kParts ? 1 : kBins;
  typedef typename RowReader<T>::Piece Piece;
  union Shared {
    RowShared<W> row;
    struct { unsigned long long mass[kBinsHere]; unsigned count[kBinsHere]; } bins;
    struct { unsigned long long order[kCap]; unsigned long long tile[kTiles]; } list;
  };
  __shared__ Shared sh;
  __shared__ Piece held[kParts ? 1 : ROW / 16];
  __shared__ unsigned long long part_mass[W], found_before;
  __shared__ unsigned part_count[W], n_found;
  __shared__ Part wave_part[W];
  __shared__ int found;
  __shared__ double table[kTable];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const RowSettings s = settings_of(a, row);
  const bool cut = needs_cut(a, s);
  const RowReader<T> in(a, row);
  const int shift = in.shift, n_pieces = (a.vocab + shift + kPer - 1) / kPer, tile_pieces = (n_pieces + 4 * W - 1) / (4 * W);
  const int tile_len = kParts ? plan.tile_len : tile_pieces * kPer, n_tiles = kParts ? 4 * plan.wave_tiles * plan.parts : 4 * W;
  Part x{-INFINITY, INFINITY, 0x7fffffff, 0};
  Cuts c{};
  int n_list = 0;
  // (what the other kernels left, in one trip to memory; what this row does not use is not looked at)
  uint2 listed{0, 0};
  unsigned long long tile_mass = 0;
  unsigned tile_kept = 0;
  if constexpr (kParts) {
    const RowScratch& ws = scratch[row];
    c = ws.cuts;
    listed = ws.list[tid];
    if (tid < n_tiles) { tile_mass = ws.tile_mass[tid]; tile_kept = ws.tile_kept[tid]; }
    x = row_extremes(ws, plan.parts);
  } else {
    constexpr int kAhead = 4;
    for (int b = tid; b < kBins; b += kThreads) { sh.bins.count[b] = 0; sh.bins.mass[b] = 0; }
    if (tid == 0) n_found = 0;
    for (int p0 = tid; p0 < n_pieces; p0 += kAhead * kThreads) {
      Piece v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = (p0 + j * kThreads) * kPer - shift;
        if (i >= 0 && i + kPer <= a.vocab) v[j] = *reinterpret_cast<const Piece*>(in.row + i);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int p = p0 + j * kThreads, i = p * kPer - shift;
        if (p >= n_pieces) break;
        const bool inside = i >= 0 && i + kPer <= a.vocab;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          if (!inside) v[j][e] = i + e >= 0 && i + e < a.vocab ? in.row[i + e] : static_cast<T>(-INFINITY);
          const float z = to_float(v[j][e]);
          if (z > x.top) { x.top = z; x.top_idx = i + e; }
          if (z > -INFINITY) x.low = fminf(x.low, z);
        }
        held[p] = v[j];
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float t = __shfl_xor(x.top, o, 64);
      const int i = __shfl_xor(x.top_idx, o, 64);
      if (ahead(t, i, x.top, x.top_idx)) { x.top = t; x.top_idx = i; }
      x.low = fminf(x.low, __shfl_xor(x.low, o, 64));
    }
    if (lane == 0) wave_part[wave] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const Part o = wave_part[w];
      if (ahead(o.top, o.top_idx, x.top, x.top_idx)) { x.top = o.top; x.top_idx = o.top_idx; }
      x.low = fminf(x.low, o.low);
    }
  }
  const uint32_t top = logit_key(x.top);
  if (top <= kKeyNone || s.greedy) {                   // (nothing to draw; or nothing else than the largest)
    if (tid == 0) {
      const bool none = top <= kKeyNone;
      a.token[row] = none ? -1 : x.top_idx;
      if (a.logprob != nullptr) a.logprob[row] = none ? -INFINITY : 0.f;
      if (a.n_kept != nullptr) a.n_kept[row] = none ? 0 : 1;
    }
    return;
  }
  const Bins bins(x.top, x.low, s.inv_t);
  bool whole = top == kKeyInf || (cut && !bins.usable);        // the list does not hold the candidates
  const Weights weights(x.top, s, a.shift, table);
  __syncthreads();
  if constexpr (!kParts)
    if (!whole && cut) {
      const bool weigh = s.top_p < 1.0;
      for (int p = tid; p < n_pieces; p += kThreads) {
        const Piece v = held[p];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const float z = to_float(v[e]);
          if (!(z > -INFINITY)) continue;
          const int b = bins.of(z);
          atomicAdd(&sh.bins.count[b], 1u);
          if (weigh) atomicAdd(&sh.bins.mass[b], Weights::whole(weights.scaled(z)));
        }
      }
      __syncthreads();
      c = find_cuts<kThreads>(sh.bins.count, sh.bins.mass, s, bins.far);
    }
  if (!whole && cut) {
    whole = c.listed > kCap;
    n_list = static_cast<int>(c.listed);
  }
  if (whole) {
    __syncthreads();
    sample_row<T, W>(a, row, s, top, sh.row);
    return;
  }
  if constexpr (kParts) {
    for (int i = tid; i < n_list; i += kThreads) {
      const uint2 v = i == tid ? listed : scratch[row].list[i];
      sh.list.order[i] = (static_cast<unsigned long long>(v.x) << 32) | ~v.y;
    }
    if (tid < n_tiles) sh.list.tile[tid] = tile_mass;   // (n_tiles is at most the number of threads)
  } else {
    const Sieve sieve(s, weights, bins, c, cut);
    __syncthreads();                                   // (the bins' place is the list's)
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int tile = wave * 4 + t, q1 = min((tile + 1) * tile_pieces, n_pieces);
      unsigned kept = 0;
      unsigned long long sum = 0;
      for (int p = tile * tile_pieces + lane; p < q1; p += 64) {
        const Piece v = held[p];
        float most = to_float(v[0]);
#pragma unroll
        for (int e = 1; e < kPer; ++e) most = fmaxf(most, to_float(v[e]));
        if (most < sieve.floor) continue;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const float z = to_float(v[e]);
          if (z > -INFINITY)
            sieve.take(z, kept, sum, [&]() __attribute__((always_inline)) {
              sh.list.order[atomicAdd(&n_found, 1u)] = (static_cast<unsigned long long>(logit_key(z)) << 32) | ~static_cast<uint32_t>(p * kPer + e - shift);
            });
        }
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) { kept += __shfl_xor(kept, o, 64); sum += __shfl_xor(sum, o, 64); }
      if (lane == 0) { sh.list.tile[tile] = sum; tile_kept += kept; }
    }
  }
  // ---- the candidates in order
  int n_pow = 1;
  while (n_pow < n_list) n_pow <<= 1;
  for (int i = n_list + tid; i < n_pow; i += kThreads) sh.list.order[i] = 0ull;
  __syncthreads();
  if (n_pow <= kThreads) sort_down<1, kThreads>(sh.list.order, n_pow);
  else if constexpr (kCap > kThreads) {
    if (n_pow == 2 * kThreads) sort_down<2, kThreads>(sh.list.order, n_pow);
    else if (n_pow == 4 * kThreads) sort_down<4, kThreads>(sh.list.order, n_pow);
    else if (n_pow == 8 * kThreads) sort_down<8, kThreads>(sh.list.order, n_pow);
    else sort_down<16, kThreads>(sh.list.order, n_pow);
  }
  // ---- the cut among them.  This thread's are own .. own + per
  const int per = max(1, n_pow / kThreads), own = tid * per;
  auto weight_at = [&](int i) { return weights.scaled(logit_of(static_cast<uint32_t>(sh.list.order[i] >> 32))); };
  int n_cand = n_list, kept_list = 0;
  if (cut) {
    const bool by_k = c.k_bin < kBins;
    // tokens that pass top-k: the list's first n_k.  (Candidates of p_lo .. p_hi come first; k_bin is among or behind them.)
    const int base_k = c.k_bin <= c.p_hi ? static_cast<int>(c.count_k - c.count_lo) : static_cast<int>(c.count_hi - c.count_lo);
    const int n_k = by_k ? base_k + s.top_k - static_cast<int>(c.count_k) : n_cand;
    unsigned long long in_k = 0, mine = 0;
    for (int i = own; i < min(own + per, n_cand); ++i) {
      const unsigned long long w = Weights::whole(weight_at(i));
      mine += w;
      if (i >= base_k && i < n_k) in_k += w;
    }
    unsigned long long mass_k = 0;
    if (s.top_p < 1.0) {
      mass_k = block_sum<W>(in_k, part_mass);
      mass_k = !by_k ? c.mass_all : c.mass_k + mass_k;
    }
    unsigned long long before = c.mass_lo + block_before<W>(mine, part_mass);
    const double target = s.top_p * static_cast<double>(mass_k);
    unsigned kept = 0;
    for (int i = own; i < min(own + per, n_cand); ++i) {
      const double w = weight_at(i);
      const unsigned long long f = Weights::whole(w);
      const bool first = i == 0 && c.p_lo == 0;        // rank 0
      if (first || (i < n_k && (s.top_p >= 1.0 || static_cast<double>(before) < target) && w >= weights.least)) {
        ++kept;
        const int e = static_cast<int>(~static_cast<uint32_t>(sh.list.order[i])) + shift;
        atomicAdd(&sh.list.tile[e / tile_len], f);
      }
      before += f;
    }
    kept_list = static_cast<int>(block_sum<W>(kept, part_count));
  }
  const unsigned long long last = kept_list > 0 ? sh.list.order[kept_list - 1] : ~0ull;     // (key, ~index) of the last kept candidate
  __syncthreads();
  // ---- the tile the number falls into
  const unsigned long long here = tid < n_tiles ? sh.list.tile[tid] : 0ull;
  const unsigned long long front = block_before<W>(here, part_mass), total = block_sum<W>(here, part_mass);
  const unsigned n_kept = block_sum<W>(tile_kept, part_count) + kept_list + (cut ? c.unlisted : 0u);
  const double target = s.u * static_cast<double>(total);
  if (static_cast<double>(front) <= target && static_cast<double>(front + here) > target) { found = tid; found_before = front; }
  __syncthreads();
  const int share = (tile_len + kThreads - 1) / kThreads, e0 = found * tile_len + tid * share, e1 = min(min(e0 + share, (found + 1) * tile_len), a.vocab + shift);
  auto kept_weight = [&](int e) {
    const int i = e - shift;
    if (i < 0) return 0.0;
    const float z = to_float(kParts ? in.row[i] : reinterpret_cast<const T*>(held)[e]);
    if (!(z > -INFINITY)) return 0.0;
    if (cut && bins.of(z) >= c.p_lo && ((static_cast<unsigned long long>(logit_key(z)) << 32) | ~static_cast<uint32_t>(i)) < last) return 0.0;
    const double w = weights.scaled(z);
    return w >= weights.least ? w : 0.0;
  };
  unsigned long long sum = 0;
  for (int e = e0; e < e1; ++e) sum += Weights::whole(kept_weight(e));
  unsigned long long before = found_before + block_before<W>(sum, part_mass);
  if (static_cast<double>(before) <= target && static_cast<double>(before + sum) > target)
    for (int e = e0; e < e1; ++e) {
      const double w = kept_weight(e);
      before += Weights::whole(w);
      if (static_cast<double>(before) > target) {
        a.token[row] = e - shift;
        if (a.logprob != nullptr) a.logprob[row] = static_cast<float>(log(w / static_cast<double>(total)));
        if (a.n_kept != nullptr) a.n_kept[row] = static_cast<int>(n_kept);
        break;
      }
    }
}

// Rows of up to 12 Ki logits are one kernel's, which holds them in LDS (smaller ones in less of it, so that several workgroups share a compute unit).  1, 32 and 256 rows
// of 5000 fp32 logits 14.7, 24.7 and 27.2 us, in parts 17.0, 26.4 and 31.6; of 16000 16.3, 28.7 and 32.8, in parts 16.8, 26.1 and 39.2; one row of 32000
// 29.4 and 23.8 (a compute unit alone takes 5 us for the weights of so many).
constexpr int kSmallRow = 16384, kLargeRow = 49152, kRowLogits = (kLargeRow - 32) / 4;     // bytes of LDS, of which 32 are for a row's beginning and end inside pieces

// Parts of 2048 to 8192 logits, so many that a call has about a thousand workgroups (four on a compute unit), at most 64 a row.  32 x 128256 with 1024
// workgroups 36 us, with 512 or 2048 43; 256 x 128001 in parts of 8192 113 us, of 4096 or 16384 126 (rows differ in work: shorter parts even it
// out, and each part has its cuts to find).  Workgroups of 16 wavefronts took longer throughout (1 x 32000 27.7 us instead of 23.5, 64 x 128256 57 instead of 49).
SamplePlan sample_plan(int n_rows, int vocab) {
  SamplePlan p{0, 0, 0, 0};
  if (vocab <= kRowLogits) return p;
  const long long wanted = std::max(1, std::min(kMaxParts, 1024 / std::max(1, n_rows)));
  const long long most = (vocab + 8 + kMaxParts - 1) / kMaxParts;                  // (8: a row's beginning inside a piece)
  const long long len = std::max(most, std::min<long long>(std::max((vocab + 8 + wanted - 1) / wanted, 2048ll), 8192));
  p.part_len = static_cast<int>((len + 2047) / 2048 * 2048);
  p.parts = (vocab + 8 + p.part_len - 1) / p.part_len;
  // (tiles of 1024 logits and more: what the last kernel reads of the row once more is a tile)
  p.wave_tiles = p.parts <= kTiles / 16 && p.part_len >= 16384 ? 4 : p.parts <= kTiles / 8 && p.part_len >= 8192 ? 2 : 1;
  p.tile_len = p.part_len / (4 * p.wave_tiles);
  return p;
}

}  // namespace

size_t sample_bytes(int n_rows, int vocab) { return sample_plan(n_rows, vocab).parts > 0 ? static_cast<size_t>(n_rows) * sizeof(RowScratch) : 0; }

template <typename T>
static void launch_sample_t(const SampleArgs& a, const SamplePlan& plan, RowScratch* ws, hipStream_t stream) {
  const dim3 grid(plan.parts, a.n_rows);
  if (plan.parts > 0) {
    hipLaunchKernelGGL(sample_max_kernel<T>, grid, dim3(256), 0, stream, a, plan, ws);
    if (a.top_k != nullptr || a.top_p != nullptr) hipLaunchKernelGGL(sample_hist_kernel<T>, grid, dim3(256), 0, stream, a, plan, ws);
    hipLaunchKernelGGL(sample_tiles_kernel<T>, grid, dim3(256), 0, stream, a, plan, ws);
  }
  // (behind other kernels a workgroup of four wavefronts: its barriers and sums over wavefronts are most of its time, and four of them have fewer)
  if (plan.parts > 0) hipLaunchKernelGGL((sample_draw_kernel<T, 4, 0>), dim3(a.n_rows), dim3(256), 0, stream, a, plan, ws);
  else if (a.vocab * sizeof(T) + 32 <= kSmallRow) hipLaunchKernelGGL((sample_draw_kernel<T, 16, kSmallRow>), dim3(a.n_rows), dim3(1024), 0, stream, a, plan, ws);
  else hipLaunchKernelGGL((sample_draw_kernel<T, 16, kLargeRow>), dim3(a.n_rows), dim3(1024), 0, stream, a, plan, ws);
}

void launch_sample(const void* logits, int logits_dtype, int n_rows, int vocab, long long stride, const float* temperature,
                   const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token, float* logprob,
                   int32_t* n_kept, void* workspace, hipStream_t stream) {
  int bits = 0;
  while ((1ll << bits) < vocab) ++bits;
  const SampleArgs a{logits, n_rows, vocab, stride, temperature, top_k, top_p, min_p, u, token, logprob, n_kept, std::min(50, 62 - bits)};
  const SamplePlan plan = sample_plan(n_rows, vocab);
  RowScratch* ws = static_cast<RowScratch*>(workspace);
  if (logits_dtype == CC_BF16) launch_sample_t<bf16_t>(a, plan, ws, stream);
  else launch_sample_t<float>(a, plan, ws, stream);
}

}  // namespace cc
