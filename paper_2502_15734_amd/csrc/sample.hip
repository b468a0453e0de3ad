// cc_sample: one token per row of logits.
//
// With x_i = (z_i - max z) / T the weights are w_i = exp(x_i), taken in 64 bits and held as whole multiples of 2^-shift
// (shift = 62 - ceil(log2 vocab), so that a row's sum stays below 2^62): sums of whole numbers come out the same in every order, so the
// drawn token does not depend on how a row is divided, and an error of 2^-46 per weight does not move a border that a float would.
// The kept tokens are the first ranks of the order (logit descending, index ascending); a rank cut is a logit and a number of
// its ties, found by a radix descent over the logits' ordered bit patterns with counts and weights per digit.
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
  s.greedy = !(t > 0.f);
  s.inv_t = s.greedy ? 1.0 : 1.0 / static_cast<double>(t);
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  s.top_k = s.greedy ? 1 : (k <= 0 || k > a.vocab) ? a.vocab : k;
  const float p = a.top_p != nullptr ? a.top_p[row] : 1.f, m = a.min_p != nullptr ? a.min_p[row] : 0.f, u = a.u[row];
  s.top_p = p < 1.f ? fmax(static_cast<double>(p), 0.0) : 1.0;                  // (a NaN: off)
  s.min_p = m > 0.f ? static_cast<double>(m) : 0.0;
  s.u = u > 0.f ? fmin(static_cast<double>(u), 1.0 - 0x1p-24) : 0.0;
  return s;
}

// weight of a logit against the row's largest one
__device__ __forceinline__ double weight_of(uint32_t key, uint32_t top, double inv_t) {
  if (key == top) return 1.0;
  if (key <= kKeyNone || top == kKeyInf) return 0.0;
  return exp((static_cast<double>(logit_of(key)) - static_cast<double>(logit_of(top))) * inv_t);
}
__device__ __forceinline__ unsigned long long fixed_of(double w, int shift) { return static_cast<unsigned long long>(ldexp(w, shift) + 0.5); }

template <typename T>
__device__ __forceinline__ uint32_t key_at(const SampleArgs& a, int row, int i) {
  return logit_key(to_float(static_cast<const T*>(a.logits)[static_cast<size_t>(row) * a.stride + i]));
}

struct Cut {              // the ranks above it: logits above key, and the first `ties` (by index) of those equal to it
  uint32_t key;
  unsigned ties;
};

constexpr int kWaves = 16;

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(64 * kWaves) void sample_row_kernel(SampleArgs a) {
  __shared__ unsigned count[256];
  __shared__ unsigned long long mass[256];
  __shared__ uint32_t wave_key[kWaves];
  __shared__ int wave_idx[kWaves];
  __shared__ unsigned wave_ties[kWaves], wave_kept[kWaves];
  __shared__ unsigned long long wave_mass[kWaves];
  __shared__ unsigned found_digit, found_count;
  __shared__ unsigned long long found_mass;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = a.vocab;
  const RowSettings s = settings_of(a, row);

  // ---- the largest logit and its lowest index
  uint32_t top = 0;
  int top_idx = 0x7fffffff;
  for (int i = tid; i < n; i += 64 * kWaves) {
    const uint32_t k = key_at<T>(a, row, i);
    if (k > top) { top = k; top_idx = i; }
  }
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t k = __shfl_xor(top, o, 64);
    const int i = __shfl_xor(top_idx, o, 64);
    if (k > top || (k == top && i < top_idx)) { top = k; top_idx = i; }
  }
  if (lane == 0) { wave_key[wave] = top; wave_idx[wave] = top_idx; }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w)
    if (wave_key[w] > top || (wave_key[w] == top && wave_idx[w] < top_idx)) { top = wave_key[w]; top_idx = wave_idx[w]; }
  if (top <= kKeyNone || s.greedy) {                   // (nothing to draw; or nothing else than the largest)
    if (tid == 0) {
      const bool none = top <= kKeyNone;
      a.token[row] = none ? -1 : top_idx;
      if (a.logprob != nullptr) a.logprob[row] = none ? -INFINITY : 0.f;
      if (a.n_kept != nullptr) a.n_kept[row] = none ? 0 : 1;
    }
    return;
  }

  // ---- radix descent: the cut behind the rank at which the count reaches `want` or the weights in front reach `target`
  unsigned long long set_mass = 0;                     // weights above the cut, its kept ties included
  auto descend = [&](bool by_mass, unsigned want, double target) {
    uint32_t prefix = 0;
    unsigned above = 0;
    unsigned long long above_mass = 0;
    for (int digit = 3; digit >= 0; --digit) {
      if (tid < 256) { count[tid] = 0; mass[tid] = 0; }
      __syncthreads();
      for (int i = tid; i < n; i += 64 * kWaves) {
        const uint32_t k = key_at<T>(a, row, i);
        if (k <= kKeyNone || (digit < 3 && (k >> (8 * digit + 8)) != prefix)) continue;
        atomicAdd(&count[(k >> (8 * digit)) & 255], 1u);
        atomicAdd(&mass[(k >> (8 * digit)) & 255], fixed_of(weight_of(k, top, s.inv_t), a.shift));
      }
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
        found_digit = at; found_count = c; found_mass = m;
      }
      __syncthreads();
      prefix = (prefix << 8) | found_digit;
      above = found_count;
      above_mass = found_mass;
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
  const int share = (n + kWaves - 1) / kWaves, i0 = wave * share, i1 = min(n, i0 + share);
  auto weight = [&](uint32_t k) {
    const double w = k > kKeyNone ? weight_of(k, top, s.inv_t) : 0.0;
    return w >= s.min_p || k == top ? w : 0.0;
  };
  const bool tie_in = cut.key > kKeyNone && (weight(cut.key) > 0.0 || s.min_p == 0.0);
  const unsigned long long each = tie_in ? fixed_of(weight(cut.key), a.shift) : 0;
  unsigned kept = 0, ties = 0;
  unsigned long long sum = 0;
  for (int i = i0 + lane; i < i1; i += 64) {
    const uint32_t k = key_at<T>(a, row, i);
    if (k <= kKeyNone) continue;
    if (k == cut.key) ++ties;
    else if (k > cut.key) {
      const double w = weight_of(k, top, s.inv_t);
      if (w >= s.min_p || k == top) { ++kept; sum += fixed_of(w, a.shift); }
    }
  }
  for (int o = 32; o > 0; o >>= 1) { kept += __shfl_xor(kept, o, 64); ties += __shfl_xor(ties, o, 64); sum += __shfl_xor(sum, o, 64); }
  if (lane == 0) { wave_ties[wave] = ties; wave_kept[wave] = kept; wave_mass[wave] = sum; }
  __syncthreads();
  unsigned ties_before = 0, n_kept = 0, first_ties = 0;
  unsigned long long total = 0;
  for (int w = 0; w < kWaves; ++w) {
    const unsigned left = cut.ties > ties_before ? cut.ties - ties_before : 0, t = tie_in ? min(left, wave_ties[w]) : 0;
    if (w == wave) first_ties = ties_before;
    n_kept += wave_kept[w] + t;
    total += wave_mass[w] + each * t;
    ties_before += wave_ties[w];
  }
  // (the largest logit with min_p above 1: it alone)
  const bool alone = s.min_p > 1.0;
  if (alone) {
    if (tid == 0) {
      a.token[row] = top_idx;
      if (a.logprob != nullptr) a.logprob[row] = 0.f;
      if (a.n_kept != nullptr) a.n_kept[row] = 1;
    }
    return;
  }
  const double target = s.u * static_cast<double>(total);
  unsigned long long before = 0;
  unsigned tb = 0;
  int mine = -1;
  for (int w = 0; w < kWaves; ++w) {
    const unsigned left = cut.ties > tb ? cut.ties - tb : 0, t = tie_in ? min(left, wave_ties[w]) : 0;
    const unsigned long long m = wave_mass[w] + each * t;
    tb += wave_ties[w];
    if (static_cast<double>(before + m) > target) { mine = w; break; }
    before += m;
  }
  if (wave != mine) return;
  unsigned seen = first_ties;
  for (int base = i0; base < i1; base += 64) {
    const int i = base + lane;
    const uint32_t k = i < i1 ? key_at<T>(a, row, i) : 0;
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

}  // namespace

size_t sample_bytes(int, int) { return 0; }

void launch_sample(const void* logits, int logits_dtype, int n_rows, int vocab, long long stride, const float* temperature,
                   const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* token, float* logprob,
                   int32_t* n_kept, void* workspace, hipStream_t stream) {
  int bits = 0;
  while ((1ll << bits) < vocab) ++bits;
  const SampleArgs a{logits, n_rows, vocab, stride, temperature, top_k, top_p, min_p, u, token, logprob, n_kept, 62 - bits};
  if (logits_dtype == CC_BF16) hipLaunchKernelGGL(sample_row_kernel<bf16_t>, dim3(n_rows), dim3(64 * kWaves), 0, stream, a);
  else hipLaunchKernelGGL(sample_row_kernel<float>, dim3(n_rows), dim3(64 * kWaves), 0, stream, a);
}

}  // namespace cc
