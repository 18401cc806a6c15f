// HIP kernels (gfx950) of token log probabilities, entropies and alternatives
// (mca_token_logprobs) and their gradient (mca_token_logprobs_grad).
//
// With powers of two: y_v = z_v log2 e, reference M = y of the largest logit (of
// what has been read), s = sum 2^(y_v - M), w = sum (y_v - M) 2^(y_v - M).  Then
//   lse = ln 2 (M + log2 s),  logprob = ln 2 ((y_t - M) - log2 s),
//   entropy = ln 2 (log2 s - w / s),
// where M cancels from all but lse, so that large logits cost no precision.
// y - M is one fma with M = fl(m log2 e) of the largest logit m, the same for all
// parts of the row.  For |m| above 2^20, where M's rounding would show in the
// exponents (and for a row of nothing but the type's lowest value, where the
// product overflows), it is (z - m) log2 e instead.
#include <algorithm>

#include "device_common.hpp"
#include "lm_device.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

constexpr int kLpThreads = 256;
constexpr int kLpWaves = kLpThreads / 64;
constexpr int kLpUnroll = 4;     // 16-byte loads that a lane has in flight
constexpr int kLpBuf = 128;      // chunks that a wave holds as candidates: thinned when over 64
// Largest vocabulary of the wave-per-row kernel (fp32, 8192 rows of 1000, 0, 5 and 20
// alternatives: 9, 18 and 46 us; workgroup per row: 20, 39 and 40; 16 rows: 4, 9 and 22
// against 5, 9 and 9).
constexpr int kLpSmall = 1024;
constexpr int kLpSplits = 64;    // most parts of a row
// Symbols of a part at least (bf16, 8 rows of 128000 in parts of 4096, 8192, 16384 and
// 32768 at least: without alternatives 7.8, 7.9, 9.5 and 11.8 us; 20 of them 17, 15, 15
// and 20).
constexpr int64_t kLpPart = 8192;
constexpr float kLowest = -3.402823466e38f;
constexpr float kFar = -1e30f;   // below every exponent; times 0 it is 0
constexpr float kHuge = 1e38f;   // logits of this size times log2 e stay finite
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Order of floats as positive numbers (equal for the two zeros), and back.
__device__ __forceinline__ uint32_t sort_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return max(b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u), 1u);
}
// The part of the order that a type's values differ in: its last bits are all
// zeros (or, of negative values, ones), and a bisection does without them.
template <int TYPE>
__device__ __forceinline__ uint32_t short_key(float x) {
  constexpr int kSame = TYPE == MCA_TYPE_F32 ? 0 : (TYPE == MCA_TYPE_BF16 ? 16 : 13);
  return max(sort_key(x) >> kSame, 1u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
// Larger value first, then lower index; 0 is nothing.
__device__ __forceinline__ uint64_t rank_key(uint32_t key, uint32_t index) { return ((uint64_t)key << 32) | (uint32_t)~index; }

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
// How many of n keys in LDS go before `key`; behind the n, zeros up to a multiple
// of 8, so that eight are under way at a time.
__device__ __forceinline__ int keys_above(const uint64_t* keys, int n, uint64_t key) {
  int before = 0;
  for (int i = 0; i < n; i += 8) {
    uint64_t x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = keys[i + u];
#pragma unroll
    for (int u = 0; u < 8; ++u) before += x[u] > key;
  }
  return before;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
  return x;
}

// The sums of part of a row (m: its largest logit), and two parts joined.
struct Sums {
  float m, s, w;
};
__device__ __forceinline__ bool ordinary(float m) { return fabsf(m) < 0x1p20f; }
// y - M of logit z for the maximum m
__device__ __forceinline__ float exponent(float z, float m, bool plain) {
  return plain ? fmaf(z, kLog2e, -(m * kLog2e)) : (z - m) * kLog2e;
}
__device__ __forceinline__ Sums moved(Sums a, float m) {
  // the difference of the two references, the rounding of those that are products included
  const bool from = ordinary(a.m), to = ordinary(m);
  float e = (a.m - m) * kLog2e;
  if (from && to) e = a.m * kLog2e - m * kLog2e;
  else if (from) e += fmaf(-a.m, kLog2e, a.m * kLog2e);
  else if (to) e -= fmaf(-m, kLog2e, m * kLog2e);
  const float d = fmaxf(e, kFar), f = __builtin_amdgcn_exp2f(d);
  return {m, a.s * f, f * fmaf(d, a.s, a.w)};
}
__device__ __forceinline__ Sums join(Sums a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  a = moved(a, m);
  b = moved(b, m);
  return {m, a.s + b.s, a.w + b.w};
}
__device__ __forceinline__ Sums wave_join(Sums a) {
  const float m = wave_max(a.m);
  a = moved(a, m);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    a.s += __shfl_xor(a.s, d, 64);
    a.w += __shfl_xor(a.w, d, 64);
  }
  return a;
}

__device__ __forceinline__ int64_t token_of(const void* tokens, int bytes, int64_t t) {
  return bytes == 8 ? ((const int64_t*)tokens)[t] : (int64_t)((const int32_t*)tokens)[t];
}
// log probability of logit z in a row of sums a
__device__ __forceinline__ float logprob_of(const Sums& a, float z) {
  if (a.s == 0.f) return -__builtin_huge_valf();
  const float l2 = __builtin_amdgcn_logf(a.s);
  return ordinary(a.m) && fabsf(z) < kHuge ? kLn2 * (exponent(z, a.m, true) - l2) : (z - a.m) - kLn2 * l2;
}
// a row's three numbers (one thread)
template <int TYPE>
__device__ __forceinline__ void finish_row(const mca_token_logprobs_args& p, int64_t t, const Sums& a) {
  const bool none = a.s == 0.f;
  const float l2 = __builtin_amdgcn_logf(a.s);
  p.lse[t] = none ? -__builtin_huge_valf() : (ordinary(a.m) ? kLn2 * (a.m * kLog2e + l2) : a.m + kLn2 * l2);
  p.entropy[t] = none ? 0.f : kLn2 * (l2 - a.w / a.s);
  const int64_t tok = token_of(p.tokens, p.token_bytes, t);
  const typename Elem<TYPE>::Raw* row = (const typename Elem<TYPE>::Raw*)p.logits + t * p.logits_row;
  p.logprob[t] = tok < 0 || tok >= p.n_vocab ? 0.f : logprob_of(a, to_f32<TYPE>(row[tok]));
}

// an alternative that a row (with NaN) lacks
__device__ __forceinline__ void no_choice(const mca_token_logprobs_args& p, int64_t t, int n) {
  p.top_logprob[t * p.n_top + n] = __builtin_nanf("");
  p.top_id[t * p.n_top + n] = 0;
}

// A key that at least k and, if they are not equal, at most `most` of the wave's
// 64 keys reach, by bisection.
__device__ __forceinline__ uint32_t reached_by(uint32_t key, int k, int most) {
  uint32_t lo = key, hi = key;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    lo = min(lo, (uint32_t)__shfl_xor(lo, d, 64));
    hi = max(hi, (uint32_t)__shfl_xor(hi, d, 64));
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  int reach = 64;
  while (reach > most && lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    const int c = __popcll(__ballot(key >= mid));
    if (c >= k) {
      lo = mid;
      reach = c;
    } else {
      hi = mid - 1;
    }
  }
  return lo;
}

// Of cnt <= 64 N (key, id) pairs in LDS, ids rising, keeps at most `most` among
// which are the k with the largest keys, of equal ones the first; the order stays.
// One wave.  *least becomes a key that at least k of them reach.  It is found by
// bisection, which ends as soon as few enough reach it; only where so many keys are
// equal that none does are those thinned by their order.
template <int N>
__device__ __forceinline__ int keep_largest(uint32_t* key, uint32_t* id, int cnt, int k, int most, uint32_t* least) {
  const int lane = threadIdx.x & 63;
  wave_sync();
  if (cnt <= most) return cnt;
  uint32_t kk[N], ii[N], lo = 0xffffffffu, hi = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = 64 * i + lane;
    kk[i] = p < cnt ? key[p] : 0;
    ii[i] = p < cnt ? id[p] : 0;
    lo = min(lo, p < cnt ? kk[i] : 0xffffffffu);
    hi = max(hi, kk[i]);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    lo = min(lo, (uint32_t)__shfl_xor(lo, d, 64));
    hi = max(hi, (uint32_t)__shfl_xor(hi, d, 64));
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  int reach = cnt;  // keys of at least lo; fewer than k are above hi
  while (reach > most && lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) c += __popcll(__ballot(kk[i] >= mid));
    if (c >= k) {
      lo = mid;
      reach = c;
    } else {
      hi = mid - 1;
    }
  }
  int equal = reach;  // how many keys equal to lo are kept
  if (reach > most) {
    equal = k;
#pragma unroll
    for (int i = 0; i < N; ++i) equal -= __popcll(__ballot(kk[i] > lo));
  }
  int eq = 0, out = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool same = kk[i] == lo && 64 * i + lane < cnt;
    const uint64_t es = __ballot(same);
    const bool keep = kk[i] > lo || (same && eq + lanes_below(es) < equal);
    const uint64_t ks = __ballot(keep);
    if (keep) {
      const int at = out + lanes_below(ks);
      key[at] = kk[i];
      id[at] = ii[i];
    }
    eq += __popcll(es);
    out += __popcll(ks);
  }
  wave_sync();
  *least = lo;
  return out;
}

}  // namespace

// Rows of more than kLpSmall symbols: one workgroup per row, or per part of a
// row (grid y), in one pass over the logits.
//
// Alternatives.  The row is cut into chunks: its 16-byte vectors, and the values
// before the first and behind the last whole one.  The k largest values lie in
// the k chunks of largest maximum (equal ones: the first), because each of
// those maxima is a value.  So the pass compares one maximum per chunk with the
// k-th largest so far, and only larger ones go to the wave's buffer, which is
// thinned to about k when it is full; the chunks left are read again at the end.
//
// Bound by memory without alternatives (4096 rows of 50001, fp16, 410 MB: 77 us, 5.3
// TB/s), with 5 of them also by the comparisons and the thinning (96 us); few rows by
// latency (8 of 128000, bf16, 20 alternatives: 11 us and 5 of joining).
template <int TYPE, bool TOP>
__global__ __launch_bounds__(kLpThreads) void k_lm_logprobs(mca_token_logprobs_args p, int splits, Sums* part,
                                                            uint64_t* part_keys) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  typedef typename Elem<TYPE>::Raw Raw;
  __shared__ uint32_t s_key[TOP ? kLpWaves : 1][TOP ? kLpBuf : 1], s_id[TOP ? kLpWaves : 1][TOP ? kLpBuf : 1];
  __shared__ __attribute__((aligned(16))) uint64_t s_rank[TOP ? 64 * kLpWaves * VE + 8 : 1];
  __shared__ uint32_t s_least[kLpWaves];
  __shared__ int s_found;
  __shared__ Sums s_sums[kLpWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const int split = blockIdx.y, k = p.n_top, V = (int)p.n_vocab;
  const Raw* row = (const Raw*)p.logits + t * p.logits_row;
  const int head = (int)(((16 - ((uintptr_t)row & 15)) & 15) / EL);  // V > kLpSmall > 8
  const int nvec = (V - head) / VE, tail = V - head - nvec * VE;
  const u32x4* vec = (const u32x4*)(row + head);
  const int per = (nvec + splits - 1) / splits, v0 = min(split * per, nvec), v1 = min(nvec, v0 + per);
  Sums a = {kLowest, 0.f, 0.f};
  int cnt = 0;       // chunks held
  uint32_t thr = 0;  // only maxima of larger keys are taken: the wave has k that reach it
  // one chunk a lane; `here` lanes have one
  auto take = [&](const float (&f)[VE], bool here, int id) {
    float cm = f[0];
#pragma unroll
    for (int i = 1; i < VE; ++i) cm = fmaxf(cm, f[i]);
    if (__ballot(here && cm > a.m) != 0) a = moved(a, wave_max(here ? fmaxf(cm, a.m) : a.m));
    // 0 times the exponent of a logit of -inf has to be 0, which a bound on the
    // exponent gives; only chunks with such logits pay for it
    float low = f[0];
#pragma unroll
    for (int i = 1; i < VE; ++i) low = fminf(low, f[i]);
    auto add = [&](bool plain, bool bounded) {
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float y = exponent(f[i], a.m, plain), e = __builtin_amdgcn_exp2f(y);
        a.s += e;
        a.w = fmaf(e, bounded ? fmaxf(y, kFar) : y, a.w);
      }
    };
    if (ordinary(a.m) && __ballot(here && low < kFar) == 0) {
      if (here) add(true, false);
    } else if (here) {
      if (ordinary(a.m)) add(true, true); else add(false, true);
    }
    if constexpr (TOP) {
      const uint32_t key = short_key<TYPE>(cm);
      const uint64_t mask = __ballot(here && key > thr);
      if (mask != 0) {
        if ((mask >> lane) & 1) {
          const int at = cnt + lanes_below(mask);
          s_key[wave][at] = key;
          s_id[wave][at] = (uint32_t)id;
        }
        cnt += __popcll(mask);
        if (cnt > kLpBuf - 64) {
          cnt = keep_largest<kLpBuf / 64>(s_key[wave], s_id[wave], cnt, k, max(k + 8, 16), &thr);
        }
      }
    }
  };
  // `n` values from v on as lane 0's chunk
  auto take_part = [&](int v, int n, int id) {
    float f[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) f[i] = lane == 0 && i < n ? to_f32<TYPE>(row[v + i]) : -__builtin_huge_valf();
    take(f, lane == 0, id);
  };
  if (head > 0 && split == 0 && wave == 0) take_part(0, head, 0);
  for (int b = v0 + wave * 64 * kLpUnroll; b < v1; b += kLpWaves * 64 * kLpUnroll) {
    u32x4 x[kLpUnroll];
#pragma unroll
    for (int u = 0; u < kLpUnroll; ++u) x[u] = gload(vec + min(b + 64 * u + lane, v1 - 1));
    if (TOP && thr == 0 && b + 64 * kLpUnroll <= v1) {
      // the first whole round: at least k lanes reach the k-th largest of the lanes'
      // maxima, which spares the buffer most of the round
      float top = -__builtin_huge_valf();
#pragma unroll
      for (int u = 0; u < kLpUnroll; ++u) {
        float f[VE];
        unpack<TYPE>(x[u], f);
#pragma unroll
        for (int i = 0; i < VE; ++i) top = fmaxf(top, f[i]);
      }
      thr = reached_by(short_key<TYPE>(top), k, max(k + 8, 16)) - 1;  // that key itself is taken
    }
#pragma unroll
    for (int u = 0; u < kLpUnroll; ++u) {
      const int v = b + 64 * u + lane;
      float f[VE];
      unpack<TYPE>(x[u], f);
      take(f, v < v1, 1 + v);
    }
  }
  if (tail > 0 && split == splits - 1 && wave == kLpWaves - 1) take_part(V - tail, tail, nvec + 1);
  a = wave_join(a);
  if (lane == 0) s_sums[wave] = a;
  uint32_t mine = 0;
  if constexpr (TOP) {
    // the wave's chunks, at most 64, one a lane, and a key that k of them reach
    wave_sync();
    mine = lane < cnt ? s_key[wave][lane] : 0;
    const uint32_t least = cnt >= k ? reached_by(mine, k, k + 8) : 0;
    if (lane == 0) s_least[wave] = least;
    if (tid == 0) s_found = 0;
  }
  __syncthreads();
  a = s_sums[0];
#pragma unroll
  for (int w = 1; w < kLpWaves; ++w) a = join(a, s_sums[w]);
  if (tid == 0) {
    if (splits == 1)
      finish_row<TYPE>(p, t, a);
    else
      part[t * splits + split] = a;
  }
  if constexpr (TOP) {
    // The largest of those keys is one that k values reach, so only values that do
    // are ranked: k and a few, but for equal ones.
    uint32_t least = s_least[0];
#pragma unroll
    for (int w = 1; w < kLpWaves; ++w) least = max(least, s_least[w]);
    if (mine != 0 && mine >= least) {
      const int id = (int)s_id[wave][lane];
      const int v = id == 0 ? 0 : head + (id - 1) * VE;
      float f[VE];
      if (id == 0 || id > nvec) {
        const int n = id == 0 ? head : tail;
#pragma unroll
        for (int i = 0; i < VE; ++i) f[i] = to_f32<TYPE>(row[v + min(i, n - 1)]);
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (i < n && short_key<TYPE>(f[i]) >= least) s_rank[atomicAdd(&s_found, 1)] = rank_key(sort_key(f[i]), (uint32_t)(v + i));
      } else {
        unpack<TYPE>(gload(vec + id - 1), f);
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (short_key<TYPE>(f[i]) >= least) s_rank[atomicAdd(&s_found, 1)] = rank_key(sort_key(f[i]), (uint32_t)(v + i));
      }
    }
    __syncthreads();
    const int found = s_found;
    if (tid < 8) s_rank[found + tid] = 0;
    // behind the last: nothing of a part, and in a row with NaN something in bounds
    if (tid >= found && tid < k) {
      if (splits > 1) part_keys[(t * splits + split) * k + tid] = 0; else no_choice(p, t, tid);
    }
    __syncthreads();
    for (int i = tid; i < found; i += kLpThreads) {
      const uint64_t key = s_rank[i];
      const int before = keys_above(s_rank, found, key);
      if (before >= k) continue;
      if (splits == 1) {
        p.top_logprob[t * k + before] = logprob_of(a, key_value((uint32_t)(key >> 32)));
        p.top_id[t * k + before] = (int32_t)~(uint32_t)key;
      } else {
        part_keys[(t * splits + split) * k + before] = key;
      }
    }
  }
}

// The parts of a row joined.  Part lists are in falling order, so with
// j = ceil(k / splits) the least of the lists' j-th keys has at least k keys
// at or above it: only those are ranked.
template <int TYPE>
__global__ __launch_bounds__(kLpThreads) void k_lm_logprobs_join(mca_token_logprobs_args p, int splits, const Sums* part,
                                                                 const uint64_t* part_keys) {
  __shared__ __attribute__((aligned(16))) uint64_t s_rank[kLpSplits * MCA_MAX_TOP + 8];
  __shared__ int s_cnt;
  const int tid = threadIdx.x, lane = tid & 63, k = p.n_top;
  const int64_t t = blockIdx.x;
  // every wave joins the sums for itself
  Sums a = lane < splits ? part[t * splits + lane] : Sums{kLowest, 0.f, 0.f};
  a = wave_join(a);
  if (tid == 0) finish_row<TYPE>(p, t, a);
  if (k == 0) return;
  const uint64_t* keys = part_keys + t * splits * k;
  const int j = (k + splits - 1) / splits;
  uint64_t bound = lane < splits ? keys[lane * k + j - 1] : ~0ull;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t o = ((uint64_t)__shfl_xor((uint32_t)(bound >> 32), d, 64) << 32) | __shfl_xor((uint32_t)bound, d, 64);
    bound = min(bound, o);
  }
  if (tid == 0) s_cnt = 0;
  __syncthreads();
  for (int i = tid; i < splits * k; i += kLpThreads) {
    const uint64_t key = keys[i];
    if (key != 0 && key >= bound) s_rank[atomicAdd(&s_cnt, 1)] = key;
  }
  __syncthreads();
  const int n = s_cnt;
  if (tid < 8) s_rank[n + tid] = 0;
  if (tid >= n && tid < k) no_choice(p, t, tid);
  __syncthreads();
  for (int i = tid; i < n; i += kLpThreads) {
    const uint64_t key = s_rank[i];
    const int before = keys_above(s_rank, n, key);
    if (before < k) {
      p.top_logprob[t * k + before] = logprob_of(a, key_value((uint32_t)(key >> 32)));
      p.top_id[t * k + before] = (int32_t)~(uint32_t)key;
    }
  }
}

// Rows of at most 64 N symbols: a wave per row, the row in registers; the
// alternatives one after the other, each the wave's largest of what is left.
template <int TYPE, int N>
__global__ __launch_bounds__(kLpThreads) void k_lm_logprobs_small(mca_token_logprobs_args p) {
  typedef typename Elem<TYPE>::Raw Raw;
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * kLpWaves + (threadIdx.x >> 6);
  if (t >= p.n_rows) return;
  const int V = (int)p.n_vocab, k = p.n_top;
  const Raw* row = (const Raw*)p.logits + t * p.logits_row;
  float z[N];
  Sums a = {kLowest, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; ++i) z[i] = lane + 64 * i < V ? to_f32<TYPE>(row[lane + 64 * i]) : -__builtin_huge_valf();
#pragma unroll
  for (int i = 0; i < N; ++i) a.m = fmaxf(a.m, z[i]);
  a.m = wave_max(a.m);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = exponent(z[i], a.m, ordinary(a.m)), e = __builtin_amdgcn_exp2f(y);
    a.s += e;
    a.w = fmaf(e, fmaxf(y, kFar), a.w);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    a.s += __shfl_xor(a.s, d, 64);
    a.w += __shfl_xor(a.w, d, 64);
  }
  if (lane == 0) finish_row<TYPE>(p, t, a);
  uint32_t key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) key[i] = lane + 64 * i < V ? sort_key(z[i]) : 0;
  for (int n = 0; n < k; ++n) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < N; ++i) best = max(best, key[i]);
    uint32_t top = best;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor(top, d, 64));
    // the first of equal ones: the lowest register, then the lowest lane
    bool open = true;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint64_t mask = __ballot(open && key[i] == top);
      if (open && mask != 0) {
        const int at = __ffsll((unsigned long long)mask) - 1;
        if (lane == at) {
          key[i] = 0;
          p.top_logprob[t * k + n] = logprob_of(a, key_value(top));
          p.top_id[t * k + n] = 64 * i + at;
        }
        open = false;
      }
    }
  }
}

// One value of the gradient from its logit: lse = 0 and g = ge = 0 for rows of
// nothing but -inf.
struct RowGrad {
  float lse, entropy, g, ge;
  int64_t token;
};
__device__ __forceinline__ RowGrad row_grad(const mca_token_logprobs_grad_args& p, int64_t t) {
  RowGrad r;
  r.lse = p.lse[t];
  r.g = p.grad_logprob != nullptr ? p.grad_logprob[t] : 0.f;
  r.ge = p.grad_entropy != nullptr ? p.grad_entropy[t] : 0.f;
  r.entropy = p.grad_entropy != nullptr ? p.entropy[t] : 0.f;
  r.token = p.grad_logprob != nullptr ? token_of(p.tokens, p.token_bytes, t) : -1;
  if (r.token < 0 || r.token >= p.n_vocab) {
    r.token = -1;
    r.g = 0.f;
  }
  if (r.lse == -__builtin_huge_valf()) {
    r.lse = r.g = r.ge = 0.f;
    r.token = -1;
  }
  return r;
}
__device__ __forceinline__ float grad_of(const RowGrad& r, float z, bool token) {
  // a bound below which probabilities are 0, so that 0 times the logarithm is 0
  const float lp = fmaxf(z - r.lse, -1e4f);
  // NaN must stay: the maximum drops it from lp, not from the probability
  const float q = __builtin_amdgcn_exp2f((z - r.lse) * kLog2e);
  // q first: a probability of 0 gives 0 whatever finite number ge is
  const float d = -fmaf(q * (lp + r.entropy), r.ge, q * r.g);
  return token ? d + r.g : d;
}

// Long rows: a workgroup takes 256 x kLpUnroll vectors of one row.  Bound by memory
// (4096 rows of 50001, bf16, 819 MB read and written: 143 us, 5.7 TB/s).
template <int TYPE>
__global__ __launch_bounds__(kLpThreads) void k_lm_logprobs_grad(mca_token_logprobs_grad_args p) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  typedef typename Elem<TYPE>::Raw Raw;
  const int tid = threadIdx.x, V = (int)p.n_vocab;
  const int64_t t = blockIdx.y;
  const Raw* row = (const Raw*)p.logits + t * p.logits_row;
  Raw* out = (Raw*)p.grad + t * p.grad_row;
  const int head = (int)(((16 - ((uintptr_t)row & 15)) & 15) / EL);
  const int nvec = (V - head) / VE, tail = V - head - nvec * VE;
  const RowGrad r = row_grad(p, t);
  const u32x4* vec = (const u32x4*)(row + head);
  u32x4* vout = (u32x4*)(out + head);
  const int b = blockIdx.x * kLpThreads * kLpUnroll + tid;
  u32x4 x[kLpUnroll];
#pragma unroll
  for (int u = 0; u < kLpUnroll; ++u)
    if (b + kLpThreads * u < nvec) x[u] = gload(vec + b + kLpThreads * u);
#pragma unroll
  for (int u = 0; u < kLpUnroll; ++u) {
    const int v = b + kLpThreads * u;
    if (v >= nvec) continue;
    float f[VE];
    unpack<TYPE>(x[u], f);
    const int64_t at = r.token - head - (int64_t)v * VE;
    u32x4 y;
#pragma unroll
    for (int i = 0; i < VE; ++i) f[i] = grad_of(r, f[i], at == i);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (TYPE == MCA_TYPE_F32)
        y[i] = __float_as_uint(f[i]);
      else
        y[i] = from_f32<TYPE>(f[2 * i]) | ((uint32_t)from_f32<TYPE>(f[2 * i + 1]) << 16);
    }
    gstore(vout + v, y);
  }
  if (blockIdx.x == 0 && tid < head + tail) {
    const int v = tid < head ? tid : V - tail + (tid - head);
    out[v] = from_f32<TYPE>(grad_of(r, to_f32<TYPE>(row[v]), r.token == v));
  }
}

// Short rows, and rows whose logits and gradient are not aligned alike: a
// workgroup takes `rows` whole rows, value by value.  8192 rows of 65, fp32: 4.4 us.
// Long rows pay for it: bf16, 4096 of 50257 values, the logits' 50304 apart and the
// gradient's 50257, 537 us, and 142 with the gradient's 50304 apart too; 8 of 128000,
// 128001 apart and 128000, 190 us and 4.5.
template <int TYPE>
__global__ __launch_bounds__(kLpThreads) void k_lm_logprobs_grad_flat(mca_token_logprobs_grad_args p, int rows) {
  typedef typename Elem<TYPE>::Raw Raw;
  const unsigned V = (unsigned)p.n_vocab;
  const int64_t t0 = (int64_t)blockIdx.x * rows;
  const unsigned todo = (unsigned)min((int64_t)rows, p.n_rows - t0) * V;
  for (unsigned e = threadIdx.x; e < todo; e += kLpThreads) {
    const unsigned n = e / V, v = e - n * V;
    const int64_t t = t0 + n;
    const RowGrad r = row_grad(p, t);
    const float z = to_f32<TYPE>(((const Raw*)p.logits)[t * p.logits_row + v]);
    ((Raw*)p.grad)[t * p.grad_row + v] = from_f32<TYPE>(grad_of(r, z, r.token == (int64_t)v));
  }
}

LogprobsPlan lm_logprobs_plan(const mca_token_logprobs_args& a) {
  LogprobsPlan p{1, 0};
  if (a.n_vocab <= 2 * kLpPart || a.n_rows == 0) return p;
  // about 1024 workgroups (bf16, 20 alternatives, 600 rows of 50001 in 512, 1024 and 2048
  // workgroups at least: 32, 37 and 40 us, without alternatives 19, 20 and 21; 256 rows
  // without 12.8, 12.0 and 12.5; 64 of 128000 10.2, 9.9 and 9.8)
  const int64_t want = (1024 + a.n_rows - 1) / a.n_rows, most = (a.n_vocab + kLpPart - 1) / kLpPart;
  p.splits = (int32_t)std::clamp<int64_t>(std::min(want, most), 1, kLpSplits);
  if (p.splits > 1) p.bytes = (size_t)a.n_rows * p.splits * (sizeof(uint64_t) * a.n_top + sizeof(Sums));
  return p;
}

namespace {

template <int TYPE>
void launch_logprobs(const mca_token_logprobs_args& a, const LogprobsPlan& plan, hipStream_t s) {
  const dim3 threads(kLpThreads);
  if (a.n_vocab <= kLpSmall) {
    const dim3 grid((unsigned)((a.n_rows + kLpWaves - 1) / kLpWaves));
    if (a.n_vocab <= 128)
      hipLaunchKernelGGL((k_lm_logprobs_small<TYPE, 2>), grid, threads, 0, s, a);
    else if (a.n_vocab <= 256)
      hipLaunchKernelGGL((k_lm_logprobs_small<TYPE, 4>), grid, threads, 0, s, a);
    else if (a.n_vocab <= 512)
      hipLaunchKernelGGL((k_lm_logprobs_small<TYPE, 8>), grid, threads, 0, s, a);
    else
      hipLaunchKernelGGL((k_lm_logprobs_small<TYPE, 16>), grid, threads, 0, s, a);
    return;
  }
  uint64_t* keys = (uint64_t*)a.workspace;
  Sums* sums = (Sums*)(keys + (size_t)a.n_rows * plan.splits * a.n_top);
  const dim3 grid((unsigned)a.n_rows, (unsigned)plan.splits);
  if (a.n_top > 0)
    hipLaunchKernelGGL((k_lm_logprobs<TYPE, true>), grid, threads, 0, s, a, plan.splits, sums, keys);
  else
    hipLaunchKernelGGL((k_lm_logprobs<TYPE, false>), grid, threads, 0, s, a, plan.splits, sums, keys);
  if (plan.splits > 1)
    hipLaunchKernelGGL((k_lm_logprobs_join<TYPE>), dim3((unsigned)a.n_rows), threads, 0, s, a, plan.splits, sums, keys);
}

template <int TYPE>
void launch_grad(const mca_token_logprobs_grad_args& a, hipStream_t s) {
  const int el = Elem<TYPE>::kSize;
  const bool alike = (((uintptr_t)a.logits - (uintptr_t)a.grad) & 15) == 0 &&
                     (((a.logits_row - a.grad_row) * el) & 15) == 0;
  // (8192 rows of 256, fp32: 8.6 us with a workgroup or more a row, 7.2 value by value;
  // of 400 9.5 and 10.6, of 1000 13.3 and 21.4)
  if (a.n_vocab >= 512 && alike) {
    const int64_t per = (int64_t)kLpThreads * kLpUnroll * Elem<TYPE>::kPer;
    for (int64_t t0 = 0; t0 < a.n_rows; t0 += 65535) {  // grid y
      mca_token_logprobs_grad_args b = a;
      b.n_rows = std::min<int64_t>(65535, a.n_rows - t0);
      b.logits = (const char*)a.logits + t0 * a.logits_row * el;
      b.grad = (char*)a.grad + t0 * a.grad_row * el;
      b.tokens = a.tokens != nullptr ? (const char*)a.tokens + t0 * a.token_bytes : nullptr;
      b.lse += t0;
      if (b.entropy != nullptr) b.entropy += t0;
      if (b.grad_logprob != nullptr) b.grad_logprob += t0;
      if (b.grad_entropy != nullptr) b.grad_entropy += t0;
      hipLaunchKernelGGL((k_lm_logprobs_grad<TYPE>), dim3((unsigned)((a.n_vocab + per - 1) / per), (unsigned)b.n_rows),
                         dim3(kLpThreads), 0, s, b);
    }
  } else {
    const int rows = (int)std::max<int64_t>(1, 1024 / a.n_vocab);
    hipLaunchKernelGGL((k_lm_logprobs_grad_flat<TYPE>), dim3((unsigned)((a.n_rows + rows - 1) / rows)), dim3(kLpThreads),
                       0, s, a, rows);
  }
}

}  // namespace

hipError_t lm_launch_logprobs(const mca_token_logprobs_args& a, const LogprobsPlan& plan, hipStream_t s) {
  if (a.n_rows == 0) return hipSuccess;
  switch (a.dtype) {
    case MCA_TYPE_F32: launch_logprobs<MCA_TYPE_F32>(a, plan, s); break;
    case MCA_TYPE_BF16: launch_logprobs<MCA_TYPE_BF16>(a, plan, s); break;
    default: launch_logprobs<MCA_TYPE_F16>(a, plan, s); break;
  }
  return hipGetLastError();
}

hipError_t lm_launch_logprobs_grad(const mca_token_logprobs_grad_args& a, hipStream_t s) {
  if (a.n_rows == 0) return hipSuccess;
  switch (a.dtype) {
    case MCA_TYPE_F32: launch_grad<MCA_TYPE_F32>(a, s); break;
    case MCA_TYPE_BF16: launch_grad<MCA_TYPE_BF16>(a, s); break;
    default: launch_grad<MCA_TYPE_F16>(a, s); break;
  }
  return hipGetLastError();
}

}  // namespace mca
