// HIP kernels (gfx950) of distillation from a teacher's most probable symbols
// (mca_distill) and its gradient (mca_distill_grad).
//
// The teacher's part of a row is at most 32 entries, worked on in 64 bits by one
// wave; the student's is one pass over the logits for a sum of exponentials.  With
// `rest` that is the sum over the symbols that are none of the teacher's, relative to
// the largest of those, and the teacher's are added behind the pass: the loss takes the
// logarithm of the first, which a difference of nearly equal sums, or exponentials relative
// to the largest logit of all, would lose where the teacher's symbols have nearly all
// weight.
//
// Bound by the logits' bytes for large vocabularies: bf16, 4096 rows of 50001 symbols, 20
// entries and rest, are 79 us (410 MB, 5.2 TB/s) and with the gradient 148 more (820 MB read and
// written, 5.5 TB/s); a large copy reaches 5.1 TB/s on this card.  For small ones by the entries'
// 64-bit chains of a wave: 8192 rows of 65, 7.5 and 7.0 us (2.2 MB read, as much written).
#include <algorithm>

#include "device_common.hpp"
#include "lm_device.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

constexpr int kDsThreads = 256;
constexpr int kDsWaves = kDsThreads / 64;
constexpr int kDsUnroll = 4;
constexpr int kDsSmall = 1024;     // largest vocabulary of the wave-per-row kernels
constexpr int64_t kDsFew = 1024;   // rows up to which that is kDsSmall / 2
constexpr int kDsSplits = 64;      // most parts of a row
constexpr int64_t kDsPart = 8192;  // symbols of a part at least
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;

// The sum s of exp(scale (z - m)) over a part of a row, m the largest logit of it (with
// `rest` of the symbols that are none of the teacher's).
struct Sums {
  float m, s;
  __device__ __forceinline__ void move(float to, float k2) {
    s *= __builtin_amdgcn_exp2f((m - to) * k2);
    m = to;
  }
  __device__ __forceinline__ void join(float m2, float s2, float k2) {
    move(fmaxf(m, m2), k2);
    s += s2 * __builtin_amdgcn_exp2f((m2 - m) * k2);
  }
};

// A wave's lane j: entry j of row t (-1: none).
struct Entry {
  int id;
  float logprob;
};
template <class Args>
__device__ __forceinline__ Entry entry_of(const Args& p, int64_t t, int lane) {
  Entry e{-1, 0.f};
  if (lane < p.n_top) {
    const int id = p.ids[t * p.n_top + lane];
    if (id >= 0 && id < p.n_vocab) e = {id, p.logprob[t * p.n_top + lane]};
  }
  return e;
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
  return x;
}
// A number of lane `from`, in all lanes.
__device__ __forceinline__ double lane_of(double x, int from) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, from), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), from);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
// Logarithms of the teacher's probabilities, relative to the largest without rest: no
// entry has any if that is -inf (`none`).
struct Logs {
  double x;
  bool any, none;
};
template <class Args>
__device__ __forceinline__ Logs logs_of(const Args& p, const Entry& e) {
  const float lp = e.id >= 0 ? e.logprob : -__builtin_huge_valf();
  Logs r;
  r.any = __ballot(e.id >= 0) != 0;
  r.none = false;
  r.x = (double)lp;
  if (p.rest == 0) {
    float top = lp;
    for (int d = 1; d < p.n_top; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(top)));
    r.none = top == -__builtin_huge_valf() && __ballot(lp != lp) == 0;
    r.x = r.none ? -__builtin_huge_val() : (double)p.scale * ((double)lp - (double)top);
  }
  return r;
}
// exp of a number that is at most 700 if it counts: what passes that (a logprob that is no
// logarithm of a probability) becomes NaN, as +inf does
__device__ __forceinline__ double prob_of(double x) { return x > 700.0 ? __builtin_nan("") : exp_of(x); }

// What the loss needs of a row's entries (one wave, entry j in lane j): with q_j
// their probabilities under the teacher, z_j their logits and m the largest of those
//   loss = part + q (la + k (top - m)) + other (log other - log s_r),
// part = sum q_j (log q_j - k (z_j - m)), q = sum q_j, for a sum over all symbols of
// exp(la + k top); with `rest`, s is that of exp(k (z - m)) over the entries' symbols.
struct Known {
  double part, q, other, s, norm;  // (without rest, log norm is still to be taken off part)
  float m;
  bool any;
};
template <int TYPE>
__device__ __forceinline__ Known known_of(const mca_distill_args& p, int64_t t, const Entry& e) {
  const int lane = threadIdx.x & 63, K = p.n_top;
  const double k = p.scale;
  const float z = e.id >= 0 ? to_f32<TYPE>(((const typename Elem<TYPE>::Raw*)p.logits)[t * p.logits_row + e.id]) : -__builtin_huge_valf();
  const Logs lp = logs_of(p, e);
  Known r;
  r.any = lp.any;
  float m = z;
  for (int d = 1; d < K; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  m = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(m)));
  r.m = m;
  const double y = k * ((double)z - (double)(m == -__builtin_huge_valf() ? 0.f : m));
  // The entries' probabilities in lanes 0 to 31, in lanes 32 on their exponentials under the
  // student: one stream of instructions for both.
  double x = lp.x;
  if (p.rest != 0) {
    bool first = e.id >= 0;  // a symbol counts once
    for (int j = 0; j < K; ++j) {
      const int id = __builtin_amdgcn_readlane(e.id, j);
      if (j < lane && id == e.id) first = false;
    }
    const double mine = first ? y : -__builtin_huge_val(), other = __shfl(mine, lane & 31, 64);
    x = lane < 32 ? x : other;
  }
  double sum = prob_of(x);
  double part = lane < 32 && (sum > 0 || sum != sum) ? sum * (x - y) : 0.0;
  if (p.rest == 0 && lane >= 32) sum = 0;
  for (int d = 1; d < K; d <<= 1) {
    sum += __shfl_xor(sum, d, 64);
    part += __shfl_xor(part, d, 64);
  }
  const double q = lane_of(sum, 0);
  part = lane_of(part, 0);
  r.s = lane_of(sum, 32);
  r.norm = 1;
  if (p.rest != 0) {
    r.q = q;
    r.other = fmax(1.0 - q, 0.0);
    r.part = part;
  } else {
    r.q = lp.none ? 0.0 : (q != q ? q : 1.0);
    r.other = 0;
    r.norm = lp.none ? 1.0 : q;
    r.part = lp.none ? 0.0 : part / q;
  }
  return r;
}
// The loss of row t from the pass's sum s relative to m, in lane 0.
__device__ __forceinline__ void finish(const mca_distill_args& p, int64_t t, const Known& e, float m, double s) {
  const int lane = threadIdx.x & 63;
  const double k = p.scale, inf = __builtin_huge_val();
  const bool rest = p.rest != 0;
  const double top = rest ? fmax((double)m, (double)e.m) : (double)m;
  double all = s;
  if (rest) {
    // exponentials of both maxima, a lane each
    const double f = exp_of(k * ((double)(lane == 0 ? m : e.m) - top));
    all = s * lane_of(f, 0) + (e.s == 0 ? 0.0 : e.s * lane_of(f, 1));
  }
  // logarithms beside k times the largest, which cancels from the loss; of three numbers
  // in a lane each
  const double l = log_of(lane == 0 ? all : (lane == 1 ? (rest ? s : e.norm) : (e.other > 0x1p-100 ? e.other : 1.0)));
  const double la = all == 0 ? -inf : lane_of(l, 0), ls = s == 0 ? -inf : lane_of(l, 1);
  const double part = rest ? e.part : e.part - lane_of(l, 1);
  double loss = 0;
  if (e.q != e.q)
    loss = e.q;
  else if (part == inf)
    loss = inf;
  else if (!(e.q == 0))
    loss = part + e.q * (la + k * (top - (e.m == -__builtin_huge_valf() ? 0.0 : (double)e.m)));
  if (e.other > 0) loss += s == 0 ? inf : e.other * (lane_of(l, 2) - (k * ((double)m - top) + ls - la));
  if (all != all) loss = all;
  if (lane == 0) {
    p.loss[t] = e.any ? (float)loss : 0.f;
    p.lse[t] = (float)(all == 0 ? -inf : k * top + la);
    if (rest) p.lse_rest[t] = (float)(s == 0 ? -inf : k * (double)m + ls);
  }
}

}  // namespace

// Larger rows: a workgroup per row, or per part of one (grid y), in one pass of its first
// four waves; the fifth has the row's entries meanwhile (behind the pass they cost 15 us of the
// 79).  With `rest` the teacher's symbols leave the pass in the registers: a ballot finds those
// among a round's 8192 bytes, mostly none (compared with each vector, they cost 40 us).
template <int TYPE>
__global__ __launch_bounds__(kDsThreads + 64) void k_lm_distill(mca_distill_args p, int splits, Sums* parts) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  typedef typename Elem<TYPE>::Raw Raw;
  __shared__ Sums s_sums[kDsWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const int split = blockIdx.y, V = (int)p.n_vocab;
  const float k2 = p.scale * kLog2e;
  const Raw* row = (const Raw*)p.logits + t * p.logits_row;
  const int head = (int)(((16 - ((uintptr_t)row & 15)) & 15) / EL);
  const int nvec = (V - head) / VE, tail = V - head - nvec * VE;
  const u32x4* vec = (const u32x4*)(row + head);
  const int per = (nvec + splits - 1) / splits, v0 = min(split * per, nvec), v1 = min(nvec, v0 + per);
  const Entry e = entry_of(p, t, lane);       // every wave has them
  const int mine = p.rest != 0 ? e.id : -1;  // to be left out
  if (wave == kDsWaves) {
    Known known{};
    if (splits == 1) known = known_of<TYPE>(p, t, e);
    __syncthreads();
    Sums a = s_sums[0];
#pragma unroll
    for (int w = 1; w < kDsWaves; ++w) a.join(s_sums[w].m, s_sums[w].s, k2);
    if (splits == 1)
      finish(p, t, known, a.m, a.s);
    else if (lane == 0)
      parts[t * splits + split] = a;
    return;
  }
  Sums a = {kLowest, 0.f};
  // `n` values from v on, of one lane
  auto take_some = [&](int v, int n) {
    for (int i = 0; i < n; ++i) {
      const bool out = __ballot(mine == v + i) != 0;
      const float z = to_f32<TYPE>(row[v + i]);
      if (lane == 0 && !out) a.join(z < kLowest ? kLowest : z, __builtin_amdgcn_exp2f((z - (z < kLowest ? kLowest : z)) * k2), k2);
    }
  };
  for (int b = v0 + wave * 64 * kDsUnroll; b < v1; b += kDsWaves * 64 * kDsUnroll) {
    u32x4 x[kDsUnroll];
#pragma unroll
    for (int u = 0; u < kDsUnroll; ++u) x[u] = gload(vec + min(b + 64 * u + lane, v1 - 1));
    // the teacher's symbols among these: their values become -inf, in every lane that holds
    // their vector (those behind the last vector hold it, too)
    const int s0 = head + b * VE;
    for (uint64_t some = __ballot(mine >= s0 && mine - s0 < 64 * kDsUnroll * VE); some != 0; some &= some - 1) {
      const int in = __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(some)) - s0, v = in / VE, word = in % VE * EL / 4;
      const uint32_t low = TYPE == MCA_TYPE_F32 ? 0xff800000u : (TYPE == MCA_TYPE_BF16 ? 0xff80u : 0xfc00u);
      const int shift = EL == 4 ? 0 : 16 * (in & 1);
      const uint32_t keep = EL == 4 ? 0u : 0xffff0000u >> shift;
#pragma unroll
      for (int u = 0; u < kDsUnroll; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool this_one = v == min(64 * u + lane, v1 - 1 - b) && i == word;
          x[u][i] = this_one ? (x[u][i] & keep) | (low << shift) : x[u][i];
        }
    }
    float top = -__builtin_huge_valf();
#pragma unroll
    for (int u = 0; u < kDsUnroll; ++u) {
      float f[VE];
      unpack<TYPE>(x[u], f);
#pragma unroll
      for (int i = 0; i < VE; ++i) top = fmaxf(top, f[i]);
    }
    // (lanes behind the last vector hold that one: its maximum is theirs)
    if (top > a.m) a.move(top, k2);
    float sum[kDsUnroll];
#pragma unroll
    for (int u = 0; u < kDsUnroll; ++u) {
      float f[VE];
      unpack<TYPE>(x[u], f);
      sum[u] = 0.f;
#pragma unroll
      for (int i = 0; i < VE; ++i) sum[u] += __builtin_amdgcn_exp2f((f[i] - a.m) * k2);
      sum[u] = b + 64 * u + lane < v1 ? sum[u] : 0.f;
    }
    a.s += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  static_assert(kDsUnroll == 4, "sums of a round");
  if (head > 0 && split == 0 && wave == 0) take_some(0, head);
  if (tail > 0 && split == splits - 1 && wave == kDsWaves - 1) take_some(V - tail, tail);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) a.join(__shfl_xor(a.m, d, 64), __shfl_xor(a.s, d, 64), k2);
  if (lane == 0) s_sums[wave] = a;
  __syncthreads();
}

template <int TYPE>
__global__ __launch_bounds__(64) void k_lm_distill_join(mca_distill_args p, int splits, const Sums* parts) {
  const int lane = threadIdx.x;
  const int64_t t = blockIdx.x;
  const Sums x = lane < splits ? parts[t * splits + lane] : Sums{kLowest, 0.f};
  float m = x.m;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  const double f = exp((double)p.scale * ((double)x.m - (double)m));
  finish(p, t, known_of<TYPE>(p, t, entry_of(p, t, lane)), m, wave_sum(f * x.s));
}

// Rows of at most 64 N symbols: a wave per row, the row in registers.  Bound by the
// entries' chain (an exponential, two logarithms of 64 bits and the sums over lanes), which
// waves of other rows fill.
template <int TYPE, int N>
__global__ __launch_bounds__(kDsThreads) void k_lm_distill_small(mca_distill_args p) {
  typedef typename Elem<TYPE>::Raw Raw;
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * kDsWaves + (threadIdx.x >> 6);
  if (t >= p.n_rows) return;
  const int V = (int)p.n_vocab;
  const Raw* row = (const Raw*)p.logits + t * p.logits_row;
  const float k2 = p.scale * kLog2e;
  const Entry e = entry_of(p, t, lane);
  float z[N], m = kLowest, s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) z[i] = lane + 64 * i < V ? to_f32<TYPE>(row[lane + 64 * i]) : -__builtin_huge_valf();
  if (p.rest != 0) {
    uint32_t mine = 0;  // which of the lane's symbols are the teacher's
    for (int j = 0; j < p.n_top; ++j) {
      const int id = __builtin_amdgcn_readlane(e.id, j);
      if (id >= 0 && (id & 63) == lane) mine |= 1u << (id >> 6);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = (mine >> i) & 1 ? -__builtin_huge_valf() : z[i];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, z[i]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
#pragma unroll
  for (int i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f((z[i] - m) * k2);
  finish(p, t, known_of<TYPE>(p, t, e), m, wave_sum((double)s));
}

namespace {

// A row's gradient: factors of exp(scale z - lse) for symbols of the teacher's and of
// exp(scale z - lse_other) for others, both at most 1, and what is taken off the teacher's.
struct RowGrad {
  float lse, lse_other, known, other;
  bool zero;
};
__device__ __forceinline__ RowGrad row_grad(const mca_distill_grad_args& p, int64_t t, const Entry& e, float* off) {
  RowGrad r;
  const int lane = threadIdx.x & 63;
  const double g = (double)p.grad_loss[t] * (double)p.scale;
  const bool rest = p.rest != 0;
  const Logs lp = logs_of(p, e);
  r.lse = r.lse_other = p.lse[t];
  const float lr = rest ? p.lse_rest[t] : 0.f;
  const bool nothing = rest && lr == -__builtin_huge_valf();  // then the others' exponentials are 0
  // the entries' probabilities, and in lane 63 the student's of the others
  const double q = prob_of(rest && lane == 63 ? (double)(nothing ? 0.f : lr) - (double)r.lse : lp.x);
  double sum = lane < 32 ? q : 0.0;
  for (int d = 1; d < p.n_top; d <<= 1) sum += __shfl_xor(sum, d, 64);
  sum = lane_of(sum, 0);
  const bool undefined = sum != sum || r.lse != r.lse;  // so is the loss
  r.zero = !lp.any || (r.lse == -__builtin_huge_valf() && !undefined);
  const double left = rest ? fmax(1.0 - sum, 0.0) : 0.0;
  // (without rest the entries' sum to 1, if any has some)
  const double total = rest ? (sum != sum ? sum : sum + left) : (lp.none ? 0.0 : (sum != sum ? sum : 1.0));
  r.known = r.other = (float)(g * total);
  if (rest) {
    r.lse_other = nothing ? 0.f : lr;
    r.other = nothing ? (undefined ? __builtin_nanf("") : 0.f) : (float)(g * (total * lane_of(q, 63) - left));
  }
  *off = (float)(lp.none ? 0.0 : g * (rest ? q : q / sum));
  return r;
}
__device__ __forceinline__ float prob(float z, float scale, float lse) {
  return __builtin_amdgcn_exp2f(fmaf(z, scale, -lse) * kLog2e);
}

}  // namespace

// Long rows: a workgroup takes 256 x kDsUnroll vectors of one row.  Which of them hold a
// teacher's symbol is a bit each in LDS, so that the entries are compared only with those
// vectors' values.
template <int TYPE>
__global__ __launch_bounds__(kDsThreads) void k_lm_distill_grad(mca_distill_grad_args p) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  typedef typename Elem<TYPE>::Raw Raw;
  __shared__ uint32_t s_flag[kDsThreads * kDsUnroll / 32];
  __shared__ int s_id[MCA_MAX_TOP];
  __shared__ float s_off[MCA_MAX_TOP];
  __shared__ RowGrad s_row;
  const int tid = threadIdx.x, lane = tid & 63, V = (int)p.n_vocab, K = p.n_top;
  const int64_t t = blockIdx.y;
  const Raw* row = (const Raw*)p.logits + t * p.logits_row;
  Raw* out = (Raw*)p.grad + t * p.grad_row;
  const int head = (int)(((16 - ((uintptr_t)row & 15)) & 15) / EL);
  const int nvec = (V - head) / VE, tail = V - head - nvec * VE;
  const u32x4* vec = (const u32x4*)(row + head);
  u32x4* vout = (u32x4*)(out + head);
  const int c0 = blockIdx.x * kDsThreads * kDsUnroll, b = c0 + tid;
  u32x4 x[kDsUnroll];
#pragma unroll
  for (int u = 0; u < kDsUnroll; ++u)
    if (b + kDsThreads * u < nvec) x[u] = gload(vec + b + kDsThreads * u);
  if (tid < kDsThreads * kDsUnroll / 32) s_flag[tid] = 0;
  __syncthreads();
  if (tid < 64) {
    const Entry e = entry_of(p, t, lane);
    float off;
    const RowGrad r = row_grad(p, t, e, &off);
    if (lane < K) {
      s_id[lane] = e.id;
      s_off[lane] = off;
    }
    if (lane == 0) s_row = r;
    if (e.id >= head) {
      const int v = (e.id - head) / VE - c0;
      if (v >= 0 && v < kDsThreads * kDsUnroll) atomicOr(&s_flag[v >> 5], 1u << (v & 31));
    }
  }
  __syncthreads();
  const RowGrad r = s_row;
  auto grads = [&](float (&f)[VE], int first, bool known) {
    float y[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) y[i] = r.zero ? 0.f : prob(f[i], p.scale, r.lse_other) * r.other;
    if (known && !r.zero) {
      uint32_t mine = 0;
      for (int j = 0; j < K; ++j) {
        const int at = s_id[j] - first;
        if (s_id[j] < 0 || at < 0 || at >= VE) continue;
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (i == at) y[i] = ((mine >> i) & 1 ? y[i] : prob(f[i], p.scale, r.lse) * r.known) - s_off[j];
        mine |= 1u << at;
      }
    }
#pragma unroll
    for (int i = 0; i < VE; ++i) f[i] = y[i];
  };
#pragma unroll
  for (int u = 0; u < kDsUnroll; ++u) {
    const int v = b + kDsThreads * u;
    if (v >= nvec) continue;
    float f[VE];
    unpack<TYPE>(x[u], f);
    grads(f, head + v * VE, (s_flag[(v - c0) >> 5] >> ((v - c0) & 31)) & 1);
    u32x4 y;
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
    float f[VE];
    f[0] = to_f32<TYPE>(row[v]);
#pragma unroll
    for (int i = 1; i < VE; ++i) f[i] = 0.f;
    // (of the VE values from v on only the first counts)
    grads(f, v, true);
    out[v] = from_f32<TYPE>(f[0]);
  }
}

// Short rows, and rows whose logits and gradient are not aligned alike: a wave per row,
// value by value.
template <int TYPE>
__global__ __launch_bounds__(kDsThreads) void k_lm_distill_grad_rows(mca_distill_grad_args p) {
  typedef typename Elem<TYPE>::Raw Raw;
  const int lane = threadIdx.x & 63, V = (int)p.n_vocab;
  const int64_t t = (int64_t)blockIdx.x * kDsWaves + (threadIdx.x >> 6);
  if (t >= p.n_rows) return;
  const Raw* row = (const Raw*)p.logits + t * p.logits_row;
  Raw* out = (Raw*)p.grad + t * p.grad_row;
  const Entry e = entry_of(p, t, lane);
  float off;
  const RowGrad r = row_grad(p, t, e, &off);
  for (int v0 = 0; v0 < V; v0 += 64) {
    const int v = v0 + lane;
    const float z = v < V ? to_f32<TYPE>(row[v]) : 0.f;
    float y = prob(z, p.scale, r.lse_other) * r.other;
    bool known = false;
    // the entries among these 64 symbols
    for (uint64_t some = __ballot(e.id >= v0 && e.id < v0 + 64); some != 0; some &= some - 1) {
      const int j = __builtin_ctzll(some);
      const int id = __shfl(e.id, j, 64);
      const float o = __shfl(off, j, 64);
      if (id != v) continue;
      y = (known ? y : prob(z, p.scale, r.lse) * r.known) - o;
      known = true;
    }
    if (v < V) out[v] = from_f32<TYPE>(r.zero ? 0.f : y);
  }
}

// Rows of more than 65536 symbols are split while they are fewer than 512.  (us whole and
// split, bf16: one row of 128000 12.2 and 7.4, 64 rows 15.7 and 10.6, 128 of them in fp32 22.5 and
// 16.9; but 300 rows 20.6 and 20.9, and of 50000 symbols one to 16 rows 7.7 and 8.1, 128 9.3 and 10.4:
// the second launch costs more than the first one's pass.  For 1024 workgroups and more, 600
// rows of 128000 take 36.6 for 32.6.)
LogprobsPlan lm_distill_plan(const mca_distill_args& a) {
  LogprobsPlan p{1, 0};
  if (a.n_vocab <= 8 * kDsPart || a.n_rows == 0) return p;
  const int64_t want = (512 + a.n_rows - 1) / a.n_rows, most = (a.n_vocab + kDsPart - 1) / kDsPart;
  p.splits = (int32_t)std::clamp<int64_t>(std::min(want, most), 1, kDsSplits);
  if (p.splits > 1) p.bytes = (size_t)a.n_rows * p.splits * sizeof(Sums);
  return p;
}

namespace {

// A wave per row up to kDsSmall symbols, of few rows up to half of that.  (us of a wave and of
// a workgroup a row, bf16: 4096 rows of 512 symbols 7.3 and 15.3, of 1000 11.6 and 15.4; 1024 rows
// of 512 5.9 and 5.8, of 1000 6.9 and 5.8; 16 rows of 300 5.5 and 5.7, of 1000 6.7 and 5.2.)
template <int TYPE>
void launch_distill(const mca_distill_args& a, const LogprobsPlan& plan, hipStream_t s) {
  const dim3 threads(kDsThreads), grid((unsigned)((a.n_rows + kDsWaves - 1) / kDsWaves));
  if (a.n_vocab <= 128)
    hipLaunchKernelGGL((k_lm_distill_small<TYPE, 2>), grid, threads, 0, s, a);
  else if (a.n_vocab <= 256)
    hipLaunchKernelGGL((k_lm_distill_small<TYPE, 4>), grid, threads, 0, s, a);
  else if (a.n_vocab <= 512)
    hipLaunchKernelGGL((k_lm_distill_small<TYPE, 8>), grid, threads, 0, s, a);
  else if (a.n_vocab <= kDsSmall && a.n_rows > kDsFew)
    hipLaunchKernelGGL((k_lm_distill_small<TYPE, 16>), grid, threads, 0, s, a);
  else {
    Sums* parts = (Sums*)a.workspace;
    constexpr int64_t kMost = 1 << 23;  // rows of a launch: a grid has less than 2^32 threads in x (rows in parts are few)
    for (int64_t t0 = 0; t0 < a.n_rows; t0 += kMost) {
      mca_distill_args b = a;
      b.n_rows = std::min(kMost, a.n_rows - t0);
      b.logits = (const char*)a.logits + t0 * a.logits_row * Elem<TYPE>::kSize;
      b.logprob += t0 * a.n_top;
      b.ids += t0 * a.n_top;
      b.loss += t0;
      b.lse += t0;
      if (b.lse_rest != nullptr) b.lse_rest += t0;
      hipLaunchKernelGGL((k_lm_distill<TYPE>), dim3((unsigned)b.n_rows, (unsigned)plan.splits), dim3(kDsThreads + 64), 0, s, b, plan.splits, parts);
    }
    if (plan.splits > 1)
      hipLaunchKernelGGL((k_lm_distill_join<TYPE>), dim3((unsigned)a.n_rows), dim3(64), 0, s, a, plan.splits, parts);
  }
}

// Vectors from 768 symbols on, where logits and gradient allow.  (us of a wave a row, value
// by value, and of vectors, bf16: 4096 rows of 512 symbols 6.4 and 9.0, of 700 8.8 and 11.4, of 1000
// 11.4 and 10.5, of 2000 18.9 and 12.6; 16 rows of 300 4.5 and 5.6, of 1000 6.6 and 4.7.)
template <int TYPE>
void launch_distill_grad(const mca_distill_grad_args& a, hipStream_t s) {
  const int el = Elem<TYPE>::kSize;
  const bool alike = (((uintptr_t)a.logits - (uintptr_t)a.grad) & 15) == 0 &&
                     (((a.logits_row - a.grad_row) * el) & 15) == 0;
  if (a.n_vocab >= 768 && alike) {
    const int64_t per = (int64_t)kDsThreads * kDsUnroll * Elem<TYPE>::kPer;
    for (int64_t t0 = 0; t0 < a.n_rows; t0 += 65535) {  // grid y
      mca_distill_grad_args b = a;
      b.n_rows = std::min<int64_t>(65535, a.n_rows - t0);
      b.logits = (const char*)a.logits + t0 * a.logits_row * el;
      b.grad = (char*)a.grad + t0 * a.grad_row * el;
      b.logprob += t0 * a.n_top;
      b.ids += t0 * a.n_top;
      b.lse += t0;
      if (b.lse_rest != nullptr) b.lse_rest += t0;
      b.grad_loss += t0;
      hipLaunchKernelGGL((k_lm_distill_grad<TYPE>), dim3((unsigned)((a.n_vocab + per - 1) / per), (unsigned)b.n_rows),
                         dim3(kDsThreads), 0, s, b);
    }
  } else {
    hipLaunchKernelGGL((k_lm_distill_grad_rows<TYPE>), dim3((unsigned)((a.n_rows + kDsWaves - 1) / kDsWaves)), dim3(kDsThreads),
                       0, s, a);
  }
}

}  // namespace

hipError_t lm_launch_distill(const mca_distill_args& a, const LogprobsPlan& plan, hipStream_t s) {
  switch (a.dtype) {
    case MCA_TYPE_F32: launch_distill<MCA_TYPE_F32>(a, plan, s); break;
    case MCA_TYPE_BF16: launch_distill<MCA_TYPE_BF16>(a, plan, s); break;
    default: launch_distill<MCA_TYPE_F16>(a, plan, s); break;
  }
  return hipGetLastError();
}

hipError_t lm_launch_distill_grad(const mca_distill_grad_args& a, hipStream_t s) {
  switch (a.dtype) {
    case MCA_TYPE_F32: launch_distill_grad<MCA_TYPE_F32>(a, s); break;
    case MCA_TYPE_BF16: launch_distill_grad<MCA_TYPE_BF16>(a, s); break;
    default: launch_distill_grad<MCA_TYPE_F16>(a, s); break;
  }
  return hipGetLastError();
}

}  // namespace mca
