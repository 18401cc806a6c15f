// HIP kernels (gfx950) of the verification of drafted tokens (mca_verify_drafts).
//
// With p and q the softmax of a node's target and draft logits, what a node's
// children and the token behind them are drawn from after j rejections is
// max(p - c_j q, 0) / S_j: max(max(p - c q, 0) / S - q, 0) is max(p - (c + S) q, 0) / S,
// so c_{j+1} = c_j + S_j, and one number a node stands for all that was rejected.
//
// Four steps: sums of exponentials of all rows (nothing hangs on what is accepted, and
// it reads nearly all of the bytes), the walk of each request, and for the node that it
// ends at the sums again in 64 bits and the draw.  The draw compares a random number
// with sums over the vocabulary, whose borders lie close: exponentials of 32 bits move
// them by 1e-8, which at 128000 symbols would give another token once in a thousand draws,
// those of 64 by 1e-16.
#include <algorithm>

#include "device_common.hpp"
#include "lm_device.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

constexpr int kVThreads = 256;
constexpr int kVWaves = kVThreads / 64;
constexpr int kVUnroll = 4;
constexpr int kVMaxSplits = 64;   // parts of a row
constexpr int64_t kVPart = 8192;  // symbols of a part at least
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;

// A part of a row: its largest logit, and the sum of exp(scale (z - m)); of greedy
// calls the first symbol of that logit.  s is NaN if the part has NaN or +inf.
struct RowPart {
  float m, s;
  int32_t at, reserved;
};
// Where a request's path ends: what its token is drawn from.
struct End {
  int64_t row;  // of the logits; -1: no token
  double c;     // 0: p alone
  float mp, mq;  // largest logits
  int32_t first, node, gone, reserved;  // given drafts: this many of the node's children were rejected
};

struct VerifyDev {
  mca_verify_drafts_args a;
  int32_t splits, cuts;  // parts of a row in the first and in the last steps
  RowPart* parts;        // [n_rows][1 or 2][splits]
  End* ends;             // [n_req]
  double* sums;          // [n_req][2][cuts]: sums of exponentials
  double* left;          // [n_req][cuts]: sums of what is drawn from
  int32_t* tickets;      // [n_req]
  int32_t* paths;        // [n_rows]
};

// 16 bytes at any address
template <int TYPE>
__device__ __forceinline__ void load_any(const char* p, float (&f)[Elem<TYPE>::kPer]) {
  struct __attribute__((packed)) Any {
    u32x4 x;
  };
  unpack<TYPE>(((const Any*)p)->x, f);
}
// symbols v .. v + kPer - 1 of a row of V; behind it -inf
template <int TYPE>
__device__ __forceinline__ void load_symbols(const char* row, int v, int V, float (&f)[Elem<TYPE>::kPer]) {
  constexpr int VE = Elem<TYPE>::kPer;
  if (v + VE <= V) {
    load_any<TYPE>(row + (int64_t)v * Elem<TYPE>::kSize, f);
  } else {
#pragma unroll
    for (int i = 0; i < VE; ++i)
      f[i] = v + i < V ? to_f32<TYPE>(((const typename Elem<TYPE>::Raw*)row)[v + i]) : -__builtin_huge_valf();
  }
}
template <class T>
__device__ __forceinline__ T wave_sum(T x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
  return x;
}
// the workgroup's sum, in a fixed order, for all its threads
template <int WAVES>
__device__ __forceinline__ double group_sum(double x, double* s) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
  __syncthreads();
  x = s[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) x += s[w];
  return x;
}

// Request of row t, by 64 at a time; -1 if it is none's.
__device__ __forceinline__ int row_request(const int32_t* offsets, int n_req, int64_t t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_req;
  while (true) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int c = __popcll(__ballot(at < hi && offsets[min(at, hi - 1)] <= t));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    hi = min(hi, lo + step);
    if (step == 1) return t < offsets[lo + 1] ? lo : -1;
  }
}
__device__ __forceinline__ bool nodes_of(const mca_verify_drafts_args& a, int r, int* first, int* n) {
  const int64_t f = a.offsets[r], e = a.offsets[r + 1];
  *first = (int)f;
  *n = (int)(e - f);
  return f >= 0 && e > f && e <= a.n_rows && e - f <= a.max_nodes;
}

}  // namespace

// Sums of a row's part: grid (rows, parts of the target's, then of the draft's).  Rows
// of no request, and draft rows of nodes without children, are left out.
template <int TYPE, bool GREEDY>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_rows(VerifyDev p) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  typedef typename Elem<TYPE>::Raw Raw;
  const mca_verify_drafts_args& a = p.a;
  __shared__ float s_m[kVWaves], s_s[kVWaves];
  __shared__ int s_at[kVWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const int which = blockIdx.y / p.splits, split = blockIdx.y - which * p.splits, V = (int)a.n_vocab;
  const int r = row_request(a.offsets, a.n_req, t);
  if (r < 0) return;
  if (which == 1) {
    int first, n;
    if (!nodes_of(a, r, &first, &n)) return;
    const int node = (int)(t - first);
    bool child = false;
    for (int i = node + 1 + lane; i < n; i += 64) child = child || a.parents[first + i] == node;
    if (__ballot(child) == 0) return;
  }
  const float k2 = (float)((which ? a.draft_scale : a.scale) * 1.4426950408889634);
  const Raw* row = (const Raw*)(which ? a.draft : a.target) + t * (which ? a.draft_row : a.target_row);
  const int head = min(V, (int)(((16 - ((uintptr_t)row & 15)) & 15) / EL));
  const int nvec = (V - head) / VE, tail = V - head - nvec * VE;
  const u32x4* vec = (const u32x4*)(row + head);
  const int per = (nvec + p.splits - 1) / p.splits, v0 = min(split * per, nvec), v1 = min(nvec, v0 + per);
  float m = kLowest, s = 0.f;
  int at = 0;
  auto take = [&](const float (&f)[VE], bool here, int first) {
    if constexpr (GREEDY) {
      if (here) {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          s += f[i] < __builtin_huge_valf() ? 0.f : __builtin_nanf("");
          if (f[i] > m) {
            m = f[i];
            at = first + i;
          }
        }
      }
    } else {
      float cm = f[0];
#pragma unroll
      for (int i = 1; i < VE; ++i) cm = fmaxf(cm, f[i]);
      if (here && cm > m) {
        s *= __builtin_amdgcn_exp2f((m - cm) * k2);
        m = cm;
      }
      if (here) {
#pragma unroll
        for (int i = 0; i < VE; ++i) s += __builtin_amdgcn_exp2f((f[i] - m) * k2);
      }
    }
  };
  auto take_some = [&](int v, int n) {
    float f[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) f[i] = i < n ? to_f32<TYPE>(row[v + i]) : -__builtin_huge_valf();
    take(f, lane == 0, v);
  };
  if (GREEDY) m = -__builtin_huge_valf();
  if (head > 0 && split == 0 && wave == 0) take_some(0, head);
  for (int b = v0 + wave * 64 * kVUnroll; b < v1; b += kVWaves * 64 * kVUnroll) {
    u32x4 x[kVUnroll];
#pragma unroll
    for (int u = 0; u < kVUnroll; ++u) x[u] = gload(vec + min(b + 64 * u + lane, v1 - 1));
#pragma unroll
    for (int u = 0; u < kVUnroll; ++u) {
      const int v = b + 64 * u + lane;
      float f[VE];
      unpack<TYPE>(x[u], f);
      take(f, v < v1, head + v * VE);
    }
  }
  if (tail > 0 && split == p.splits - 1 && wave == kVWaves - 1) take_some(V - tail, tail);
  // lanes, then waves; equal logits: the first symbol
  auto join = [&](float m2, float s2, int at2) {
    if constexpr (GREEDY) {
      if (m2 > m || (m2 == m && at2 < at)) {
        m = m2;
        at = at2;
      }
      s += s2;
    } else {
      const float mn = fmaxf(m, m2);
      s = s * __builtin_amdgcn_exp2f((m - mn) * k2) + s2 * __builtin_amdgcn_exp2f((m2 - mn) * k2);
      m = mn;
    }
  };
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) join(__shfl_xor(m, d, 64), __shfl_xor(s, d, 64), __shfl_xor(at, d, 64));
  if (lane == 0) {
    s_m[wave] = m;
    s_s[wave] = s;
    s_at[wave] = at;
  }
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int w = 1; w < kVWaves; ++w) join(s_m[w], s_s[w], s_at[w]);
    const int both = a.draft != nullptr && !GREEDY ? 2 : 1;
    p.parts[(t * both + which) * p.splits + split] = {m, s, at, 0};
  }
}

// A request's walk, by one workgroup; every wave takes the same steps.
template <int TYPE, bool GREEDY>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_walk(VerifyDev p) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  typedef typename Elem<TYPE>::Raw Raw;
  const mca_verify_drafts_args& a = p.a;
  const bool drawn = a.draft != nullptr && !GREEDY;
  __shared__ float s_m[2][MCA_MAX_NODES];
  __shared__ double s_sum[2][MCA_MAX_NODES];  // 0: no softmax; of greedy calls 1
  __shared__ int s_best[MCA_MAX_NODES];
  __shared__ int s_up[MCA_MAX_NODES], s_tok[MCA_MAX_NODES];
  __shared__ float s_u[MCA_MAX_NODES];
  __shared__ double s_p[MCA_MAX_NODES], s_q[MCA_MAX_NODES];  // of a node's token at its parent
  __shared__ double s_red[kVWaves];
  const int tid = threadIdx.x, lane = tid & 63, r = blockIdx.x, V = (int)a.n_vocab;
  int first, n;
  if (tid == 0) p.tickets[r] = 0;
  if (!nodes_of(a, r, &first, &n)) {
    if (tid == 0) {
      a.new_len[r] = a.lengths[r];
      a.token[r] = -1;
      p.ends[r].row = -1;
    }
    return;
  }
  // every node's sums, parent and token
  for (int x = tid; x < n * (drawn ? 2 : 1); x += kVThreads) {
    const int which = x >= n, i = x - which * n;
    const RowPart* part = p.parts + ((int64_t)(first + i) * (drawn ? 2 : 1) + which) * p.splits;
    bool parent = which == 0;
    if (which)
      for (int j = i + 1; j < n; ++j) parent = parent || a.parents[first + j] == i;
    float m = kLowest;
    double s = 0;
    int at = -1;
    if (GREEDY) m = -__builtin_huge_valf();
    if (parent) {
      for (int y = 0; y < p.splits; ++y) {
        const RowPart u = part[y];
        if constexpr (GREEDY) {
          if (u.m > m) {
            m = u.m;
            at = u.at;
          }
          s += u.s;
        } else {
          m = fmaxf(m, u.m);
        }
      }
      if constexpr (GREEDY) {
        s = s == 0 && at >= 0 ? 1.0 : 0.0;
      } else {
        const double k = which ? a.draft_scale : a.scale;
        for (int y = 0; y < p.splits; ++y) s += (double)part[y].s * exp(k * ((double)part[y].m - (double)m));
      }
    }
    s_m[which][i] = m;
    s_sum[which][i] = s > 0 ? s : 0.0;  // NaN: none
    if (which == 0) s_best[i] = at;
  }
  if (tid < n) {
    const int up = a.parents[first + tid];
    s_up[tid] = tid > 0 && up >= 0 && up < tid ? up : -1;
    s_tok[tid] = a.tokens[first + tid];
    if constexpr (!GREEDY) s_u[tid] = a.accept[first + tid];
  }
  __syncthreads();
  if (!GREEDY && tid < n && s_up[tid] >= 0 && s_tok[tid] >= 0 && s_tok[tid] < V) {
    const int up = s_up[tid];
    const int64_t row = first + up;
    const float z = to_f32<TYPE>(((const Raw*)a.target)[row * a.target_row + s_tok[tid]]);
    s_p[tid] = exp(a.scale * ((double)z - (double)s_m[0][up])) / s_sum[0][up];
    if (drawn) {
      const float d = to_f32<TYPE>(((const Raw*)a.draft)[row * a.draft_row + s_tok[tid]]);
      s_q[tid] = exp(a.draft_scale * ((double)d - (double)s_m[1][up])) / s_sum[1][up];
    }
  }
  __syncthreads();
  const int up0 = lane < n ? s_up[lane] : -1, up1 = lane + 64 < n ? s_up[lane + 64] : -1;
  const bool legal0 = lane < n && s_tok[lane] >= 0 && s_tok[lane] < V;
  const bool legal1 = lane + 64 < n && s_tok[lane + 64] >= 0 && s_tok[lane + 64] < V;
  int node = 0, count = 1, gone = 0;
  double c = 0;
  bool ok = true;
  if (tid == 0) p.paths[first] = first;
  while (true) {
    // its children in their order
    uint64_t kids[2] = {__ballot(up0 == node), __ballot(up1 == node)};
    ok = s_sum[0][node] > 0 && (!drawn || (kids[0] | kids[1]) == 0 || s_sum[1][node] > 0);
    if (!ok) break;
    kids[0] &= __ballot(legal0);
    kids[1] &= __ballot(legal1);
    int go = -1;
    double sum = 1;
    c = 0;
    gone = 0;
    while (true) {
      const int i = kids[0] ? __builtin_ctzll(kids[0]) : (kids[1] ? 64 + __builtin_ctzll(kids[1]) : -1);
      if (i < 0) break;
      if (i < 64) kids[0] &= kids[0] - 1; else kids[1] &= kids[1] - 1;
      if constexpr (GREEDY) {
        if (s_tok[i] == s_best[node]) {
          go = i;
          break;
        }
      } else if (drawn) {
        if ((double)s_u[i] * sum * s_q[i] < s_p[i] - c * s_q[i]) {
          go = i;
          break;
        }
        c += sum;
        if (kids[0] | kids[1]) {
          const char* zt = (const char*)a.target + (first + node) * a.target_row * EL;
          const char* zd = (const char*)a.draft + (first + node) * a.draft_row * EL;
          const float mp = s_m[0][node], mq = s_m[1][node];
          const float kp = (float)a.scale * kLog2e, kq = (float)a.draft_scale * kLog2e;
          const float fp = (float)(1.0 / s_sum[0][node]), fq = (float)(c / s_sum[1][node]);
          double mine = 0;
          for (int v = tid * VE; v < V; v += kVThreads * VE) {
            float x[VE], y[VE], w = 0.f;
            load_symbols<TYPE>(zt, v, V, x);
            load_symbols<TYPE>(zd, v, V, y);
#pragma unroll
            for (int e = 0; e < VE; ++e)
              w += fmaxf(fmaf(__builtin_amdgcn_exp2f((x[e] - mp) * kp), fp, -(__builtin_amdgcn_exp2f((y[e] - mq) * kq) * fq)), 0.f);
            mine += (double)w;
          }
          sum = group_sum<kVWaves>(mine, s_red);
        }
      } else {
        // a symbol that was rejected before has nothing left
        bool again = false;
        for (int j = node + 1; j < i; ++j) again = again || (s_up[j] == node && s_tok[j] == s_tok[i]);
        const double left = again ? 0.0 : s_p[i];
        if ((double)s_u[i] * sum < left) {
          go = i;
          break;
        }
        sum -= left;
        gone = i + 1;
      }
    }
    if (go < 0) break;
    node = go;
    if (tid == 0) p.paths[first + count] = first + node;
    ++count;
  }
  if (tid == 0) {
    a.new_len[r] = a.lengths[r] + count;
    a.token[r] = GREEDY && ok ? s_best[node] : -1;
    p.ends[r] = {ok && !GREEDY ? first + (int64_t)node : -1, c, s_m[0][node], drawn ? s_m[1][node] : 0.f, first, node, gone, 0};
  }
}

// Symbols of a cut of a row.
__device__ __forceinline__ void cut_of(const VerifyDev& p, int cut, int* lo, int* hi) {
  const int V = (int)p.a.n_vocab, per = ((V + p.cuts - 1) / p.cuts + 7) / 8 * 8;
  *lo = (int)min((int64_t)cut * per, (int64_t)V);
  *hi = min(V, *lo + per);
}

// Where something was rejected: the sums of both softmaxes again, in 64 bits.
template <int TYPE>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_sums(VerifyDev p) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  const mca_verify_drafts_args& a = p.a;
  __shared__ double s_red[kVWaves];
  const int r = blockIdx.x, cut = blockIdx.y;
  const End e = p.ends[r];
  if (e.row < 0 || e.c == 0) return;
  int lo, hi;
  cut_of(p, cut, &lo, &hi);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const char* row = (const char*)(which ? a.draft : a.target) + e.row * (which ? a.draft_row : a.target_row) * EL;
    const double k = which ? a.draft_scale : a.scale, m = which ? e.mq : e.mp;
    double mine = 0;
    for (int v = lo + (int)threadIdx.x * VE; v < hi; v += kVThreads * VE) {
      float f[VE];
      load_symbols<TYPE>(row, v, hi, f);
#pragma unroll
      for (int i = 0; i < VE; ++i) mine += exp(k * ((double)f[i] - m));
    }
    const double sum = group_sum<kVWaves>(mine, s_red);
    if (threadIdx.x == 0) p.sums[((int64_t)r * 2 + which) * p.cuts + cut] = sum;
  }
}

// The rows accepted, request after request (one workgroup).
__device__ void compact(const VerifyDev& p, int* s_wave) {
  const mca_verify_drafts_args& a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t base = 0;
  for (int r0 = 0; r0 < a.n_req; r0 += kVThreads) {
    const int r = r0 + tid;
    const int n = r < a.n_req ? a.new_len[r] - a.lengths[r] : 0;
    int run = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(run, d, 64);
      if (lane >= d) run += up;
    }
    if (lane == 63) s_wave[wave] = run;
    __syncthreads();
    int all = 0, pre = run - n;
#pragma unroll
    for (int w = 0; w < kVWaves; ++w) {
      if (w < wave) pre += s_wave[w];
      all += s_wave[w];
    }
    const int first = n > 0 ? a.offsets[r] : 0;
    for (int i = 0; i < n; ++i)
      if (base + pre + i < a.n_rows) a.rows[base + pre + i] = p.paths[first + i];
    base += all;
    __syncthreads();
  }
  for (int64_t t = base + tid; t < a.n_rows; t += kVThreads) a.rows[t] = -1;
}

__global__ __launch_bounds__(kVThreads) void k_lm_verify_compact(VerifyDev p) {
  __shared__ int s_wave[kVWaves];
  compact(p, s_wave);
}

// The draw: every cut's sum of what is drawn from; the request's last workgroup finds
// the cut, then the symbol.  Workgroup (n_req, 0) puts the rows together.
template <int TYPE>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_draw(VerifyDev p) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  const mca_verify_drafts_args& a = p.a;
  __shared__ double s_red[kVWaves];
  __shared__ double s_all[kVMaxSplits], s_scan[kVThreads];
  __shared__ int s_wave[kVWaves];
  __shared__ int s_last, s_found;
  const int tid = threadIdx.x, r = blockIdx.x, cut = blockIdx.y;
  if (r == a.n_req) {
    if (cut == 0) compact(p, s_wave);
    return;
  }
  const End e = p.ends[r];
  if (e.row < 0) return;
  const char* zt = (const char*)a.target + e.row * a.target_row * EL;
  const char* zd = (const char*)a.draft + (a.draft != nullptr ? e.row * a.draft_row * EL : 0);
  double ip = 1, iq = 0;
  if (e.c != 0) {
    double sp = 0, sq = 0;
    for (int x = 0; x < p.cuts; ++x) {
      sp += p.sums[((int64_t)r * 2) * p.cuts + x];
      sq += p.sums[((int64_t)r * 2 + 1) * p.cuts + x];
    }
    ip = 1 / sp;
    iq = e.c / sq;
  }
  // what symbols v .. are drawn from; `plain`: from p
  auto weights = [&](int v, int hi, bool plain, double (&w)[VE]) {
    float x[VE];
    load_symbols<TYPE>(zt, v, hi, x);
#pragma unroll
    for (int i = 0; i < VE; ++i) w[i] = exp(a.scale * ((double)x[i] - (double)e.mp)) * ip;
    if (e.c != 0 && !plain) {
      load_symbols<TYPE>(zd, v, hi, x);
#pragma unroll
      for (int i = 0; i < VE; ++i) w[i] = fmax(w[i] - iq * exp(a.draft_scale * ((double)x[i] - (double)e.mq)), 0.0);
    }
    if (e.gone > 0 && !plain) {
      for (int j = e.node + 1; j < e.gone; ++j) {
        const int out = a.tokens[e.first + j] - v;
        if (a.parents[e.first + j] == e.node && out >= 0 && out < VE) {
#pragma unroll
          for (int i = 0; i < VE; ++i) w[i] = i == out ? 0.0 : w[i];
        }
      }
    }
  };
  int lo, hi;
  cut_of(p, cut, &lo, &hi);
  double mine = 0;
  for (int v = lo + tid * VE; v < hi; v += kVThreads * VE) {
    double w[VE];
    weights(v, hi, false, w);
#pragma unroll
    for (int i = 0; i < VE; ++i) mine += w[i];
  }
  const double sum = group_sum<kVWaves>(mine, s_red);
  if (p.cuts > 1) {
    if (tid == 0) {
      __hip_atomic_store(&p.left[(int64_t)r * p.cuts + cut], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_last = __hip_atomic_fetch_add(&p.tickets[r], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == p.cuts - 1;
    }
    __syncthreads();
    if (!s_last) return;
    if (tid < p.cuts) s_all[tid] = __hip_atomic_load(&p.left[(int64_t)r * p.cuts + tid], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  } else if (tid == 0) {
    s_all[0] = sum;
  }
  __syncthreads();
  double total = 0;
  for (int x = 0; x < p.cuts; ++x) total += s_all[x];
  const bool plain = !(total > 0);  // nothing is left: from p itself
  if (plain) {
    for (int x = 0; x < p.cuts; ++x) {
      int l, h;
      cut_of(p, x, &l, &h);
      double m2 = 0;
      for (int v = l + tid * VE; v < h; v += kVThreads * VE) {
        double w[VE];
        weights(v, h, true, w);
#pragma unroll
        for (int i = 0; i < VE; ++i) m2 += w[i];
      }
      m2 = group_sum<kVWaves>(m2, s_red);
      if (tid == 0) s_all[x] = m2;
    }
    __syncthreads();
    total = 0;
    for (int x = 0; x < p.cuts; ++x) total += s_all[x];
  }
  const float u = a.sample[r];
  const double goal = (u >= 0.f ? (double)fminf(u, 0x1.fffffep-1f) : 0.0) * total;
  // the cut: the first behind which the sum is past the goal, or the last that has any
  int at = -1, some = 0;
  double before = 0, run = 0;
  for (int x = 0; x < p.cuts; ++x) {
    const double next = run + s_all[x];
    if (next > goal && at < 0) {
      at = x;
      before = run;
    }
    if (s_all[x] > 0) some = x;
    run = next;
  }
  const bool rounded = at < 0;  // by the order of the sums alone
  if (rounded) at = some;
  cut_of(p, at, &lo, &hi);
  // a thread's symbols lie side by side
  const int each = ((hi - lo + kVThreads - 1) / kVThreads + VE - 1) / VE * VE, v0 = lo + tid * each, v1 = min(hi, v0 + each);
  mine = 0;
  for (int v = v0; v < v1; v += VE) {
    double w[VE];
    weights(v, v1, plain, w);
#pragma unroll
    for (int i = 0; i < VE; ++i) mine += w[i];
  }
  s_scan[tid] = mine;
  if (tid == 0) s_found = 0x7fffffff;
  __syncthreads();
  for (int x = 0; x < tid; ++x) before += s_scan[x];
  int last = -1;  // the thread's last symbol that has any
  if (mine > 0) {
    bool done = false;
    for (int v = v0; v < v1 && !done; v += VE) {
      double w[VE];
      weights(v, v1, plain, w);
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        before += w[i];
        if (w[i] > 0) last = v + i;
        if (!done && !rounded && w[i] > 0 && before > goal) {
          atomicMin(&s_found, v + i);
          done = true;
        }
      }
    }
  }
  __syncthreads();
  if (s_found == 0x7fffffff) {
    // the sums' rounding leaves none: the last symbol that has any
    __syncthreads();
    if (tid == 0) s_found = -1;
    __syncthreads();
    atomicMax(&s_found, last);
    __syncthreads();
  }
  if (tid == 0) a.token[r] = s_found;
}

namespace {

int row_splits(const mca_verify_drafts_args& a) {
  const int64_t rows = std::max<int64_t>(1, a.n_rows) * (a.draft != nullptr && !a.greedy ? 2 : 1);
  return (int)std::clamp<int64_t>(std::min((2048 + rows - 1) / rows, a.n_vocab / kVPart), 1, kVMaxSplits);
}
int end_cuts(const mca_verify_drafts_args& a) {
  const int64_t reqs = std::max(1, a.n_req);
  return (int)std::clamp<int64_t>(std::min((1024 + reqs - 1) / reqs, a.n_vocab / 2048), 1, kVMaxSplits);
}
size_t room(size_t n) { return (n + 255) / 256 * 256; }

// The workspace's regions; returns its size.
size_t lay_out(const mca_verify_drafts_args& a, VerifyDev* d) {
  const int both = a.draft != nullptr && !a.greedy ? 2 : 1;
  const int splits = row_splits(a), cuts = end_cuts(a);
  char* at = (char*)a.workspace;
  size_t n = 0;
  auto take = [&](size_t bytes) {
    char* p = at + n;
    n += room(bytes);
    return p;
  };
  d->a = a;
  d->splits = splits;
  d->cuts = cuts;
  d->parts = (RowPart*)take((size_t)a.n_rows * both * splits * sizeof(RowPart));
  d->ends = (End*)take((size_t)a.n_req * sizeof(End));
  d->sums = (double*)take((size_t)a.n_req * 2 * cuts * sizeof(double));
  d->left = (double*)take((size_t)a.n_req * cuts * sizeof(double));
  d->tickets = (int32_t*)take((size_t)a.n_req * sizeof(int32_t));
  d->paths = (int32_t*)take((size_t)a.n_rows * sizeof(int32_t));
  return n;
}

template <int TYPE>
void launch(const VerifyDev& d, hipStream_t s) {
  const mca_verify_drafts_args& a = d.a;
  const dim3 threads(kVThreads);
  const unsigned both = a.draft != nullptr && !a.greedy ? 2 : 1;
  const dim3 rows((unsigned)a.n_rows, both * (unsigned)d.splits);
  if (a.n_req == 0) {  // no row is anyone's
    hipLaunchKernelGGL(k_lm_verify_compact, dim3(1), threads, 0, s, d);
    return;
  }
  if (a.greedy) {
    if (a.n_rows > 0) hipLaunchKernelGGL((k_lm_verify_rows<TYPE, true>), rows, threads, 0, s, d);
    hipLaunchKernelGGL((k_lm_verify_walk<TYPE, true>), dim3((unsigned)a.n_req), threads, 0, s, d);
    hipLaunchKernelGGL(k_lm_verify_compact, dim3(1), threads, 0, s, d);
    return;
  }
  if (a.n_rows > 0) hipLaunchKernelGGL((k_lm_verify_rows<TYPE, false>), rows, threads, 0, s, d);
  hipLaunchKernelGGL((k_lm_verify_walk<TYPE, false>), dim3((unsigned)a.n_req), threads, 0, s, d);
  if (both == 2) hipLaunchKernelGGL((k_lm_verify_sums<TYPE>), dim3((unsigned)a.n_req, (unsigned)d.cuts), threads, 0, s, d);
  hipLaunchKernelGGL((k_lm_verify_draw<TYPE>), dim3((unsigned)a.n_req + 1, (unsigned)d.cuts), threads, 0, s, d);
}

}  // namespace

size_t lm_verify_plan(const mca_verify_drafts_args& a) {
  VerifyDev d;
  return lay_out(a, &d);
}

hipError_t lm_launch_verify(const mca_verify_drafts_args& a, hipStream_t s) {
  VerifyDev d;
  lay_out(a, &d);
  switch (a.dtype) {
    case MCA_TYPE_F32: launch<MCA_TYPE_F32>(d, s); break;
    case MCA_TYPE_BF16: launch<MCA_TYPE_BF16>(d, s); break;
    default: launch<MCA_TYPE_F16>(d, s); break;
  }
  return hipGetLastError();
}

}  // namespace mca
