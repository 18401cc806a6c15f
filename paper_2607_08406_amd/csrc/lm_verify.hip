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
// those of 64 by 1e-14.  So where children were rejected at that node, c is made again from
// sums of 64 bits, one step of all of the chip for each of the first rejections.
//
// What bounds it: only the first step moves many bytes.  The others are chains of short
// kernels, whose time is their launch, the spread of their workgroups and 64-bit
// arithmetic (about 25 operations a symbol).  bf16, 32 requests of up to 9 nodes, 128000
// symbols: rows 21 us (82 MB, 3.9 TB/s), walk 19, sums 11, draw 23, its further steps 16, 4
// and 3: 93 us in a graph.
#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "lm_device.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

constexpr int kVThreads = 256;
constexpr int kVWaves = kVThreads / 64;
constexpr int kWalkThreads = 1024;  // of the walk over large vocabularies, whose passes one workgroup makes
constexpr int kVUnroll = 4;
constexpr int kVMaxSplits = 64;   // parts of a row
constexpr int64_t kVPart = 8192;  // symbols of a part at least
constexpr int kVSteps = 3;        // further steps of the draw
constexpr int kVSide = 8;         // symbols side by side in a thread of the draw
constexpr int kVCut = 2048;       // symbols of a cut of the draw at least
constexpr int kVSegment = 256;    // symbols that a wave weighs at a time in the kernel of whole requests
constexpr int kVWhole = 32 * kVSegment;  // its largest vocabulary (64 segments at most)
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;

// A part of a row: its largest logit, and the sum of exp(scale (z - m)); of greedy
// calls the first symbol of that logit.  s is NaN if the part has NaN or +inf.
struct RowPart {
  double s;
  float m;
  int32_t at;
};
// What sums a lane's part of a row: exponentials of 32 bits, a vector at a time, in 64 (in 32 they
// lose up to half a step each: 50 steps at 70000 symbols; of 64 costs the call less than
// 1 %: 300 requests of 9 nodes, 128000 bf16 symbols, 443 and 445 us).  Of greedy calls NaN or 0.
template <bool GREEDY>
using Sum = std::conditional_t<GREEDY, float, double>;
// Where a request's path ends: what its token is drawn from.
struct End {
  int64_t row;  // of the logits; -1: no token
  double c;     // 0: p alone; 1 behind the first rejection
  float mp, mq;  // largest logits
  int32_t first, node, gone;  // given drafts: the children before this one were rejected
  int32_t more;               // drawn ones: rejections whose S is still to be added to c
};

struct VerifyDev {
  mca_verify_drafts_args a;
  int32_t splits, cuts;  // parts of a row in the first and in the last steps
  RowPart* parts;        // [n_rows][1 or 2][splits]
  End* ends;             // [n_req]
  double* sums;          // [n_req][2][cuts]: sums of exponentials
  double* left;          // [n_req][cuts]: sums of what is drawn from
  int32_t* tickets;      // [n_req]
  int32_t* active;       // [kVSteps][1 + n_req]: requests of the draw's further steps, behind their number
  int32_t* paths;        // [n_rows]
};

// 16 bytes at any address
__device__ __forceinline__ u32x4 any_vector(const char* p) {
  struct __attribute__((packed)) Any {
    u32x4 x;
  };
  return ((const Any*)p)->x;
}
// symbols v .. v + kPer - 1 of a row of V; behind it -inf
template <int TYPE>
__device__ __forceinline__ void load_symbols(const char* row, int v, int V, float (&f)[Elem<TYPE>::kPer]) {
  constexpr int VE = Elem<TYPE>::kPer;
  if (v + VE <= V) {
    unpack<TYPE>(any_vector(row + (int64_t)v * Elem<TYPE>::kSize), f);
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
// of no request, and draft rows of nodes without children, are left out.  Bound by the
// loads: four of 16 bytes a lane in flight, the running maximum kept by each lane so that
// nothing waits for another before the end.
template <int TYPE, bool GREEDY>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_rows(VerifyDev p) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  typedef typename Elem<TYPE>::Raw Raw;
  const mca_verify_drafts_args& a = p.a;
  __shared__ float s_m[kVWaves];
  __shared__ Sum<GREEDY> s_s[kVWaves];
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
  float m = kLowest;
  Sum<GREEDY> s = 0;
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
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < VE; ++i) w += __builtin_amdgcn_exp2f((f[i] - m) * k2);
        s += w;
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
  auto join = [&](float m2, Sum<GREEDY> s2, int at2) {
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
    p.parts[(t * both + which) * p.splits + split] = {s, m, at};
  }
}

namespace {

// What a walk needs of its nodes, in LDS.
struct Nodes {
  float m[2][MCA_MAX_NODES];      // largest logits of the target and the draft
  double sum[2][MCA_MAX_NODES];   // 0: no softmax; of greedy calls 1
  int best[MCA_MAX_NODES];        // of greedy calls the first symbol of the largest logit
  int up[MCA_MAX_NODES], tok[MCA_MAX_NODES];
  float u[MCA_MAX_NODES];
  double p[MCA_MAX_NODES], q[MCA_MAX_NODES];  // of a node's token at its parent
  uint8_t parent[MCA_MAX_NODES];  // whether a node has children
  double red[kWalkThreads / 64];
};

// Parents, tokens and random numbers of a request's nodes (THREADS >= MCA_MAX_NODES).
template <bool GREEDY>
__device__ __forceinline__ void load_nodes(const mca_verify_drafts_args& a, int first, int n, Nodes& s) {
  const int tid = threadIdx.x;
  int up = -1;
  if (tid < n) {
    up = a.parents[first + tid];
    up = tid > 0 && up >= 0 && up < tid ? up : -1;
    s.up[tid] = up;
    s.tok[tid] = a.tokens[first + tid];
    if constexpr (!GREEDY) s.u[tid] = a.accept[first + tid];
    s.parent[tid] = 0;
  }
  __syncthreads();
  if (up >= 0) s.parent[up] = 1;
}

// The sum of max(p - c q, 0) over the vocabulary at a node.
template <int TYPE, int THREADS>
__device__ __forceinline__ double left_sum(const mca_verify_drafts_args& a, int first, int node, double c, Nodes& s) {
  constexpr int VE = Elem<TYPE>::kPer, EL = Elem<TYPE>::kSize;
  const int V = (int)a.n_vocab;
  const char* zt = (const char*)a.target + (first + node) * a.target_row * EL;
  const char* zd = (const char*)a.draft + (first + node) * a.draft_row * EL;
  const float mp = s.m[0][node], mq = s.m[1][node];
  const float kp = (float)a.scale * kLog2e, kq = (float)a.draft_scale * kLog2e;
  // logarithms (base 2) of the factors of the exponentials
  const float fp = -__builtin_amdgcn_logf((float)s.sum[0][node]), fq = __builtin_amdgcn_logf((float)(c / s.sum[1][node]));
  double mine = 0;
  auto weigh = [&](const float (&x)[VE], const float (&y)[VE]) {
    float w = 0.f;
#pragma unroll
    for (int e = 0; e < VE; ++e)
      w += fmaxf(__builtin_amdgcn_exp2f(fmaf(x[e] - mp, kp, fp)) - __builtin_amdgcn_exp2f(fmaf(y[e] - mq, kq, fq)), 0.f);
    mine += (double)w;
  };
  // All loads of a round before its sums.  A thread's last vectors are moved up to the row's
  // end, and what was there before them (all of those that lie behind it) is left out.
  const int v0 = (int)threadIdx.x * VE;
  if (V < VE) {
    float x[VE], y[VE];
    load_symbols<TYPE>(zt, v0, V, x);
    load_symbols<TYPE>(zd, v0, V, y);
    if (v0 == 0) weigh(x, y);
    return group_sum<THREADS / 64>(mine, s.red);
  }
#pragma unroll 1
  for (int b = 0; b < V; b += kVUnroll * THREADS * VE) {
    u32x4 xs[kVUnroll], ys[kVUnroll];
#pragma unroll
    for (int u = 0; u < kVUnroll; ++u) {
      const int at = min(b + v0 + u * THREADS * VE, V - VE);
      xs[u] = any_vector(zt + (int64_t)at * EL);
      ys[u] = any_vector(zd + (int64_t)at * EL);
    }
#pragma unroll
    for (int u = 0; u < kVUnroll; ++u) {
      float x[VE], y[VE];
      unpack<TYPE>(xs[u], x);
      unpack<TYPE>(ys[u], y);
      const int skip = b + v0 + u * THREADS * VE - (V - VE);
      if (skip > 0) {
#pragma unroll
        for (int e = 0; e < VE; ++e) x[e] = e < skip ? -__builtin_huge_valf() : x[e];
      }
      weigh(x, y);
    }
  }
  return group_sum<THREADS / 64>(mine, s.red);
}

// A request's walk, by one workgroup, whose waves all take the same steps; s.m, s.sum
// and s.best are there.  Writes the path and new_len, and the token where no draw follows.
template <int TYPE, bool GREEDY, int THREADS>
__device__ __forceinline__ End walk(const VerifyDev& d, int r, int first, int n, Nodes& s) {
  typedef typename Elem<TYPE>::Raw Raw;
  const mca_verify_drafts_args& a = d.a;
  const bool drawn = a.draft != nullptr && !GREEDY;
  const int tid = threadIdx.x, lane = tid & 63, V = (int)a.n_vocab;
  if (!GREEDY && tid < n && s.up[tid] >= 0 && s.tok[tid] >= 0 && s.tok[tid] < V) {
    const int up = s.up[tid];
    const int64_t row = first + up;
    const float z = to_f32<TYPE>(((const Raw*)a.target)[row * a.target_row + s.tok[tid]]);
    s.p[tid] = exp_of(a.scale * ((double)z - (double)s.m[0][up])) / s.sum[0][up];
    if (drawn) {
      const float y = to_f32<TYPE>(((const Raw*)a.draft)[row * a.draft_row + s.tok[tid]]);
      s.q[tid] = exp_of(a.draft_scale * ((double)y - (double)s.m[1][up])) / s.sum[1][up];
    }
  }
  __syncthreads();
  const int up0 = lane < n ? s.up[lane] : -1, up1 = lane + 64 < n ? s.up[lane + 64] : -1;
  const bool legal0 = lane < n && s.tok[lane] >= 0 && s.tok[lane] < V;
  const bool legal1 = lane + 64 < n && s.tok[lane + 64] >= 0 && s.tok[lane + 64] < V;
  int node = 0, count = 1, gone = 0, lost = 0;
  bool ok = true;
  if (tid == 0) d.paths[first] = first;
  while (true) {
    // its children in their order
    uint64_t kids[2] = {__ballot(up0 == node), __ballot(up1 == node)};
    ok = s.sum[0][node] > 0 && (!drawn || (kids[0] | kids[1]) == 0 || s.sum[1][node] > 0);
    if (!ok) break;
    kids[0] &= __ballot(legal0);
    kids[1] &= __ballot(legal1);
    int go = -1;
    double sum = 1, c = 0;
    gone = lost = 0;
    while (true) {
      const int i = kids[0] ? __builtin_ctzll(kids[0]) : (kids[1] ? 64 + __builtin_ctzll(kids[1]) : -1);
      if (i < 0) break;
      if (i < 64) kids[0] &= kids[0] - 1; else kids[1] &= kids[1] - 1;
      if constexpr (GREEDY) {
        if (s.tok[i] == s.best[node]) {
          go = i;
          break;
        }
      } else if (drawn) {
        if ((double)s.u[i] * sum * s.q[i] < s.p[i] - c * s.q[i]) {
          go = i;
          break;
        }
        c += sum;
        ++lost;
        if (kids[0] | kids[1]) sum = left_sum<TYPE, THREADS>(a, first, node, c, s);
      } else {
        // a symbol that was rejected before has nothing left
        bool again = false;
        for (int j = node + 1; j < i; ++j) again = again || (s.up[j] == node && s.tok[j] == s.tok[i]);
        const double left = again ? 0.0 : s.p[i];
        if ((double)s.u[i] * sum < left) {
          go = i;
          break;
        }
        sum -= left;
        gone = i + 1;
      }
    }
    if (go < 0) break;
    node = go;
    if (tid == 0) d.paths[first + count] = first + node;
    ++count;
  }
  if (tid == 0) {
    a.new_len[r] = a.lengths[r] + count;
    if (GREEDY || !ok) a.token[r] = ok ? s.best[node] : -1;
  }
  return {ok && !GREEDY ? first + (int64_t)node : -1, lost > 0 ? 1.0 : 0.0, s.m[0][node], drawn ? s.m[1][node] : 0.f, first, node, gone, max(lost - 1, 0)};
}
// of a request that has no nodes, or too many
__device__ __forceinline__ void no_walk(const mca_verify_drafts_args& a, int r) {
  a.new_len[r] = a.lengths[r];
  a.token[r] = -1;
}

// What the token is drawn from: ip times exp(scale (z - mp)) less iq times the draft's, or
// none of some symbols.
struct Weights {
  const char *zt, *zd;
  double k, kd, mp, mq, ip, iq;
  const int* gone;  // in LDS
  int n_gone;
};
// Of given drafts, the symbols that were rejected at the node, to LDS (all threads).
__device__ __forceinline__ int gone_symbols(const mca_verify_drafts_args& a, const End& e, int* s_gone, int* s_count) {
  if (e.gone == 0) return 0;
  if (threadIdx.x == 0) *s_count = 0;
  __syncthreads();
  const int j = e.node + 1 + (int)threadIdx.x;
  if (j < e.gone && a.parents[e.first + j] == e.node) s_gone[atomicAdd(s_count, 1)] = a.tokens[e.first + j];
  __syncthreads();
  return *s_count;
}
template <int TYPE>
__device__ __forceinline__ Weights weights_of(const mca_verify_drafts_args& a, const End& e, double sp, double sq, const int* gone, int n_gone) {
  constexpr int EL = Elem<TYPE>::kSize;
  return {(const char*)a.target + e.row * a.target_row * EL,
          (const char*)a.draft + (a.draft != nullptr ? e.row * a.draft_row * EL : 0),
          a.scale, a.draft_scale, (double)e.mp, (double)e.mq, e.c != 0 ? 1 / sp : 1.0, e.c != 0 ? e.c / sq : 0.0, gone, n_gone};
}
// The E symbols of a thread from v on, below hi (behind it -inf).
template <int TYPE, int E>
__device__ __forceinline__ void symbols(const char* row, int v, int hi, float (&x)[E]) {
  typedef typename Elem<TYPE>::Raw Raw;
  struct __attribute__((packed)) Any {
    Raw x[E];
  };
  if (v + E <= hi) {
    const Any y = *(const Any*)(row + (int64_t)v * Elem<TYPE>::kSize);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = to_f32<TYPE>(y.x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = v + i < hi ? to_f32<TYPE>(((const Raw*)row)[v + i]) : -__builtin_huge_valf();
  }
}
// their weights; `plain`: of p alone
template <int TYPE, int E>
__device__ __forceinline__ void weigh(const Weights& f, int v, int hi, bool plain, double (&w)[E]) {
  const bool both = f.iq != 0 && !plain;
  float x[E], y[E];
  symbols<TYPE, E>(f.zt, v, hi, x);
  if (both) symbols<TYPE, E>(f.zd, v, hi, y);
#pragma unroll
  for (int i = 0; i < E; ++i) w[i] = 0;
#pragma unroll 1
  for (int which = 0; which < (both ? 2 : 1); ++which) {
    const double k = which ? f.kd : f.k, m = which ? f.mq : f.mp, by = which ? -f.iq : f.ip;
    double e[E];
#pragma unroll
    for (int i = 0; i < E; ++i) e[i] = k * ((double)(which ? y[i] : x[i]) - m);
    exps_of(e);
#pragma unroll
    for (int i = 0; i < E; ++i) w[i] += e[i] * by;  // (both products rounded: equal ones leave nothing)
  }
#pragma unroll
  for (int i = 0; i < E; ++i) w[i] = w[i] < 0 ? 0.0 : w[i];
  if (!plain)
    for (int j = 0; j < f.n_gone; ++j) {
      const int out = f.gone[j] - v;
#pragma unroll
      for (int i = 0; i < E; ++i) w[i] = i == out ? 0.0 : w[i];
    }
}
// The sums of both softmaxes' exponentials over symbols lo .. hi - 1.
template <int TYPE, int E, int THREADS>
__device__ __forceinline__ void exp_sums(const Weights& f, int lo, int hi, double* s_red, double* sp, double* sq) {
  double sum[2] = {0, 0};
#pragma unroll 1
  for (int v = lo + (int)threadIdx.x * E; v < hi; v += THREADS * E) {
    float x[E], y[E];
    symbols<TYPE, E>(f.zt, v, hi, x);
    symbols<TYPE, E>(f.zd, v, hi, y);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
      const double k = which ? f.kd : f.k, m = which ? f.mq : f.mp;
      double e[E], mine = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) e[i] = k * ((double)(which ? y[i] : x[i]) - m);
      exps_of(e);
#pragma unroll
      for (int i = 0; i < E; ++i) mine += e[i];
      sum[0] += which ? 0.0 : mine;
      sum[1] += which ? mine : 0.0;
    }
  }
  *sp = group_sum<THREADS / 64>(sum[0], s_red);
  *sq = group_sum<THREADS / 64>(sum[1], s_red);
}

__device__ __forceinline__ double goal_of(const mca_verify_drafts_args& a, int r, double total) {
  const float u = a.sample[r];
  return (u >= 0.f ? (double)fminf(u, 0x1.fffffep-1f) : 0.0) * total;
}
// Of the workgroup's next symbols, E side by side in a thread from v0 on, with weights w:
// the first with which the sum, *before in front of them, is past the goal; 0x7fffffff if
// none is.  *before moves behind them, *last becomes the thread's last of any weight.
template <int E>
__device__ __forceinline__ int past_goal(const double (&w)[E], int v0, double goal, double* before, int* last, double* s_wave, int* s_found) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  double mine = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    mine += w[i];
    if (w[i] > 0) *last = v0 + i;
  }
  double run = mine;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const double up = __shfl_up(run, x, 64);
    if (lane >= x) run += up;
  }
  __syncthreads();
  if (lane == 63) s_wave[wave] = run;
  if (tid == 0) *s_found = 0x7fffffff;
  __syncthreads();
  double at = *before;
#pragma unroll
  for (int x = 0; x < kVWaves; ++x) {
    if (x < wave) at += s_wave[x];
    *before += s_wave[x];
  }
  at += run - mine;
  int mark = 0x7fffffff;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    at += w[i];
    if (w[i] > 0 && at > goal) mark = min(mark, v0 + i);
  }
  if (mark != 0x7fffffff) atomicMin(s_found, mark);
  __syncthreads();
  return *s_found;
}
// Where only the rounding of the sums leaves none: the last of any weight (-1: none has).
__device__ __forceinline__ int last_of(int last, int* s_found) {
  __syncthreads();
  if (threadIdx.x == 0) *s_found = -1;
  __syncthreads();
  atomicMax(s_found, last);
  __syncthreads();
  return *s_found;
}

}  // namespace

// A request's walk over a large vocabulary, from the rows' parts.  One workgroup, as
// whether a child is accepted decides which row is read next; a pass for S over 128000
// symbols at one rejection takes it 6 us (8 where a thread's loads waited for its sums, 15 in
// 4 waves).  Only children behind a rejected one need such a pass.
template <int TYPE, bool GREEDY>
__global__ __launch_bounds__(kWalkThreads) void k_lm_verify_walk(VerifyDev d) {
  const mca_verify_drafts_args& a = d.a;
  const bool drawn = a.draft != nullptr && !GREEDY;
  __shared__ Nodes s;
  const int tid = threadIdx.x, r = blockIdx.x;
  int first, n;
  if (tid == 0) d.tickets[r] = 0;
  if (r == 0 && tid < kVSteps) d.active[tid * (1 + a.n_req)] = 0;
  if (!nodes_of(a, r, &first, &n)) {
    if (tid == 0) {
      no_walk(a, r);
      d.ends[r].row = -1;
    }
    return;
  }
  load_nodes<GREEDY>(a, first, n, s);
  __syncthreads();
  for (int x = tid; x < n * (drawn ? 2 : 1); x += kWalkThreads) {
    const int which = x >= n, i = x - which * n;
    const RowPart* part = d.parts + ((int64_t)(first + i) * (drawn ? 2 : 1) + which) * d.splits;
    float m = GREEDY ? -__builtin_huge_valf() : kLowest;
    double sum = 0;
    int at = -1;
    if (which == 0 || s.parent[i]) {
#pragma unroll 4
      for (int y = 0; y < d.splits; ++y) {
        const RowPart u = part[y];
        if constexpr (GREEDY) {
          if (u.m > m) {
            m = u.m;
            at = u.at;
          }
          sum += u.s;  // (0 or NaN)
        } else {
          m = fmaxf(m, u.m);
        }
      }
      if constexpr (GREEDY) {
        sum = sum == 0 && at >= 0 ? 1.0 : 0.0;
      } else {
        const double k = which ? a.draft_scale : a.scale;
#pragma unroll 4
        for (int y = 0; y < d.splits; ++y) sum += part[y].s * exp_of(k * ((double)part[y].m - (double)m));
      }
    }
    s.m[which][i] = m;
    s.sum[which][i] = sum > 0 ? sum : 0.0;  // NaN: none
    if (which == 0) s.best[i] = at;
  }
  __syncthreads();
  const End e = walk<TYPE, GREEDY, kWalkThreads>(d, r, first, n, s);
  if (tid == 0) d.ends[r] = e;
}

// Symbols of a cut of a row.
__device__ __forceinline__ void cut_of(const VerifyDev& d, int cut, int* lo, int* hi) {
  const int V = (int)d.a.n_vocab, per = ((V + d.cuts - 1) / d.cuts + 7) / 8 * 8;
  *lo = (int)min((int64_t)cut * per, (int64_t)V);
  *hi = (int)min((int64_t)*lo + per, (int64_t)V);
}

// Where something was rejected: the sums of both softmaxes again, in 64 bits.
template <int TYPE>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_sums(VerifyDev d) {
  __shared__ double s_red[kVWaves];
  const int r = blockIdx.x, cut = blockIdx.y;
  const End e = d.ends[r];
  if (e.row < 0 || e.c == 0) return;
  int lo, hi;
  cut_of(d, cut, &lo, &hi);
  double sp, sq;
  exp_sums<TYPE, kVSide, kVThreads>(weights_of<TYPE>(d.a, e, 1, 1, nullptr, 0), lo, hi, s_red, &sp, &sq);
  if (threadIdx.x == 0) {
    d.sums[(int64_t)r * 2 * d.cuts + cut] = sp;
    d.sums[((int64_t)r * 2 + 1) * d.cuts + cut] = sq;
  }
}

// The rows accepted, request after request (one workgroup).
__device__ void compact(const VerifyDev& d, int* s_wave) {
  const mca_verify_drafts_args& a = d.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t base = 0;
  for (int r0 = 0; r0 < a.n_req; r0 += kVThreads) {
    const int r = r0 + tid;
    const int n = r < a.n_req ? a.new_len[r] - a.lengths[r] : 0;
    int run = n;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int up = __shfl_up(run, x, 64);
      if (lane >= x) run += up;
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
      if (base + pre + i < a.n_rows) a.rows[base + pre + i] = d.paths[first + i];
    base += all;
    __syncthreads();
  }
  for (int64_t t = base + tid; t < a.n_rows; t += kVThreads) a.rows[t] = -1;
}

__global__ __launch_bounds__(kVThreads) void k_lm_verify_compact(VerifyDev d) {
  __shared__ int s_wave[kVWaves];
  compact(d, s_wave);
}

namespace {

struct DrawShared {
  double red[kVWaves], all[kVMaxSplits];
  int gone[MCA_MAX_NODES];
  int last, found;
};

// A step of the draw for one request and cut: the cut's sum of what is left by c.  The
// request's last workgroup adds the sums to c while there are more rejections; behind them
// it finds the cut, then the symbol.  In the last step it goes through further rejections
// by itself.
template <int TYPE>
__device__ __forceinline__ void draw_cut(const VerifyDev& d, int r, int cut, int step, int steps, DrawShared& s) {
  const mca_verify_drafts_args& a = d.a;
  const int tid = threadIdx.x, lane = tid & 63;
  End e = d.ends[r];
  if (e.row < 0) return;
  // (every wave for itself, a cut a lane)
  double sp = 1, sq = 1;
  if (e.c != 0) {
    const double* sums = d.sums + (int64_t)r * 2 * d.cuts;
    sp = wave_sum(lane < d.cuts ? sums[lane] : 0.0);
    sq = wave_sum(lane < d.cuts ? sums[d.cuts + lane] : 0.0);
  }
  Weights f = weights_of<TYPE>(a, e, sp, sq, s.gone, gone_symbols(a, e, s.gone, &s.found));
  int lo, hi;
  cut_of(d, cut, &lo, &hi);
  // First this cut's sum; then, of the request's last workgroup, sums over all cuts where
  // it has to go on alone (more rejections, or nothing is left and p itself is drawn from),
  // and the cut in which the goal lies.  One body serves them all: nothing here runs often
  // enough to pay for more instructions.
  bool plain = false, finding = false, alone = false;
  int x = 0, last = -1;
  double before = 0, goal = 0;
  while (true) {
    double mine = 0;
#pragma unroll 1
    for (int b = lo; b < hi; b += kVThreads * kVSide) {
      const int v0 = b + tid * kVSide;
      double w[kVSide];
      weigh<TYPE, kVSide>(f, v0, hi, plain, w);
      if (finding) {
        const int found = past_goal<kVSide>(w, v0, goal, &before, &last, s.red, &s.found);
        if (found == 0x7fffffff) continue;
        if (tid == 0) a.token[r] = found;
        return;
      }
#pragma unroll
      for (int i = 0; i < kVSide; ++i) mine += w[i];
    }
    if (finding) {
      const int found = last_of(last, &s.found);
      if (tid == 0) a.token[r] = found;
      return;
    }
    mine = group_sum<kVWaves>(mine, s.red);
    if (!alone) {
      if (tid == 0) {
        // The sums are written and read past the caches (agent scope), so that the ticket
        // only has to wait for its own: no cache is written back or emptied for it.
        __hip_atomic_store(&d.left[(int64_t)r * d.cuts + cut], mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        s.last = __hip_atomic_fetch_add(&d.tickets[r], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == d.cuts - 1;
      }
      __syncthreads();
      if (!s.last) return;
      mine = lane < d.cuts ? __hip_atomic_load(&d.left[(int64_t)r * d.cuts + lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    } else {
      if (tid == 0) s.all[x] = mine;
      if (++x < d.cuts) {
        cut_of(d, x, &lo, &hi);
        continue;
      }
      __syncthreads();
      mine = lane < d.cuts ? s.all[lane] : 0.0;
      __syncthreads();
    }
    const double total = wave_sum(mine);
    if (e.more > 0 || (!plain && !(total > 0))) {
      if (e.more > 0) {
        e.c += total;
        --e.more;
        if (step < steps - 1) {
          if (tid == 0) {
            d.ends[r].c = e.c;
            d.ends[r].more = e.more;
            d.tickets[r] = 0;
            int32_t* list = d.active + (int64_t)step * (1 + a.n_req);
            list[1 + atomicAdd(list, 1)] = r;
          }
          return;
        }
        f.iq = e.c / sq;
      } else {
        plain = true;
      }
      alone = true;
      x = 0;
      cut_of(d, 0, &lo, &hi);
      continue;
    }
    goal = goal_of(a, r, total);
    // the cut: the first with which the sum is past the goal, or the last that has any
    double run = mine;
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) {
      const double up = __shfl_up(run, y, 64);
      if (lane >= y) run += up;
    }
    uint64_t some = __ballot(mine > 0 && run > goal);
    if (some == 0) {
      goal = __builtin_huge_val();
      some = 1ull << (63 - __builtin_clzll(__ballot(mine > 0) | 1));
    }
    const int at = __builtin_ctzll(some);
    before = __shfl(run - mine, at, 64);
    cut_of(d, at, &lo, &hi);
    finding = true;
  }
}

}  // namespace

// The first step, of all requests and cuts: 13 us from the first workgroup to the last
// (their weights take 3 to 4, the other 7 pass until the last one has started), 5 for the
// request's last workgroup to find the symbol.  Workgroup (n_req, 0) puts the rows together.
template <int TYPE>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_draw(VerifyDev d, int steps) {
  __shared__ DrawShared s;
  __shared__ int s_wave[kVWaves];
  if ((int)blockIdx.x == d.a.n_req) {
    if (blockIdx.y == 0) compact(d, s_wave);
    return;
  }
  draw_cut<TYPE>(d, blockIdx.x, blockIdx.y, 0, steps, s);
}

// Further ones, of the requests that the step before has named, by as many workgroups as
// run together (with two steps 97 us in the above; where all of them start again, most to end
// at once, 101).
template <int TYPE>
__global__ __launch_bounds__(kVThreads) void k_lm_verify_draw_more(VerifyDev d, int step, int steps) {
  __shared__ DrawShared s;
  const int32_t* list = d.active + (int64_t)(step - 1) * (1 + d.a.n_req);
  const int64_t items = (int64_t)list[0] * d.cuts;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    draw_cut<TYPE>(d, list[1 + x / d.cuts], (int)(x % d.cuts), step, steps, s);
    __syncthreads();
  }
}

// All of a request in one workgroup, but for its place among the rows: a wave a node's
// sums, the walk, the weights of 256 symbols a wave, and of those in which the goal lies
// once more.  The sums of few values are of 64 bits from the start.
template <int TYPE, bool GREEDY>
__global__ __launch_bounds__(kWalkThreads) void k_lm_verify_whole(VerifyDev d) {
  constexpr int THREADS = kWalkThreads, WAVES = THREADS / 64, EACH = kVSegment / 64;
  const mca_verify_drafts_args& a = d.a;
  const bool drawn = a.draft != nullptr && !GREEDY;
  __shared__ Nodes s;
  __shared__ int s_count, s_gone[MCA_MAX_NODES];
  __shared__ double s_seg[64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x, V = (int)a.n_vocab;
  int first, n;
  if (!nodes_of(a, r, &first, &n)) {
    if (tid == 0) no_walk(a, r);
    return;
  }
  load_nodes<GREEDY>(a, first, n, s);
  const int rows = n * (drawn ? 2 : 1);
  const bool exact = !GREEDY && rows * V <= 1 << 14;
  // (also of draft rows that no child was drawn from: nothing looks at them)
  for (int x = wave; x < rows; x += WAVES) {
    const int which = x >= n, i = x - which * n;
    const char* row = (const char*)(which ? a.draft : a.target) +
                      (int64_t)(first + i) * (which ? a.draft_row : a.target_row) * Elem<TYPE>::kSize;
    const double k = which ? a.draft_scale : a.scale;
    const float k2 = (float)(k * 1.4426950408889634);
    float m = GREEDY ? -__builtin_huge_valf() : kLowest;
    Sum<GREEDY> sum = 0;
    int at = V;
#pragma unroll 4
    for (int v = lane * EACH; v < V; v += kVSegment) {
      float z[EACH];
      symbols<TYPE, EACH>(row, v, V, z);
      if constexpr (GREEDY) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
          sum += z[j] < __builtin_huge_valf() ? 0.f : __builtin_nanf("");
          if (z[j] > m) {
            m = z[j];
            at = v + j;
          }
        }
      } else {
        float top = m;
#pragma unroll
        for (int j = 0; j < EACH; ++j) top = fmaxf(top, z[j]);
        sum *= __builtin_amdgcn_exp2f((m - top) * k2);
        m = top;
        float w = 0.f;
#pragma unroll
        for (int j = 0; j < EACH; ++j) w += __builtin_amdgcn_exp2f((z[j] - m) * k2);
        sum += w;
      }
    }
    float own = m;
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) {
      const float m2 = __shfl_xor(m, y, 64);
      if constexpr (GREEDY) {
        const int at2 = __shfl_xor(at, y, 64);
        if (m2 > m || (m2 == m && at2 < at)) at = at2;
      }
      m = fmaxf(m, m2);
    }
    double total = 0;
    if (exact) {
#pragma unroll 1
      for (int v = lane * EACH; v < V; v += kVSegment) {
        float z[EACH];
        symbols<TYPE, EACH>(row, v, V, z);
        double e[EACH];
#pragma unroll
        for (int j = 0; j < EACH; ++j) e[j] = k * ((double)z[j] - (double)m);
        exps_of(e);
#pragma unroll
        for (int j = 0; j < EACH; ++j) total += e[j];
      }
    } else {
      total = GREEDY ? (double)sum : sum * (double)__builtin_amdgcn_exp2f((own - m) * k2);
    }
    total = wave_sum(total);
    if constexpr (GREEDY) total = total == 0 && at < V ? 1.0 : 0.0;
    if (lane == 0) {
      s.m[which][i] = m;
      s.sum[which][i] = total > 0 ? total : 0.0;  // NaN: none
      if (which == 0) s.best[i] = at;
    }
  }
  __syncthreads();
  const End e = walk<TYPE, GREEDY, THREADS>(d, r, first, n, s);
  if (GREEDY || e.row < 0) return;
  double sp = s.sum[0][e.node], sq = s.sum[1][e.node];
  if (e.c != 0 && !exact) exp_sums<TYPE, EACH, THREADS>(weights_of<TYPE>(a, e, 1, 1, nullptr, 0), 0, V, s.red, &sp, &sq);
  Weights f = weights_of<TYPE>(a, e, sp, sq, s_gone, gone_symbols(a, e, s_gone, &s_count));
  const int segments = (V + kVSegment - 1) / kVSegment;
  int more = e.more, plain = 0;  // rejections to be added to c; nothing is left, from p itself
  double c = e.c;
  while (true) {
#pragma unroll 1
    for (int x = wave; x < segments; x += WAVES) {
      double w[EACH];
      weigh<TYPE, EACH>(f, x * kVSegment + lane * EACH, V, plain, w);
      double mine = 0;
#pragma unroll
      for (int j = 0; j < EACH; ++j) mine += w[j];
      mine = wave_sum(mine);
      if (lane == 0) s_seg[x] = mine;
    }
    __syncthreads();
    const double mine = lane < segments ? s_seg[lane] : 0.0;
    double run = mine;
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) {
      const double up = __shfl_up(run, y, 64);
      if (lane >= y) run += up;
    }
    const double total = __shfl(run, 63, 64);
    if (more > 0 || (!(total > 0) && plain == 0)) {
      if (more > 0) {
        c += total;
        --more;
        f.iq = c / sq;
      } else {
        plain = 1;
      }
      __syncthreads();
      continue;
    }
    if (wave != 0) return;
    double goal = goal_of(a, r, total);
    uint64_t some = __ballot(mine > 0 && run > goal);
    if (some == 0) {  // by the sums' rounding alone: the last that has any weight
      goal = __builtin_huge_val();
      some = 1ull << (63 - __builtin_clzll(__ballot(mine > 0) | 1));
    }
    const int seg = __builtin_ctzll(some);
    double at = __shfl(run - mine, seg, 64), w[EACH], own = 0;
    const int v0 = seg * kVSegment + lane * EACH;
    weigh<TYPE, EACH>(f, v0, V, plain, w);
#pragma unroll
    for (int j = 0; j < EACH; ++j) own += w[j];
    double ends = own;
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) {
      const double up = __shfl_up(ends, y, 64);
      if (lane >= y) ends += up;
    }
    at += ends - own;
    int hit = 0x7fffffff, last = -1;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      at += w[j];
      if (w[j] > 0) {
        last = v0 + j;
        if (at > goal) hit = min(hit, v0 + j);
      }
    }
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) {
      hit = min(hit, __shfl_xor(hit, y, 64));
      last = max(last, __shfl_xor(last, y, 64));
    }
    if (lane == 0) a.token[r] = hit != 0x7fffffff ? hit : last;
    return;
  }
}

namespace {

// Parts of a row in the first step: enough for 2048 workgroups, of 8192 symbols or more.
// (us of the whole call for 512, 2048 and 8192: trees of 9 nodes for 32 requests, 128000 bf16
// symbols 102.5, 97.2 and 99.7; with parts of 4096 one request of 5 nodes 30.3 for 28.1.)
int row_splits(const mca_verify_drafts_args& a) {
  const int64_t rows = std::max<int64_t>(1, a.n_rows) * (a.draft != nullptr && !a.greedy ? 2 : 1);
  return (int)std::clamp<int64_t>(std::min((2048 + rows - 1) / rows, a.n_vocab / kVPart), 1, kVMaxSplits);
}
// Parts of a row in the draw: enough for four workgroups a compute unit, of 2048 symbols or
// more.  (Us, bf16, with 256, 512, 1024 and 2048 workgroups: 32 requests of trees, 128000 symbols
// 133, 107, 100 and 105; 150 chains of 4 drafts, 32000 symbols 87, 70, 68 and 69.  With parts of 4096 symbols
// and of 2048: one request of 128000 symbols 30.5 and 28.7, 8 of 50000 35.6 and 31.5, 32 of 32000 with four
// children a node 111 and 116.  Half as many workgroups of 512 threads take 104 for 94, of 1024 122.)
int end_cuts(const mca_verify_drafts_args& a) {
  const int64_t reqs = std::max(1, a.n_req), cuts = (a.n_vocab + kVCut - 1) / kVCut;
  return (int)std::clamp<int64_t>(std::min(cuts, (1024 + reqs - 1) / reqs), 1, kVMaxSplits);
}
size_t room(size_t n) { return (n + 255) / 256 * 256; }
// A request in one workgroup, while its rows are few values in all.  (bf16, 32 requests,
// us with one workgroup a request and over all of the chip: drafts of 5, 1000 symbols 18 and
// 25; trees of 8, 2000 symbols 22 and 26, 5000 30 and 31, 16000 72 and 36; 8 requests of 47
// nodes, 500 symbols 25 and 27; 200 drafts of 4, 6000 symbols 32 and 40; but 4 of one
// node, 16000 symbols 37 and 27.  Greedy calls need no draw: 64 drafts of 4, 8000 symbols 17
// and 12.  Four waves instead of 16 are slower: 22 for 18, 46 for 30.)
bool is_whole(const mca_verify_drafts_args& a) {
  const int64_t values = a.n_vocab * a.max_nodes * (a.draft != nullptr && !a.greedy ? 2 : 1);
  return a.n_vocab <= kVWhole && values <= (a.greedy ? 1 << 13 : 1 << 16);
}

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
  d->active = (int32_t*)take((size_t)kVSteps * (1 + a.n_req) * sizeof(int32_t));
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
  if (is_whole(a)) {
    if (a.greedy)
      hipLaunchKernelGGL((k_lm_verify_whole<TYPE, true>), dim3((unsigned)a.n_req), dim3(kWalkThreads), 0, s, d);
    else
      hipLaunchKernelGGL((k_lm_verify_whole<TYPE, false>), dim3((unsigned)a.n_req), dim3(kWalkThreads), 0, s, d);
    hipLaunchKernelGGL(k_lm_verify_compact, dim3(1), threads, 0, s, d);
    return;
  }
  if (a.greedy) {
    if (a.n_rows > 0) hipLaunchKernelGGL((k_lm_verify_rows<TYPE, true>), rows, threads, 0, s, d);
    hipLaunchKernelGGL((k_lm_verify_walk<TYPE, true>), dim3((unsigned)a.n_req), dim3(kWalkThreads), 0, s, d);
    hipLaunchKernelGGL(k_lm_verify_compact, dim3(1), threads, 0, s, d);
    return;
  }
  if (a.n_rows > 0) hipLaunchKernelGGL((k_lm_verify_rows<TYPE, false>), rows, threads, 0, s, d);
  hipLaunchKernelGGL((k_lm_verify_walk<TYPE, false>), dim3((unsigned)a.n_req), dim3(kWalkThreads), 0, s, d);
  if (both == 2) hipLaunchKernelGGL((k_lm_verify_sums<TYPE>), dim3((unsigned)a.n_req, (unsigned)d.cuts), threads, 0, s, d);
  // A node has at most max_nodes - 1 children.  (us with 1, 2 and 3 further steps: 32 requests
  // of trees of 9 nodes with four children each, 32000 symbols 150, 119 and 86, with two 96.5, 97.3
  // and 99.8, 128000 symbols; of chains of 5, which need none, 41, 43 and 44.)
  const int steps = 1 + (both == 2 ? std::clamp(a.max_nodes - 2, 0, kVSteps) : 0);
  hipLaunchKernelGGL((k_lm_verify_draw<TYPE>), dim3((unsigned)a.n_req + 1, (unsigned)d.cuts), threads, 0, s, d, steps);
  for (int i = 1; i < steps; ++i)
    hipLaunchKernelGGL((k_lm_verify_draw_more<TYPE>), dim3((unsigned)std::min<int64_t>(512, (int64_t)a.n_req * d.cuts)), threads, 0, s, d, i, steps);
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
