// HIP kernels (gfx950) of the attention of drafted tokens over a paged cache
// (mca_tree_attention).
#include <algorithm>

#include "device_common.hpp"
#include "lm_device.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / 64;
constexpr int kTilePos = 32;  // cached tokens that a wave takes at a time
constexpr int kMaskWords = MCA_MAX_NODES / 32;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// The running maximum follows the scores only when one passes it by more than
// this (in powers of two): weights then reach 2^8 at most, which fp16 holds, and
// the sums of the products are rescaled a few times in all, not once a tile.
constexpr float kSlack = 8.0f;

template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 v = {a, b};
  if constexpr (TYPE == MCA_TYPE_BF16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
template <int TYPE>
__device__ __forceinline__ f32x4 mma32(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (TYPE == MCA_TYPE_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
}
// whether one of a dword's values is infinite or NaN
template <int TYPE>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  if constexpr (TYPE == MCA_TYPE_F32) return (w & 0x7f800000u) == 0x7f800000u;
  constexpr uint32_t e = TYPE == MCA_TYPE_BF16 ? 0x7f80u : 0x7c00u;
  return (w & e) == e || (w & (e << 16)) == (e << 16);
}
template <int TYPE>
__device__ __forceinline__ float part_of(uint32_t w, int half) {
  if constexpr (TYPE == MCA_TYPE_F32) return __uint_as_float(w);
  if constexpr (TYPE == MCA_TYPE_BF16) return __uint_as_float(half ? w & 0xffff0000u : w << 16);
  return (float)__builtin_bit_cast(f16x2, w)[half];
}

template <int N>
__device__ __forceinline__ void load_words(const char* p, uint32_t* out) {
  if constexpr (N == 1) {
    out[0] = gload((const uint32_t*)p);
  } else if constexpr (N == 2) {
    const u32x2 v = gload((const u32x2*)p);
    out[0] = v[0];
    out[1] = v[1];
  } else {
    const u32x4 v = gload((const u32x4*)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = v[i];
  }
}

struct AttnDev {
  mca_tree_attention_args a;
  int32_t group, row_tiles, chunk, splits;  // query heads per key head
  float* part_o;                            // [n_rows][n_head][splits][head_dim], each split's result
  float* part_l;                            // [n_rows][n_head][splits], log2 of its sum of exponentials
};

// Chunks of a request (at least one).
__device__ __forceinline__ int chunks_of(int len, int chunk) { return max(1, (len + chunk - 1) / chunk); }

}  // namespace

// A workgroup takes 16 QT rows (node, head of the group) of one request and key
// head against one chunk of the cached tokens; its 4 waves take tiles of 32
// tokens in turn, each with a running maximum, sum and result of its own, which
// are joined in LDS at the end, and chunks in a second launch.
//
// Everything stays in registers.  The products are transposed: S^T = K Q^T gives
// lane (q, li) the scores of query li with tokens 4 q + v and 16 + 4 q + v of the
// tile, which is already the operand layout of O^T = V^T P^T if the product's
// index 8 q + j means token 4 q + j (j < 4) or 16 + 4 q + j - 4.  V comes in as
// rows: a lane loads the same few dimensions of its 8 tokens, so 16 lanes read
// a whole row, and pairs of tokens are put together by one byte permutation per
// word; the result's row li then is dimension li * (dimensions of a lane) + e.
// fp32 takes v_mfma_f32_16x16x4f32 with one token of a lane a step.
//
// The last chunk's workgroup also takes the drafted tokens, each wave a tile
// of 32 nodes, with a mask of ancestors for each row (pointer doubling in LDS).
//
// PAD: head_dim is below DP; the missing dimensions are zero.
template <int TYPE, int DP, int QT, bool PAD>
__global__ __launch_bounds__(kAttnThreads) void k_lm_attn(AttnDev p) {
  constexpr bool f32 = TYPE == MCA_TYPE_F32;
  constexpr int EL = f32 ? 4 : 2;
  constexpr int KL = DP * EL / 64;        // 16-byte loads of a K row
  constexpr int VD = DP * EL / 64;        // words of a V row in a lane
  constexpr int CD = VD < 4 ? VD : 4;     // words of one load
  constexpr int NC = VD / CD;
  constexpr int EW = 4 / EL;              // values of a word
  constexpr int OT = DP / 16;             // 16-dimension tiles of the result
  const mca_tree_attention_args& a = p.a;
  __shared__ int s_par[2][MCA_MAX_NODES];
  __shared__ uint32_t s_mask[2][MCA_MAX_NODES][kMaskWords];
  __shared__ float s_o[2][OT * 4 * QT][64];
  __shared__ float s_ml[2][2 * QT][64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, q = lane >> 4, li = lane & 15;
  const int G = p.group, H = a.n_kv_head, D = a.head_dim, B = a.block_size;
  const int rt = blockIdx.x % p.row_tiles, rh = blockIdx.x / p.row_tiles, h = rh % H, r = rh / H;
  int first, n;
  if (!rows_of(a, r, &first, &n)) return;
  const int row0 = rt * 16 * QT;
  if (row0 >= n * G) return;
  const int len = cached_of(a, r), nchunk = chunks_of(len, p.chunk), split = blockIdx.y;
  if (split >= nchunk) return;
  const bool tree = split == nchunk - 1;
  const int dbytes = D * EL;
  // queries of the lane: column li of each of QT groups of 16 rows
  int node[QT], head[QT];
  u32x4 qf[QT][KL];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int row = row0 + 16 * t + li;
    node[t] = row / G;
    head[t] = h * G + (row - node[t] * G);
    const char* qp = (const char*)a.q + ((int64_t)(first + min(node[t], n - 1)) * a.q_row + (int64_t)head[t] * a.q_head) * EL;
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const bool ok = !PAD || 64 * i + 16 * q < dbytes;
      qf[t][i] = ok ? gload((const u32x4*)(qp + 64 * i + 16 * q)) : u32x4{0, 0, 0, 0};
    }
  }
  float m[QT], l[QT];
  f32x4 o[QT][OT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    m[t] = kLowest;
    l[t] = 0.f;
#pragma unroll
    for (int e = 0; e < OT; ++e) o[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float c2 = a.scale * kLog2e;

  u32x4 kf[2][KL];
  uint32_t vf[8][VD];
  // the wave's tile: token (lane & 31) in row `row` of kb and vb
  auto load_tile = [&](int64_t row, const char* kb, int64_t ks, const char* vb, int64_t vs) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int64_t rw = __shfl(row, 16 * x + li, 64);
      const char* kp = kb + rw * ks + 16 * q;
#pragma unroll
      for (int i = 0; i < KL; ++i)
        kf[x][i] = (!PAD || 64 * i + 16 * q < dbytes) ? gload((const u32x4*)(kp + 64 * i)) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t rw = __shfl(row, 4 * q + (j & 3) + 16 * (j >> 2), 64);
      const char* vp = vb + rw * vs + li * CD * 4;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (!PAD || (c * 16 + li) * CD * 4 < dbytes) {
          load_words<CD>(vp + c * 64 * CD, &vf[j][c * CD]);
        } else {
#pragma unroll
          for (int w = 0; w < CD; ++w) vf[j][c * CD + w] = 0;
        }
      }
    }
  };
  // One tile: valid has a bit for each token that is there; see[t] for each that
  // the lane's query t sees.
  f32x4 s[QT][2];
  auto scores = [&](uint32_t all, const uint32_t (&see)[QT]) {
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        s[t][x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          if constexpr (f32) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
              s[t][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[x][i][u]), __uint_as_float(qf[t][i][u]),
                                                             s[t][x], 0, 0, 0);
          } else {
            s[t][x] = mma32<TYPE>(kf[x][i], qf[t][i], s[t][x]);
          }
        }
      }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float top = -__builtin_huge_valf();
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          float z = s[t][x][v] * c2;
          if (all != 0xffffffffu) z = (see[t] >> (16 * x + 4 * q + v)) & 1 ? z : -__builtin_huge_valf();
          s[t][x][v] = z;
          top = fmaxf(top, z);
        }
      if (__ballot(top > m[t] + kSlack) != 0) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = fmaxf(m[t], top), f = __builtin_amdgcn_exp2f(m[t] - mn);
        m[t] = mn;
        l[t] *= f;
#pragma unroll
        for (int e = 0; e < OT; ++e) o[t][e] *= f;
      }
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float w = __builtin_amdgcn_exp2f(s[t][x][v] - m[t]);
          s[t][x][v] = w;
          l[t] += w;
        }
    }
  };
  auto products = [&]() {
    if constexpr (f32) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < OT; ++e)
#pragma unroll
          for (int t = 0; t < QT; ++t)
            o[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[j][e]), s[t][j >> 2][j & 3], o[t][e], 0, 0, 0);
    } else {
      u32x4 w[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          w[t][2 * x] = pack2<TYPE>(s[t][x][0], s[t][x][1]);
          w[t][2 * x + 1] = pack2<TYPE>(s[t][x][2], s[t][x][3]);
        }
#pragma unroll
      for (int d = 0; d < VD; ++d)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j)  // tokens 2 j and 2 j + 1, the low or high half of word d
            v[j] = __builtin_amdgcn_perm(vf[2 * j + 1][d], vf[2 * j][d], b ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int t = 0; t < QT; ++t) o[t][2 * d + b] = mma32<TYPE>(v, w[t], o[t][2 * d + b]);
        }
    }
  };
  // values of tokens that are not there (or not finite) do not enter the products
  auto clear_values = [&](uint32_t keep) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool ok = (keep >> (4 * q + (j & 3) + 16 * (j >> 2))) & 1;
#pragma unroll
      for (int w = 0; w < VD; ++w) vf[j][w] = ok ? vf[j][w] : 0u;
    }
  };

  {
    const int32_t* tab = a.table + (int64_t)r * a.table_stride;
    const int end = min(len, (split + 1) * p.chunk);
    for (int p0 = split * p.chunk + wave * kTilePos; p0 < end; p0 += kAttnWaves * kTilePos) {
      const int pos = p0 + (lane & 31);
      const int blk = pos < end ? tab[(unsigned)pos / (unsigned)B] : -1;
      const bool ok = blk >= 0 && blk < a.n_blocks;
      const int64_t row = ok ? ((int64_t)blk * H + h) * B + (unsigned)pos % (unsigned)B : 0;
      const uint32_t valid = (uint32_t)__ballot(ok);
      load_tile(row, (const char*)a.k_cache, dbytes, (const char*)a.v_cache, dbytes);
      uint32_t see[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) see[t] = valid;
      if (valid != 0xffffffffu) clear_values(valid);
      scores(valid, see);
      products();
    }
  }
  if (tree) {
    // masks of ancestors: a node's mask takes in that of the node its pointer
    // stands at, and the pointer moves on to where that one's stands
    if (tid < n) {
      const int up = a.parents[first + tid];
      s_par[0][tid] = up >= 0 && up < tid ? up : -1;
#pragma unroll
      for (int w = 0; w < kMaskWords; ++w) s_mask[0][tid][w] = (tid >> 5) == w ? 1u << (tid & 31) : 0u;
    }
    int from = 0;
    for (int d = 1; d < n; d <<= 1) {
      __syncthreads();
      if (tid < n) {
        const int up = s_par[from][tid];
        s_par[from ^ 1][tid] = up >= 0 ? s_par[from][up] : -1;
#pragma unroll
        for (int w = 0; w < kMaskWords; ++w)
          s_mask[from ^ 1][tid][w] = s_mask[from][tid][w] | (up >= 0 ? s_mask[from][up][w] : 0u);
      }
      from ^= 1;
    }
    __syncthreads();
    const int w0 = wave;  // a wave's 32 nodes
    if (32 * w0 < n) {
      const int nd = 32 * w0 + (lane & 31);
      const uint32_t valid = (uint32_t)__ballot(nd < n);
      const char* kb = (const char*)a.k + ((int64_t)first * a.k_row + (int64_t)h * a.k_head) * EL;
      const char* vb = (const char*)a.v + ((int64_t)first * a.v_row + (int64_t)h * a.v_head) * EL;
      load_tile(nd < n ? nd : 0, kb, a.k_row * EL, vb, a.v_row * EL);
      uint32_t see[QT];
#pragma unroll
      for (int t = 0; t < QT; ++t) see[t] = s_mask[from][min(node[t], n - 1)][w0];
      // A node that some rows do not see may hold anything: values that are not
      // finite are left out of the products and added for the rows that see them.
      uint32_t odd = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        bool nf = false;
#pragma unroll
        for (int w = 0; w < VD; ++w) nf = nf || not_finite<TYPE>(vf[j][w]);
        const uint64_t any = __ballot(nf);
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if ((any >> (16 * g)) & 0xffff) odd |= 1u << (4 * g + (j & 3) + 16 * (j >> 2));
      }
      clear_values(valid & ~odd);
      scores(0, see);
      products();
      for (odd &= valid; odd != 0; odd &= odd - 1) {
        const int at = __builtin_ctz(odd), x = at >> 4, src = ((at >> 2) & 3) * 16 + li;
        const char* vp = vb + (int64_t)(32 * w0 + at) * a.v_row * EL;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
          float w = 0.f;
#pragma unroll
          for (int xx = 0; xx < 2; ++xx)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const float y = __shfl(s[t][xx][v], src, 64);
              if (xx == x && v == (at & 3)) w = y;
            }
          if (((see[t] >> at) & 1) == 0) continue;
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int off = (c * 16 + 4 * q + v) * CD * 4;
              if (PAD && off >= dbytes) continue;
              uint32_t vals[CD];
              load_words<CD>(vp + off, vals);
#pragma unroll
              for (int d = 0; d < CD; ++d)
#pragma unroll
                for (int b = 0; b < EW; ++b)
                  o[t][(c * CD + d) * EW + b][v] = fmaf(w, part_of<TYPE>(vals[d], b), o[t][(c * CD + d) * EW + b][v]);
            }
        }
      }
    }
  }
  // join the waves: 2, 3 into 0, 1, then 1 into 0
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] += __shfl_xor(l[t], 16, 64);
    l[t] += __shfl_xor(l[t], 32, 64);
  }
#pragma unroll
  for (int half = kAttnWaves / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        s_ml[wave - half][2 * t][lane] = m[t];
        s_ml[wave - half][2 * t + 1][lane] = l[t];
#pragma unroll
        for (int e = 0; e < OT; ++e)
#pragma unroll
          for (int v = 0; v < 4; ++v) s_o[wave - half][(t * OT + e) * 4 + v][lane] = o[t][e][v];
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const float m2 = s_ml[wave][2 * t][lane], l2 = s_ml[wave][2 * t + 1][lane];
        const float mn = fmaxf(m[t], m2);
        const float f1 = __builtin_amdgcn_exp2f(m[t] - mn), f2 = __builtin_amdgcn_exp2f(m2 - mn);
        m[t] = mn;
        l[t] = l[t] * f1 + l2 * f2;
#pragma unroll
        for (int e = 0; e < OT; ++e)
#pragma unroll
          for (int v = 0; v < 4; ++v) o[t][e][v] = o[t][e][v] * f1 + s_o[wave][(t * OT + e) * 4 + v][lane] * f2;
      }
    }
  }
  if (wave != 0) return;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (node[t] >= n) continue;
    // a chunk without a token that is there weighs nothing
    const bool none = l[t] == 0.f;
    const float inv = none ? 0.f : 1.0f / l[t];
    const float lse2 = none ? -__builtin_huge_valf() : m[t] + __builtin_amdgcn_logf(l[t]);
    const int64_t out_row = (int64_t)(first + node[t]);
    if (nchunk > 1) {
      const int64_t at = (out_row * a.n_head + head[t]) * p.splits + split;
      if (q == 0) p.part_l[at] = lse2;
      float* po = p.part_o + at * D;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int d0 = (c * 16 + 4 * q + v) * CD * EW;
          if (PAD && d0 >= D) continue;
#pragma unroll
          for (int e = 0; e < CD * EW; ++e) po[d0 + e] = o[t][c * CD * EW + e][v] * inv;
        }
    } else {
      if (a.lse != nullptr && q == 0) a.lse[out_row * a.n_head + head[t]] = lse2 * kLn2;
      char* op = (char*)a.out + (out_row * a.out_row + (int64_t)head[t] * a.out_head) * EL;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int off = (c * 16 + 4 * q + v) * CD * 4;
          if (PAD && off >= dbytes) continue;
#pragma unroll
          for (int w = 0; w < CD; ++w) {
            uint32_t x;
            if constexpr (f32)
              x = __float_as_uint(o[t][c * CD + w][v] * inv);
            else
              x = pack2<TYPE>(o[t][(c * CD + w) * 2][v] * inv, o[t][(c * CD + w) * 2 + 1][v] * inv);
            gstore((uint32_t*)(op + off) + w, x);
          }
        }
    }
  }
}

// The results of a request's chunks joined: a wave per row and head, weights
// 2^(l_s - max l).
template <int TYPE>
__global__ __launch_bounds__(256) void k_lm_attn_join(AttnDev p) {
  const mca_tree_attention_args& a = p.a;
  const int r = blockIdx.y, lane = threadIdx.x & 63;
  int first, n;
  if (!rows_of(a, r, &first, &n)) return;
  const int nchunk = chunks_of(cached_of(a, r), p.chunk);
  const int item = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (nchunk == 1 || item >= n * a.n_head) return;
  const int64_t at = ((int64_t)first * a.n_head + item) * p.splits;
  const float* pl = p.part_l + at;
  const float* po = p.part_o + at * a.head_dim;
  float top = -__builtin_huge_valf();
  for (int s = lane; s < nchunk; s += 64) top = fmaxf(top, pl[s]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  float sum = 0.f;
  for (int s = lane; s < nchunk; s += 64) sum += __builtin_amdgcn_exp2f(pl[s] - top);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
  const int node = item / a.n_head, head = item - node * a.n_head;
  const float inv = 1.0f / sum;
  const int64_t row = (int64_t)first + node;
  if (a.lse != nullptr && lane == 0) a.lse[row * a.n_head + head] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
  for (int d = lane; d < a.head_dim; d += 64) {
    float acc = 0.f;
#pragma unroll 4
    for (int s = 0; s < nchunk; ++s) acc = fmaf(__builtin_amdgcn_exp2f(pl[s] - top), po[(int64_t)s * a.head_dim + d], acc);
    const int64_t to = row * a.out_row + (int64_t)head * a.out_head + d;
    if constexpr (TYPE == MCA_TYPE_F32)
      ((float*)a.out)[to] = acc * inv;
    else
      ((uint16_t*)a.out)[to] = (uint16_t)pack2<TYPE>(acc * inv, 0.f);
  }
}

namespace {

int row_group(const mca_tree_attention_args& a) {
  const int rows = a.max_nodes * (a.n_head / a.n_kv_head);
  return rows <= 16 || a.head_dim > 128 || (a.dtype == MCA_TYPE_F32 && a.head_dim > 64) ? 1 : 2;
}
int row_tiles(const mca_tree_attention_args& a) {
  const int rows = a.max_nodes * (a.n_head / a.n_kv_head), t = 16 * row_group(a);
  return (rows + t - 1) / t;
}

template <int TYPE, int DP, int QT>
void launch_dim(const AttnDev& p, dim3 grid, hipStream_t s) {
  if (p.a.head_dim == DP)
    hipLaunchKernelGGL((k_lm_attn<TYPE, DP, QT, false>), grid, dim3(kAttnThreads), 0, s, p);
  else
    hipLaunchKernelGGL((k_lm_attn<TYPE, DP, QT, true>), grid, dim3(kAttnThreads), 0, s, p);
}
template <int TYPE>
void launch_type(const AttnDev& p, dim3 grid, hipStream_t s) {
  const int D = p.a.head_dim, qt = row_group(p.a);
  constexpr int kBig = TYPE == MCA_TYPE_F32 ? 1 : 2;
  if (D <= 32) {
    qt == 1 ? launch_dim<TYPE, 32, 1>(p, grid, s) : launch_dim<TYPE, 32, 2>(p, grid, s);
  } else if (D <= 64) {
    qt == 1 ? launch_dim<TYPE, 64, 1>(p, grid, s) : launch_dim<TYPE, 64, 2>(p, grid, s);
  } else if (D <= 128) {
    qt == 1 ? launch_dim<TYPE, 128, 1>(p, grid, s) : launch_dim<TYPE, 128, kBig>(p, grid, s);
  } else {
    launch_dim<TYPE, 256, 1>(p, grid, s);
  }
  if (p.splits > 1)
    hipLaunchKernelGGL((k_lm_attn_join<TYPE>), dim3((unsigned)((p.a.max_nodes * p.a.n_head + 3) / 4), (unsigned)p.a.n_req),
                       dim3(256), 0, s, p);
}

}  // namespace

AttnPlan lm_attention_plan(const mca_tree_attention_args& a) {
  // chunks of at least two tiles a wave, as many as give the chip a few
  // workgroups per CU
  const int64_t wgs = (int64_t)row_tiles(a) * a.n_kv_head * a.n_req;
  const int64_t least = 2 * kAttnWaves * kTilePos;
  const int64_t want = std::clamp<int64_t>((2048 + wgs - 1) / wgs, 1, 256);
  int64_t chunk = std::max<int64_t>(least, (a.max_len + want - 1) / want);
  chunk = (chunk + kAttnWaves * kTilePos - 1) / (kAttnWaves * kTilePos) * (kAttnWaves * kTilePos);
  AttnPlan p;
  p.chunk = (int32_t)chunk;
  p.splits = (int32_t)std::max<int64_t>(1, (a.max_len + chunk - 1) / chunk);
  p.bytes = p.splits > 1 ? (size_t)a.n_rows * a.n_head * p.splits * (a.head_dim + 1) * sizeof(float) : 0;
  return p;
}

hipError_t lm_launch_attention(const mca_tree_attention_args& a, const AttnPlan& plan, hipStream_t s) {
  if (a.n_req == 0 || a.n_rows == 0) return hipSuccess;
  AttnDev p;
  p.a = a;
  p.group = a.n_head / a.n_kv_head;
  p.row_tiles = row_tiles(a);
  p.chunk = plan.chunk;
  p.splits = plan.splits;
  p.part_o = (float*)a.workspace;
  p.part_l = p.part_o + (size_t)a.n_rows * a.n_head * plan.splits * a.head_dim;
  const dim3 grid((unsigned)((int64_t)p.row_tiles * a.n_kv_head * a.n_req), (unsigned)plan.splits);
  switch (a.dtype) {
    case MCA_TYPE_F32: launch_type<MCA_TYPE_F32>(p, grid, s); break;
    case MCA_TYPE_BF16: launch_type<MCA_TYPE_BF16>(p, grid, s); break;
    default: launch_type<MCA_TYPE_F16>(p, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace mca
