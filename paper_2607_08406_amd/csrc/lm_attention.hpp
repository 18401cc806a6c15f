// HIP kernels (gfx950) of the attention of drafted tokens over a paged cache, in the
// type of the queries (mca_tree_attention, lm_attention.hip) or in 8 bits
// (mca_tree_attention8, lm_attention8.hip; C8 below).
#pragma once

#include <algorithm>

#include "device_common.hpp"
#include "lm_device.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

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
// Weights are powers of two relative to a reference that follows a row's scores only
// where a tile's largest leaves a window around it, so that the sums of the products
// are rescaled a few times in all, not once a tile.  With 8 exponent bits (fp32, bf16)
// the reference is the running maximum and follows what passes it by more than 2^8:
// smaller weights lose nothing until they are 2^-126.
//
// fp16 holds 2^-14 to 2^15 in full and steps of 2^-24 below, while the tokens that
// make the result may all lie far below the largest weight (a first token that takes
// nearly all weight and whose value is 0).  So the reference goes down as well: a
// tile's largest weight is put at 2^11, where a single one is exact (below that, by less
// than a power, on the way down), and stays between 2^-8 and 2^15.  A weight then
// is off by half a step of its own, or by 2^-25 where it is below 2^-14; over a tile
// of 64 tokens the latter is 2^-11 of the tile's largest weight at the most, and
// 2^-29 of it in a tile that has moved the reference.  It moves down by whole powers,
// which round nothing, and not below what leaves the sums under 2^80: tokens that lie
// further down weigh less than 2^-69 of their row's together.  (The second
// comparison costs 1 % at most, 4 % where scores are 4 times as large and references move
// often: 16 drafts of 48, 192 to 384 rows, head_dim 128, 273 us with and without, 284
// against 273.)
template <int TYPE>
struct Window {
  static constexpr bool kMoves = TYPE == MCA_TYPE_F16;
  static constexpr float kAbove = kMoves ? 15.0f : 8.0f, kBelow = 8.0f, kPut = 11.0f, kMost = 0x1p80f;
};
// Units of a workgroup that shares the work: fewer are not worth the joining.  (One
// request of 4096 tokens, 128 rows a key head, 4 of them, bf16, head_dim 128: 33 us
// with 2, 35 with 4, 54 with 16; 16 requests of 16384: 138, 136 and 139 us.)
constexpr int kLeastUnits = 4;

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
  // results of the parts of a row that several workgroups work on, and log2 of
  // their sums of exponentials: [n_rows][n_head][splits] of few rows, [2 share
  // workgroups][rows of a tile] of many (Share)
  float* part_o;
  float* part_l;
  int32_t sharers, rows;  // workgroups that share the work (0: one a tile of rows), rows of a tile
  int32_t* first_unit;    // [n_req + 1]
  const uint8_t *k_scale, *v_scale;  // of a cache of 8-bit values, [n_blocks][n_kv_head]
};

// Chunks of a request (at least one).
__device__ __forceinline__ int chunks_of(int len, int chunk) { return max(1, (len + chunk - 1) / chunk); }

// The rows of a wave, 16 QT of them (node, head of the group), against tiles of
// 32 NH tokens.  The products are transposed:
// S^T = K Q^T gives lane (q, li) the scores of query li with tokens 4 q + v and
// 16 + 4 q + v of the tile, which is already the operand layout of
// O^T = V^T P^T if the product's index 8 q + j means token 4 q + j (j < 4) or
// 16 + 4 q + j - 4.  V comes in as rows: a lane has the same few dimensions of
// its 8 tokens, so 16 lanes read a whole row, and pairs of tokens are put
// together by one byte permutation per word; the result's row li then is
// dimension li * (dimensions of a lane) + e.  So no score and no value passes through
// LDS to change its layout.  fp32 takes v_mfma_f32_16x16x4f32 with one token of a
// lane a step.
//
// A tile is worked on in registers as far as they go.  By the compiler's remarks the
// wide kernels of 16-bit values spill 13 to 17 (4 waves) or 31 to 35 (8) of 256 at
// head_dim 65 to 128 with 32 rows a wave, 10 to 24 above 128, none below 65; and the
// narrow fp32 kernel above 128 keeps whole arrays in 1152 bytes of scratch memory a lane
// (100 requests of 2000, one row a head, 4 key heads: 2.1 TB/s at 256, 4.2 at 128).
//
// DP is head_dim rounded up; with PAD the missing dimensions are zero.  A lane's
// parts of a K row lie 64 bytes apart, unless the row comes in 8 bits straight from
// memory: then they are those of the same bytes, LB of them a load (scores do not
// depend on the order of the dimensions).
template <int TYPE, int DP, int QT, int NH, bool PAD, int LB = 0>
struct Rows {
  static constexpr bool kF32 = TYPE == MCA_TYPE_F32;
  static constexpr int EL = kF32 ? 4 : 2;
  static constexpr int KL = DP * EL / 64;     // 16-byte parts of a K row in a lane
  static constexpr int VD = DP * EL / 64;     // words of a V row in a lane
  static constexpr int CD = VD < 4 ? VD : 4;  // words of one load
  static constexpr int NC = VD / CD;
  static constexpr int EW = 4 / EL;           // values of a word
  static constexpr int OT = DP / 16;          // 16-dimension tiles of the result

  // where 16-byte part i of lane q's dimensions lies in a row
  static __device__ __forceinline__ int part_at(int i, int q) {
    if constexpr (LB == 0) return 64 * i + 16 * q;
    constexpr int PP = LB == 0 ? 1 : LB * EL / 16;  // parts of a load
    return (i / PP * 4 + q) * LB * EL + i % PP * 16;
  }

  int q, li, first, n, dbytes;
  int node[QT], head[QT];
  u32x4 qf[QT][KL];
  typedef Window<TYPE> W;
  float m[QT], l[QT], c2;  // reference of the weights (scores times c2) and their sum so far
  f32x4 o[QT][OT];
  f32x4 s[QT][2 * NH];     // a tile's scores
  // and its weights: 16-bit ones in pairs, as operands of their products
  static constexpr int PW = kF32 ? 2 : 1;
  u32x4 pw[QT][PW * NH];

  // rows row0 .. row_end - 1 of request rows first_ ..
  __device__ __forceinline__ void begin(const mca_tree_attention_args& a, int h, int group, int row0, int row_end, int first_, int n_) {
    const int lane = threadIdx.x & 63;
    q = lane >> 4;
    li = lane & 15;
    first = first_;
    n = n_;
    dbytes = a.head_dim * EL;
    // a negative scale turns the queries round, so that larger scores weigh more;
    // a scale of 0 makes them 0, so that the -inf of a masked score stays
    const uint32_t turn = a.scale < 0.f ? (kF32 ? 0x80000000u : 0x80008000u) : 0u;
    const uint32_t stay = a.scale == 0.f ? 0u : 0xffffffffu;
    c2 = a.scale == 0.f ? kLog2e : fabsf(a.scale) * kLog2e;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int row = row0 + 16 * t + li;
      node[t] = row / group;
      head[t] = h * group + (row - node[t] * group);
      if (row >= row_end) node[t] = n;
      const char* qp = (const char*)a.q + ((int64_t)(first + min(node[t], n - 1)) * a.q_row + (int64_t)head[t] * a.q_head) * EL;
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        const int at = part_at(i, q);
        const bool ok = !PAD || at < dbytes;
        qf[t][i] = ok ? gload((const u32x4*)(qp + at)) : u32x4{0, 0, 0, 0};
        qf[t][i] = (qf[t][i] ^ turn) & stay;
      }
      m[t] = kLowest;
      l[t] = 0.f;
#pragma unroll
      for (int e = 0; e < OT; ++e) o[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // scores of 16 tokens: part i of row li of theirs is k(i)
  template <class K>
  __device__ __forceinline__ void score(int x, K k) {
#pragma unroll
    for (int t = 0; t < QT; ++t) s[t][x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const u32x4 kf = k(i);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        if constexpr (kF32) {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            s[t][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[u]), __uint_as_float(qf[t][i][u]), s[t][x], 0, 0, 0);
        } else {
          s[t][x] = mma32<TYPE>(kf, qf[t][i], s[t][x]);
        }
      }
    }
  }
  // weights of the tile; see[t][h] has a bit for each token of the h-th 32 that
  // query t sees, all of them if `every`.  The 16-bit types' weights are rounded to
  // 16 bits, as their products take them; the sum takes them in 32.  A result is off by
  // half a step of sum p |v| for that, and fp16's by what Window says; fp32 weights
  // would cost the products at a sixteenth of the rate.
  __device__ __forceinline__ void weigh(bool every, const uint32_t (&see)[QT][NH]) {
    if (!every) {
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int x = 0; x < 2 * NH; ++x)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            s[t][x][v] = (see[t][x >> 1] >> (16 * (x & 1) + 4 * q + v)) & 1 ? s[t][x][v] : -__builtin_huge_valf();
    }
    float top[QT];
    bool over = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      top[t] = s[t][0][0];
#pragma unroll
      for (int x = 0; x < 2 * NH; ++x)
#pragma unroll
        for (int v = 0; v < 4; ++v) top[t] = fmaxf(top[t], s[t][x][v]);
      top[t] *= c2;
      over = over || top[t] > m[t] + W::kAbove;
      if constexpr (W::kMoves) over = over || top[t] < m[t] - W::kBelow;
    }
    if (__ballot(over) != 0) {
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        top[t] = fmaxf(top[t], __shfl_xor(top[t], 16, 64));
        top[t] = fmaxf(top[t], __shfl_xor(top[t], 32, 64));
        float mn = fmaxf(m[t], top[t]), by = m[t] - mn;
        if constexpr (W::kMoves) {
          float sum = l[t] + __shfl_xor(l[t], 16, 64);
          sum += __shfl_xor(sum, 32, 64);
          const float put = top[t] - W::kPut, whole = floorf(m[t] - put);
          // (not so if nothing is seen or a score is NaN)
          const bool down = top[t] < m[t] - W::kBelow && sum * __builtin_amdgcn_exp2f(whole) <= W::kMost;
          const bool up = top[t] > m[t] + W::kAbove;
          by = up ? m[t] - put : (down ? whole : 0.f);
          mn = up ? put : m[t] - (down ? whole : 0.f);
        }
        const float f = __builtin_amdgcn_exp2f(by);
        m[t] = mn;
        l[t] *= f;
#pragma unroll
        for (int e = 0; e < OT; ++e) o[t][e] *= f;
      }
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 2 * NH; ++x) {
        float y[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          y[v] = __builtin_amdgcn_exp2f(fmaf(s[t][x][v], c2, -m[t]));
          sum[v] += y[v];
        }
        if constexpr (kF32) {
#pragma unroll
          for (int v = 0; v < 4; ++v) pw[t][x][v] = __float_as_uint(y[v]);
        } else {
          pw[t][x >> 1][2 * (x & 1)] = pack2<TYPE>(y[0], y[1]);
          pw[t][x >> 1][2 * (x & 1) + 1] = pack2<TYPE>(y[2], y[3]);
        }
      }
      l[t] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
  }
  // values of tokens that are not in `keep` become zero
  __device__ __forceinline__ void clear(uint32_t (&vf)[8][VD], uint32_t keep) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool ok = (keep >> (4 * q + (j & 3) + 16 * (j >> 2))) & 1;
#pragma unroll
      for (int w = 0; w < VD; ++w) vf[j][w] = ok ? vf[j][w] : 0u;
    }
  }
  // the values of the h-th 32 tokens, weighed; word d of a lane's row j of theirs is v(j, d)
  template <class V>
  __device__ __forceinline__ void add_words(int h, V word) {
    if constexpr (kF32) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < OT; ++e)
#pragma unroll
          for (int t = 0; t < QT; ++t)
            o[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(j, e)),
                                                           __uint_as_float(pw[t][2 * h + (j >> 2)][j & 3]), o[t][e], 0, 0, 0);
    } else {
#pragma unroll
      for (int d = 0; d < VD; ++d) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = word(j, d);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j)  // tokens 2 j and 2 j + 1, the low or high half of word d
            v[j] = __builtin_amdgcn_perm(w[2 * j + 1], w[2 * j], b ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int t = 0; t < QT; ++t) o[t][2 * d + b] = mma32<TYPE>(v, pw[t][h], o[t][2 * d + b]);
        }
      }
    }
  }
  __device__ __forceinline__ void add(int h, const uint32_t (&vf)[8][VD]) {
    add_words(h, [&](int j, int d) { return vf[j][d]; });
  }
  // the same of values that are operands already: value(e) is those of the lane's dimension e
  template <class V>
  __device__ __forceinline__ void add_operands(int h, V value) {
#pragma unroll
    for (int e = 0; e < OT; ++e) {
      const u32x4 v = value(e);
#pragma unroll
      for (int t = 0; t < QT; ++t) o[t][e] = mma32<TYPE>(v, pw[t][h], o[t][e]);
    }
  }
  // Drafted nodes: one that some rows do not see may hold anything.  Values that
  // are not finite (bits of `odd`) are left out of the products and added for the
  // rows that see them; value(at) is node `at`'s row of V in memory.
  __device__ __forceinline__ uint32_t odd_of(const uint32_t (&vf)[8][VD]) {
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
    return odd;
  }
  template <class Value>
  __device__ __forceinline__ void add_odd(int h, uint32_t odd, const uint32_t (&see)[QT][NH], Value value) {
    for (; odd != 0; odd &= odd - 1) {
      const int at = __builtin_ctz(odd), x = at >> 4, src = ((at >> 2) & 3) * 16 + li;
      const char* vp = value(at);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * PW; ++i) {
          const uint32_t y = __shfl(pw[t][PW * h + (i >> 2)][i & 3], src, 64);
          if (i == (4 * x + (at & 3)) / EW) w = part_of<TYPE>(y, at & (EW - 1));
        }
        if (((see[t][h] >> at) & 1) == 0) continue;
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
  __device__ __forceinline__ void sum_lanes() {
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      l[t] += __shfl_xor(l[t], 16, 64);
      l[t] += __shfl_xor(l[t], 32, 64);
    }
  }
  // results: to the call's output, or to place part(t) of the parts
  template <class Part>
  __device__ __forceinline__ void write(const AttnDev& p, bool whole, Part part) {
    const mca_tree_attention_args& a = p.a;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (node[t] >= n) continue;
      // A part that no weight falls to (none of its tokens is there, or every score is
      // -inf) weighs nothing.  A whole row sees itself: it has no weights only if every
      // score is -inf, and then softmax has no value, as the parts joined have none.
      const bool none = l[t] == 0.f;
      const float inv = none && !whole ? 0.f : 1.0f / l[t];
      const float lse2 = none ? (whole ? __builtin_nanf("") : -__builtin_huge_valf()) : m[t] + __builtin_amdgcn_logf(l[t]);
      const int64_t out_row = (int64_t)(first + node[t]);
      if (!whole) {
        const int64_t at = part(t);
        if (q == 0) p.part_l[at] = lse2;
        float* po = p.part_o + at * a.head_dim;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int d0 = (c * 16 + 4 * q + v) * CD * EW;
            if (PAD && d0 >= a.head_dim) continue;
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
              if constexpr (kF32)
                x = __float_as_uint(o[t][c * CD + w][v] * inv);
              else
                x = pack2<TYPE>(o[t][(c * CD + w) * 2][v] * inv, o[t][(c * CD + w) * 2 + 1][v] * inv);
              gstore((uint32_t*)(op + off) + w, x);
            }
          }
      }
    }
  }
};

// Cached token pos < end: its block, as the table has it (another's behind the
// end, so that the load needs no branch), and with that its row of the cache (one
// key head's token), -1 if it is not there.  The two are apart because a table's
// entry has to be under way before the tile in front of it is worked on.
__device__ __forceinline__ int cache_block(const mca_tree_attention_args& a, const int32_t* tab, int pos, int end) {
  return gload(tab + (unsigned)min(pos, end - 1) / (unsigned)a.block_size);
}
__device__ __forceinline__ int cache_row(const mca_tree_attention_args& a, int blk, int h, int pos, int end) {
  const int in = (int)((unsigned)pos % (unsigned)a.block_size);
  const bool ok = pos < end && blk >= 0 && blk < a.n_blocks;
  return ok ? (blk * a.n_kv_head + h) * a.block_size + in : -1;
}

// Masks of ancestors of a request's n nodes (all threads of the workgroup): a
// node's mask takes in that of the node its pointer stands at, and the pointer
// moves on to where that one's stands.  Returns which of the two buffers has them.
__device__ __forceinline__ int ancestors(const int32_t* parents, int n, int (&s_par)[2][MCA_MAX_NODES],
                                         uint32_t (&s_mask)[2][MCA_MAX_NODES][kMaskWords]) {
  const int tid = threadIdx.x;
  if (tid < n) {
    const int up = parents[tid];
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
  return from;
}

// The workgroup's tile of rows, key head, request and chunk: workgroups go round
// the 8 XCDs, so those that read the same cached tokens (the tiles of rows of one
// request, key head and chunk) are 8 apart, which puts them behind one L2.
__device__ __forceinline__ bool place(const AttnDev& p, int* rt, int* h, int* r, int* split) {
  const unsigned of = blockIdx.x / 8, pairs = (unsigned)p.a.n_req * p.a.n_kv_head;
  *rt = (int)(of % p.row_tiles);
  const unsigned item = of / p.row_tiles * 8 + blockIdx.x % 8, rh = item % pairs;
  *split = (int)(item / pairs);
  *h = (int)(rh % p.a.n_kv_head);
  *r = (int)(rh / p.a.n_kv_head);
  return *split < p.splits;
}

// The kernel's arguments, read anew: what they hold would otherwise stay in scalar
// registers for the whole kernel, more than there are, and crowd out a tile's vectors.
__device__ __forceinline__ const AttnDev& again() {
  auto k = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(k));
  return *(const AttnDev*)k;
}

// Many rows, long contexts: the work is cut into units, one tile of tokens
// against one tile of rows, in the order of requests, key heads, tiles of rows and
// tiles of tokens, and each workgroup takes `per` units in a row, so that all
// end together whatever the lengths are.  At most two of a workgroup's items
// are cut, its first (place 2 g of the parts) and its last (2 g + 1).
struct Share {
  int tiles, row_tiles, rows;  // of an item: tiles of tokens; of a request and key head: tiles of rows, and a tile's
  __device__ __forceinline__ Share(const AttnDev& p, int len, int n, int TP) {
    const int all = n * p.group;
    tiles = (len + TP - 1) / TP + (n + TP - 1) / TP;
    row_tiles = (all + p.rows - 1) / p.rows;
    rows = row_tiles == 0 ? 0 : ((all + row_tiles - 1) / row_tiles + 15) / 16 * 16;  // evenly
  }
  // (their number fits 32 bits: lm_attention_plan)
  static __device__ __forceinline__ int units(const AttnDev& p, int r, int TP) {
    int first, n;
    if (!rows_of(p.a, r, &first, &n)) return 0;
    const Share s(p, cached_of(p.a, r), n, TP);
    return p.a.n_kv_head * s.row_tiles * s.tiles;
  }
  static __device__ __forceinline__ int per(const AttnDev& p, int all) {
    const int even = (all + p.sharers - 1) / p.sharers;
    return even > kLeastUnits ? even : kLeastUnits;
  }
};

// Where the workgroup's share begins: its units and the place of its first part;
// s_begin has the request and the units before that.  False if there are none.
template <int TP, int NW>
__device__ __forceinline__ bool share_begin(const AttnDev& p, int (&s_wave)[NW], int (&s_begin)[2], int* unit, int* end, int* part) {
  constexpr int THREADS = 64 * NW;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n_req = p.a.n_req;
  // each thread's requests, then the sums of those before them
  const int some = (n_req + THREADS - 1) / THREADS;
  int mine = 0;
  for (int x = tid * some; x < (tid + 1) * some && x < n_req; ++x) mine += Share::units(p, x, TP);
  int run = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(run, d, 64);
    if (lane >= d) run += up;
  }
  if (lane == 63) s_wave[wave] = run;
  __syncthreads();
  int all = 0, pre = run - mine;
#pragma unroll
  for (int x = 0; x < NW; ++x) {
    if (x < wave) pre += s_wave[x];
    all += s_wave[x];
  }
  // workgroups on one XCD (every eighth) take neighbouring units
  const int g = (int)(blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8), per = Share::per(p, all);
  // g per < sharers (all / sharers + 1) + the least units of all: below 2^31
  const int u0 = g * per, u1 = min(all, u0 + per);
  for (int x = tid * some; x < (tid + 1) * some && x < n_req; ++x) {
    const int u = Share::units(p, x, TP);
    if (blockIdx.x == 0) p.first_unit[x] = pre;
    if (u0 >= pre && u0 < pre + u) {
      s_begin[0] = x;
      s_begin[1] = pre;
    }
    pre += u;
  }
  if (blockIdx.x == 0 && tid == 0) p.first_unit[n_req] = all;
  if (u0 >= u1) return false;
  *unit = u0;
  *end = u1;
  *part = 2 * g;
  __syncthreads();
  return true;
}

}  // namespace

// Few rows: a workgroup takes 16 rows of one request and key head against one
// chunk of the cached tokens; its 4 waves take tiles in turn, straight from memory
// into registers, each with a reference, sum and result of its own, which are
// joined in LDS at the end, and chunks in a second launch.  The last chunk's
// workgroup also takes the drafted tokens, each wave 32 nodes.
//
// Bound by memory where there is enough to read: a cached value is read once and
// used 16 times, and nothing is shared between the waves that LDS would save (200
// requests of 1000 to 2000, one row a head, 4 key heads of 128, bf16: 0.6 GB in
// 131 us).  Small calls are bound by the chain of table entry, K, scores, V (64 drafts
// of up to 8 nodes over at most 120 tokens, 4 heads of 32, fp32: 8.5 us).
// Over codes the same; a code's conversion and scale are one instruction for two, which
// memory still hides: 32 single tokens behind 8192 to 32768, 8 key heads of 128, 4 rows a
// head, bf16 (1.33 GB): 250 us and 10 of joining, 5.3 TB/s; the drafts of 8 8.1 us.

// Waves of a SIMD that its registers are for, of 8-bit caches; of shared work (head_dim above
// 64) few enough that nothing of the loop around the items goes to scratch memory.
constexpr int resident8(int type, int dp, bool share) {
  if (share) return dp <= 128 ? 2 : 1;
  return dp <= 64 ? (type == MCA_TYPE_F32 ? 3 : 4) : (dp <= 128 ? (type == MCA_TYPE_F32 ? 2 : 3) : 1);
}
template <int TYPE, int DP, bool PAD, bool C8, bool SHARE = false>
__global__ __launch_bounds__(kAttnThreads, C8 ? resident8(TYPE, DP, SHARE) : 1) void k_lm_attn(AttnDev args) {
  constexpr int LB = DP / 4 < 16 ? DP / 4 : 16;  // bytes of a load of 8-bit keys
  typedef Rows<TYPE, DP, 1, 1, PAD, C8 ? LB : 0> R;
  constexpr int EL = R::EL, KL = R::KL, VD = R::VD, CD = R::CD, NC = R::NC, OT = R::OT;
  __shared__ int s_par[2][MCA_MAX_NODES];
  __shared__ uint32_t s_mask[2][MCA_MAX_NODES][kMaskWords];
  __shared__ float s_o[2][OT * 4][64];
  __shared__ float s_ml[2][2][64];
  __shared__ int s_wave[kAttnWaves], s_begin[2];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  constexpr int TP = kAttnWaves * kTilePos;  // tokens of a unit of shared work
  constexpr bool shared = SHARE;
  int rt = 0, h = 0, r = 0, split = 0, first, n;
  int unit = 0, unit_end = 0, before = 0, part = 0;
  if (shared) {
    if (!share_begin<TP, kAttnWaves>(again(), s_wave, s_begin, &unit, &unit_end, &part)) return;
    r = __builtin_amdgcn_readfirstlane(s_begin[0]);
    before = __builtin_amdgcn_readfirstlane(s_begin[1]);
  } else if (!place(args, &rt, &h, &r, &split)) {
    return;
  }
  // one item, or those of the workgroup's share
  while (true) {
    const AttnDev& p = SHARE ? again() : args;
    const mca_tree_attention_args& a = p.a;
    int from_token, end, parts;  // the cached tokens, and in how many parts the rows are worked on
    bool drafted;
    if (shared) {
      if (unit >= unit_end) return;
      for (int units = Share::units(p, r, TP); unit >= before + units; units = Share::units(p, r, TP)) {
        before += units;
        ++r;
      }
      rows_of(a, r, &first, &n);
      const int len = cached_of(a, r);
      const Share sh(p, len, n, TP);
      h = (unit - before) / sh.tiles;
      const int tile0 = unit - before - h * sh.tiles, tile1 = min(sh.tiles, tile0 + (unit_end - unit));
      unit += tile1 - tile0;
      from_token = tile0 * TP;
      end = min(len, tile1 * TP);
      drafted = tile1 * TP > len && tile1 == sh.tiles;
      parts = tile0 == 0 && tile1 == sh.tiles ? 1 : 2;
    } else {
      if (!rows_of(a, r, &first, &n) || rt * 16 >= n * p.group) return;
      const int len = cached_of(a, r);
      parts = chunks_of(len, p.chunk);
      if (split >= parts) return;
      from_token = split * p.chunk;
      end = min(len, (split + 1) * p.chunk);
      drafted = split == parts - 1;
    }
    const int row0 = rt * 16;
    R w;
    w.begin(a, h, p.group, row0, n * p.group, first, n);
    const int q = w.q, li = w.li;
    u32x4 kf[2][KL];
    uint32_t vf[8][VD];
    // the tile's tokens: token (lane & 31) is row `row` of kb and vb
    auto load_tile = [&](int row, const char* kb, uint32_t ks, const char* vb, uint32_t vs) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const char* kp = kb + (uint64_t)(uint32_t)__shfl(row, 16 * x + li, 64) * ks;
#pragma unroll
        for (int i = 0; i < KL; ++i)
          kf[x][i] = (!PAD || w.part_at(i, q) < w.dbytes) ? gload((const u32x4*)(kp + w.part_at(i, q))) : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const char* vp = vb + (uint64_t)(uint32_t)__shfl(row, 4 * q + (j & 3) + 16 * (j >> 2), 64) * vs + li * CD * 4;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          if (!PAD || (c * 16 + li) * CD * 4 < w.dbytes) {
            load_words<CD>(vp + c * 64 * CD, &vf[j][c * CD]);
          } else {
#pragma unroll
            for (int d = 0; d < CD; ++d) vf[j][c * CD + d] = 0;
          }
        }
      }
    };
    auto scores = [&]() {
#pragma unroll
      for (int x = 0; x < 2; ++x) w.score(x, [&](int i) { return kf[x][i]; });
    };
    uint32_t see[1][1];
    {
      const int32_t* tab = a.table + (int64_t)r * a.table_stride;
      int p0 = from_token + wave * kTilePos;
      int blk = p0 < end ? cache_block(a, tab, p0 + (lane & 31), end) : 0;
      if constexpr (C8) {
        // A tile's codes are requested while the one before is worked on (a value takes
        // half the registers that it would in 16 bits), and widened, times its block's
        // scale, where its product takes it.
        constexpr int NK = DP / 4 / LB, VB = CD * 4 / EL, VW = VB < 4 ? 1 : VB / 4;  // loads of a K row, bytes and words of one of V
        uint32_t kc[2][NK][LB / 4], vc[8][NC][VW], nk[2][NK][LB / 4], nv[8][NC][VW];
        int row = -1, ks = 0, vs = 0;
        auto request = [&](int at) {
          row = cache_row(a, blk, h, at + (lane & 31), end);
          const int of = row >= 0 ? blk * a.n_kv_head + h : 0, from = max(row, 0);
          ks = gload(p.k_scale + of);
          vs = gload(p.v_scale + of);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const char* kp = (const char*)a.k_cache + (uint64_t)(uint32_t)__shfl(from, 16 * x + li, 64) * a.head_dim + LB * q;
#pragma unroll
            for (int i = 0; i < NK; ++i) {
              if (!PAD || 4 * LB * i + LB * q < a.head_dim) {
                load_codes<LB>(kp + 4 * LB * i, nk[x][i]);
              } else {
#pragma unroll
                for (int d = 0; d < LB / 4; ++d) nk[x][i][d] = 0;
              }
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const char* vp = (const char*)a.v_cache + (uint64_t)(uint32_t)__shfl(from, 4 * q + (j & 3) + 16 * (j >> 2), 64) * a.head_dim + VB * li;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              if (!PAD || (c * 16 + li) * VB < a.head_dim) {
                load_codes<VB>(vp + c * 16 * VB, nv[j][c]);
              } else {
#pragma unroll
                for (int d = 0; d < VW; ++d) nv[j][c][d] = 0;
              }
            }
          }
          blk = cache_block(a, tab, at + kAttnWaves * kTilePos + (lane & 31), end);
        };
        if (p0 < end) request(p0);
        for (; p0 < end; p0 += kAttnWaves * kTilePos) {
          const uint32_t valid = (uint32_t)__ballot(row >= 0);
          const int ksc = ks, vsc = vs;
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < NK; ++i)
#pragma unroll
              for (int d = 0; d < LB / 4; ++d) kc[x][i][d] = nk[x][i][d];
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
              for (int d = 0; d < VW; ++d) vc[j][c][d] = nv[j][c][d];
          if (p0 + kAttnWaves * kTilePos < end) request(p0 + kAttnWaves * kTilePos);
          see[0][0] = valid;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float f = scale_of((uint32_t)__shfl(ksc, 16 * x + li, 64));
            constexpr int PP = LB * EL / 16, PC = 16 / EL / 4;  // parts of a load, words of codes of a part
            w.score(x, [&](int i) { return wide_part<TYPE>(&kc[x][i / PP][i % PP * PC], f); });
          }
          w.weigh(valid == 0xffffffffu, see);
          float f[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            f[j] = scale_of((uint32_t)__shfl(vsc, 4 * q + (j & 3) + 16 * (j >> 2), 64));
            if (valid != 0xffffffffu) {
              const bool ok = (valid >> (4 * q + (j & 3) + 16 * (j >> 2))) & 1;
#pragma unroll
              for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int d = 0; d < VW; ++d) vc[j][c][d] = ok ? vc[j][c][d] : 0u;
            }
          }
          w.add_words(0, [&](int j, int d) {
            const int c = d / CD, x = d % CD;
            if constexpr (TYPE == MCA_TYPE_F32)
              return x & 2 ? wide2_f32<true>(vc[j][c][0], f[j])[x & 1] : wide2_f32<false>(vc[j][c][0], f[j])[x & 1];
            else
              return x & 1 ? wide2<TYPE, true>(vc[j][c][x / 2], f[j]) : wide2<TYPE, false>(vc[j][c][x / 2], f[j]);
          });
        }
      } else {
        for (; p0 < end; p0 += kAttnWaves * kTilePos) {
          const int row = cache_row(a, blk, h, p0 + (lane & 31), end);
          blk = cache_block(a, tab, p0 + kAttnWaves * kTilePos + (lane & 31), end);
          const uint32_t valid = (uint32_t)__ballot(row >= 0);
          load_tile(max(row, 0), (const char*)a.k_cache, w.dbytes, (const char*)a.v_cache, w.dbytes);
          see[0][0] = valid;
          if (valid != 0xffffffffu) w.clear(vf, valid);
          scores();
          w.weigh(valid == 0xffffffffu, see);
          w.add(0, vf);
        }
      }
    }
    if (drafted) {
      const int from = ancestors(a.parents + first, n, s_par, s_mask);
      const int n0 = kTilePos * wave;
      if (n0 < n) {
        const int nd = n0 + (lane & 31);
        const uint32_t valid = (uint32_t)__ballot(nd < n);
        const char* kb = (const char*)a.k + ((int64_t)first * a.k_row + (int64_t)h * a.k_head) * EL;
        const char* vb = (const char*)a.v + ((int64_t)first * a.v_row + (int64_t)h * a.v_head) * EL;
        load_tile(nd < n ? nd : 0, kb, (uint32_t)(a.k_row * EL), vb, (uint32_t)(a.v_row * EL));
        see[0][0] = s_mask[from][min(w.node[0], n - 1)][wave];
        const uint32_t odd = w.odd_of(vf) & valid;
        w.clear(vf, valid & ~odd);
        scores();
        w.weigh(false, see);
        w.add(0, vf);
        w.add_odd(0, odd, see, [&](int at) { return vb + (int64_t)(n0 + at) * a.v_row * EL; });
      }
    }
    // join the waves: 2, 3 into 0, 1, then 1 into 0
    w.sum_lanes();
#pragma unroll
    for (int half = kAttnWaves / 2; half > 0; half >>= 1) {
      __syncthreads();
      if (wave >= half && wave < 2 * half) {
        s_ml[wave - half][0][lane] = w.m[0];
        s_ml[wave - half][1][lane] = w.l[0];
#pragma unroll
        for (int e = 0; e < OT; ++e)
#pragma unroll
          for (int v = 0; v < 4; ++v) s_o[wave - half][e * 4 + v][lane] = w.o[0][e][v];
      }
      __syncthreads();
      if (wave < half) {
        const float m2 = s_ml[wave][0][lane], l2 = s_ml[wave][1][lane];
        const float mn = fmaxf(w.m[0], m2);
        const float f1 = __builtin_amdgcn_exp2f(w.m[0] - mn), f2 = __builtin_amdgcn_exp2f(m2 - mn);
        w.m[0] = mn;
        w.l[0] = w.l[0] * f1 + l2 * f2;
#pragma unroll
        for (int e = 0; e < OT; ++e)
#pragma unroll
          for (int v = 0; v < 4; ++v) w.o[0][e][v] = w.o[0][e][v] * f1 + s_o[wave][e * 4 + v][lane] * f2;
      }
    }
    if (wave == 0)
      w.write(p, parts == 1, [&](int t) {
        return shared ? (int64_t)part * p.rows + li : ((int64_t)(first + w.node[t]) * a.n_head + w.head[t]) * p.splits + split;
      });
    if (!shared) return;
    part |= 1;  // a workgroup's later items are its last, if they are cut
  }
}

// Many rows: each of the NW waves takes 16 QT rows of its own, and all read the
// same tiles of TP tokens from LDS, two buffers of them: a tile's rows are
// requested while the one before is worked on, and stored behind it, with one
// barrier a tile.  A row's 16-byte parts change places with the row, so that the
// 16 lanes that read one part of 16 rows take all 64 banks.
//
// Bound by the matrix and vector units together: a 16-bit score takes head_dim / 256
// cycles of a SIMD's matrix core over both products and about 8 vector instructions
// (maximum, exponential, sum, packing) of a sixteenth of a cycle, which only another
// wave's products hide.  16 requests of 4096 to 16384, 192 to 384 rows, 4 key heads of 128,
// fp16 (95 GFLOP): 258 us and 27 of joining, 340 TFLOP/s of the 1213 that a large
// product reaches; of 16384, 512 rows, 8 key heads, bf16 830 and fp16 800.  One request of 262144, 96 rows,
// 2 key heads of 64, bf16 (134 MB): 41 and 10.  16 rows of a wave, 32 requests of 8192
// to 32768, one row a head, 8 key heads of 128, bf16 (2.63 GB): 465 and 8, 5.6 TB/s.
// Codes are widened once, on their way into LDS, so that the products are the same: the
// drafts above over them 220 to 244 us and 26 of joining.
template <int TYPE, int DP, int QT, int NW, bool PAD, bool C8>
__global__ __launch_bounds__(64 * NW, DP * (TYPE == MCA_TYPE_F32 ? 2 : 1) > 256 ? 1 : 2) void k_lm_attn_wide(AttnDev) {
  constexpr int EL = TYPE == MCA_TYPE_F32 ? 4 : 2;
  constexpr int RB = DP * EL, NCH = RB / 16;   // bytes and parts of a row
  constexpr int NH = RB <= 256 ? 2 : 1, TP = 32 * NH;  // tokens of a tile
  typedef Rows<TYPE, DP, QT, NH, PAD> R;
  constexpr int VD = R::VD, CD = R::CD, NC = R::NC;
  constexpr int THREADS = 64 * NW;
  constexpr int PER = (TP * NCH + THREADS - 1) / THREADS;  // parts of K and of V that a thread stages
  constexpr bool EVEN = TP * NCH % THREADS == 0;
  static_assert(EVEN || PER == 1, "whole rounds");
  const AttnDev& p = again();
  const mca_tree_attention_args& a = p.a;
  __shared__ int s_par[2][MCA_MAX_NODES];
  __shared__ uint32_t s_mask[2][MCA_MAX_NODES][kMaskWords];
  __shared__ __attribute__((aligned(1024))) char s_kv[2][2][TP * RB];
  __shared__ int s_wave[NW];
  // where the workgroup stands, in LDS so that it takes no registers beside a tile's:
  // its next and last unit, its request and the units before that, its next place
  __shared__ int s_unit, s_end, s_begin[2], s_part;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  int rt = 0, h = 0, r = 0, part = 0;
  if (p.sharers == 0) {
    if (!place(p, &rt, &h, &r, &part)) return;
  } else {
    int unit, end;
    if (!share_begin<TP, NW>(p, s_wave, s_begin, &unit, &end, &part)) return;
    if (tid == 0) {
      s_unit = unit;
      s_end = end;
      s_part = part;
    }
    __syncthreads();
  }
  auto place_of = [](int row, int part) {
    return row * RB + ((part ^ ((RB < 256 ? row * RB / 256 : row) & (NCH < 16 ? NCH - 1 : 15))) << 4);
  };
  constexpr auto vkey = [](int j) { return RB >= 256 ? j : (RB == 128 ? j >> 1 : 0); };
  const int col = lane & (TP - 1);
  while (true) {
    const AttnDev& p = again();
    const mca_tree_attention_args& a = p.a;
    int first, n, tile0 = 0, tile1 = 0;
    if (p.sharers > 0) {
      int before = __builtin_amdgcn_readfirstlane(s_begin[1]);
      const int unit = __builtin_amdgcn_readfirstlane(s_unit), end = __builtin_amdgcn_readfirstlane(s_end);
      part = __builtin_amdgcn_readfirstlane(s_part);
      r = __builtin_amdgcn_readfirstlane(s_begin[0]);
      if (unit >= end) return;
      for (int units = Share::units(p, r, TP); unit >= before + units; units = Share::units(p, r, TP)) {
        before += units;
        ++r;
      }
      rows_of(a, r, &first, &n);
      const Share sh(p, cached_of(a, r), n, TP);
      const int in = unit - before, item = in / sh.tiles;
      tile0 = in - item * sh.tiles;
      tile1 = min(sh.tiles, tile0 + (end - unit));
      h = item / sh.row_tiles;
      rt = item - h * sh.row_tiles;
      __syncthreads();
      if (tid == 0) {
        s_unit = unit + (tile1 - tile0);
        s_begin[0] = r;
        s_begin[1] = before;
        s_part = part | 1;  // a workgroup's later items are its last, if they are cut
      }
    } else if (!rows_of(a, r, &first, &n)) {
      return;
    }
    const int len = cached_of(a, r);
    const Share sh(p, len, n, TP);
    if (p.sharers == 0) {
      if (rt >= sh.row_tiles) return;
      tile1 = sh.tiles;
    }
    const int row0 = rt * sh.rows, row_end = min(n * p.group, row0 + sh.rows), mine = row0 + wave * 16 * QT;
    const bool busy = mine < row_end;
    R w;
    w.begin(a, h, p.group, busy ? mine : row0, row_end, first, n);
    const int q = w.q, li = w.li;
    const int cached = (len + TP - 1) / TP;
    int from = 0;
    if (tile1 > cached) from = ancestors(a.parents + first, n, s_par, s_mask);
    const int32_t* tab = a.table + (int64_t)r * a.table_stride;
    const char* nk = (const char*)a.k + ((int64_t)first * a.k_row + (int64_t)h * a.k_head) * EL;
    const char* nv = (const char*)a.v + ((int64_t)first * a.v_row + (int64_t)h * a.v_head) * EL;
    // K and V of a tile are staged apart: V one tile behind K, as they are used
    u32x4 sk[PER], sv[PER];
    auto fetch = [&](const char* base, uint32_t stride, int row, u32x4 (&to)[PER]) {
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int e = tid + THREADS * u, c = e % NCH;
        const uint64_t rw = (uint32_t)__shfl(max(row, 0), (e / NCH) % TP, 64);
        const bool ok = (!PAD || c * 16 < w.dbytes) && (EVEN || e < TP * NCH);
        to[u] = ok ? gload((const u32x4*)(base + rw * stride + c * 16)) : u32x4{0, 0, 0, 0};
      }
    };
    auto store = [&](char* buf, const u32x4 (&from_)[PER]) {
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int e = tid + THREADS * u;
        if (!EVEN && e >= TP * NCH) break;
        *(u32x4*)&buf[place_of(e / NCH, e % NCH)] = from_[u];
      }
    };
    // the same of rows in 8 bits, which are widened on their way into LDS, times the
    // scale whose byte lane (row) of the wave has
    constexpr int CB = 16 / EL, CW = CB / 4;  // codes of a part, their words
    uint32_t ck[C8 ? PER : 1][CW], cv[C8 ? PER : 1][CW];
    auto fetch8 = [&](const char* base, int row, uint32_t (&to)[C8 ? PER : 1][CW]) {
      if constexpr (C8) {
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const int e = tid + THREADS * u, c = e % NCH;
          const uint64_t rw = (uint32_t)__shfl(max(row, 0), (e / NCH) % TP, 64);
          const bool ok = (!PAD || c * CB < a.head_dim) && (EVEN || e < TP * NCH);
          if (ok) {
            load_codes<CB>(base + rw * (uint32_t)a.head_dim + c * CB, to[u]);
          } else {
#pragma unroll
            for (int d = 0; d < CW; ++d) to[u][d] = 0;
          }
        }
      }
    };
    auto store8 = [&](char* buf, const uint32_t (&from_)[C8 ? PER : 1][CW], int scale) {
      if constexpr (C8) {
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const int e = tid + THREADS * u;
          const float f = scale_of((uint32_t)__shfl(scale, (e / NCH) % TP, 64));
          if (!EVEN && e >= TP * NCH) break;
          *(u32x4*)&buf[place_of(e / NCH, e % NCH)] = wide_part<TYPE>(from_[u], f);
        }
      }
    };
    // V of codes in the order of its product's operand, of head_dim 128 in 16 bits: a part
    // is a dimension's 8 tokens 4 q .. 4 q + 3 and 16 + those of half a tile, dimension 8 x + y
    // in place 16 y + x, so that the 16 lanes of one read have neighbours.  A thread takes
    // PER neighbouring tokens' 8 dimensions; tokens that are not there become zeros.  That
    // saves the 64 permutations of a tile's values in each wave for 16 of each thread (16 requests of up
    // to 16384, bf16, 1024 rows a key head 575 and 622 us, fp16, 64 rows 90 and 92), but not where
    // four waves of 32 rows fill their registers: the reads then wait for each product, while
    // permutations pass behind products (192 to 384 rows 283 and 269).
    constexpr bool OPERAND = C8 && TYPE != MCA_TYPE_F32 && DP == 128 && (QT == 1 || NW == 8);
    uint64_t v_there = 0;  // which tokens of the values on their way are there
    // (a wave's threads store whole parts, so that they take all banks)
    const int vc = tid % NCH, vx = tid / NCH / (PER == 2 ? 2 : 1);
    const int vt = 4 * ((vx >> 3) * 8 + (vx & 1) * 4 + (vx >> 1 & 3)) + (PER == 2 ? tid / NCH % 2 * 2 : 0);
    auto fetch_v8 = [&](const char* base, int row) {
      if constexpr (OPERAND) {
        v_there = __ballot(row >= 0);
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const uint64_t rw = (uint32_t)__shfl(max(row, 0), vt + u, 64);
          if (!PAD || vc * CB < a.head_dim) {
            load_codes<CB>(base + rw * (uint32_t)a.head_dim + vc * CB, cv[u]);
          } else {
#pragma unroll
            for (int d = 0; d < CW; ++d) cv[u][d] = 0;
          }
        }
      } else {
        fetch8(base, row, cv);
      }
    };
    auto store_v8 = [&](char* buf, int scale) {
      if constexpr (OPERAND) {
        static_assert(PER == 2 || PER == 4, "pairs of tokens");
        uint32_t w[PER][4];
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const u32x4 x = wide_part<TYPE>(cv[u], scale_of((uint32_t)__shfl(scale, vt + u, 64)));
#pragma unroll
          for (int d = 0; d < 4; ++d) w[u][d] = x[d];
        }
        if (v_there != ~0ull) {
#pragma unroll
          for (int u = 0; u < PER; ++u)
#pragma unroll
            for (int d = 0; d < 4; ++d) w[u][d] = (v_there >> (vt + u)) & 1 ? w[u][d] : 0u;
        }
        const int g = vt / 4, q_ = g & 3, at = (((g >> 3) * 4 + q_) * DP + vc) * 16 + (g >> 2 & 1) * 8 + (vt & 2) * 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t y[PER / 2];
#pragma unroll
          for (int u = 0; u < PER / 2; ++u)
            y[u] = __builtin_amdgcn_perm(w[2 * u + 1][e >> 1], w[2 * u][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
          if constexpr (PER == 4)
            *(u32x2*)&buf[at + e * 256] = u32x2{y[0], y[1]};
          else
            *(uint32_t*)&buf[at + e * 256] = y[0];
        }
      } else {
        store8(buf, cv, scale);
      }
    };
    // what a lane reads of the first 16 rows: part i of row li is at k0 ^ 64 i, its
    // words of row 4 q + j at (v0 ^ 16 vkey(j)) + j RB; 16 rows on, the places are the same
    const int k0 = place_of(li, q), v0 = place_of(4 * q, li * CD / 4) + (li * CD * 4 & 15);
    constexpr uint64_t kAll = NH == 2 ? ~0ull : 0xffffffffull;
    auto scores = [&](const char* K) {
      // nothing moves over the marks: what is read ahead has to fit the registers
#pragma unroll
      for (int x = 0; x < 2 * NH; ++x) {
        w.score(x, [&](int k) { return *(const u32x4*)&K[(k0 ^ (64 * k)) + 16 * x * RB]; });
        if (x & 1) __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto values = [&](const char* V, int half, uint32_t (&vf)[8][VD]) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const char* vp = &V[(v0 ^ (16 * vkey(j & 3))) + (32 * half + 16 * (j >> 2) + (j & 3)) * RB + c * 256];
          if constexpr (CD == 4) {
            const u32x4 y = *(const u32x4*)vp;
#pragma unroll
            for (int d = 0; d < 4; ++d) vf[j][c * 4 + d] = y[d];
          } else if constexpr (CD == 2) {
            const u32x2 y = *(const u32x2*)vp;
            vf[j][0] = y[0];
            vf[j][1] = y[1];
          } else {
            vf[j][0] = *(const uint32_t*)vp;
          }
        }
    };
    // The cached tiles pass in two phases: first the products of the tile before and
    // the scores of this one (matrix cores), then its weights (vector units) and the
    // staging.  With 8 waves a SIMD has two, and the second four waves run one phase
    // behind, so that each unit has work from one of them while the other uses the
    // other unit.  A phase ends at a barrier; with the lag, tile i's keys (and tile
    // i - 1's values) are read in phases 2 i and 2 i + 1 and stored in 2 i - 2 and
    // 2 i - 1, when nothing reads that buffer.  Tiles behind the last are staged like
    // others (of whatever tokens, or row 0), so that the loop has no branches around
    // loads in flight; nothing uses them.
    constexpr bool LAG = NW == 8;
    const int last = min(tile1, cached);  // behind the last cached tile
    if (tile0 < last) {
      const bool late = LAG && wave >= NW / 2;
      auto block_at = [&](int i) -> int { return cache_block(a, tab, i * TP + col, len); };
      auto row_at = [&](int i, int blk) -> int { return cache_row(a, blk, h, i * TP + col, len); };
      const int blk0 = block_at(tile0), blk1 = block_at(tile0 + 1);
      int row_v = row_at(tile0, blk0), row_k = row_at(tile0 + 1, blk1);
      int blk = block_at(tile0 + 2);
      // the bytes of scales of a lane's token: of the keys that are on their way, of the
      // values of the same tile, and of the values that are on their way
      int k_of_k = 0, v_of_k = 0, v_of_v = 0;
      auto scales_of = [&](int b, int row, int* ks, int* vs) {
        const int of = row >= 0 ? b * a.n_kv_head + h : 0;
        *ks = gload(p.k_scale + of);
        *vs = gload(p.v_scale + of);
      };
      // which tokens of a tile are there: of the one whose products are next, the one
      // whose scores are, and those behind it
      uint64_t t_prod = 0, t_now = __ballot(row_v >= 0), t_1 = __ballot(row_k >= 0), t_2 = 0, t_3 = 0;
      const char *kc = (const char*)a.k_cache, *v_cache = (const char*)a.v_cache;
      // stores tile i's keys and tile i - 1's values and requests the next ones
      auto stage = [&](int i) {
        if constexpr (C8) {
          store8(s_kv[i & 1][0], ck, k_of_k);
          store_v8(s_kv[(i - 1) & 1][1], v_of_v);
        } else {
          store(s_kv[i & 1][0], sk);
          store(s_kv[(i - 1) & 1][1], sv);
        }
        row_v = row_k;
        row_k = row_at(i + 1, blk);
        t_2 = __ballot(row_k >= 0);
        if constexpr (C8) {
          v_of_v = v_of_k;
          scales_of(blk, row_k, &k_of_k, &v_of_k);
          fetch8(kc, row_k, ck);
          fetch_v8(v_cache, row_v);
        } else {
          fetch(kc, w.dbytes, row_k, sk);
          fetch(v_cache, w.dbytes, row_v, sv);
        }
        blk = block_at(i + 2);
      };
      auto products = [&](int i) {
        const char* V = s_kv[i & 1][1];
#pragma unroll
        for (int half = 0; half < NH; ++half) {
          if constexpr (OPERAND) {
            w.add_operands(half, [&](int e) { return *(const u32x4*)&V[((half * 4 + q) * DP + e * 16 + li) * 16]; });
            __builtin_amdgcn_sched_barrier(0);
            continue;
          }
          uint32_t vf[8][VD];
          values(V, half, vf);
          if ((t_prod & kAll) != kAll) w.clear(vf, (uint32_t)(t_prod >> (32 * half)));
          w.add(half, vf);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if constexpr (C8) {
        scales_of(blk0, row_v, &k_of_k, &v_of_v);
        fetch8(kc, row_v, ck);
        store8(s_kv[tile0 & 1][0], ck, k_of_k);
        scales_of(blk1, row_k, &k_of_k, &v_of_k);
        fetch8(kc, row_k, ck);
        fetch_v8(v_cache, row_v);
      } else {
        fetch(kc, w.dbytes, row_v, sk);
        store(s_kv[tile0 & 1][0], sk);
        fetch(kc, w.dbytes, row_k, sk);
        fetch(v_cache, w.dbytes, row_v, sv);
      }
      __syncthreads();
      if (late) {
        stage(tile0 + 1);
        t_3 = t_2;
        __syncthreads();
      }
      for (int i = tile0; i < last; ++i) {
        if (busy) {
          if (i > tile0) products(i - 1);
          scores(s_kv[i & 1][0]);
        }
        if (LAG) __syncthreads();
        if (busy) {
          uint32_t see[QT][NH];
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int half = 0; half < NH; ++half) see[t][half] = (uint32_t)(t_now >> (32 * half));
          w.weigh((t_now & kAll) == kAll, see);
        }
        stage(i + (late ? 2 : 1));
        t_prod = t_now;
        t_now = t_1;
        t_1 = late ? t_3 : t_2;
        t_3 = t_2;
        __syncthreads();
      }
      if (busy) products(last - 1);
      if (LAG && !late) __syncthreads();
      __syncthreads();
    }
    // the drafted tiles, one after the other
    for (int i = max(tile0, cached); i < tile1; ++i) {
      const int n0 = (i - cached) * TP, nd = n0 + col;
      const uint64_t there = __ballot(nd < n);
      fetch(nk, (uint32_t)(a.k_row * EL), nd < n ? nd : 0, sk);
      fetch(nv, (uint32_t)(a.v_row * EL), nd < n ? nd : 0, sv);
      store(s_kv[0][0], sk);
      store(s_kv[0][1], sv);
      __syncthreads();
      if (busy) {
        uint32_t see[QT][NH];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int half = 0; half < NH; ++half)
            see[t][half] = (uint32_t)(there >> (32 * half)) &
                           s_mask[from][min(w.node[t], n - 1)][min(n0 / 32 + half, kMaskWords - 1)];
        scores(s_kv[0][0]);
        w.weigh(false, see);
#pragma unroll
        for (int half = 0; half < NH; ++half) {
          const uint32_t valid = (uint32_t)(there >> (32 * half));
          uint32_t vf[8][VD];
          values(s_kv[0][1], half, vf);
          const uint32_t odd = w.odd_of(vf) & valid;
          w.clear(vf, valid & ~odd);
          w.add(half, vf);
          w.add_odd(half, odd, see, [&](int at) { return nv + (int64_t)(n0 + 32 * half + at) * a.v_row * EL; });
        }
      }
      __syncthreads();
    }
    if (busy) {
      w.sum_lanes();
      const bool whole = tile0 == 0 && tile1 == sh.tiles;
      const AttnDev& p = again();
      w.write(p, whole, [&](int t) { return (int64_t)part * p.rows + wave * 16 * QT + 16 * t + li; });
    }
    if (p.sharers == 0) return;
    __syncthreads();  // the buffers and masks are free
  }
}

// The chunks of a row and head joined: a wave each, weights 2^(l_s - max l).
template <int TYPE>
__global__ __launch_bounds__(256) void k_lm_attn_join(AttnDev p) {
  const mca_tree_attention_args& a = p.a;
  const int r = blockIdx.y, lane = threadIdx.x & 63;
  int first, n;
  if (!rows_of(a, r, &first, &n)) return;
  const int parts = chunks_of(cached_of(a, r), p.chunk);
  const int item = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (parts == 1 || item >= n * a.n_head) return;
  const int64_t at = ((int64_t)first * a.n_head + item) * p.splits;
  const float* pl = p.part_l + at;
  const float* po = p.part_o + at * a.head_dim;
  float top = -__builtin_huge_valf();
  for (int s = lane; s < parts; s += 64) top = fmaxf(top, pl[s]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  float sum = 0.f;
  for (int s = lane; s < parts; s += 64) sum += __builtin_amdgcn_exp2f(pl[s] - top);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
  const int node = item / a.n_head, head = item - node * a.n_head;
  const float inv = 1.0f / sum;
  const int64_t row = (int64_t)first + node;
  if (a.lse != nullptr && lane == 0) a.lse[row * a.n_head + head] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
  for (int d = lane; d < a.head_dim; d += 64) {
    float acc = 0.f;
#pragma unroll 8
    for (int s = 0; s < parts; ++s) acc = fmaf(__builtin_amdgcn_exp2f(pl[s] - top), gload(po + (int64_t)s * a.head_dim + d), acc);
    const int64_t to = row * a.out_row + (int64_t)head * a.out_head + d;
    if constexpr (TYPE == MCA_TYPE_F32)
      ((float*)a.out)[to] = acc * inv;
    else
      ((uint16_t*)a.out)[to] = (uint16_t)pack2<TYPE>(acc * inv, 0.f);
  }
}

// The parts of shared work joined: a workgroup takes 4 `fours` rows of one tile of
// rows, which are cut in the same places, 4 at a time: their weights are made in
// LDS, then its NW waves take parts in turn and are added there.  head_dim is at
// most 64 NI.
constexpr int kMaxSharers = 512;  // workgroups: two a compute unit
template <int TYPE, int NI, int NW>
__global__ __launch_bounds__(64 * NW) void k_lm_attn_join_shared(AttnDev p, int TP, int fours) {
  const mca_tree_attention_args& a = p.a;
  __shared__ float s_w[4][kMaxSharers];
  __shared__ float s_acc[NW][4 * 64 * NI];
  const int groups = p.rows / (4 * fours), tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int tile = blockIdx.x / groups, rt = tile % p.row_tiles, rh = tile / p.row_tiles;
  const int h = rh % a.n_kv_head, r = rh / a.n_kv_head;
  int first, n;
  if (!rows_of(a, r, &first, &n)) return;
  const Share sh(p, cached_of(a, r), n, TP);
  const int rows = min(sh.rows, n * p.group - rt * sh.rows);  // of the tile; none behind the last
  int row0 = (blockIdx.x - tile * groups) * 4 * fours;
  if (rt >= sh.row_tiles || row0 >= rows) return;
  const int per = Share::per(p, p.first_unit[a.n_req]);
  const int u0 = p.first_unit[r] + (h * sh.row_tiles + rt) * sh.tiles, g0 = u0 / per;
  const int parts = (u0 + sh.tiles - 1) / per - g0 + 1;
  if (parts == 1) return;
  // places of part s: a workgroup's first item, but for the first part its last item, unless that is its first
  const int late = u0 != g0 * per;
  auto at = [&](int s) { return (int64_t)(2 * (g0 + s) + (s == 0 ? late : 0)) * p.rows + row0; };
  const int D = a.head_dim, all = 4 * D;  // a multiple of 16
  for (int four = 0; four < fours && row0 < rows; ++four, row0 += 4) {
    if (wave < 4) {
      const bool here = row0 + wave < rows;
      float top = -__builtin_huge_valf(), sum = 0.f;
      for (int s = lane; s < parts; s += 64) {
        const float l = here ? p.part_l[at(s) + wave] : 0.f;
        s_w[wave][s] = l;
        top = fmaxf(top, l);
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
      for (int s = lane; s < parts; s += 64) {
        const float w = __builtin_amdgcn_exp2f(s_w[wave][s] - top);
        s_w[wave][s] = w;
        sum += w;
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
      const float inv = 1.0f / sum;
      for (int s = lane; s < parts; s += 64) s_w[wave][s] *= inv;
      const int row = rt * sh.rows + row0 + wave, node = row / p.group;
      if (a.lse != nullptr && lane == 0 && here)
        a.lse[(int64_t)(first + node) * a.n_head + h * p.group + (row - node * p.group)] =
            (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    __syncthreads();
    // a lane's values: 4 (lane + 64 i) on of the four rows one after the other.  It
    // loads without asking whether there are any (the parts have room for whole tiles
    // of rows), so that the loads of several parts are under way together.
    f32x4 acc[NI];
    int at_e[NI], of_e[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      at_e[i] = min(4 * (lane + 64 * i), all - 4);
      of_e[i] = at_e[i] / D;
    }
#pragma unroll 8
    for (int s = wave; s < parts; s += NW) {
      const float* po = p.part_o + at(s) * D;
#pragma unroll
      for (int i = 0; i < NI; ++i) acc[i] += s_w[of_e[i]][s] * gload((const f32x4*)(po + at_e[i]));
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (4 * (lane + 64 * i) < all) *(f32x4*)&s_acc[wave][at_e[i]] = acc[i];
    __syncthreads();
    for (int e = tid; e < all; e += 64 * NW) {
      const int of = e / D, row = rt * sh.rows + row0 + of, node = row / p.group;
      if (row0 + of >= rows) break;
      float x = s_acc[0][e];
#pragma unroll
      for (int u = 1; u < NW; ++u) x += s_acc[u][e];
      const int64_t to = (int64_t)(first + node) * a.out_row + (int64_t)(h * p.group + (row - node * p.group)) * a.out_head + (e - of * D);
      if constexpr (TYPE == MCA_TYPE_F32)
        ((float*)a.out)[to] = x;
      else
        ((uint16_t*)a.out)[to] = (uint16_t)pack2<TYPE>(x, 0.f);
    }
    __syncthreads();
  }
}

namespace {

constexpr int kCUs = 256;

// Rows that share a key head's cached tokens.
int shared_rows(const mca_tree_attention_args& a) { return a.max_nodes * (a.n_head / a.n_kv_head); }
// Whether 16 rows of a wave, not 32, are all that its registers hold.
bool big_rows(const mca_tree_attention_args& a) { return a.head_dim > (a.dtype == MCA_TYPE_F32 ? 64 : 128); }
// The wide kernel reads a tile once for all rows; the narrow one, which reads it for
// 16, splits the tokens finer and starts and joins faster.  So wide is what reads
// enough, earlier if the (request, key head) pairs alone fill the chip.  (4 key heads,
// head_dim 128, bf16, wide and narrow, us; in brackets thousands of cached tokens
// times key heads times 16 rows.  One request of 500 tokens, 128 rows 28 and 15 (17);
// 16 of 1024, 128 rows 44 and 30 (541); one of 60000, 24 rows 48 and 40 (480), 48 rows
// 51 and 55 (720); 16 of 8192, 64 rows 60 and 87 (2100).  Pairs that fill the chip: 64
// of 600, 24 rows 26 and 23 (309), 48 rows 27 and 36 (470).)
//
// One group of 16 rows is wide only over long contexts in plenty, where its shares end
// together (8 key heads, 4 rows: 32 of 8192 to 32768 457 and 483, 8 of 100000 483 and
// 504, but 128 of 8000 593 and 576).  Narrow fp32 rows are more work for the matrix
// units than for memory, and a wide workgroup's waves without rows do none of it: 32
// rows stay narrow (head_dim 64, 200 requests of 2000: 257 and 185; 64 rows 278 and 325).
//
// Where the rule takes the slower one (the one taken, and the other): it does not look
// at head_dim, and above 128 a narrow workgroup's registers leave a CU one wave a SIMD
// (256, 64 requests of 300, 24 rows 37 and 27, fp32 162 and 71, 48 rows 50 and 30; 8 of
// 100000, 4 key heads, 4 rows 557 and 484, at 128 270 and 245); and many fp32 rows over
// short contexts are too little for the wide kernel (16 of 1024, 256 rows, head_dim 64 91
// and 65, 32 52 and 35; of 2048, 64 100 and 116).
template <bool C8>
bool is_wide(const mca_tree_attention_args& a) {
  const int rows = shared_rows(a);
  const int64_t pairs = (int64_t)a.n_req * a.n_kv_head, reads = pairs * ((int64_t)a.max_len + a.max_nodes);
  if (a.dtype == MCA_TYPE_F32 && !big_rows(a) && rows <= 32) return false;
  if (C8 && rows <= 16) return false;
  if (rows <= 16) return a.max_len >= (1 << 14) && reads >= (1 << 22);
  return reads * ((rows + 15) / 16) > (pairs >= kCUs ? 3 << 17 : 5 << 17);
}
// 16-row groups of a wave of the wide kernel: one while that is enough for 4 waves
// (64 rows, bf16, head_dim 128: 65 us against 78 of two; fp32, 64: 102 against 160)
int row_group(const mca_tree_attention_args& a) { return big_rows(a) || shared_rows(a) <= 64 ? 1 : 2; }
// Waves of the wide kernel.  Eight, which overlap matrix and vector phases and halve
// the reads of a tile, where one row group is all that fits (bf16, head_dim 256, 128
// rows: 232 us against 324 of four; fp32, 128: 503 against 522), and of the others
// where a tile takes long enough and nearly all of a tile's rows are there (bf16,
// head_dim 128, 64 requests of 8192: 256 rows 346 us against 389, 512 623 against 727,
// but 128 279 against 235, 384 567 against 580; fp16, head_dim 64: 256 rows 225
// against 229, 128 184 against 133).  Wider fp32 rows leave no registers for eight.
template <bool C8>
int wide_waves(const mca_tree_attention_args& a) {
  const int rows = shared_rows(a), tiles = (rows + 255) / 256;
  if (big_rows(a)) return rows > 64 && (a.dtype != MCA_TYPE_F32 || a.head_dim <= 128) ? 8 : 4;
  return a.dtype != MCA_TYPE_F32 && a.head_dim > 64 && 8 * rows >= 7 * 256 * tiles ? 8 : 4;
}
// rows of a workgroup, and the tokens of the wide kernel's tiles
template <bool C8>
int tile_rows(const mca_tree_attention_args& a) { return is_wide<C8>(a) ? 16 * row_group(a) * wide_waves<C8>(a) : 16; }
int tile_tokens(const mca_tree_attention_args& a) {
  const int el = a.dtype == MCA_TYPE_F32 ? 4 : 2, d = a.head_dim <= 32 ? 32 : (a.head_dim <= 64 ? 64 : (a.head_dim <= 128 ? 128 : 256));
  return d * el <= 256 ? 64 : 32;
}
template <bool C8>
int row_tiles(const mca_tree_attention_args& a) { return (shared_rows(a) + tile_rows<C8>(a) - 1) / tile_rows<C8>(a); }
template <bool C8>
int64_t wide_items(const mca_tree_attention_args& a) { return (int64_t)row_tiles<C8>(a) * a.n_kv_head * a.n_req; }

template <int TYPE, int DP, bool PAD, bool C8>
void launch_pad(const AttnDev& p, dim3 grid, hipStream_t s) {
  constexpr bool kBig = DP > (TYPE == MCA_TYPE_F32 ? 64 : 128);             // big_rows()
  constexpr bool kEight = TYPE == MCA_TYPE_F32 ? DP == 128 : DP >= 128;     // wide_waves() may be 8
  if (!is_wide<C8>(p.a)) {
    if constexpr (C8 && DP > 64)
      if (p.sharers > 0) {
        hipLaunchKernelGGL((k_lm_attn<TYPE, DP, PAD, C8, true>), grid, dim3(kAttnThreads), 0, s, p);
        return;
      }
    hipLaunchKernelGGL((k_lm_attn<TYPE, DP, PAD, C8>), grid, dim3(kAttnThreads), 0, s, p);
    return;
  }
  if constexpr (kEight)
    if (wide_waves<C8>(p.a) == 8) {
      hipLaunchKernelGGL((k_lm_attn_wide<TYPE, DP, kBig ? 1 : 2, 8, PAD, C8>), grid, dim3(512), 0, s, p);
      return;
    }
  if constexpr (!kBig)
    if (row_group(p.a) == 2) {
      hipLaunchKernelGGL((k_lm_attn_wide<TYPE, DP, 2, 4, PAD, C8>), grid, dim3(256), 0, s, p);
      return;
    }
  hipLaunchKernelGGL((k_lm_attn_wide<TYPE, DP, 1, 4, PAD, C8>), grid, dim3(256), 0, s, p);
}
template <int TYPE, int DP, bool C8>
void launch_dim(const AttnDev& p, dim3 grid, hipStream_t s) {
  if (p.a.head_dim == DP)
    launch_pad<TYPE, DP, false, C8>(p, grid, s);
  else
    launch_pad<TYPE, DP, true, C8>(p, grid, s);
}
// 16 waves of a workgroup where there are few, each with many parts to read, else 4
// (with the attention, 16 and 4 waves: one request of 60000, 64 rows, 4 key heads, bf16,
// head_dim 128, 64 workgroups, 48 and 51 us, head_dim 256 89 and 115; 4 requests of
// 8192, 128 rows, head_dim 128, 512 workgroups, 58 and 54).
template <int TYPE, int NI, bool C8>
void launch_join(const AttnDev& p, dim3 groups, int fours, hipStream_t s) {
  const int tokens = is_wide<C8>(p.a) ? tile_tokens(p.a) : kAttnWaves * kTilePos;
  if (groups.x <= kCUs)
    hipLaunchKernelGGL((k_lm_attn_join_shared<TYPE, NI, 16>), groups, dim3(1024), 0, s, p, tokens, fours);
  else
    hipLaunchKernelGGL((k_lm_attn_join_shared<TYPE, NI, 4>), groups, dim3(256), 0, s, p, tokens, fours);
}
template <int TYPE, bool C8>
void launch_type(const AttnDev& p, dim3 grid, hipStream_t s) {
  const int D = p.a.head_dim;
  if (D <= 32)
    launch_dim<TYPE, 32, C8>(p, grid, s);
  else if (D <= 64)
    launch_dim<TYPE, 64, C8>(p, grid, s);
  else if (D <= 128)
    launch_dim<TYPE, 128, C8>(p, grid, s);
  else
    launch_dim<TYPE, 256, C8>(p, grid, s);
  if (p.splits > 1)
    hipLaunchKernelGGL((k_lm_attn_join<TYPE>), dim3((unsigned)((p.a.max_nodes * p.a.n_head + 3) / 4), (unsigned)p.a.n_req),
                       dim3(256), 0, s, p);
  else if (p.sharers > 0) {
    // 16 rows a workgroup once that fills the chip (what they read first they read
    // once), else 4 (64 requests of 4096, 128 rows, bf16, head_dim 128: 150 us against
    // 162 of attention and joining; one of 60000: 81 against 66)
    const int fours = wide_items<C8>(p.a) * p.rows / 16 >= 4 * kCUs ? 4 : 1;
    const dim3 groups((unsigned)(wide_items<C8>(p.a) * (p.rows / (4 * fours))));
    if (D <= 64)
      launch_join<TYPE, 1, C8>(p, groups, fours, s);
    else if (D <= 128)
      launch_join<TYPE, 2, C8>(p, groups, fours, s);
    else
      launch_join<TYPE, 4, C8>(p, groups, fours, s);
  }
}

template <bool C8>
AttnPlan attention_plan(const mca_tree_attention_args& a) {
  AttnPlan p{};
  if (a.n_req == 0) return p;
  const int64_t wgs = (int64_t)row_tiles<C8>(a) * a.n_kv_head * a.n_req;
  if (is_wide<C8>(a)) {
    // Shared, if that saves more than the joining costs.  A workgroup for each tile of
    // rows takes as many rounds of `tiles` as the chip needs for them all; shared, a
    // part of a round counts as such.  An fp32 tile counts twice, as its products do.
    // The joining costs about the time of 12 tiles and of the parts, two a workgroup.
    // (128 rows, 4 key heads, bf16, head_dim 128, shared and not: one request of 512
    // tokens 33 and 28 us, of 1024 33 and 41; 16 of 1024 52 and 43, of 2048 58 and 71;
    // 64 of 4096 147 and 133, of 16384 380 and 464.)
    const bool one = wide_waves<C8>(a) == 8 || (a.dtype == MCA_TYPE_F32 && a.head_dim > 128);  // LDS or registers of a CU
    const int tokens = tile_tokens(a), resident = kCUs * (one ? 1 : 2);
    const int64_t tiles = (a.max_len + tokens - 1) / tokens;
    p.chunk = a.max_len;
    p.splits = 1;
    const int64_t idle = (wgs + resident - 1) / resident * resident - wgs;
    const bool saves = (a.dtype == MCA_TYPE_F32 ? 2 : 1) * tiles * idle / resident > 12 + std::min<int64_t>(wgs, resident) / 8;
    if (saves && wgs * (tiles + MCA_MAX_NODES / 32) < (1 << 30)) {
      p.sharers = (int32_t)std::min<int64_t>(resident, (wgs * (tiles + MCA_MAX_NODES / 32) / kLeastUnits + 8) / 8 * 8);
      p.bytes = ((size_t)a.n_req + 1 + 63) / 64 * 256 + (size_t)2 * p.sharers * tile_rows<C8>(a) * (a.head_dim + 1) * sizeof(float);
    }
    return p;
  }
  if (C8 && row_tiles<C8>(a) == 1 && a.head_dim > 64) {
    // Shared, over long contexts: the chunks of ragged ones leave the chip idle behind the
    // last (chunks and shares, us, one row or four a head, 8 key heads of 128, bf16: 32 of
    // 8192 to 32768 271 and 259, 8 of 100000 218 and 190, one 64 and 53; but 256 of 2000 154
    // and 169, 8 of 8000 32 and 39, and head_dim 64, 32 of 32768 142 and 146).  Wider fp32
    // rows, whose chunks' kernel works in scratch memory, always: 32 of 8192 531 and 364, of
    // 1000 131 and 108.
    const bool big = a.dtype == MCA_TYPE_F32 && a.head_dim > 128;
    const int64_t units = wgs * ((a.max_len + kAttnWaves * kTilePos - 1) / (kAttnWaves * kTilePos) + 1);
    static_assert(2 * kCUs <= kMaxSharers, "shared work's weights in LDS");
    const int resident = kCUs * resident8(a.dtype, a.head_dim, true);
    if ((big || a.max_len >= 1 << 14) && units >= 8 * resident && units < (1 << 30)) {
      p.chunk = a.max_len;
      p.splits = 1;
      p.sharers = resident;
      p.bytes = ((size_t)a.n_req + 1 + 63) / 64 * 256 + (size_t)2 * p.sharers * 16 * (a.head_dim + 1) * sizeof(float);
      return p;
    }
  }
  // Chunks of at least two tiles a wave while there are fewer than two workgroups a
  // CU; behind that of 1536 tokens, up to 16 workgroups a CU, which evens out requests
  // of different lengths.  (Workgroups in all of 512, 1024, 2048 and 4096, bf16,
  // head_dim 128, 8 key heads: one request of 200000 162, 170, 185 and 185 us; 32 of
  // 8192 to 32768 526, 500, 478 and 470.)
  const int64_t step = kAttnWaves * kTilePos;
  const int64_t first = std::min<int64_t>((512 + wgs - 1) / wgs, (a.max_len + 2 * step - 1) / (2 * step));
  const int64_t more = std::min<int64_t>((4096 + wgs - 1) / wgs, (a.max_len + 1535) / 1536);
  const int64_t want = std::clamp<int64_t>(std::max(first, more), 1, 256);
  const int64_t chunk = (a.max_len + want - 1) / want;
  p.chunk = (int32_t)std::max<int64_t>(step, (chunk + step - 1) / step * step);
  p.splits = (int32_t)std::max<int64_t>(1, ((int64_t)a.max_len + p.chunk - 1) / p.chunk);
  p.bytes = p.splits > 1 ? (size_t)a.n_rows * a.n_head * p.splits * (a.head_dim + 1) * sizeof(float) : 0;
  return p;
}

template <bool C8>
hipError_t launch_attention(const mca_tree_attention_args& a, const AttnPlan& plan, const uint8_t* k_scale, const uint8_t* v_scale,
                            hipStream_t s) {
  if (a.n_req == 0 || a.n_rows == 0) return hipSuccess;
  AttnDev p;
  p.a = a;
  p.group = a.n_head / a.n_kv_head;
  p.row_tiles = row_tiles<C8>(a);
  p.chunk = plan.chunk;
  p.splits = plan.splits;
  p.sharers = plan.sharers;
  p.rows = tile_rows<C8>(a);
  p.first_unit = (int32_t*)a.workspace;
  p.part_o = (float*)a.workspace;
  size_t parts = (size_t)a.n_rows * a.n_head * plan.splits;
  if (plan.sharers > 0) {
    p.part_o = (float*)((char*)a.workspace + ((size_t)a.n_req + 1 + 63) / 64 * 256);
    parts = (size_t)2 * plan.sharers * p.rows;
  }
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.part_l = p.part_o + parts * a.head_dim;
  const dim3 grid((unsigned)(plan.sharers > 0 ? plan.sharers
                                              : ((int64_t)a.n_kv_head * a.n_req * plan.splits + 7) / 8 * 8 * p.row_tiles));
  switch (a.dtype) {
    case MCA_TYPE_F32: launch_type<MCA_TYPE_F32, C8>(p, grid, s); break;
    case MCA_TYPE_BF16: launch_type<MCA_TYPE_BF16, C8>(p, grid, s); break;
    default: launch_type<MCA_TYPE_F16, C8>(p, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace

}  // namespace mca
