// HIP kernels (gfx950) of the paged cache of 8-bit values: rows quantised into
// their places (mca_cache8_append) and read back (mca_cache8_read).
//
// A code is an e4m3 value, and a block's scale 2^e for one key head, so that a code
// is one conversion from its value and back, a larger scale changes kept codes only
// where they become subnormal, and neither the order nor the pieces in which a
// block's tokens arrive change anything else.
//
// Both are bound by memory, and of few tokens by a chain of loads (offsets, the block's
// number, its scale, the rows): bf16, 8 heads of 128, 60500 rows of 32 requests'
// prompts are 80 us (248 MB read, 124 written, 4.6 TB/s), the values of 51200 tokens 72 us
// (105 MB read, 210 written, 4.4 TB/s); 64 requests of 8 rows, 4 heads of 32 fp32, 5.0 and 4.7 us.
#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "lm_device.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Pages and heads of a workgroup whose waves take one each; W > 1 waves that take one
// together are a workgroup.
constexpr int kC8Pages = 4;
template <int W>
constexpr int kC8Threads = 64 * (W == 1 ? kC8Pages : W);
constexpr int kC8Loads = 4;  // 16-byte loads of K and of V that a lane has in flight

// Exponents of scales: the least (below it fp16 values would be no codes' values any
// more; the others' stay normal numbers), and the one from which 256 times the scale
// is past the type's largest value.
template <int TYPE>
struct Scale {
  static constexpr int kLeast = TYPE == MCA_TYPE_F16 ? -15 : -100, kFull = TYPE == MCA_TYPE_F16 ? 8 : 120;
};

// The largest code's value that, times 2^e, the type holds: the one below 2^(kFull + 8 - e).
template <int TYPE>
__device__ __forceinline__ float most_of(int e) {
  const int t = Scale<TYPE>::kFull + 8 - e;
  return t > 8 ? 448.f : fmaxf(__builtin_ldexpf(1.f, t) - __builtin_ldexpf(1.f, max(t - 4, -9)), 0.f);
}

// The pages of all requests laid end to end with room to spare: request r's begin at
// offsets[r] / B + 2 r, which leaves each at least its (tokens / B) + 2, and `items` of
// the whole call can be had from what the host knows.  A wave looks 64 requests up
// at a time.
__device__ __forceinline__ int64_t first_item(const int32_t* offsets, int r, int B) {
  return (int64_t)max(offsets[r], 0) / (unsigned)B + 2 * (int64_t)r;
}
__device__ __forceinline__ int request_of(const int32_t* offsets, int n_req, int B, int64_t item) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_req;
  while (true) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int c = __popcll(__ballot(at < hi && first_item(offsets, at, B) <= item));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    hi = min(hi, lo + step);
    if (step == 1) return lo;
  }
}

// A request's page: its first row among the call's, positions and block.
struct Page {
  int64_t row0;  // of position `from`
  int from, to;  // positions of the call's tokens in the page
  int start, block;
};
template <class Args>
__device__ __forceinline__ bool page_of(const Args& a, const int32_t* before, int64_t item, Page* p) {
  const int r = request_of(a.offsets, a.n_req, a.block_size, item);
  if (r < 0) return false;
  const int64_t o0 = a.offsets[r], o1 = a.offsets[r + 1], len = before[r];
  if (o0 < 0 || o1 <= o0 || o1 > a.n || len < 0) return false;
  const int64_t page = len / a.block_size + (item - first_item(a.offsets, r, a.block_size));
  const int64_t lo = max(len, page * a.block_size), hi = min(len + (o1 - o0), (page + 1) * a.block_size);
  if (lo >= hi) return false;
  p->row0 = o0 + (lo - len);
  // positions behind max_blocks need not fit 32 bits
  const bool in = page < a.max_blocks;
  p->start = in ? (int)(page * a.block_size) : 0;
  p->from = in ? (int)lo : 0;
  p->to = p->from + (int)(hi - lo);
  p->block = in ? a.table[(int64_t)r * a.table_stride + page] : -1;
  if (p->block >= a.n_blocks) p->block = -1;
  return true;
}

__device__ __forceinline__ bool finite_bits(uint32_t b) { return (b & 0x7f800000u) != 0x7f800000u; }
// four codes, rounded to nearest, of values times 2^-e, none above `most`
__device__ __forceinline__ uint32_t codes_of(const float* f, int e, float most) {
  float y[4];
  uint32_t nan = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool ok = finite_bits(__float_as_uint(f[i]));
    y[i] = fminf(fmaxf(ok ? __builtin_ldexpf(f[i], -e) : 0.f, -most), most);
    nan |= ok ? 0u : 0x7fu << (8 * i);
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return nan == 0 ? (uint32_t)w : ((uint32_t)w & ~(nan * 2 + (nan & 0x01010101u))) | nan;
}
// the same of finite values that are at most 448 times 2^e: `by` is 2^-e
__device__ __forceinline__ uint32_t codes_of(const float* f, float by) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * by, f[1] * by, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * by, f[3] * by, w, true);
  return (uint32_t)w;
}
// Largest magnitudes, as numbers' bits without their signs: of 16-bit types of two halves
// side by side.  Infinities and NaN come out on top.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int TYPE>
__device__ __forceinline__ uint32_t larger(uint32_t top, uint32_t x) {
  if constexpr (TYPE == MCA_TYPE_F32) {
    return max(top, x & 0x7fffffffu);
  } else {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                                  __builtin_bit_cast(u16x2, x & 0x7fff7fffu)));
  }
}
// the magnitude in 32 bits (infinities and NaN stay such)
template <int TYPE>
__device__ __forceinline__ uint32_t magnitude(uint32_t top) {
  if constexpr (TYPE == MCA_TYPE_F32) return top;
  const uint32_t x = max(top & 0xffffu, top >> 16);
  if constexpr (TYPE == MCA_TYPE_BF16) return x << 16;
  return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)x));
}
// four kept codes in a scale 2^down times theirs (down <= 0); NaN stays as it is
__device__ __forceinline__ uint32_t recoded(uint32_t codes, float by) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, by, false);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, by, true);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(b[0], b[1], w, true);
  uint32_t nan = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (((codes >> (8 * i)) & 0x7f) == 0x7f) nan |= 0xffu << (8 * i);
  return ((uint32_t)w & ~nan) | (codes & nan);
}

}  // namespace

// W waves take one page of a request and one key head: largest values of K and V
// first, from all their new rows, then codes.  What fits kC8Loads loads of a lane (64
// rows of 128, 16-bit, of 4 waves) stays in registers between the two, so that each row
// is read once; only pages of more are read again, from the last part to the first, of
// which the caches still hold the end.
template <int TYPE, int W>
__global__ __launch_bounds__(kC8Threads<W>) void k_lm_append8(mca_cache8_append_args a, int64_t units) {
  constexpr int EL = TYPE == MCA_TYPE_F32 ? 4 : 2, VE = 16 / EL, T = 64 * W;
  typedef Scale<TYPE> S;
  __shared__ uint32_t s_top[2][W];
  const int wave = threadIdx.x >> 6, tid = threadIdx.x % T;
  const int64_t unit = W == 1 ? (int64_t)blockIdx.x * kC8Pages + wave : (int64_t)blockIdx.x;
  Page pg{};
  const bool any = unit < units && page_of(a, a.lengths, unit / a.n_kv_head, &pg) && pg.block >= 0;
  if (!any) return;  // the same for all waves of a unit
  const int h = (int)(unit % a.n_kv_head);
  const int per = a.head_dim / VE, tokens = pg.to - pg.from, all = tokens * per;
  const int64_t at = ((int64_t)pg.block * a.n_kv_head + h);
  const int keep = max(0, pg.from - pg.start);
  const uint32_t was_k = a.k_scale[at], was_v = a.v_scale[at];
  u32x4 kx[kC8Loads], vx[kC8Loads];
  const int step_t = T / per, step_part = T - step_t * per;
  auto load = [&](int c) {
    int t = (c + tid) / per, part = c + tid - t * per;
#pragma unroll
    for (int u = 0; u < kC8Loads; ++u) {
      kx[u] = vx[u] = u32x4{0, 0, 0, 0};
      if (t < tokens) {
        const int64_t row = a.rows != nullptr ? (int64_t)a.rows[pg.row0 + t] : pg.row0 + t;
        if (row >= 0 && row < a.n_src) {
          kx[u] = gload((const u32x4*)((const char*)a.k + (row * a.k_row + h * a.k_head) * EL) + part);
          vx[u] = gload((const u32x4*)((const char*)a.v + (row * a.v_row + h * a.v_head) * EL) + part);
        }
      }
      t += step_t;
      part += step_part;
      if (part >= per) {
        part -= per;
        ++t;
      }
    }
  };
  const int last = (all - 1) / (T * kC8Loads) * (T * kC8Loads);
  // the unit's largest of what its lanes found
  auto join = [&](uint32_t& x, uint32_t& y) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      x = max(x, (uint32_t)__shfl_xor(x, d, 64));
      y = max(y, (uint32_t)__shfl_xor(y, d, 64));
    }
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) {
        s_top[0][wave] = x;
        s_top[1][wave] = y;
      }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < W; ++w) {
        x = max(x, s_top[0][w]);
        y = max(y, s_top[1][w]);
      }
    }
  };
  uint32_t top_k = 0, top_v = 0;
  for (int c = 0; c <= last; c += T * kC8Loads) {
    load(c);
#pragma unroll
    for (int u = 0; u < kC8Loads; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top_k = larger<TYPE>(top_k, kx[u][i]);
        top_v = larger<TYPE>(top_v, vx[u][i]);
      }
  }
  top_k = magnitude<TYPE>(top_k);
  top_v = magnitude<TYPE>(top_v);
  join(top_k, top_v);
  const bool finite = finite_bits(top_k) && finite_bits(top_v);
  if (!finite) {  // the same for all waves of a unit: once more, of finite values alone
    top_k = top_v = 0;
    auto look = [&](u32x4 x, uint32_t* top) {
      float f[VE];
      unpack<TYPE>(x, f);
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const uint32_t b = __float_as_uint(f[i]) & 0x7fffffffu;
        *top = max(*top, finite_bits(b) ? b : 0u);
      }
    };
    for (int c = 0; c <= last; c += T * kC8Loads) {
      if (last > 0) load(c);
#pragma unroll
      for (int u = 0; u < kC8Loads; ++u) {
        look(kx[u], &top_k);
        look(vx[u], &top_v);
      }
    }
    if constexpr (W > 1) __syncthreads();  // s_top is free
    join(top_k, top_v);
  }
  // 448 is 1.75 times 2^8
  auto exponent = [&](uint32_t top, uint32_t was, int* before) {
    const int e = max((int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), S::kLeast);
    *before = (int)min(max(was, 1u), 254u) - 127;
    return keep > 0 ? max(e, *before) : e;
  };
  int old_k, old_v;
  const int ek = exponent(top_k, was_k, &old_k), ev = exponent(top_v, was_v, &old_v);
  if (tid == 0) {
    a.k_scale[at] = (uint8_t)(ek + 127);
    a.v_scale[at] = (uint8_t)(ev + 127);
  }
  uint8_t* kc = a.k_cache + at * a.block_size * a.head_dim;
  uint8_t* vc = a.v_cache + at * a.block_size * a.head_dim;
  auto write = [&](auto plain) {
    const float most_k = most_of<TYPE>(ek), most_v = most_of<TYPE>(ev);
    const float by_k = __builtin_ldexpf(1.f, -ek), by_v = __builtin_ldexpf(1.f, -ev);
    for (int c = last; c >= 0; c -= T * kC8Loads) {
      if (c != last) load(c);
#pragma unroll
      for (int u = 0; u < kC8Loads; ++u) {
        const int e = c + tid + T * u;
        if (e >= all) continue;
        const int64_t to = (int64_t)(pg.from - pg.start) * a.head_dim + (int64_t)e * VE;
        auto put = [&](u32x4 x, uint8_t* cache, int ex, float most, float by) {
          float f[VE];
          unpack<TYPE>(x, f);
          uint32_t w[VE / 4];
#pragma unroll
          for (int i = 0; i < VE / 4; ++i) w[i] = plain ? codes_of(f + 4 * i, by) : codes_of(f + 4 * i, ex, most);
          if constexpr (VE == 4)
            gstore((uint32_t*)(cache + to), w[0]);
          else
            gstore((u32x2*)(cache + to), u32x2{w[0], w[1]});
        };
        put(kx[u], kc, ek, most_k, by_k);
        put(vx[u], vc, ev, most_v, by_v);
      }
    }
  };
  if (finite && max(ek, ev) < S::kFull)
    write(std::true_type());
  else
    write(std::false_type());
  if (keep > 0) {
    auto again = [&](uint8_t* cache, int down) {
      if (down >= 0) return;
      const float by = __builtin_ldexpf(1.0f, max(down, -60));  // smaller: all codes 0 as well
      for (int e = tid; e < keep * a.head_dim / 16; e += T) {
        u32x4 x = gload((const u32x4*)cache + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = recoded(x[i], by);
        gstore((u32x4*)cache + e, x);
      }
    };
    again(kc, old_k - ek);
    again(vc, old_v - ev);
  }
}

// W waves take one page of a request and one key head: VE codes of K and of V a lane
// and round, their values to the request's rows.
template <int TYPE, int W>
__global__ __launch_bounds__(kC8Threads<W>) void k_lm_read8(mca_cache8_read_args a, int64_t units) {
  constexpr int EL = TYPE == MCA_TYPE_F32 ? 4 : 2, VE = 16 / EL, CW = VE / 4, T = 64 * W;
  const int wave = threadIdx.x >> 6, tid = threadIdx.x % T;
  const int64_t unit = W == 1 ? (int64_t)blockIdx.x * kC8Pages + wave : (int64_t)blockIdx.x;
  Page pg{};
  if (unit >= units || !page_of(a, a.start, unit / a.n_kv_head, &pg)) return;
  const int h = (int)(unit % a.n_kv_head);
  const int per = a.head_dim / VE, all = (pg.to - pg.from) * per;
  const bool there = pg.block >= 0;
  const int64_t at = (int64_t)max(pg.block, 0) * a.n_kv_head + h;
  const float fk = scale_of(a.k_scale[at]), fv = scale_of(a.v_scale[at]);
  const int64_t base = at * a.block_size * a.head_dim + (int64_t)(pg.from - pg.start) * a.head_dim;
  for (int c = tid; c < all; c += T * kC8Loads) {
    uint32_t kx[kC8Loads][CW], vx[kC8Loads][CW];
#pragma unroll
    for (int u = 0; u < kC8Loads; ++u) {
      const int e = c + T * u;
#pragma unroll
      for (int i = 0; i < CW; ++i) kx[u][i] = vx[u][i] = 0;
      if (there && e < all) {
        load_codes<VE>((const char*)a.k_cache + base + (int64_t)e * VE, kx[u]);
        load_codes<VE>((const char*)a.v_cache + base + (int64_t)e * VE, vx[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kC8Loads; ++u) {
      const int e = c + T * u;
      if (e >= all) continue;
      const int t = e / per, part = e - t * per;
      const int64_t row = pg.row0 + t;
      gstore((u32x4*)((char*)a.k + (row * a.k_row + h * a.k_head) * EL) + part, wide_part<TYPE>(kx[u], fk));
      gstore((u32x4*)((char*)a.v + (row * a.v_row + h * a.v_head) * EL) + part, wide_part<TYPE>(vx[u], fv));
    }
  }
}

namespace {

// Waves of a page and head: one while its loads in flight are all of a page's new rows, else
// four.  (us with one and four, 8 heads, bf16: 32 requests of 8 rows of 128 5.8 and 6.5, of 24 7.8
// and 5.9, of 40 10.2 and 6.1; the 60500 rows above in blocks of 64 101 and 80, of 32 85 and 79, of 16
// 77 and 100, of 256 141 and 107; read back 51200 tokens of blocks of 64 73 and 72, of 32 70 and 71, of
// 16 68 and 84; 120 of 4 heads of 32 fp32 4.7 and 6.3.)  The host knows only how many rows a
// request has on average.  (The same of mixed calls, appended: one prompt of 3000 among 255 single
// tokens, blocks of 16 10.3 and 17.5, of 64 14.2 and 14.9, of 256 43 and 15, where the rule takes the slower;
// among 30 of 8 rows 7.2 and 10.2, 7.7 and 7.6, 13.5 both.  Rows behind the last request count as rows: 64 of 8
// and 60000 such, blocks of 16, 12.8 and 34.8, of 64 12.2 both.)
template <class Args>
int waves_of(const Args& a) {
  const int64_t tokens = std::min<int64_t>(a.block_size, (a.n + a.n_req - 1) / a.n_req);
  return tokens * a.head_dim / (a.dtype == MCA_TYPE_F32 ? 4 : 8) <= 64 * kC8Loads ? 1 : 4;
}
template <int TYPE>
void append(const mca_cache8_append_args& a, int waves, int64_t units, dim3 grid, hipStream_t s) {
  if (waves == 1)
    hipLaunchKernelGGL((k_lm_append8<TYPE, 1>), grid, dim3(kC8Threads<1>), 0, s, a, units);
  else
    hipLaunchKernelGGL((k_lm_append8<TYPE, 4>), grid, dim3(kC8Threads<4>), 0, s, a, units);
}
template <int TYPE>
void read(const mca_cache8_read_args& a, int waves, int64_t units, dim3 grid, hipStream_t s) {
  if (waves == 1)
    hipLaunchKernelGGL((k_lm_read8<TYPE, 1>), grid, dim3(kC8Threads<1>), 0, s, a, units);
  else
    hipLaunchKernelGGL((k_lm_read8<TYPE, 4>), grid, dim3(kC8Threads<4>), 0, s, a, units);
}
template <class Args, class F32, class BF16, class F16>
hipError_t launch(const Args& a, hipStream_t s, F32 f32, BF16 bf16, F16 f16) {
  const int64_t units = (a.n / a.block_size + 2 * (int64_t)a.n_req) * a.n_kv_head;
  const int waves = waves_of(a), each = waves == 1 ? kC8Pages : 1;
  const dim3 grid((unsigned)((units + each - 1) / each));
  switch (a.dtype) {
    case MCA_TYPE_F32: f32(a, waves, units, grid, s); break;
    case MCA_TYPE_BF16: bf16(a, waves, units, grid, s); break;
    default: f16(a, waves, units, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t lm_launch_append8(const mca_cache8_append_args& a, hipStream_t s) {
  return launch(a, s, append<MCA_TYPE_F32>, append<MCA_TYPE_BF16>, append<MCA_TYPE_F16>);
}

hipError_t lm_launch_read8(const mca_cache8_read_args& a, hipStream_t s) {
  return launch(a, s, read<MCA_TYPE_F32>, read<MCA_TYPE_BF16>, read<MCA_TYPE_F16>);
}

}  // namespace mca
