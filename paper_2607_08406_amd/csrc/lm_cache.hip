// HIP kernels (gfx950) of the paged cache of keys and values: block tables and
// slot map from the requests' lengths, and rows into their slots.
#include <algorithm>

#include "device_common.hpp"
#include "lm_kernels.hpp"

namespace mca {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTabThreads = 512;
constexpr int kTabEntries = 4096;  // prefix sums kept in LDS: one for every n_req / 4096 requests
constexpr int kTabPer = kTabEntries / kTabThreads;
constexpr int kTabSlots = 4;       // consecutive slots of a thread
constexpr int kAppendThreads = 256;
constexpr int kAppendUnits = 4;    // units of K and of V that a thread has in flight

// a + b, at most 2^31 - 1 (a, b in [0, 2^31 - 1])
__device__ __forceinline__ int add_sat(int a, int b) {
  const unsigned s = (unsigned)a + (unsigned)b;
  return (int)(s < 0x7fffffffu ? s : 0x7fffffffu);
}

struct Change {
  int add, grow, back, held;  // new tokens, blocks taken, blocks given up, blocks held before
};
__device__ __forceinline__ Change plus(const Change& a, const Change& b) {
  return {add_sat(a.add, b.add), add_sat(a.grow, b.grow), add_sat(a.back, b.back), add_sat(a.held, b.held)};
}

}  // namespace

// Every workgroup sums the lengths of all requests for itself (they are few and
// come from L2), so that one launch does: no sums pass between workgroups, and
// n_free follows from the lengths.  What one writes no other reads: needed
// blocks are popped from below n_free or are given-up ones, whose numbers are
// read from the tables of shrinking requests; tables are written for growing
// ones only; given-up blocks that stay free go to n_free and above.
//
// Sums saturate at 2^31 - 1, above every limit they are compared with
// (max_tokens and n_blocks are at most 2^31 - 2).
//
// Bound by latency: lengths, two barriers of sums, then a search in LDS and a chain of
// two loads for an item.  256 decoding requests: 9.4 us, 4001 of a serving step with
// room for 924 thousand slots 26 us.
__global__ __launch_bounds__(kTabThreads) void k_lm_tables(TablesArgs a) {
  __shared__ int s_add[kTabEntries + 1], s_grow[kTabEntries + 1], s_back[kTabEntries + 1];
  __shared__ Change s_wave[kTabThreads / 64];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int R = a.n_req, B = a.block_size;
  const int per = (R + kTabEntries - 1) / kTabEntries;  // requests of an entry
  const int ne = (R + per - 1) / per;
  const int most = a.max_blocks * B;  // below 2^31 (checked on the host)
  auto change_of = [&](int o, int n, int* bad) -> Change {
    if (o < 0 || o > most || n < 0 || n > most) {
      *bad = 1;
      return {0, 0, 0, 0};
    }
    const int have = (int)(((unsigned)o + B - 1) / (unsigned)B), want = (int)(((unsigned)n + B - 1) / (unsigned)B);
    return {n > o ? n - o : 0, want > have ? want - have : 0, have > want ? have - want : 0, have};
  };
  auto change = [&](int r, int* bad) -> Change { return change_of(a.old_len[r], a.new_len[r], bad); };
  const int pt = (ne + kTabThreads - 1) / kTabThreads;  // entries of a thread
  if (tid == 0) s_bad = 0;
  __syncthreads();
  int bad = 0;
  Change mine{0, 0, 0, 0};
  Change ent[kTabPer];
  if (per == 1) {
    // all of a thread's lengths requested before the first is looked at
    int o[kTabPer], n[kTabPer];
#pragma unroll
    for (int u = 0; u < kTabPer; ++u) {
      const int r = min(tid * pt + (u < pt ? u : 0), R - 1);
      o[u] = gload(a.old_len + r);
      n[u] = gload(a.new_len + r);
    }
#pragma unroll
    for (int u = 0; u < kTabPer; ++u) {
      ent[u] = {0, 0, 0, 0};
      if (u < pt && tid * pt + u < R) ent[u] = change_of(o[u], n[u], &bad);
      mine = plus(mine, ent[u]);
    }
  } else {
#pragma unroll
    for (int u = 0; u < kTabPer; ++u) {
      const int e = tid * pt + u;
      ent[u] = {0, 0, 0, 0};
      for (int r = e * per; u < pt && r < (e + 1) * per && r < R; ++r) ent[u] = plus(ent[u], change(r, &bad));
      mine = plus(mine, ent[u]);
    }
  }
  if (bad) s_bad = 1;
  Change run = mine;  // inclusive over the wave's threads
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Change up = {__shfl_up(run.add, d, 64), __shfl_up(run.grow, d, 64), __shfl_up(run.back, d, 64),
                       __shfl_up(run.held, d, 64)};
    if (lane >= d) run = plus(run, up);
  }
  if (lane == 63) s_wave[wave] = run;
  Change before = {__shfl_up(run.add, 1, 64), __shfl_up(run.grow, 1, 64), __shfl_up(run.back, 1, 64), 0};
  if (lane == 0) before = {0, 0, 0, 0};
  __syncthreads();
  Change total{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < kTabThreads / 64; ++w) {
    if (w == wave) before = plus(before, total);
    total = plus(total, s_wave[w]);
  }
#pragma unroll
  for (int u = 0; u < kTabPer; ++u) {
    const int e = tid * pt + u;
    if (u < pt && e < ne) {
      s_add[e] = before.add;
      s_grow[e] = before.grow;
      s_back[e] = before.back;
    }
    before = plus(before, ent[u]);
  }
  if (tid == 0) {
    s_add[ne] = total.add;
    s_grow[ne] = total.grow;
    s_back[ne] = total.back;
  }
  __syncthreads();
  int code = MCA_TABLES_OK;
  const int n_free = a.n_blocks - total.held;
  if (s_bad || total.held > a.n_blocks) code = MCA_TABLES_LENGTH;
  else if (total.add > a.max_tokens) code = MCA_TABLES_SLOTS;
  else if (total.grow > add_sat(n_free, total.back)) code = MCA_TABLES_EXHAUSTED;
  const int64_t step = (int64_t)gridDim.x * kTabThreads, first = (int64_t)blockIdx.x * kTabThreads + tid;
  if (first == 0) {
    a.status[0] = code;
    a.status[1] = code == MCA_TABLES_OK ? n_free + total.back - total.grow : max(n_free, 0);
    a.status[2] = code == MCA_TABLES_OK ? total.add : 0;
    a.status[3] = code == MCA_TABLES_OK ? total.grow : 0;
  }
  if (code != MCA_TABLES_OK) {
    for (int64_t r = first; r <= R; r += step) a.offsets[r] = 0;
    for (int64_t i = first; i < a.max_tokens; i += step) a.slots[i] = -1;
    return;
  }
  // the request that item i of a prefix sum falls to, and the sum before it
  auto find = [&](const int* pre, int i, int which, int* start) -> int {
    int lo = 0, hi = ne;  // pre[lo] <= i < pre[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] <= i) lo = mid; else hi = mid;
    }
    int r = lo * per, at = pre[lo], dummy = 0;
    for (; per > 1; ++r) {
      const Change c = change(r, &dummy);
      const int n = which == 0 ? c.add : (which == 1 ? c.grow : c.back);
      if (i < at + n || r + 1 >= R) break;
      at += n;
    }
    *start = at;
    return r;
  };
  auto blocks = [&](int len) -> int { return (int)(((unsigned)len + B - 1) / (unsigned)B); };
  // given-up block number i, and needed block number i, in the order of requests
  auto given = [&](int i) -> int {
    int at;
    const int r = find(s_back, i, 2, &at);
    return a.table[(int64_t)r * a.table_stride + blocks(a.new_len[r]) + (i - at)];
  };
  auto popped = [&](int i) -> int {
    const int p = n_free + total.back - 1 - i;
    return p < n_free ? a.free_list[p] : given(p - n_free);
  };
  for (int64_t e = first; e < ne; e += step) {
    int at = s_add[e], dummy = 0;
    for (int r = (int)e * per; r < ((int)e + 1) * per && r < R; ++r) {
      a.offsets[r] = at;
      if (per > 1) at += change(r, &dummy).add;
    }
  }
  if (first == 0) a.offsets[R] = total.add;
  for (int64_t i0 = first * kTabSlots; i0 < a.max_tokens; i0 += step * kTabSlots) {
    int r = 0, at = 0, end = -1, o = 0, have = 0, page = -1;
    int64_t block = 0;
    for (int u = 0; u < kTabSlots && i0 + u < a.max_tokens; ++u) {
      const int64_t i = i0 + u;
      if (i >= total.add) {
        a.slots[i] = -1;
        continue;
      }
      if ((int)i >= end) {
        r = find(s_add, (int)i, 0, &at);
        o = a.old_len[r];
        end = at + (a.new_len[r] - o);
        have = blocks(o);
        page = -1;
      }
      const int pos = o + ((int)i - at), pg = (int)((unsigned)pos / (unsigned)B);
      if (pg != page) {
        page = pg;
        if (pg < have) {
          block = a.table[(int64_t)r * a.table_stride + pg];
        } else {
          int g = s_grow[r / per], dummy = 0;
          for (int x = r / per * per; per > 1 && x < r; ++x) g += change(x, &dummy).grow;
          block = popped(g + pg - have);
        }
      }
      a.slots[i] = block * B + (pos - pg * B);
    }
  }
  for (int64_t i = first; i < total.grow; i += step) {
    int at;
    const int r = find(s_grow, (int)i, 1, &at);
    a.table[(int64_t)r * a.table_stride + blocks(a.old_len[r]) + ((int)i - at)] = popped((int)i);
  }
  for (int64_t i = first; i < (int64_t)total.back - total.grow; i += step) a.free_list[n_free + i] = given((int)i);
}

hipError_t lm_launch_tables(const TablesArgs& a, hipStream_t s) {
  const int64_t items = std::max<int64_t>(a.max_tokens / kTabSlots, a.n_req);
  const int64_t nb = std::min<int64_t>(512, (items + kTabThreads - 1) / kTabThreads);
  hipLaunchKernelGGL(k_lm_tables, dim3((unsigned)std::max<int64_t>(nb, 1)), dim3(kTabThreads), 0, s, a);
  return hipGetLastError();
}

// Copies units of sizeof(U) bytes: a row has n_kv_head * per_head of them in K
// and as many in V.  A workgroup takes rows_per_group rows.  Bound by memory: a
// thread has kAppendUnits units of K and of V in flight.  65000 rows of 8 heads of 128,
// bf16 (533 MB read and written): 104 us, 5.1 TB/s; 256 rows of 4 heads of 32, fp32: 5.5
// us.  Units of 4 and of 2 bytes are for heads and strides that are no multiples of 16.
template <class U>
__global__ __launch_bounds__(kAppendThreads) void k_lm_append(mca_cache_append_args a, int per_head, int scale,
                                                              int rows_per_group) {
  const int row_units = a.n_kv_head * per_head;
  const int64_t i0 = (int64_t)blockIdx.x * rows_per_group;
  const int nrows = (int)min((int64_t)rows_per_group, a.n - i0);
  const int64_t n_slots = (int64_t)a.n_blocks * a.block_size;
  const int todo = nrows * row_units;
  for (int e0 = threadIdx.x; e0 < todo; e0 += kAppendThreads * kAppendUnits) {
    U kv[kAppendUnits], vv[kAppendUnits];
    int64_t to[kAppendUnits];
#pragma unroll
    for (int u = 0; u < kAppendUnits; ++u) {
      const int e = e0 + u * kAppendThreads;
      to[u] = -1;
      if (e < todo) {
        const int row = e / row_units, c = e - row * row_units, h = c / per_head, d = c - h * per_head;
        const int64_t i = i0 + row, slot = a.slots[i];
        const int64_t src = a.rows != nullptr ? (int64_t)a.rows[i] : i;
        if (slot >= 0 && slot < n_slots && src >= 0 && src < a.n_src) {
          const int64_t blk = slot / a.block_size, in = slot - blk * a.block_size;
          to[u] = ((blk * a.n_kv_head + h) * a.block_size + in) * per_head + d;
          kv[u] = gload((const U*)a.k + (src * a.k_row + h * a.k_head) / scale + d);
          vv[u] = gload((const U*)a.v + (src * a.v_row + h * a.v_head) / scale + d);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAppendUnits; ++u)
      if (to[u] >= 0) {
        gstore((U*)a.k_cache + to[u], kv[u]);
        gstore((U*)a.v_cache + to[u], vv[u]);
      }
  }
}

hipError_t lm_launch_append(const mca_cache_append_args& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  const int el = a.dtype == MCA_TYPE_F32 ? 4 : 2;
  // the widest unit that every row and address is a multiple of
  const uint64_t all = (uint64_t)a.k | (uint64_t)a.v | (uint64_t)a.k_cache | (uint64_t)a.v_cache |
                       (uint64_t)(a.k_row * el) | (uint64_t)(a.k_head * el) | (uint64_t)(a.v_row * el) |
                       (uint64_t)(a.v_head * el) | (uint64_t)((int64_t)a.head_dim * el);
  const int unit = all % 16 == 0 ? 16 : (all % 4 == 0 ? 4 : 2);
  const int per_head = a.head_dim * el / unit;
  const int64_t row_units = (int64_t)a.n_kv_head * per_head;
  const int rows = (int)std::max<int64_t>(1, kAppendThreads * kAppendUnits / row_units);
  const dim3 grid((unsigned)((a.n + rows - 1) / rows));
  if (unit == 16)
    hipLaunchKernelGGL(k_lm_append<u32x4>, grid, dim3(kAppendThreads), 0, s, a, per_head, unit / el, rows);
  else if (unit == 4)
    hipLaunchKernelGGL(k_lm_append<uint32_t>, grid, dim3(kAppendThreads), 0, s, a, per_head, unit / el, rows);
  else
    hipLaunchKernelGGL(k_lm_append<uint16_t>, grid, dim3(kAppendThreads), 0, s, a, per_head, unit / el, rows);
  return hipGetLastError();
}

}  // namespace mca
