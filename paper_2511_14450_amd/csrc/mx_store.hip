// Writing rows into caches of 8 and 4 bits, and reading them back.
#include "mx_format.h"

namespace hyp {
namespace {

// value of another lane of the same four
template <int X> __device__ __forceinline__ unsigned quad_xor(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, X == 1 ? 0xb1 : 0x4e, 0xf, 0xf, true);  // quad_perm [1,0,3,2], [2,3,0,1]
}

// Features f .. f + 7 of a row of d, zeros from d on.  WIDE: whole pieces of 16 bytes; no branch is in the way of requesting several.
template <typename T, bool WIDE> struct Eight {
  static constexpr int N = sizeof(T) / 2;
  uint4 w[N];
  __device__ __forceinline__ void load(const T *row, int f, int d) {
    if constexpr (WIDE) {
      const uint4 *at = (const uint4 *)(row + min(f, d - 8));
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load((const f32x4_t *)at + i));
    } else {
      T x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = f + i < d ? row[f + i] : (T)0;
      __builtin_memcpy(w, x, sizeof(x));
    }
  }
  __device__ __forceinline__ void get(int f, int d, float (&x)[8]) const {
    T y[8];
    __builtin_memcpy(y, w, sizeof(y));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = !WIDE || f < d ? load_f32(y + i) : 0.f;
  }
};

// Rows are read and written once here and are larger than what the caches hold: streaming loads and stores leave those to the codes (reading
// four caches of 6007 to 8192 keys back 41 us without, 30 with; 4 x 8192 rows into 4 bits 72 and 62).
__device__ __forceinline__ float low_of(unsigned pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high_of(unsigned pair) { return __uint_as_float(pair & 0xffff0000u); }
template <typename T, bool WIDE> __device__ __forceinline__ void store8(T *row, int f, int d, const unsigned (&pairs)[4]) {
  if constexpr (WIDE) {
    if (f >= d) return;
    if constexpr (sizeof(T) == 2) {
      const uint4 v = make_uint4(pairs[0], pairs[1], pairs[2], pairs[3]);
      __builtin_nontemporal_store(__builtin_bit_cast(f32x4_t, v), (f32x4_t *)(row + f));
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        __builtin_nontemporal_store(f32x4_t{low_of(pairs[2 * i]), high_of(pairs[2 * i]), low_of(pairs[2 * i + 1]), high_of(pairs[2 * i + 1])}, (f32x4_t *)(row + f + 4 * i));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (f + i < d) store_f32(row + f + i, i & 1 ? high_of(pairs[i >> 1]) : low_of(pairs[i >> 1]));
  }
}

// Largest magnitude of a group, which lies in four lanes of eight features, as bits: those of a NaN are the highest.
__device__ __forceinline__ unsigned group_most(const float (&x)[8]) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  m = max(m, quad_xor<1>(m));
  return max(m, quad_xor<2>(m));
}

// Codes and scale of eight features, and the numbers that are stored.
template <int F> __device__ __forceinline__ unsigned put8(uint8_t *codes, uint8_t *scales, int within, int64_t group_stride, const float (&x)[8], unsigned (&pairs)[4]) {
  const unsigned scale = mx_scale_byte<F>(group_most(x));
  unsigned w[2];
  mx_quantise<F>(x, scale, w, pairs);
  if constexpr (F == HYP_E4M3) *(uint2 *)(codes + 8 * within) = make_uint2(w[0], w[1]);
  else *(unsigned *)(codes + 4 * within) = w[0];
  if ((within & 3) == 0) scales[(within >> 2) * group_stride] = (uint8_t)scale;
  return scale;
}

constexpr int kThreads = 256, kBatch = 4;

// Rows mine, mine + step, ... below n of one KV head to codes, and, where `out` is given, to the numbers that these stand for; seen(numbers, whether they
// are NaN) gets them too.
template <typename T, int F, bool WIDE, typename Seen>
__device__ __forceinline__ void write_rows(const T *in, int64_t in_stride, T *out, int64_t out_stride, uint8_t *codes, int64_t key_stride, uint8_t *scales, int64_t group_stride,
                                           int within, int mine, int step, int n, int d, Seen &&seen) {
  const int f = 8 * within;
  // kBatch keys of a thread are requested before the first is worked on; those behind the last one again as the last
  for (int base = mine; base < n; base += kBatch * step) {
    Eight<T, WIDE> raw[kBatch];
#pragma unroll
    for (int x = 0; x < kBatch; ++x) raw[x].load(in + min(base + x * step, n - 1) * in_stride, f, d);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      const int r = base + x * step;
      if (r >= n) break;
      float y[8];
      unsigned pairs[4];
      raw[x].get(f, d, y);
      const unsigned scale = put8<F>(codes + (uint64_t)(unsigned)r * (unsigned)key_stride, scales + r, within, group_stride, y, pairs);
      seen(pairs, scale == 255u);
      if (out) store8<T, WIDE>(out + r * out_stride, f, d, pairs);
    }
  }
}

// One block of keys of one request and KV head, which lie in one page: half of the threads take the keys, half the values, 4 lanes a group, `groups`
// of them a key, as many keys at a time as there are threads.  What is stored also goes to k_out / v_out, and each feature's least and largest number
// to the block's bounds, joined over the threads in LDS and with the bounds that the block had if it was begun before.  Bytes bound large calls: 4 x 8192
// rows of 8 heads into 4 bits, the stored numbers and bounds with them, 60 us, 5.1 TB/s (keys and values in turn in workgroups of half as many
// threads, and rows through the caches: 72).  Small ones are a chain of reads (starts and lengths, page, rows) and the quantising of four rows a
// thread: 2107 rows of 16 prompts 12 us, a row each of 32 requests 6.7 in the kernel.
template <typename T, bool WIDE, int KF, int VF> __global__ void __launch_bounds__(2 * kThreads) k_mx_write(const MxWriteCall p) {
  extern __shared__ float lds[];  // bounds: [keys at a time][features], least numbers, then largest
  __shared__ int begins[2 * kThreads + 1], lens[2 * kThreads];
  const hyp_mx_cache_t &c = p.m.c;
  const int tid = threadIdx.x, tile = blockIdx.x % p.tiles, head = blockIdx.x / p.tiles;
  const int rows = (int)p.r.n_rows, n = c.n_requests;
  int b = tile, q0, q1, len;
  if (!p.r.q_start) {
    q0 = b;
    q1 = b + 1;
    len = mx_len(c, b);
  } else {
    // the last request whose tiles begin at or before this one; starts and lengths of up to 512 requests are read at once
    auto start = [&](int i) { return mx_clamped(p.r.q_start[i], 0, rows); };
    const bool few = n <= 2 * kThreads;
    int count = 0;
    for (int i = tid; i - tid < n; i += 2 * kThreads) {
      const int begin = i < n ? start(i) : 0;
      if (few && i < n) {
        lens[i] = mx_len(c, i);
        begins[i] = begin;
        if (i == n - 1) begins[n] = start(n);
      }
      count += __syncthreads_count(i < n && (begin >> p.block_shift) + 2 * i <= tile);
    }
    b = count - 1;
    if (b < 0) return;
    q0 = few ? begins[b] : start(b);
    q1 = few ? begins[b + 1] : start(b + 1);
    len = few ? lens[b] : mx_len(c, b);
    q0 = __builtin_amdgcn_readfirstlane(q0);
    q1 = __builtin_amdgcn_readfirstlane(q1);
    len = __builtin_amdgcn_readfirstlane(len);
  }
  const int first = len - (q1 - q0), from = max(first, 0);  // key of the first row
  if (q1 <= q0 || from >= len) return;
  // wrong values in q_start give a block that the request does not touch
  const int64_t blk = p.r.q_start ? (int64_t)(from >> p.block_shift) + tile - ((q0 >> p.block_shift) + 2 * b) : from >> p.block_shift;
  if (blk < from >> p.block_shift || blk > (len - 1) >> p.block_shift) return;
  const int begin = (int)blk << p.block_shift, j0 = max(from, begin), j1 = min(len - 1, begin + ((1 << p.block_shift) - 1)) + 1;
  const int64_t page = c.page_table ? mx_clamped(c.page_table[(int64_t)b * c.pages_per_request + (j0 >> p.m.shift)], 0, c.n_pages - 1) : b;
  const int at0 = c.page_table ? j0 & (c.page_keys - 1) : j0;
  const bool values = __builtin_amdgcn_readfirstlane(tid / kThreads);
  const int per = 4 * p.m.groups, step = kThreads / per, within = tid % kThreads % per, mine = tid % kThreads / per, f = 8 * within, d = c.head_dim;
  const bool bounds = c.lo != nullptr;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = INFINITY;
    hi[i] = -INFINITY;
  }
  bool bad = false;
  if (mine < step) {
    const int64_t row0 = (int64_t)q0 + (j0 - first);
    if (values) {
      write_rows<T, VF, WIDE>((const T *)p.r.v + row0 * p.r.v_row_stride + head * p.r.v_head_stride, p.r.v_row_stride,
                              p.r.v_out ? (T *)p.r.v_out + row0 * p.r.v_out_row_stride + head * p.r.v_out_head_stride : nullptr, p.r.v_out_row_stride,
                              c.v + page * c.v_page_stride + head * c.v_head_stride + at0 * c.v_key_stride, c.v_key_stride,
                              c.v_scale + page * c.v_scale_page_stride + head * c.v_scale_head_stride + at0, c.v_scale_group_stride, within, mine, step, j1 - j0, d,
                              [](const unsigned (&)[4], bool) {});
    } else {
      write_rows<T, KF, WIDE>((const T *)p.r.k + row0 * p.r.k_row_stride + head * p.r.k_head_stride, p.r.k_row_stride,
                              p.r.k_out ? (T *)p.r.k_out + row0 * p.r.k_out_row_stride + head * p.r.k_out_head_stride : nullptr, p.r.k_out_row_stride,
                              c.k + page * c.k_page_stride + head * c.k_head_stride + at0 * c.k_key_stride, c.k_key_stride,
                              c.k_scale + page * c.k_scale_page_stride + head * c.k_scale_head_stride + at0, c.k_scale_group_stride, within, mine, step, j1 - j0, d,
                              [&](const unsigned (&pairs)[4], bool nan) {
                                if (!bounds) return;
                                bad |= nan;
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                  const float x = i & 1 ? high_of(pairs[i >> 1]) : low_of(pairs[i >> 1]);
                                  lo[i] = fminf(lo[i], x);
                                  hi[i] = fmaxf(hi[i], x);
                                }
                              });
    }
  }
  if (!bounds) return;
  const int width = 8 * per;
  if (mine < step && !values) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lds[mine * width + f + i] = bad ? NAN : lo[i];
      lds[(step + mine) * width + f + i] = bad ? NAN : hi[i];
    }
  }
  const int place = c.page_table ? at0 >> p.block_shift : (int)blk;
  const int64_t at = page * c.bound_page_stride + head * c.bound_head_stride + place * c.bound_block_stride;
  const bool begun = j0 > begin;
  const int used = min(step, j1 - j0);
  __syncthreads();
  for (int y = tid; y < 2 * d; y += 2 * kThreads) {
    const bool upper = y >= d;
    const int x = upper ? y - d : y;
    bf16_t *to = (bf16_t *)(upper ? c.hi : c.lo) + at + x;
    const float *of = lds + (upper ? step * width : 0) + x;
    float a = begun ? bf16_to_f32(*to) : upper ? -INFINITY : INFINITY;
    bool nan = a != a;
    for (int i = 0; i < used; ++i) {
      const float v = of[i * width];
      nan |= v != v;
      a = upper ? fmaxf(a, v) : fminf(a, v);
    }
    *to = nan ? (bf16_t)0x7fc0 : f32_to_bf16(a);
  }
}

// 64 keys of one request and KV head, kBatch of a thread at a time.  Bytes bound it: four caches of 6007 to 8192 keys of 8 heads out of 8 bits 29.5 us,
// 6.3 TB/s.
constexpr int kReadKeys = 64;
template <typename T, int F, bool WIDE> __device__ __forceinline__ void get8(uint2 codes, unsigned scale_byte, int within, T *to, int d) {
  const unsigned w[2] = {codes.x, codes.y};
  const float scale = mx_scale(scale_byte);
  unsigned pairs[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) pairs[i] = mx_pair<F>(w, i, scale);
  store8<T, WIDE>(to, 8 * within, d, pairs);
}

template <typename T, bool WIDE, int KF, int VF> __global__ void __launch_bounds__(kThreads) k_mx_read(const MxReadCall p) {
  const hyp_mx_cache_t &c = p.m.c;
  const int tid = threadIdx.x, tile = blockIdx.x % p.tiles, head = (int)(blockIdx.x / p.tiles) % c.n_kv_heads, b = (int)(blockIdx.x / p.tiles) / c.n_kv_heads;
  const int len = mx_len(c, b), first = p.first ? mx_clamped(p.first[b], 0, len) : 0;
  const int r0 = tile * kReadKeys, r1 = min(min(len - first, p.o.keys), r0 + kReadKeys);
  const int per = 4 * p.m.groups, step = kThreads / per, within = tid % per, mine = tid / per, d = c.head_dim;
  if (mine >= step) return;
  for (int base = r0 + mine; base < r1; base += kBatch * step) {
    int64_t page[kBatch];
    int at[kBatch];
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      at[x] = first + min(base + x * step, r1 - 1);
      page[x] = b;
    }
    if (c.page_table) {
#pragma unroll
      for (int x = 0; x < kBatch; ++x) page[x] = c.page_table[(int64_t)b * c.pages_per_request + (at[x] >> p.m.shift)];
#pragma unroll
      for (int x = 0; x < kBatch; ++x) {
        page[x] = mx_clamped((int)page[x], 0, c.n_pages - 1);
        at[x] &= c.page_keys - 1;
      }
    }
    uint2 k[kBatch], v[kBatch];
    unsigned ks[kBatch], vs[kBatch];
    auto codes = [&](const uint8_t *from, auto format) {
      if constexpr (decltype(format)::value == HYP_E4M3) return *(const uint2 *)(from + 8 * within);
      else return make_uint2(*(const unsigned *)(from + 4 * within), 0u);
    };
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      k[x] = codes(c.k + page[x] * c.k_page_stride + head * c.k_head_stride + at[x] * c.k_key_stride, std::integral_constant<int, KF>());
      v[x] = codes(c.v + page[x] * c.v_page_stride + head * c.v_head_stride + at[x] * c.v_key_stride, std::integral_constant<int, VF>());
      ks[x] = c.k_scale[page[x] * c.k_scale_page_stride + head * c.k_scale_head_stride + (within >> 2) * c.k_scale_group_stride + at[x]];
      vs[x] = c.v_scale[page[x] * c.v_scale_page_stride + head * c.v_scale_head_stride + (within >> 2) * c.v_scale_group_stride + at[x]];
    }
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      const int r = base + x * step;
      if (r >= r1) break;
      get8<T, KF, WIDE>(k[x], ks[x], within, (T *)p.o.k + b * p.o.k_request_stride + head * p.o.k_head_stride + r * p.o.k_key_stride, d);
      get8<T, VF, WIDE>(v[x], vs[x], within, (T *)p.o.v + b * p.o.v_request_stride + head * p.o.v_head_stride + r * p.o.v_key_stride, d);
    }
  }
}

template <typename T, bool WIDE> hipError_t read(const MxReadCall &p, hipStream_t s) {
  const unsigned blocks = (unsigned)p.tiles * p.m.c.n_kv_heads * p.m.c.n_requests;
  const bool k8 = p.m.c.k_format == HYP_E4M3, v8 = p.m.c.v_format == HYP_E4M3;
  if (k8 && v8) k_mx_read<T, WIDE, HYP_E4M3, HYP_E4M3><<<blocks, kThreads, 0, s>>>(p);
  else if (k8) k_mx_read<T, WIDE, HYP_E4M3, HYP_E2M1><<<blocks, kThreads, 0, s>>>(p);
  else if (v8) k_mx_read<T, WIDE, HYP_E2M1, HYP_E4M3><<<blocks, kThreads, 0, s>>>(p);
  else k_mx_read<T, WIDE, HYP_E2M1, HYP_E2M1><<<blocks, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T, bool WIDE> hipError_t write(const MxWriteCall &p, hipStream_t s) {
  const int per = 4 * p.m.groups, step = kThreads / per, lds = p.m.c.lo ? 2 * step * 8 * per * 4 : 0;
  const unsigned blocks = (unsigned)p.tiles * p.m.c.n_kv_heads;
  const bool k8 = p.m.c.k_format == HYP_E4M3, v8 = p.m.c.v_format == HYP_E4M3;
  if (k8 && v8) k_mx_write<T, WIDE, HYP_E4M3, HYP_E4M3><<<blocks, 2 * kThreads, lds, s>>>(p);
  else if (k8) k_mx_write<T, WIDE, HYP_E4M3, HYP_E2M1><<<blocks, 2 * kThreads, lds, s>>>(p);
  else if (v8) k_mx_write<T, WIDE, HYP_E2M1, HYP_E4M3><<<blocks, 2 * kThreads, lds, s>>>(p);
  else k_mx_write<T, WIDE, HYP_E2M1, HYP_E2M1><<<blocks, 2 * kThreads, lds, s>>>(p);
  return hipGetLastError();
}

}  // namespace

template <typename T> hipError_t mx_write(const MxWriteCall &p, hipStream_t s) {
  return p.wide ? write<T, true>(p, s) : write<T, false>(p, s);
}

template <typename T> hipError_t mx_read(const MxReadCall &p, hipStream_t s) { return p.wide ? read<T, true>(p, s) : read<T, false>(p, s); }

template hipError_t mx_write<float>(const MxWriteCall &, hipStream_t);
template hipError_t mx_write<bf16_t>(const MxWriteCall &, hipStream_t);
template hipError_t mx_read<float>(const MxReadCall &, hipStream_t);
template hipError_t mx_read<bf16_t>(const MxReadCall &, hipStream_t);

}  // namespace hyp
