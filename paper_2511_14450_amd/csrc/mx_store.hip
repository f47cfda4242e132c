// Writing rows into caches of 8 and 4 bits, and reading them back.
#include "mx_format.h"

namespace hyp {
namespace {

// value of another lane of the same four
template <int X> __device__ __forceinline__ unsigned quad_xor(unsigned v) {
  return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, X == 1 ? 0xb1 : 0x4e, 0xf, 0xf, true);  // quad_perm [1,0,3,2], [2,3,0,1]
}

// Features f .. f + 7 of a row of d, zeros from d on.
template <typename T, bool WIDE> __device__ __forceinline__ void load8(const T *row, int f, int d, float (&x)[8]) {
  if constexpr (WIDE) {  // d is a multiple of 8
    if (f >= d) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
    } else if constexpr (sizeof(T) == 2) {
      const u16x8_t v = *(const u16x8_t *)(row + f);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(v.v[i]);
    } else {
      const f32x4_t a = *(const f32x4_t *)(row + f), b = *(const f32x4_t *)(row + f + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = a[i];
        x[4 + i] = b[i];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = f + i < d ? load_f32(row + f + i) : 0.f;
  }
}

template <typename T, bool WIDE> __device__ __forceinline__ void store8(T *row, int f, int d, const float (&x)[8]) {
  if constexpr (WIDE) {
    if (f >= d) return;
    if constexpr (sizeof(T) == 2) {
      u16x8_t v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.v[i] = f32_to_bf16(x[i]);
      *(u16x8_t *)(row + f) = v;
    } else {
      *(f32x4_t *)(row + f) = f32x4_t{x[0], x[1], x[2], x[3]};
      *(f32x4_t *)(row + f + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (f + i < d) store_f32(row + f + i, x[i]);
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

// Codes and scale of eight features; x becomes the numbers that are stored.
template <int F> __device__ __forceinline__ unsigned put8(uint8_t *codes, uint8_t *scales, int within, int64_t group_stride, float (&x)[8]) {
  const unsigned scale = mx_scale_byte<F>(group_most(x));
  unsigned w[2];
  mx_quantise<F>(x, scale, w);
  if constexpr (F == HYP_E4M3) *(uint2 *)(codes + 8 * within) = make_uint2(w[0], w[1]);
  else *(unsigned *)(codes + 4 * within) = w[0];
  if ((within & 3) == 0) scales[(within >> 2) * group_stride] = (uint8_t)scale;
  return scale;
}

constexpr int kThreads = 256;

// One block of keys of one request and KV head: 4 lanes a group, `groups` of them a key, as many keys at a time as there are threads.  What is
// stored also goes to k_out / v_out, and each feature's least and largest number to the block's bounds, joined over the threads in LDS
// and with the bounds that the block had if it was begun before.
template <typename T, bool WIDE> __global__ void __launch_bounds__(kThreads) k_mx_write(const MxWriteCall p) {
  extern __shared__ float lds[];  // bounds: [keys at a time][features], least numbers, then largest
  const hyp_mx_cache_t &c = p.m.c;
  const int tid = threadIdx.x, tile = blockIdx.x % p.tiles, head = blockIdx.x / p.tiles;
  const int rows = (int)p.r.n_rows;
  int b = tile, q0, q1;
  auto start = [&](int i) { return mx_clamped(p.r.q_start[i], 0, rows); };
  if (!p.r.q_start) {
    q0 = b;
    q1 = b + 1;
  } else {
    // the last request whose tiles begin at or before this one
    int count = 0;
    for (int i = 0; i < c.n_requests; i += kThreads) {
      const bool before = i + tid < c.n_requests && (start(i + tid) >> p.block_shift) + 2 * (i + tid) <= tile;
      count += __syncthreads_count(before);
    }
    b = count - 1;
    if (b < 0) return;
    q0 = start(b);
    q1 = start(b + 1);
  }
  const int len = mx_len(c, b), first = len - (q1 - q0);  // key of the first row
  const int from = max(first, 0);
  if (q1 <= q0 || from >= len) return;
  // wrong values in q_start give a block that the request does not touch
  const int64_t blk = p.r.q_start ? (int64_t)(from >> p.block_shift) + tile - ((q0 >> p.block_shift) + 2 * b) : from >> p.block_shift;
  if (blk < from >> p.block_shift || blk > (len - 1) >> p.block_shift) return;
  const int begin = (int)blk << p.block_shift, j0 = max(from, begin), j1 = min(len - 1, begin + ((1 << p.block_shift) - 1)) + 1;
  const int per = 4 * p.m.groups, step = kThreads / per, within = tid % per, mine = tid / per, f = 8 * within, d = c.head_dim;
  const bool bounds = c.lo != nullptr;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = INFINITY;
    hi[i] = -INFINITY;
  }
  bool bad = false;
  if (mine < step) {
    for (int j = j0 + mine; j < j1; j += step) {
      int64_t page = b;
      int at = j;
      if (c.page_table) {
        page = mx_clamped(c.page_table[(int64_t)b * c.pages_per_request + (j >> p.m.shift)], 0, c.n_pages - 1);
        at = j & (c.page_keys - 1);
      }
      const int64_t row = (int64_t)q0 + (j - first);
      float k[8], v[8];
      load8<T, WIDE>((const T *)p.r.k + row * p.r.k_row_stride + head * p.r.k_head_stride, f, d, k);
      load8<T, WIDE>((const T *)p.r.v + row * p.r.v_row_stride + head * p.r.v_head_stride, f, d, v);
      uint8_t *kc = c.k + page * c.k_page_stride + head * c.k_head_stride + at * c.k_key_stride;
      uint8_t *vc = c.v + page * c.v_page_stride + head * c.v_head_stride + at * c.v_key_stride;
      uint8_t *ks = c.k_scale + page * c.k_scale_page_stride + head * c.k_scale_head_stride + at;
      uint8_t *vs = c.v_scale + page * c.v_scale_page_stride + head * c.v_scale_head_stride + at;
      const unsigned scale = c.k_format == HYP_E4M3 ? put8<HYP_E4M3>(kc, ks, within, c.k_scale_group_stride, k) : put8<HYP_E2M1>(kc, ks, within, c.k_scale_group_stride, k);
      if (c.v_format == HYP_E4M3) put8<HYP_E4M3>(vc, vs, within, c.v_scale_group_stride, v);
      else put8<HYP_E2M1>(vc, vs, within, c.v_scale_group_stride, v);
      bad |= scale == 255u;
      if (bounds) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          lo[i] = fminf(lo[i], k[i]);
          hi[i] = fmaxf(hi[i], k[i]);
        }
      }
      if (p.r.k_out) {
        store8<T, WIDE>((T *)p.r.k_out + row * p.r.k_out_row_stride + head * p.r.k_out_head_stride, f, d, k);
        store8<T, WIDE>((T *)p.r.v_out + row * p.r.v_out_row_stride + head * p.r.v_out_head_stride, f, d, v);
      }
    }
  }
  if (!bounds) return;
  const int width = 8 * per;
  if (mine < step) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lds[mine * width + f + i] = bad ? NAN : lo[i];
      lds[(step + mine) * width + f + i] = bad ? NAN : hi[i];
    }
  }
  __syncthreads();
  const int64_t page = c.page_table ? mx_clamped(c.page_table[(int64_t)b * c.pages_per_request + (j0 >> p.m.shift)], 0, c.n_pages - 1) : b;
  const int place = c.page_table ? (j0 & (c.page_keys - 1)) >> p.block_shift : (int)blk;
  const int64_t at = page * c.bound_page_stride + head * c.bound_head_stride + place * c.bound_block_stride;
  const bool begun = j0 > begin;
  const int used = min(step, j1 - j0);
  for (int x = tid; x < d; x += kThreads) {
    bf16_t *lo_p = (bf16_t *)c.lo + at + x, *hi_p = (bf16_t *)c.hi + at + x;
    float a = begun ? bf16_to_f32(*lo_p) : INFINITY, z = begun ? bf16_to_f32(*hi_p) : -INFINITY;
    bool nan = begun && (a != a || z != z);
    for (int i = 0; i < used; ++i) {
      const float l = lds[i * width + x], h = lds[(step + i) * width + x];
      nan |= l != l;
      a = fminf(a, l);
      z = fmaxf(z, h);
    }
    *lo_p = nan ? (bf16_t)0x7fc0 : f32_to_bf16(a);
    *hi_p = nan ? (bf16_t)0x7fc0 : f32_to_bf16(z);
  }
}

// 64 keys of one request and KV head.
constexpr int kReadKeys = 64;
template <typename T, int F, bool WIDE> __device__ __forceinline__ void get8(const uint8_t *codes, const uint8_t *scales, int within, int64_t group_stride, T *to, int d) {
  unsigned w[2];
  if constexpr (F == HYP_E4M3) {
    const uint2 x = *(const uint2 *)(codes + 8 * within);
    w[0] = x.x;
    w[1] = x.y;
  } else {
    w[0] = *(const unsigned *)(codes + 4 * within);
    w[1] = 0;
  }
  const float scale = mx_scale(scales[(within >> 2) * group_stride]);
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned r = mx_pair<F>(w, i, scale);
    x[2 * i] = __uint_as_float(r << 16);
    x[2 * i + 1] = __uint_as_float(r & 0xffff0000u);
  }
  store8<T, WIDE>(to, 8 * within, d, x);
}

template <typename T, bool WIDE> __global__ void __launch_bounds__(kThreads) k_mx_read(const MxReadCall p) {
  const hyp_mx_cache_t &c = p.m.c;
  const int tid = threadIdx.x, tile = blockIdx.x % p.tiles, head = (int)(blockIdx.x / p.tiles) % c.n_kv_heads, b = (int)(blockIdx.x / p.tiles) / c.n_kv_heads;
  const int len = mx_len(c, b), first = p.first ? mx_clamped(p.first[b], 0, len) : 0;
  const int most = min(len - first, p.o.keys), r0 = tile * kReadKeys;
  const int per = 4 * p.m.groups, step = kThreads / per, within = tid % per, mine = tid / per, d = c.head_dim;
  if (mine >= step) return;
  for (int r = r0 + mine; r < min(most, r0 + kReadKeys); r += step) {
    const int j = first + r;
    int64_t page = b;
    int at = j;
    if (c.page_table) {
      page = mx_clamped(c.page_table[(int64_t)b * c.pages_per_request + (j >> p.m.shift)], 0, c.n_pages - 1);
      at = j & (c.page_keys - 1);
    }
    T *k = (T *)p.o.k + b * p.o.k_request_stride + head * p.o.k_head_stride + r * p.o.k_key_stride;
    T *v = (T *)p.o.v + b * p.o.v_request_stride + head * p.o.v_head_stride + r * p.o.v_key_stride;
    const uint8_t *kc = c.k + page * c.k_page_stride + head * c.k_head_stride + at * c.k_key_stride;
    const uint8_t *vc = c.v + page * c.v_page_stride + head * c.v_head_stride + at * c.v_key_stride;
    const uint8_t *ks = c.k_scale + page * c.k_scale_page_stride + head * c.k_scale_head_stride + at;
    const uint8_t *vs = c.v_scale + page * c.v_scale_page_stride + head * c.v_scale_head_stride + at;
    if (c.k_format == HYP_E4M3) get8<T, HYP_E4M3, WIDE>(kc, ks, within, c.k_scale_group_stride, k, d);
    else get8<T, HYP_E2M1, WIDE>(kc, ks, within, c.k_scale_group_stride, k, d);
    if (c.v_format == HYP_E4M3) get8<T, HYP_E4M3, WIDE>(vc, vs, within, c.v_scale_group_stride, v, d);
    else get8<T, HYP_E2M1, WIDE>(vc, vs, within, c.v_scale_group_stride, v, d);
  }
}

template <typename T, bool WIDE> hipError_t write(const MxWriteCall &p, hipStream_t s) {
  const int per = 4 * p.m.groups, step = kThreads / per;
  k_mx_write<T, WIDE><<<(unsigned)p.tiles * p.m.c.n_kv_heads, kThreads, p.m.c.lo ? 2 * step * 8 * per * 4 : 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

template <typename T> hipError_t mx_write(const MxWriteCall &p, hipStream_t s) {
  return p.wide ? write<T, true>(p, s) : write<T, false>(p, s);
}

template <typename T> hipError_t mx_read(const MxReadCall &p, hipStream_t s) {
  const unsigned blocks = (unsigned)p.tiles * p.m.c.n_kv_heads * p.m.c.n_requests;
  if (p.wide) k_mx_read<T, true><<<blocks, kThreads, 0, s>>>(p);
  else k_mx_read<T, false><<<blocks, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

template hipError_t mx_write<float>(const MxWriteCall &, hipStream_t);
template hipError_t mx_write<bf16_t>(const MxWriteCall &, hipStream_t);
template hipError_t mx_read<float>(const MxReadCall &, hipStream_t);
template hipError_t mx_read<bf16_t>(const MxReadCall &, hipStream_t);

}  // namespace hyp
