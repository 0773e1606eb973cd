// Rows into and out of a paged cache, quantised to e4m3 or as they are.
//
// An e4m3 row (one token, one head) is d codes and one exponent: value = code * 2^k, k the least integer with
// max |x| <= 448 * 2^k.  A power of two loses nothing against a free scale but range below (e4m3 is a floating type), and
// makes everything but the rounding of the code itself exact: x * 2^-k, the exponent (taken from the bits of the largest
// magnitude), and the way back to bf16 or fp32.
//
// Both directions stream: lanes take 8 elements each (copies: 16 bytes), a row is covered by consecutive lanes, a thread has
// kUnroll rows under way.  Rows are numbered (sequence, head, token), as they lie in dense tensors and in a page.
#include "pages.h"

namespace scalekv {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// largest of x over the LANES (a power of two up to 16) neighbouring lanes, in all of them
template <int LANES>
__device__ __forceinline__ unsigned group_max(unsigned x) {
#pragma unroll
  for (int m = 1; m < LANES; m *= 2) x = max(x, (unsigned)__shfl_xor((int)x, m));
  return x;
}

// The exponent of a row whose largest finite magnitude has the fp32 bits `top`.
__device__ __forceinline__ int scale_exponent(unsigned top) {
  const int e = (int)(top >> 23) - 127;                       // top = m * 2^e, 1 <= m < 2
  const int k = (top & 0x7fffffu) <= 0x600000u ? e - 8 : e - 7;  // 448 = 1.75 * 2^8
  return min(max(k, kScaleMin), kScaleMax);
}

__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((unsigned)(k + 127) << 23); }

// Four fp32 values (as bits) to four codes.  Values above `most` are held as that: 448 is never passed but by rounding
// of nothing (k bounds them), 240 at the largest exponent keeps what is read back finite.
__device__ __forceinline__ unsigned four_codes(const unsigned* bits, float inv, float most) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = fminf(fmaxf(__uint_as_float(bits[i]) * inv, -most), most);
    y[i] = (bits[i] & 0x7fffffffu) >= 0x7f800000u ? __builtin_nanf("") : x;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}

struct Side {
  RowsView rows;
  unsigned char* pool;
  uint8_t* scale;
};

// SRC: element type of the new rows; Q8: whether the cache is e4m3 (otherwise it has the rows' type).
template <int SRC, bool Q8, int D>
__global__ __launch_bounds__(kThreads) void pages_write_kernel(Side k_side, Side v_side, PagesView c, ChunkView chunk,
                                                               int n_rows) {
  constexpr int kElem = SRC == kTypeF32 ? 4 : 2;
  constexpr int kPer = Q8 ? 8 : 16 / kElem;          // elements of a lane
  constexpr int kLanes = D / kPer;                   // lanes of a row
  constexpr int kVecs = kPer * kElem / 16;           // 16-byte vectors of a lane
  constexpr int kRowsPerWg = kThreads / kLanes;
  const Side side = SCALEKV_WG_Y ? v_side : k_side;
  const int part = threadIdx.x % kLanes;
  const int row0 = SCALEKV_WG_X * (kRowsPerWg * kUnroll) + threadIdx.x / kLanes;
  unsigned x[kUnroll][4 * kVecs];
  long long at[kUnroll], scale_at[kUnroll];          // < 0: nothing to write
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int r = row0 + u * kRowsPerWg;
    at[u] = -1;
    if (r < n_rows) {
      const int unit = r / chunk.max_new, t = r - unit * chunk.max_new;
      const int seq = unit / c.n_kv_head, head = unit - seq * c.n_kv_head;
      const int n = chunk_count(chunk, seq), p = pages_len(c, seq) - n + t;
      const long long i = (long long)chunk_first(chunk, seq) + t;
      if (t < n && p >= 0 && i >= 0 && i < side.rows.n_row) {
        const int page = c.table[(long long)seq * c.width + (p >> c.page_shift)];
        if ((unsigned)page < (unsigned)c.n_page) {
          const int slot = p & ((1 << c.page_shift) - 1);
          at[u] = page * c.page + head * c.head + (long long)slot * (Q8 ? D : D * kElem);
          scale_at[u] = page * c.scale_page + head * c.scale_head + slot;
          const u32x4* src = (const u32x4*)(side.rows.p + seq * side.rows.seq + head * side.rows.head + i * side.rows.row) +
                             part * kVecs;
#pragma unroll
          for (int w = 0; w < kVecs; ++w) *(u32x4*)&x[u][4 * w] = src[w];
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if constexpr (!Q8) {
      if (at[u] >= 0) *(u32x4*)(side.pool + at[u] + 16 * part) = *(const u32x4*)x[u];
    } else {
      unsigned bits[8], top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (SRC == kTypeF32) bits[i] = x[u][i % (4 * kVecs)];
        else bits[i] = i % 2 ? x[u][i / 2] & 0xffff0000u : x[u][i / 2] << 16;
        const unsigned m = bits[i] & 0x7fffffffu;
        top = max(top, m < 0x7f800000u ? m : 0u);
      }
      // (the lanes of a row agree on whether it is written, and the row is theirs alone)
      const int k = scale_exponent(group_max<kLanes>(top));
      const float inv = power_of_two(-k), most = k == kScaleMax ? 240.f : 448.f;
      if (at[u] >= 0) {
        const u32x2 codes = {four_codes(bits, inv, most), four_codes(bits + 4, inv, most)};
        *(u32x2*)(side.pool + at[u] + 8 * part) = codes;
        if (part == 0) side.scale[scale_at[u]] = (uint8_t)(k + 127);
      }
    }
  }
}

struct Dest {
  const unsigned char* pool;
  const uint8_t* scale;
  unsigned char* dst;
  long long seq, head;  // bytes
};

// DST: element type of the dense caches; Q8: whether the pages hold e4m3.
template <int DST, bool Q8, int D>
__global__ __launch_bounds__(kThreads) void pages_read_kernel(Dest k_side, Dest v_side, PagesView c,
                                                              const int32_t* __restrict__ idx, int n_row, int n_head,
                                                              int group, int n_rows) {
  constexpr int kElem = DST == kTypeF32 ? 4 : 2;
  constexpr int kPer = Q8 ? 8 : 16 / kElem;
  constexpr int kLanes = D / kPer;
  constexpr int kRowsPerWg = kThreads / kLanes;
  const Dest side = SCALEKV_WG_Y ? v_side : k_side;
  const int part = threadIdx.x % kLanes;
  const int row0 = SCALEKV_WG_X * (kRowsPerWg * kUnroll) + threadIdx.x / kLanes;
  unsigned x[kUnroll][4];
  unsigned scale[kUnroll];
  long long to[kUnroll];  // < 0: the row is left as it is
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int r = row0 + u * kRowsPerWg;
    to[u] = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[u][i] = 0;
    scale[u] = 127;
    if (r < n_rows) {
      const int unit = r / n_row, t = r - unit * n_row;
      const int seq = unit / n_head, head = unit - seq * n_head;
      const int p = idx ? idx[r] : t;
      if (p >= 0 && p < pages_len(c, seq)) {
        to[u] = seq * side.seq + head * side.head + (long long)t * (D * kElem);
        const int page = c.table[(long long)seq * c.width + (p >> c.page_shift)];
        if ((unsigned)page < (unsigned)c.n_page) {
          const int slot = p & ((1 << c.page_shift) - 1), kv = head / group;
          const unsigned char* src =
              side.pool + (page * c.page + kv * c.head + (long long)slot * (Q8 ? D : D * kElem));
          if constexpr (Q8) {
            *(u32x2*)x[u] = *(const u32x2*)(src + 8 * part);
            scale[u] = side.scale[page * c.scale_page + kv * c.scale_head + slot];
          } else {
            *(u32x4*)x[u] = __builtin_nontemporal_load((const u32x4*)src + part);
          }
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (to[u] < 0) continue;
    unsigned char* dst = side.dst + to[u];
    if constexpr (!Q8) {
      *(u32x4*)(dst + 16 * part) = *(const u32x4*)x[u];
    } else {
      const float s = __uint_as_float(scale[u] << 23);
      if constexpr (DST == kTypeBf16) {
        u32x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bf16x2 two = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[u][i / 2], s, true)
                                   : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[u][i / 2], s, false);
          y[i] = __builtin_bit_cast(unsigned, two);
        }
        *(u32x4*)(dst + 16 * part) = y;
      } else {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(x[u][w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(x[u][w], true);
          *(float4*)(dst + 32 * part + 16 * w) = make_float4(lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s);
        }
      }
    }
  }
}

template <typename F>
hipError_t by_shape(int dtype, bool q8, int d, F f) {
  auto dim = [&](auto type, auto quantised) {
    if (d == 64) f(type, quantised, std::integral_constant<int, 64>{});
    else f(type, quantised, std::integral_constant<int, 128>{});
  };
  auto cache = [&](auto type) {
    if (q8) dim(type, std::true_type{});
    else dim(type, std::false_type{});
  };
  if (dtype == kTypeF32) cache(std::integral_constant<int, kTypeF32>{});
  else cache(std::integral_constant<int, kTypeBf16>{});
  return hipGetLastError();
}

// workgroups of a launch over n_rows rows (threads of kPer elements)
int row_groups(int n_rows, int d, int per) {
  const int rows = kThreads / (d / per) * kUnroll;
  return (n_rows + rows - 1) / rows;
}

}  // namespace

hipError_t launch_pages_write(int dtype, int d, int n_seq, const PagesView& pages, const RowsView& k, const RowsView& v,
                              const ChunkView& chunk, hipStream_t stream) {
  const int n_rows = n_seq * pages.n_kv_head * chunk.max_new;
  if (n_rows <= 0) return hipSuccess;
  const bool q8 = pages.type == kTypeE4m3;
  const dim3 grid(row_groups(n_rows, d, q8 ? 8 : dtype == kTypeF32 ? 4 : 8), 2);
  const Side ks{k, pages.k, pages.k_scale}, vs{v, pages.v, pages.v_scale};
  return by_shape(dtype, q8, d, [&](auto type, auto quantised, auto dim) {
    hipLaunchKernelGGL((pages_write_kernel<type(), quantised(), dim()>), grid, dim3(kThreads), 0, stream, ks, vs, pages,
                       chunk, n_rows);
  });
}

hipError_t launch_pages_read(int dtype, int d, int n_seq, int n_head, const PagesView& pages, const int32_t* idx, int n_row,
                             KvView k_dst, KvView v_dst, hipStream_t stream) {
  const int n_rows = n_seq * n_head * n_row, e = dtype == kTypeF32 ? 4 : 2;
  if (n_rows <= 0) return hipSuccess;
  const bool q8 = pages.type == kTypeE4m3;
  const dim3 grid(row_groups(n_rows, d, q8 ? 8 : dtype == kTypeF32 ? 4 : 8), 2);
  const Dest ks{pages.k, pages.k_scale, (unsigned char*)k_dst.ptr, k_dst.seq_stride * e, k_dst.head_stride * e};
  const Dest vs{pages.v, pages.v_scale, (unsigned char*)v_dst.ptr, v_dst.seq_stride * e, v_dst.head_stride * e};
  return by_shape(dtype, q8, d, [&](auto type, auto quantised, auto dim) {
    hipLaunchKernelGGL((pages_read_kernel<type(), quantised(), dim()>), grid, dim3(kThreads), 0, stream, ks, vs, pages, idx,
                       n_row, n_head, n_head / pages.n_kv_head, n_rows);
  });
}

}  // namespace scalekv
