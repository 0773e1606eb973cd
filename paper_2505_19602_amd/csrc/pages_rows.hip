// Rows into and out of a paged cache, quantised to e4m3 or as they are.
//
// An e4m3 row (one token, one head) is d codes and one exponent: value = code * 2^k, k the least integer with
// max |x| <= 448 * 2^k.  A power of two loses nothing against a free scale but range below (e4m3 is a floating type), and
// makes everything but the rounding of the code itself exact: x * 2^-k, the exponent (taken from the bits of the largest
// magnitude), and the way back to bf16 or fp32.
//
// Both directions are bound by HBM.  A wave moves 16 rows that lie in one page (page sizes are multiples of 16), so that
// the page's number and the addresses of rows are scalars: with a row's place worked out by its lanes the kernels were bound
// by that.  Lanes take 8 elements each (copies: 16 bytes), a row is covered by consecutive lanes, and all rows of the wave
// are under way at once.  Rows that a list names are looked up one by one.
//
// head_dim 128: 256 units x 2304 rows bf16 into e4m3 79 to 90 us (5.8 to 5.0 TB/s; over two or many buffers in turn; with places
// worked out by lanes 129), as they are 118 us (5.1 TB/s); 256 units x 3350 rows back out of e4m3 118 us (5.6 TB/s; 191), out of
// bf16 151 us (5.8 TB/s).  A large copy reaches 5.1 TB/s.  Listed rows, 60 units x 433 of head_dim 64, 5 us, 16 times as many
// units 40 us (5.3 TB/s), 48 times 126 us (5.1 TB/s).
#include <type_traits>

#include "pages.h"

namespace scalekv {
namespace {

constexpr int kThreads = 256;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// largest of x over LANES (4, 8 or 16) neighbouring lanes, in all of them: pairs, quads, then mirrored halves
template <int LANES>
__device__ __forceinline__ unsigned group_max(unsigned x) {
  auto with = [&](auto ctrl) { return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, ctrl(), 0xf, 0xf, true)); };
  x = with(std::integral_constant<int, 0xb1>{});                            // quad_perm 1 0 3 2
  x = with(std::integral_constant<int, 0x4e>{});                            // quad_perm 2 3 0 1
  if constexpr (LANES > 4) x = with(std::integral_constant<int, 0x141>{});  // row_half_mirror
  if constexpr (LANES > 8) x = with(std::integral_constant<int, 0x140>{});  // row_mirror
  return x;
}

// The exponent of a row whose largest finite magnitude has the fp32 bits `top`.
__device__ __forceinline__ int scale_exponent(unsigned top) {
  const int e = (int)(top >> 23) - 127;                       // top = m * 2^e, 1 <= m < 2
  const int k = (top & 0x7fffffu) <= 0x600000u ? e - 8 : e - 7;  // 448 = 1.75 * 2^8
  return min(max(k, kScaleMin), kScaleMax);
}

__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((unsigned)(k + 127) << 23); }

// Eight elements of a row (fp32 bits; LANES lanes hold the row) to codes; k: the row's exponent.
template <int LANES>
__device__ __forceinline__ u32x2 quantise(const unsigned (&bits)[8], int& k) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, bits[i] & 0x7fffffffu);
  unsigned most = group_max<LANES>(top);
  const bool odd = most >= 0x7f800000u;  // something is not finite: the exponent is that of the others
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd) != 0, 0)) {
    top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned m = bits[i] & 0x7fffffffu;
      top = max(top, m < 0x7f800000u ? m : 0u);
    }
    most = group_max<LANES>(top);
  }
  k = scale_exponent(most);
  const float inv = power_of_two(-k);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(bits[i]) * inv;
  // 448 is passed by nothing that is finite; at the largest exponent 240 keeps what is read back finite
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(odd || k == kScaleMax) != 0, 0)) {
    const float limit = k == kScaleMax ? 240.f : 448.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = fminf(fmaxf(y[i], -limit), limit);
      if ((bits[i] & 0x7fffffffu) >= 0x7f800000u) y[i] = __builtin_nanf("");
    }
  }
  u32x2 codes;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const int half = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    codes[w] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], half, true);
  }
  return codes;
}

struct Side {
  RowsView rows;
  unsigned char* pool;
  uint8_t* scale;
};

constexpr int kWaves = kThreads / 64;
constexpr int kGroup = 16;  // rows of a wave

// SRC: element type of the new rows; Q8: whether the cache is e4m3 (otherwise it has the rows' type).
template <int SRC, bool Q8, int D>
__global__ __launch_bounds__(kThreads) void pages_write_kernel(Side k_side, Side v_side, PagesView c, ChunkView chunk) {
  constexpr int kElem = SRC == kTypeF32 ? 4 : 2;
  constexpr int kPer = Q8 ? 8 : 16 / kElem;          // elements of a lane
  constexpr int kLanes = D / kPer;                   // lanes of a row
  constexpr int kVecs = kPer * kElem / 16;           // 16-byte vectors of a lane
  constexpr int kRowsAtOnce = 64 / kLanes, kSteps = kGroup / kRowsAtOnce;
  constexpr int kRowBytes = Q8 ? D : D * kElem;      // in the page
  const Side side = SCALEKV_WG_Z ? v_side : k_side;
  const int unit = SCALEKV_WG_Y, seq = unit / c.n_kv_head, head = unit - seq * c.n_kv_head;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, part = lane % kLanes;
  const int len = __builtin_amdgcn_readfirstlane(pages_len(c, seq));
  const int count = __builtin_amdgcn_readfirstlane(chunk_count(chunk, seq));
  const int pos0 = len - count, from = max(pos0, 0);
  const int group0 = (from & -kGroup) + kGroup * (SCALEKV_WG_X * kWaves + wave);  // the wave's first position
  if (group0 >= len) return;
  const int page = __builtin_amdgcn_readfirstlane(c.table[(long long)seq * c.width + (group0 >> c.page_shift)]);
  if ((unsigned)page >= (unsigned)c.n_page) return;
  const int slot = group0 & ((1 << c.page_shift) - 1);
  unsigned char* const dst = side.pool + (page * c.page + head * c.head + (long long)slot * kRowBytes);
  const int row = lane / kLanes;                     // of the first step; kRowsAtOnce further on in each
  const long long token0 = (long long)__builtin_amdgcn_readfirstlane(chunk_first(chunk, seq)) + (group0 - pos0);
  const unsigned char* const src =
      side.rows.p + (seq * side.rows.seq + head * side.rows.head + token0 * side.rows.row) + 16 * kVecs * part;
  u32x4 x[kSteps][kVecs];
  bool there[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int r = row + u * kRowsAtOnce, p = group0 + r;
    there[u] = p >= from && p < len && token0 + r >= 0 && token0 + r < side.rows.n_row;
#pragma unroll
    for (int w = 0; w < kVecs; ++w) {
      x[u][w] = u32x4{0, 0, 0, 0};
      if (there[u]) x[u][w] = __builtin_nontemporal_load((const u32x4*)(src + r * side.rows.row) + w);
    }
  }
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int r = row + u * kRowsAtOnce;
    if constexpr (!Q8) {
      if (there[u]) *(u32x4*)(dst + r * kRowBytes + 16 * part) = x[u][0];
    } else {
      unsigned bits[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (SRC == kTypeF32) bits[i] = x[u][i / 4 % kVecs][i % 4];
        else bits[i] = i % 2 ? x[u][0][i / 2] & 0xffff0000u : x[u][0][i / 2] << 16;
      }
      int k;
      const u32x2 codes = quantise<kLanes>(bits, k);
      if (there[u]) {
        *(u32x2*)(dst + r * kRowBytes + 8 * part) = codes;
        if (part == 0) side.scale[page * c.scale_page + head * c.scale_head + slot + r] = (uint8_t)(k + 127);
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

// DST: element type of the dense caches; Q8: whether the pages hold e4m3; LISTED: rows by `idx`; PAST: what is written is
// more than the last-level cache holds, and goes past it.
template <int DST, bool Q8, int D, bool LISTED, bool PAST>
__global__ __launch_bounds__(kThreads) void pages_read_kernel(Dest k_side, Dest v_side, PagesView c,
                                                              const int32_t* __restrict__ idx, int n_row, int n_head,
                                                              int group) {
  constexpr int kElem = DST == kTypeF32 ? 4 : 2;
  constexpr int kPer = Q8 ? 8 : 16 / kElem;
  constexpr int kLanes = D / kPer;
  constexpr int kRowsAtOnce = 64 / kLanes, kSteps = kGroup / kRowsAtOnce;
  constexpr int kRowBytes = Q8 ? D : D * kElem;
  constexpr int kOut = kPer * kElem / 16;            // 16-byte vectors that a lane writes
  const Dest side = SCALEKV_WG_Z ? v_side : k_side;
  const int unit = SCALEKV_WG_Y, seq = unit / n_head, head = unit - seq * n_head, kv = head / group;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, part = lane % kLanes;
  const int len = __builtin_amdgcn_readfirstlane(pages_len(c, seq));
  const int row0 = kGroup * (SCALEKV_WG_X * kWaves + wave), row = row0 + lane / kLanes;
  if (row0 >= n_row || (!LISTED && row0 >= len)) return;
  const int32_t* const table = c.table + (long long)seq * c.width;
  const long long kv_ofs = kv * c.head, kv_scale = kv * c.scale_head;
  u32x4 x[kSteps];
  unsigned scale[kSteps];
  bool there[kSteps];
  int page0 = -1;
  if constexpr (!LISTED) page0 = __builtin_amdgcn_readfirstlane(table[row0 >> c.page_shift]);
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int t = row + u * kRowsAtOnce;
    x[u] = u32x4{0, 0, 0, 0};
    scale[u] = 127;
    int p = t, page = page0;
    there[u] = t < n_row;
    if constexpr (LISTED) {
      if (there[u]) p = idx[(long long)unit * n_row + t];
      there[u] = there[u] && p >= 0 && p < len;
      if (there[u]) page = table[p >> c.page_shift];
    } else {
      there[u] = there[u] && t < len;
    }
    if (there[u] && (unsigned)page < (unsigned)c.n_page) {  // (other pages read as zeros)
      const int slot = p & ((1 << c.page_shift) - 1);
      const unsigned char* src = side.pool + (page * c.page + kv_ofs) + slot * kRowBytes;
      if constexpr (Q8) {
        const u32x2 codes = __builtin_nontemporal_load((const u32x2*)src + part);
        x[u][0] = codes[0];
        x[u][1] = codes[1];
        scale[u] = side.scale[page * c.scale_page + kv_scale + slot];
      } else {
        x[u] = __builtin_nontemporal_load((const u32x4*)src + part);
      }
    }
  }
  unsigned char* const dst = side.dst + (seq * side.seq + head * side.head + (long long)row * (D * kElem)) + 16 * kOut * part;
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    if (!there[u]) continue;
    u32x4 y[kOut];
    if constexpr (!Q8) {
      y[0] = x[u];
    } else {
      const float s = __uint_as_float(scale[u] << 23);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (DST == kTypeBf16) {
          const bf16x2 two = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[u][i / 2], s, true)
                                   : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[u][i / 2], s, false);
          y[0][i] = __builtin_bit_cast(unsigned, two);
        } else {
          const auto two = i % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(x[u][i / 2], true)
                                 : __builtin_amdgcn_cvt_pk_f32_fp8(x[u][i / 2], false);
          y[i / 2 % kOut][i % 2 * 2] = __float_as_uint(two[0] * s);
          y[i / 2 % kOut][i % 2 * 2 + 1] = __float_as_uint(two[1] * s);
        }
      }
    }
#pragma unroll
    for (int w = 0; w < kOut; ++w) {
      u32x4* const to = (u32x4*)(dst + u * kRowsAtOnce * (D * kElem)) + w;
      if constexpr (PAST) __builtin_nontemporal_store(y[w], to);
      else *to = y[w];
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

}  // namespace

hipError_t launch_pages_write(int dtype, int d, int n_seq, const PagesView& pages, const RowsView& k, const RowsView& v,
                              const ChunkView& chunk, hipStream_t stream) {
  // (the first of a sequence's new tokens may lie anywhere in its group of 16 rows)
  const int groups = (chunk.max_new + kGroup - 2) / kGroup + 1;
  const dim3 grid((groups + kWaves - 1) / kWaves, n_seq * pages.n_kv_head, 2);
  const Side ks{k, pages.k, pages.k_scale}, vs{v, pages.v, pages.v_scale};
  return by_shape(dtype, pages.type == kTypeE4m3, d, [&](auto type, auto quantised, auto dim) {
    hipLaunchKernelGGL((pages_write_kernel<type(), quantised(), dim()>), grid, dim3(kThreads), 0, stream, ks, vs, pages,
                       chunk);
  });
}

hipError_t launch_pages_read(int dtype, int d, int n_seq, int n_head, const PagesView& pages, const int32_t* idx, int n_row,
                             KvView k_dst, KvView v_dst, hipStream_t stream) {
  const int e = dtype == kTypeF32 ? 4 : 2, group = n_head / pages.n_kv_head;
  const dim3 grid((n_row + kGroup * kWaves - 1) / (kGroup * kWaves), n_seq * n_head, 2);
  const Dest ks{pages.k, pages.k_scale, (unsigned char*)k_dst.ptr, k_dst.seq_stride * e, k_dst.head_stride * e};
  const Dest vs{pages.v, pages.v_scale, (unsigned char*)v_dst.ptr, v_dst.seq_stride * e, v_dst.head_stride * e};
  const bool past = rows_go_past_caches(CacheWriter::kCompact, n_seq * n_head, n_row, d * e);
  return by_shape(dtype, pages.type == kTypeE4m3, d, [&](auto type, auto quantised, auto dim) {
    auto launch = [&](auto listed, auto past_caches) {
      hipLaunchKernelGGL((pages_read_kernel<type(), quantised(), dim(), listed(), past_caches()>), grid, dim3(kThreads), 0,
                         stream, ks, vs, pages, idx, n_row, n_head, group);
    };
    if (idx) past ? launch(std::true_type{}, std::true_type{}) : launch(std::true_type{}, std::false_type{});
    else past ? launch(std::false_type{}, std::true_type{}) : launch(std::false_type{}, std::false_type{});
  });
}

}  // namespace scalekv
