// What the kernels of the attention over pages share (device code).
#pragma once
#include "pages.h"

namespace scalekv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

struct AttendArgs {
  PagesView c;
  RowsView q, out;
  ChunkView chunk;
  MaskView mask;
  int n_seq, group, n_row_group, n_split, n_wg;
  float scale_log2e, no_max;
  float *part, *stat;  // partial sums [row][split][D], their {largest logit in log2 units, sum} [row][split][2]
};

// bf16, many query rows (pages_chunk.hip): 64 row_tiles rows to a workgroup
hipError_t launch_pages_chunk(int d, bool q8, int row_tiles, const AttendArgs& a, hipStream_t stream);

// Which unit a workgroup works on, and which part of it: units are dealt out to the XCDs in turn (consecutive workgroup ids go
// round-robin over them), so that the workgroups of a unit share an L2 and the units of a long sequence do not.
__device__ __forceinline__ void unit_of(int wg, int n_wg, int per_unit, int& unit, int& part) {
  const int dealt = n_wg / per_unit / kXcds * kXcds;  // units of whole rounds; the rest one behind the other
  if (wg < dealt * per_unit) {
    const int nth = wg / kXcds;
    unit = nth / per_unit * kXcds + wg % kXcds;
    part = nth % per_unit;
  } else {
    const int rest = wg - dealt * per_unit;
    unit = dealt + rest / per_unit;
    part = rest % per_unit;
  }
}

// The query rows [first_row, first_row + rows) of a unit (rows: token t, head h of the group, number t * group + h), what
// they see, and the tiles of TN keys that hold it: those of the sinks, then those from the window's first row on.
template <int TN>
struct Seen {
  int len, count, n_rows, pos0;  // cached rows, new tokens, query rows of the unit, position of the first token
  int lo, hi, sinks;             // some row sees [lo, hi) and the first `sinks`
  int all_begin, all_end;        // all rows see [all_begin, all_end) of those (and the sinks below all_end)
  bool window;
  int causal, width;             // of the mask
  int sink_tiles, from_tile, n_tile;
  int plain_begin, plain_end;    // every row sees all of these tiles
  __device__ __forceinline__ int end_of(int p) const { return causal ? min(len, p + 1) : len; }
  __device__ __forceinline__ int begin_of(int p) const { return window ? p - width + 1 : -0x7fffffff; }
  __device__ __forceinline__ Seen(const AttendArgs& a, int seq, int first_row, int rows) {
    len = __builtin_amdgcn_readfirstlane(pages_len(a.c, seq));  // (all of this is the same in every lane: scalars)
    count = __builtin_amdgcn_readfirstlane(chunk_count(a.chunk, seq));
    n_rows = count * a.group;
    pos0 = len - count;
    causal = a.mask.causal;
    width = a.mask.window;
    window = width > 0;
    sinks = window ? a.mask.n_sink : 0;
    const int last = min(first_row + rows, n_rows) - 1;
    const int p_lo = pos0 + first_row / a.group, p_hi = pos0 + last / a.group;
    lo = begin_of(p_lo);
    hi = end_of(p_hi);
    all_begin = begin_of(p_hi);
    all_end = end_of(p_lo);
    sink_tiles = (max(min(sinks, hi), 0) + TN - 1) / TN;
    from_tile = max(max(lo, 0) / TN, sink_tiles);
    n_tile = sink_tiles + max((hi + TN - 1) / TN - from_tile, 0);
    plain_begin = window ? sink_tiles + max((max(all_begin, 0) + TN - 1) / TN - from_tile, 0) : 0;
    plain_end = sink_tiles + max(all_end, 0) / TN - from_tile;
  }
  __device__ __forceinline__ bool plain(int t) const { return t >= plain_begin && t < plain_end; }
  __device__ __forceinline__ int key0(int t) const { return (t < sink_tiles ? t : from_tile + t - sink_tiles) * TN; }
  // does some row see this position; any of [pos, pos + n); all of them
  __device__ __forceinline__ bool some(int pos) const { return pos < hi && (pos >= lo || pos < sinks); }
  __device__ __forceinline__ bool any(int pos, int n) const { return pos < hi && (pos + n > lo || pos < sinks); }
  __device__ __forceinline__ bool every(int pos, int n) const { return pos + n <= hi && (pos >= lo || pos + n <= sinks); }
  // is there a key in the tile that some rows see and others do not
  __device__ __forceinline__ bool edge(int t) const {
    const int from = key0(t), end = min(from + TN, hi);
    return end > all_end || (window && max(from, max(lo, sinks)) < min(all_begin, end));
  }
};

// an address that is the same in every lane, as a scalar
__device__ __forceinline__ const unsigned char* scalar(const unsigned char* p) {
  const unsigned long long x = (unsigned long long)p;
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)(x >> 32));
  return (const unsigned char*)((unsigned long long)hi << 32 | lo);
}

// chunk c of row r (16 bytes each) sits in slot c ^ k_flip(r) of a K row, c ^ v_flip(r) of a V row, bf16 rows in LDS:
// operand reads are free of bank conflicts (attend_pipe.hip has the reasons)
template <int D>
__device__ constexpr int k_flip_bf16(int r) {
  const int high = (r >> 4 & 1) | (r >> 3 & 1) << 1;
  return D == 128 ? (r & 3) | high << 2 : (r >> 1 & 1) | high << 1;
}
template <int D>
__device__ constexpr int v_flip_bf16(int r) {
  return D == 128 ? (r & 3) << 1 | (r >> 4 & 1) << 3 : (r >> 1 & 1) << 1 | (r >> 4 & 1) << 2;
}

// sixteen codes of a row with its scale, as the products take them
__device__ __forceinline__ void widen(const u32x4& x, float s, u32x4 (&y)[2]) {  // bf16
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i / 2][i % 2 * 2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, false));
    y[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, true));
  }
}
__device__ __forceinline__ void widen(const u32x4& x, float s, u32x4 (&y)[4]) {  // fp32
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(x[i], true);
    y[i][0] = __float_as_uint(lo[0] * s);
    y[i][1] = __float_as_uint(lo[1] * s);
    y[i][2] = __float_as_uint(hi[0] * s);
    y[i][3] = __float_as_uint(hi[1] * s);
  }
}
// zeros in the place of what is not finite; whether there was any
template <bool BF16>
__device__ __forceinline__ bool take_odd(u32x4& x) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      const bool lo = (x[i] & 0x7f80u) == 0x7f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
      odd |= lo || hi;
      x[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
    } else {
      const bool it = (x[i] & 0x7f800000u) == 0x7f800000u;
      odd |= it;
      x[i] = it ? 0u : x[i];
    }
  }
  return odd;
}

// element ch of a cached row at byte offset `at`
template <int TYPE, bool Q8>
__device__ __forceinline__ float cached_value(const unsigned char* pool, const uint8_t* scales, long long at,
                                              long long scale_at, int ch) {
  if constexpr (Q8)
    return __builtin_amdgcn_cvt_pk_f32_fp8(pool[at + ch], false)[0] * __uint_as_float((unsigned)scales[scale_at] << 23);
  else if constexpr (TYPE == kTypeBf16)
    return __uint_as_float((unsigned)((const uint16_t*)(pool + at))[ch] << 16);
  else
    return ((const float*)(pool + at))[ch];
}

// Values that are not finite have been taken out of the tiles that some rows of the workgroup see and others do not (there
// a weight of zero would make NaN of them): this adds them, for the rows that see them, to the sums of a wave.  The sums
// are in LDS meanwhile (rows of D fp32, this wave's alone), so that nothing of this is held through the tile loop.  neg: less
// the offset of row 16 b + i, in lanes 16 g + i.  Keys [from, to) of each such tile in [t0, t1) are looked at: those
// that the wave has worked on, whose offsets are no lower than their logits.  Rare, and written to be short: the logits are formed anew, a channel at a time.
template <int TYPE, bool Q8, int D, int TN, int RT>
__device__ __forceinline__ void add_odd(const AttendArgs& a, const Seen<TN>& seen, int seq, int kv, int wave_row, int t0,
                                        int t1, int from, int to, const float (&neg)[RT], float* sums) {
  const PagesView& c = a.c;
  constexpr int kElem = TYPE == kTypeBf16 ? 2 : 4;
  const int lane = threadIdx.x & 63;
  // lane r: row r of the wave
  float less = neg[0];
  if constexpr (RT == 2) less = lane & 16 ? neg[1] : neg[0];
  const int r = min(wave_row + (lane & (16 * RT - 1)), seen.n_rows - 1), tok = r / a.group, p = seen.pos0 + tok;
  const long long row = (long long)chunk_first(a.chunk, seq) + tok;
  const unsigned char* q = a.q.p + seq * a.q.seq + (kv * a.group + (r - tok * a.group)) * a.q.head + row * a.q.row;
  const bool there = row >= 0 && row < a.q.n_row;
  const int32_t* const table = c.table + (long long)seq * c.width;
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    if (!seen.edge(t)) continue;
#pragma unroll 1
    for (int key = from; key < to; ++key) {
      const int pos = seen.key0(t) + key;
      if (!seen.some(pos)) continue;
      const int page = table[pos >> c.page_shift], slot = pos & ((1 << c.page_shift) - 1);
      if ((unsigned)page >= (unsigned)c.n_page) continue;
      const long long at = page * c.page + kv * c.head + (long long)slot * (Q8 ? D : D * kElem);
      const long long scale_at = page * c.scale_page + kv * c.scale_head + slot;
      float val[D / 64];
      bool odd = false;
#pragma unroll
      for (int x = 0; x < D / 64; ++x) {
        val[x] = cached_value<TYPE, Q8>(c.v, c.v_scale, at, scale_at, 64 * x + lane);
        odd |= !(fabsf(val[x]) < INFINITY);
      }
      if (__builtin_amdgcn_ballot_w64(odd) == 0) continue;
      float s = 0.f;
      if (there)
#pragma unroll 1
        for (int ch = 0; ch < D; ++ch) {
          const float qv = TYPE == kTypeBf16 ? __uint_as_float((unsigned)((const uint16_t*)q)[ch] << 16) : ((const float*)q)[ch];
          s = fmaf(qv, cached_value<TYPE, Q8>(c.k, c.k_scale, at, scale_at, ch), s);
        }
      const float w = __builtin_amdgcn_exp2f(fmaf(s, a.scale_log2e, less));
      const bool sees = pos < seen.end_of(p) && (pos >= seen.begin_of(p) || pos < seen.sinks);
#pragma unroll 1
      for (int x = 0; x < 16 * RT; ++x) {
        const float weight = __shfl(w, x);
        if (!__shfl((int)sees, x)) continue;
#pragma unroll
        for (int y = 0; y < D / 64; ++y)
          if (!(fabsf(val[y]) < INFINITY)) sums[x * D + 64 * y + lane] += weight * val[y];
      }
    }
  }
}

// The sums of a wave (o: channels 16 c + 4 g + v of row 16 b + i, lane 16 g + i) through LDS and back, for add_odd().
template <int D, int RT>
__device__ __forceinline__ void sums_to_lds(const f32x4 (&o)[RT][D / 16], float* sums) {
  const int i = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
#pragma unroll
  for (int b = 0; b < RT; ++b)
#pragma unroll
    for (int x = 0; x < D / 16; ++x) *(f32x4*)(sums + (16 * b + i) * D + 16 * x + 4 * g) = o[b][x];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the wave's own stores have landed
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
template <int D, int RT>
__device__ __forceinline__ void sums_from_lds(f32x4 (&o)[RT][D / 16], const float* sums) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const int i = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
#pragma unroll
  for (int b = 0; b < RT; ++b)
#pragma unroll
    for (int x = 0; x < D / 16; ++x) o[b][x] = *(const f32x4*)(sums + (16 * b + i) * D + 16 * x + 4 * g);
}

}  // namespace scalekv
