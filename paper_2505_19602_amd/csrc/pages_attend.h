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
  int n_seq, group, rows, target, min_tiles;
  float scale_log2e, no_max;
  // workspace (target > 0): sums [workgroup][part_rows][D], their {offset in log2 units, sum of weights}, {first workgroup,
  // cuts} of each sequence
  float *part, *stat;
  int2* cuts;
  int part_rows;
};

// bf16, many query rows (pages_chunk.hip): 64 row_tiles rows to a workgroup
hipError_t launch_pages_chunk(int d, bool q8, int row_tiles, const AttendArgs& a, int n_wg, hipStream_t stream);

// Sum over the lanes of a wave, in all of them; sum over the lanes up to one's own.  (DPP: shifts within rows of 16 lanes,
// then the last lane of a row, and of the lower half, to those behind it.)
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_add(unsigned x) {
  return x + (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ unsigned wave_scan(unsigned x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  return dpp_add<0x143, 0xc>(x);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double x) {
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, x);
  const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)bits, CTRL, ROWS, 0xf, false);
  const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(bits >> 32), CTRL, ROWS, 0xf, false);
  return x + __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double x) {
  x = dpp_add<0x111, 0xf>(x);
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);
  x = dpp_add<0x143, 0xc>(x);
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, x);
  const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)bits, 63);
  const unsigned hi = __builtin_amdgcn_readlane((int)(unsigned)(bits >> 32), 63);
  return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}

// What a workgroup works on.  The lengths of the sequences are known to the device alone, and may differ by any factor: every
// workgroup adds up the work of all of them (tiles times row groups) and finds its own place.  A sequence's
// keys are cut into as many parts as it has multiples of `most` tiles, the work of all sequences over `target` workgroups
// (and at least min_tiles), so that a long sequence does not outlast the others, and short ones are not cut.
struct Slice {
  int seq, kv, row_group, cut, cuts;  // cuts 0: nothing
  int first_wg;                       // of the sequence
  int len, count;                     // cached rows and new tokens of the sequence
};
struct Cutter {
  const AttendArgs& a;
  int tile;   // keys of a tile
  int most;   // tiles to a workgroup
  __device__ __forceinline__ int groups(int count) const { return (count * a.group + a.rows - 1) / a.rows; }
  __device__ __forceinline__ int tiles(int len) const {
    const int all = (len + tile - 1) / tile;
    if (a.mask.window == 0 || !a.mask.causal) return all;
    const int tokens = min(a.chunk.max_new, a.rows / a.group + 1);
    return min(all, (min(a.mask.n_sink, 1 << 29) + tile - 1) / tile + (min(a.mask.window, 1 << 29) + tokens) / tile + 1);
  }
  __device__ __forceinline__ double work(int len, int count) const { return (double)groups(count) * tiles(len); }
  __device__ __forceinline__ void share(double all) {
    if (a.target) most = max(a.min_tiles, (int)min(ceil(all * a.c.n_kv_head / a.target), 1e9));
  }
  __device__ __forceinline__ int cuts(int len) const { return a.target ? max((tiles(len) + most - 1) / most, 1) : 1; }
  __device__ __forceinline__ unsigned workgroups(int len, int count) const {
    return (unsigned)(groups(count) * cuts(len)) * a.c.n_kv_head;
  }
};
template <int TN>
__device__ __forceinline__ Slice slice_of(const AttendArgs& a, unsigned wg) {
  Cutter cutter{a, TN, 1};
  const int lane = threadIdx.x & 63;
  Slice s{};
  unsigned first = 0;
  auto len_of = [&](int seq) { return pages_len(a.c, seq); };
  auto count_of = [&](int seq) { return chunk_count(a.chunk, seq); };
  if (a.n_seq == 1) {
    s.len = __builtin_amdgcn_readfirstlane(len_of(0));
    s.count = __builtin_amdgcn_readfirstlane(count_of(0));
    cutter.share(cutter.work(s.len, s.count));
    if (wg >= cutter.workgroups(s.len, s.count)) return s;
  } else if (a.n_seq <= 64) {  // a sequence to a lane, each read once
    const int len = lane < a.n_seq ? len_of(lane) : 0, count = lane < a.n_seq ? count_of(lane) : 0;
    if (a.target) cutter.share(wave_sum(cutter.work(len, count)));
    const unsigned mine = cutter.workgroups(len, count), upto = wave_scan(mine);
    const unsigned long long found = __builtin_amdgcn_ballot_w64(upto > wg);  // this lane's sequence or earlier ones
    if (found == 0) return s;
    s.seq = __builtin_ctzll(found);
    first = __builtin_amdgcn_readlane((int)(upto - mine), s.seq);
    s.len = __builtin_amdgcn_readlane(len, s.seq);
    s.count = __builtin_amdgcn_readlane(count, s.seq);
  } else {
    // Each lane walks its share of the sequences, in every workgroup: work that grows with the square of their number.  Single
    // tokens over 100 rows each, e4m3, 8 KV heads: 65 / 256 / 1024 / 2000 sequences 10.7 / 29 / 184 / 559 us, with the lengths as
    // constants 10.3 / 25 / 92 / 172; over 600 rows 25 / 81 / 345 (23 / 76 / 273) us for 65 / 256 / 1024.
    const int per_lane = (a.n_seq + 63) / 64, from = lane * per_lane, to = min(from + per_lane, a.n_seq);
    if (a.target) {
      double work = 0;
      for (int x = from; x < to; ++x) work += cutter.work(len_of(x), count_of(x));
      cutter.share(wave_sum(work));
    }
    unsigned mine = 0;
    for (int x = from; x < to; ++x) mine += cutter.workgroups(len_of(x), count_of(x));
    const unsigned upto = wave_scan(mine);
    const unsigned long long found = __builtin_amdgcn_ballot_w64(upto > wg);
    if (found == 0) return s;
    const int at = __builtin_ctzll(found);
    first = __builtin_amdgcn_readlane((int)(upto - mine), at);
    s.seq = at * per_lane;
    // (the bound holds even if lengths are changed under the call)
    for (unsigned n; s.seq + 1 < a.n_seq && wg >= first + (n = cutter.workgroups(len_of(s.seq), count_of(s.seq))); ++s.seq)
      first += n;
    s.seq = __builtin_amdgcn_readfirstlane(s.seq);
    first = __builtin_amdgcn_readfirstlane(first);
    s.len = __builtin_amdgcn_readfirstlane(len_of(s.seq));
    s.count = __builtin_amdgcn_readfirstlane(count_of(s.seq));
  }
  s.first_wg = (int)first;
  s.cuts = __builtin_amdgcn_readfirstlane(cutter.cuts(s.len));
  const int n_group = cutter.groups(s.count), per = n_group * s.cuts;
  // Eight heads at a time, dealt out in turn: consecutive workgroups go round-robin over the XCDs, so that the workgroups
  // of a head share an L2.
  const int heads = a.c.n_kv_head, dealt = heads / kXcds * kXcds;
  int j = (int)(wg - first), rest;
  if (j < dealt * per) {
    const int round = j / (kXcds * per);
    j -= round * kXcds * per;
    s.kv = round * kXcds + j % kXcds;
    rest = j / kXcds;
  } else {
    j -= dealt * per;
    s.kv = dealt + j % (heads - dealt);
    rest = j / (heads - dealt);
  }
  s.cut = rest % s.cuts;
  // under a causal mask later rows see more: they come first, so that the short ones fill up the end
  const int nth = rest / s.cuts;
  s.row_group = a.mask.causal ? n_group - 1 - nth : nth;
  if (a.target && wg == first && threadIdx.x == 0) a.cuts[s.seq] = make_int2(s.first_wg, s.cuts);
  return s;
}
// The workgroup of a part, from what slice_of() has left in the workspace: its inverse.
__device__ __forceinline__ int workgroup_of(const AttendArgs& a, int first_wg, int cuts, int n_group, int kv, int row_group,
                                            int cut) {
  const int heads = a.c.n_kv_head, dealt = heads / kXcds * kXcds, per = n_group * cuts;
  const int rest = (a.mask.causal ? n_group - 1 - row_group : row_group) * cuts + cut;
  return first_wg + (kv < dealt ? kv / kXcds * (kXcds * per) + rest * kXcds + kv % kXcds
                                : dealt * per + rest * (heads - dealt) + (kv - dealt));
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
  __device__ __forceinline__ Seen(const AttendArgs& a, const Slice& slice, int first_row, int rows) {
    len = slice.len;  // (all of this is the same in every lane: scalars)
    count = slice.count;
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
// that the wave has worked on, whose offsets are no lower than their logits.  Rare, and written to be short: the logits are
// formed anew, a channel at a time.
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

// Sixteen rows of a wave's sums (o: channels 16 c + 4 g + v of row i, lane 16 g + i) through LDS and back, for add_odd().
__device__ __forceinline__ void own_lds() {  // the wave's own stores have landed
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
template <int D>
__device__ __forceinline__ void sums_to_lds(const f32x4 (&o)[D / 16], float* sums) {
  const int i = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) *(f32x4*)(sums + i * D + 16 * x + 4 * g) = o[x];
  own_lds();
}
template <int D>
__device__ __forceinline__ void sums_from_lds(f32x4 (&o)[D / 16], const float* sums) {
  own_lds();
  const int i = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) o[x] = *(const f32x4*)(sums + i * D + 16 * x + 4 * g);
}

}  // namespace scalekv
