// Attention of a chunk of new tokens over a paged cache (bf16, fp32, or e4m3 with a power-of-two scale to each row), with
// a causal mask, a sliding window and first rows that stay visible.
//
// out_t = sum_j softmax_j(q_t . k_j * sm_scale) v_j over the rows j that token t sees, in one pass over the keys with the
// running maximum and sum of the softmax.  The query rows of a workgroup are those of ONE KV head, (token, query head of
// the group) in this order, so that the heads that share a row of the cache read it together: a single token of a group of
// eight heads is eight rows.
//
// Here: up to 16 rows to a workgroup (single tokens, short chunks), and fp32; many rows of bf16 are pages_chunk.hip's.
//
// Products, transposed as in the dense kernels: S^T[key][row] = K Q^T with K from LDS and Q in registers, O^T[channel][row]
// += V^T P^T with V^T from LDS and P^T in the registers that the first product left it in; a lane owns a query row, its
// softmax statistics are scalars of the lane.  bf16: MFMA 16x16x32, blocks of 32 keys, key order and LDS swizzle as in
// attend_pipe.hip.  fp32: MFMA 16x16x4, blocks of 16 keys.
//
// Tiles.  All waves bring in a tile of keys: whole rows, 16 bytes a lane, through registers into LDS, where e4m3 becomes
// what the products take (exactly: four significant bits and a power of two), rows that no query row of the workgroup sees
// become zeros, and the rows of the tile after it are requested before this one is worked on, their pages' numbers one
// tile earlier still.  Waves split the blocks of a tile and join their results through LDS (fp32 with many rows: they split
// the rows).  Where that leaves the chip idle the keys are split over workgroups as well; their results go to the
// workspace, and pages_join_kernel adds them up.  A workgroup walks the tiles that its rows can see: those of the first
// rows, then those from the window's first row on.
//
// What bounds it.  Few rows: HBM, each cached row being read once.  8 KV heads, head_dim 128, one token of 4 heads each: 64
// sequences x 8000 rows bf16 352 us (6.0 TB/s), e4m3 190 us (5.6 TB/s); 2 x 131072 rows bf16 200 us (5.4 TB/s; fp32 378, 5.7 TB/s),
// e4m3 113 us; 64 sequences of up to 4000 rows e4m3 78 us (3.7 TB/s: the shortest workgroups are all start and end), bf16 130 us
// (4.4 TB/s), fp32 281 us (4.1 TB/s), fp32 over e4m3 224 us.  Small calls: the chain length -> table -> rows -> products, and the
// join's launch: one sequence of 700 rows 10 us.  fp32, many rows: 24 units x 2048 causal tokens, head_dim 128, 409 us (63 TFLOP/s;
// the dense fp32 kernel 104, a large product 154; over e4m3 415 us).  It is a chain, not a pipe, that bounds this: the matrix
// pipe is busy for 46 % of the cycles, the LDS for 12 %, and waves wait 61 % of their time for an instruction to finish.
//
// Masked keys.  A weight of zero does not hide a value that is infinite or NaN from the product.  Rows hidden from all rows
// of the workgroup are zeros in LDS; in the few tiles that some of its rows see and others do not (`edge`), values that
// are not finite are taken out of the tile, remembered, and added for the rows that do see them (`add_odd`).
#include <type_traits>

#include "pages_attend.h"

namespace scalekv {
namespace {

constexpr int kThreads = 256;

// TYPE: of queries, output and arithmetic; WQ: waves that split the query rows, 16 to each.
template <int TYPE, bool Q8, int D, int WQ>
struct Form {
  static_assert(TYPE == kTypeF32 || WQ == 1, "many rows of bf16 are pages_chunk.hip's");
  static constexpr bool kBf16 = TYPE == kTypeBf16;
  static constexpr int kElem = kBf16 ? 2 : 4;
  static constexpr int WK = 4 / WQ;                      // waves that split the keys of a tile
  static constexpr int kBlock = kBf16 ? 32 : 16;         // keys of a block
  static constexpr int kBlocks = WK > 1 ? 1 : 4;         // blocks of a tile to a wave
  static constexpr int TN = kBlock * kBlocks * WK;       // keys of a tile
  static constexpr int kKeyTiles = kBlock / 16;
  static constexpr int kRowBytes = D * kElem;            // in LDS
  static constexpr int kTileBytes = TN * kRowBytes;
  // Keys in LDS as codes, widened where a wave takes them: only that wave does, and three workgroups fit a compute unit
  // instead of two (with cuts by the work of all sequences, 16 units x 131072 rows e4m3 160 -> 113 us)
  static constexpr bool kKeyCodes = kBf16 && Q8;
  static constexpr int kKeyTileBytes = kKeyCodes ? TN * D : kTileBytes;
  static constexpr int kSlabs = kRowBytes / 64;          // 16-byte operands of a query row that a lane holds
  static constexpr int kChans = D / 16;                  // 16-channel blocks of the output
  static constexpr int kSrcRow = Q8 ? D : kRowBytes;     // bytes of a cached row
  static constexpr int kSrcChunks = kSrcRow / 16;
  static constexpr int kVecs = TN * kSrcChunks / kThreads;  // 16-byte vectors of a tile of K, or of V, to a thread
  static constexpr int kRows = 16 * WQ;                  // query rows of a workgroup
  static constexpr int kWavesPerSimd = kKeyCodes ? 3 : 2;
  static constexpr int kJoinBytes = WK > 1 ? (WK - 1) * 64 * (kChans * 16 + 8) : 0;
  static constexpr int kSumBytes = 4 * 16 * D * 4;  // of all waves, for add_odd()
  static constexpr int kTilesBytes = kKeyTileBytes + kTileBytes;
  static constexpr int kLds = kTilesBytes > kJoinBytes ? kTilesBytes > kSumBytes ? kTilesBytes : kSumBytes
                                                       : kJoinBytes > kSumBytes ? kJoinBytes : kSumBytes;
  __device__ static constexpr int k_flip(int r) { return kBf16 ? k_flip_bf16<D>(r) : r & 15; }
  __device__ static constexpr int v_flip(int r) { return kBf16 ? v_flip_bf16<D>(r) : r & 15; }
  // rows of codes: the sixteen rows that lanes read eight codes of at a time differ in bits 0, 1, 3 and 4; with rows of 128
  // bytes bit 0 already tells the halves of the banks apart, with rows of 64 bytes bits 0 and 1 the quarters
  __device__ static constexpr int code_flip(int r) {
    return D == 128 ? (r >> 1 & 1) | (r >> 3 & 1) << 1 | (r >> 4 & 1) << 2 : (r >> 3 & 1) | (r >> 4 & 1) << 1;
  }
};

template <int TYPE, bool Q8, int D, int WQ>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(Form<TYPE, Q8, D, WQ>::kWavesPerSimd)))
void pages_attend_kernel(AttendArgs a) {
  using F = Form<TYPE, Q8, D, WQ>;
  constexpr bool BF16 = F::kBf16;
  constexpr int TN = F::TN, KT = F::kKeyTiles, NSL = F::kSlabs, NCB = F::kChans, NV = F::kVecs;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  __shared__ int any_odd;  // values that are not finite have been taken out of a tile
  __shared__ uint8_t key_scale[F::kKeyCodes ? TN : 1];
  const PagesView& c = a.c;

  // ---- which query rows, which tiles
  const int wg = SCALEKV_WG_X;
  const Slice slice = slice_of<TN>(a, wg);
  if (slice.cuts == 0) return;
  const int seq = slice.seq, kv = slice.kv;
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wq = wave % WQ, wk = wave / WQ;
  const int first_row = slice.row_group * F::kRows, wave_row = first_row + wq * 16;
  const Seen<TN> seen(a, slice, first_row, F::kRows);
  const int n_rows = seen.n_rows, pos0 = seen.pos0, sinks = seen.sinks;
  const int per = (seen.n_tile + slice.cuts - 1) / slice.cuts;
  const int t0 = min(slice.cut * per, seen.n_tile), t1 = min(t0 + per, seen.n_tile);

  // ---- the query rows of this lane
  const int q_row = min(wave_row + i, n_rows - 1);
  int q_end, q_begin;
  u32x4 qf[NSL];
  {
    const int t = q_row / a.group, head = kv * a.group + (q_row - t * a.group);
    q_end = seen.end_of(pos0 + t);
    q_begin = seen.begin_of(pos0 + t);
    const long long at = (long long)chunk_first(a.chunk, seq) + t;
    const u32x4* src = (const u32x4*)(a.q.p + seq * a.q.seq + head * a.q.head + at * a.q.row);
    const bool there = at >= 0 && at < a.q.n_row;
#pragma unroll
    for (int sl = 0; sl < NSL; ++sl) qf[sl] = there ? src[4 * sl + g] : u32x4{0, 0, 0, 0};
  }
  // what all rows of the wave see: [begin, end) and the first `sinks`
  const int w_end = seen.end_of(pos0 + min(wave_row, n_rows - 1) / a.group);
  const int w_begin = seen.begin_of(pos0 + min(wave_row + 15, n_rows - 1) / a.group);

  // ---- tiles: a thread's vectors of a tile lie kThreads vectors apart
  int page[NV];
  u32x4 kr[NV], vr[NV];
  uint8_t ks[NV], vs[NV];
  const int ld_row = tid / F::kSrcChunks, ld_chunk = tid % F::kSrcChunks;
  constexpr int kRowsApart = kThreads / F::kSrcChunks;
  const int32_t* const table = c.table + (long long)seq * c.width;
  const long long kv_ofs = kv * c.head, kv_scale = kv * c.scale_head;
  auto ask_pages = [&](int t) __attribute__((always_inline)) {
    const int key0 = seen.key0(t);
#pragma unroll
    for (int p = 0; p < NV; ++p) {
      const int pos = key0 + ld_row + p * kRowsApart;
      page[p] = -1;
      if (t < t1 && seen.some(pos)) page[p] = table[pos >> c.page_shift];
    }
  };
  auto ask_rows = [&](int t) __attribute__((always_inline)) {
    const int key0 = seen.key0(t);
#pragma unroll
    for (int p = 0; p < NV; ++p) {
      const int slot = (key0 + ld_row + p * kRowsApart) & ((1 << c.page_shift) - 1);
      kr[p] = vr[p] = u32x4{0, 0, 0, 0};
      ks[p] = vs[p] = 127;
      if ((unsigned)page[p] < (unsigned)c.n_page) {
        const long long at = page[p] * c.page + kv_ofs + slot * F::kSrcRow + 16 * ld_chunk;
        kr[p] = *(const u32x4*)(c.k + at);
        vr[p] = *(const u32x4*)(c.v + at);
        if constexpr (Q8) {
          const long long scale_at = page[p] * c.scale_page + kv_scale + slot;
          ks[p] = c.k_scale[scale_at];
          vs[p] = c.v_scale[scale_at];
        }
      }
    }
  };
  unsigned char* const k_lds = smem;
  unsigned char* const v_lds = smem + F::kKeyTileBytes;
  auto store_rows = [&](int t) __attribute__((always_inline)) {
    const bool edge = seen.edge(t);
    constexpr int kOut = Q8 ? F::kElem : 1;  // vectors in LDS for one of the cache
#pragma unroll
    for (int p = 0; p < NV; ++p) {
      const int row = ld_row + p * kRowsApart;
      u32x4 x[kOut], y[kOut];
      if constexpr (Q8) {
        if constexpr (F::kKeyCodes) {
          *(u32x4*)(k_lds + row * D + 16 * (ld_chunk ^ F::code_flip(row))) = kr[p];
          if (ld_chunk == 0) key_scale[row] = ks[p];
        } else {
          widen(kr[p], __uint_as_float((unsigned)ks[p] << 23), x);
        }
        widen(vr[p], __uint_as_float((unsigned)vs[p] << 23), y);
      } else {
        x[0] = kr[p];
        y[0] = vr[p];
      }
      if (edge) {
        bool odd = false;
#pragma unroll
        for (int w = 0; w < kOut; ++w) odd |= take_odd<BF16>(y[w]);
        if (odd) any_odd = 1;
      }
#pragma unroll
      for (int w = 0; w < kOut; ++w) {
        const int chunk = ld_chunk * kOut + w;
        if constexpr (!F::kKeyCodes) *(u32x4*)(k_lds + row * F::kRowBytes + 16 * (chunk ^ F::k_flip(row))) = x[w];
        *(u32x4*)(v_lds + row * F::kRowBytes + 16 * (chunk ^ F::v_flip(row))) = y[w];
      }
    }
  };

  // ---- state of the rows
  f32x4 o[NCB];
  // Less the offset of a row, its largest logit in log2 units (the same in the four lanes of a row), and this lane's share of
  // the sum.  The offset is kept as it has been rounded: factors between offsets are then exactly those between the weights
  // (formed from the logits anew they are off by the rounding of the product, 2^-24 of its magnitude).
  float neg = -(a.no_max * a.scale_log2e), l_run = 0.f;
#pragma unroll
  for (int x = 0; x < NCB; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  // key of register v of key tile t, in a block
  auto key_of = [&](int t, int v) { return BF16 ? 16 * (g & 1) + 8 * (g >> 1) + 4 * t + v : 4 * g + v; };

  auto work = [&](int t) __attribute__((always_inline)) {
    const int key0 = seen.key0(t);
    const bool masked = key0 + TN > w_end || (seen.window && key0 < w_begin && key0 + TN > sinks);
#pragma unroll 1  // (blocks side by side spill registers)
    for (int nb = 0; nb < F::kBlocks; ++nb) {
      const int block = wk * F::kBlocks + nb;
      const unsigned char* const kb = k_lds + block * F::kBlock * (F::kKeyCodes ? D : F::kRowBytes);
      const unsigned char* const vb = v_lds + block * F::kBlock * F::kRowBytes;
      f32x4 s[KT];
#pragma unroll
      for (int x = 0; x < KT; ++x) {
        const int row = BF16 ? 16 * (i >> 2 & 1) + 8 * (i >> 3) + (i & 3) + 4 * x : i;
        u32x4 kf[NSL];
#pragma unroll
        for (int sl = 0; sl < NSL; ++sl) {
          if constexpr (F::kKeyCodes) {
            const uint2 codes = *(const uint2*)(kb + row * D + 16 * ((2 * sl + g / 2) ^ F::code_flip(row)) + 8 * (g & 1));
            const float scale = __uint_as_float((unsigned)key_scale[block * F::kBlock + row] << 23);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const unsigned four = e < 2 ? codes.x : codes.y;
              const bf16x2 two = e & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, true)
                                       : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, false);
              kf[sl][e] = __builtin_bit_cast(unsigned, two);
            }
          } else {
            kf[sl] = *(const u32x4*)(kb + row * F::kRowBytes + 16 * ((4 * sl + g) ^ F::k_flip(row)));
          }
        }
        if constexpr (BF16) {
          s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int sl = 0; sl < NSL; ++sl)
            s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[sl]),
                                                           __builtin_bit_cast(bf16x8, qf[sl]), s[x], 0, 0, 0);
        } else {
          // four sums of every fourth channel: shorter chains, of instructions and of roundings
          f32x4 sum[4];
#pragma unroll
          for (int sl = 0; sl < NSL; ++sl)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sum[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[sl][e]), __uint_as_float(qf[sl][e]),
                                                            sl ? sum[e] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
          s[x] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
      }
      if (masked) {
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int pos = key0 + block * F::kBlock + key_of(x, v);
            if (pos >= q_end || (pos < q_begin && pos >= sinks)) s[x][v] = -INFINITY;
          }
      }
      // Running maximum, moved only where it has grown by more than kRescaleThreshold; in fp32 wherever it has grown, so that
      // the exponents of the weights that count are small, and with them the rounding of an exponent.
      float mx = s[0][0];
#pragma unroll
      for (int y = 1; y < 4 * KT; ++y) mx = fmaxf(mx, s[y / 4][y % 4]);
      mx = xor32_max(xor16_max(mx));
      if (__builtin_amdgcn_ballot_w64(fmaf(mx, a.scale_log2e, neg) > (BF16 ? kRescaleThreshold : 0.f)) != 0) {
        const float now = fminf(neg, -(mx * a.scale_log2e)), alpha = __builtin_amdgcn_exp2f(now - neg);
        neg = now;
        l_run *= alpha;
#pragma unroll
        for (int x = 0; x < NCB; ++x) o[x] *= alpha;
      }
      float w[4 * KT];
      u32x4 p;
#pragma unroll
      for (int y = 0; y < 4 * KT; ++y) w[y] = __builtin_amdgcn_exp2f(fmaf(s[y / 4][y % 4], a.scale_log2e, neg));
      if constexpr (BF16) {
        // (weights are rounded to bf16 for the matrix cores; the sum adds the rounded ones)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const bf16x2 two = {(__bf16)w[2 * y], (__bf16)w[2 * y + 1]}, ones = {(__bf16)1.f, (__bf16)1.f};
          l_run = __builtin_amdgcn_fdot2_f32_bf16(two, ones, l_run, false);
          p[y] = __builtin_bit_cast(unsigned, two);
        }
      } else {
#pragma unroll
        for (int y = 0; y < 4 * KT; ++y) l_run += w[y];
      }
#pragma unroll
      for (int ch = 0; ch < NCB; ++ch) {
        if constexpr (BF16) {
          typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
          const int row = 16 * (g & 1) + 8 * (g >> 1) + (i >> 2);
          const unsigned char* const at = vb + row * F::kRowBytes + 16 * (2 * ch ^ F::v_flip(row)) + 8 * (i & 3);
          const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
          const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * F::kRowBytes));
          const bf16x8 vt = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
          o[ch] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, p), o[ch], 0, 0, 0);
        } else {
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int row = 4 * g + v;
            const int chunk = (4 * ch + (i >> 2)) ^ F::v_flip(row);
            const float val = *(const float*)(vb + row * F::kRowBytes + 16 * chunk + 4 * (i & 3));
            o[ch] = __builtin_amdgcn_mfma_f32_16x16x4f32(val, w[v], o[ch], 0, 0, 0);
          }
        }
      }
    }
  };

  // ---- the tiles
  if (tid == 0) any_odd = 0;
  if (t0 < t1) {
    ask_pages(t0);
    ask_rows(t0);
    ask_pages(t0 + 1);
    __syncthreads();
    store_rows(t0);
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
      if (t + 1 < t1) {
        ask_rows(t + 1);
        ask_pages(t + 2);
      }
      if (wave_row < n_rows) work(t);  // (the others only carry their share of the tiles)
      __syncthreads();
      if (t + 1 < t1) store_rows(t + 1);
      __syncthreads();
    }
    if (any_odd && wave_row < n_rows) {
      float* const sums = (float*)smem + wave * (16 * D);
      sums_to_lds<D>(o, sums);
      constexpr int kMine = F::kBlocks * F::kBlock;
      const float less[1] = {neg};
      add_odd<TYPE, Q8, D, TN, 1>(a, seen, seq, kv, wave_row, t0, t1, wk * kMine, (wk + 1) * kMine, less, sums);
      sums_from_lds<D>(o, sums);
    }
  }

  // ---- join the waves that have split the keys: a common maximum, then the sums
  l_run = xor32_sum(xor16_sum(l_run));
  if constexpr (F::WK > 1) {
    f32x4* const part = (f32x4*)smem;                                  // [wave - 1][channel block][lane]
    float* const stat = (float*)(smem + (F::WK - 1) * NCB * 64 * 16);  // [wave - 1][2][lane]
    __syncthreads();
    if (wk > 0) {
#pragma unroll
      for (int ch = 0; ch < NCB; ++ch) part[((wk - 1) * NCB + ch) * 64 + lane] = o[ch];
      stat[(wk - 1) * 128 + lane] = neg;
      stat[(wk - 1) * 128 + 64 + lane] = l_run;
    }
    __syncthreads();
    if (wk > 0) return;
    float now = neg;
#pragma unroll
    for (int x = 0; x < F::WK - 1; ++x) now = fminf(now, stat[x * 128 + lane]);
    const float own = __builtin_amdgcn_exp2f(now - neg);
    l_run *= own;
#pragma unroll
    for (int ch = 0; ch < NCB; ++ch) o[ch] *= own;
#pragma unroll
    for (int x = 0; x < F::WK - 1; ++x) {
      const float f = __builtin_amdgcn_exp2f(now - stat[x * 128 + lane]);
      l_run += f * stat[x * 128 + 64 + lane];
#pragma unroll
      for (int ch = 0; ch < NCB; ++ch) o[ch] += f * part[(x * NCB + ch) * 64 + lane];
    }
    neg = now;
  }

  // ---- write
  if (wave_row + i >= n_rows) return;
  if (slice.cuts > 1) {
    const long long row = (long long)wg * a.part_rows + (q_row - first_row);
    if (g == 0) {
      a.stat[2 * row] = -neg;
      a.stat[2 * row + 1] = l_run;
    }
#pragma unroll
    for (int ch = 0; ch < NCB; ++ch) *(f32x4*)(a.part + row * D + 16 * ch + 4 * g) = o[ch];
    return;
  }
  const int t = q_row / a.group, head = kv * a.group + (q_row - t * a.group);
  const long long at = (long long)chunk_first(a.chunk, seq) + t;
  if (at < 0 || at >= a.out.n_row) return;
  // a row that sees nothing, or keys of weight zero only, is zero
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  unsigned char* const dst = a.out.p + seq * a.out.seq + head * a.out.head + at * a.out.row;
#pragma unroll
  for (int ch = 0; ch < NCB; ++ch) {
    const f32x4 x = l_run == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[ch] * inv;
    if constexpr (BF16) {
      const bf16x2 lo2 = {(__bf16)x[0], (__bf16)x[1]}, hi2 = {(__bf16)x[2], (__bf16)x[3]};
      *(uint2*)(dst + 32 * ch + 8 * g) = make_uint2(__builtin_bit_cast(unsigned, lo2), __builtin_bit_cast(unsigned, hi2));
    } else {
      *(f32x4*)(dst + 64 * ch + 16 * g) = x;
    }
  }
}

// Adds up what the workgroups of a row group have left: a wave to a row, D / 64 channels to a lane.  A workgroup has
// kJoinRows rows of one row group (most launches find little to do: keys are cut for long sequences alone).
constexpr int kJoinRows = 32;
template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void pages_join_kernel(AttendArgs a, int n_row_group, int join_groups) {
  constexpr int kPer = D / 64;
  const int wg = SCALEKV_WG_X, part_of = wg % join_groups, row_group = wg / join_groups % n_row_group;
  const int unit = wg / join_groups / n_row_group, seq = unit / a.c.n_kv_head, kv = unit - seq * a.c.n_kv_head;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n_rows = __builtin_amdgcn_readfirstlane(chunk_count(a.chunk, seq)) * a.group;
  const int first_row = row_group * a.rows;
  if (first_row >= n_rows) return;
  const int2 cut = a.cuts[seq];
  const int cuts = __builtin_amdgcn_readfirstlane(cut.y);
  if (cuts < 2) return;  // written already
  const int n_group = (n_rows + a.rows - 1) / a.rows;
  const int wg0 = workgroup_of(a, __builtin_amdgcn_readfirstlane(cut.x), cuts, n_group, kv, row_group, 0);
  const long long rows_apart =
      (long long)(workgroup_of(a, __builtin_amdgcn_readfirstlane(cut.x), cuts, n_group, kv, row_group, 1) - wg0) * a.part_rows;
  const int end = min(min(first_row + a.rows, n_rows), first_row + (part_of + 1) * kJoinRows);
  for (int r = first_row + part_of * kJoinRows + wave; r < end; r += kThreads / 64) {
    const int t = r / a.group, head = kv * a.group + (r - t * a.group);
    const long long at = (long long)chunk_first(a.chunk, seq) + t;
    if (at < 0 || at >= a.out.n_row) continue;
    const long long row0 = (long long)wg0 * a.part_rows + (r - first_row);
    const float* const part = a.part + row0 * D + kPer * lane;
    const float* const stat = a.stat + 2 * row0;
    float top = -INFINITY;
#pragma unroll 4
    for (int x = 0; x < cuts; ++x) top = fmaxf(top, stat[2 * x * rows_apart]);
    float sum = 0.f, o[kPer] = {};
#pragma unroll 4
    for (int x = 0; x < cuts; ++x) {  // (a part without keys has sums of zero, at an offset far below all others)
      const float f = __builtin_amdgcn_exp2f(stat[2 * x * rows_apart] - top);
      sum += f * stat[2 * x * rows_apart + 1];
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] += f * part[x * rows_apart * D + e];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    unsigned char* const dst = a.out.p + seq * a.out.seq + head * a.out.head + at * a.out.row;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const float y = sum == 0.f ? 0.f : o[e] * inv;
      if constexpr (TYPE == kTypeBf16) ((__bf16*)dst)[kPer * lane + e] = (__bf16)y;
      else ((float*)dst)[kPer * lane + e] = y;
    }
  }
}

template <int TYPE, bool Q8, int D, int WQ>
hipError_t launch_form(const AttendArgs& a, int n_wg, hipStream_t stream) {
  using F = Form<TYPE, Q8, D, WQ>;
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_dynamic_lds((const void*)pages_attend_kernel<TYPE, Q8, D, WQ>, F::kLds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((pages_attend_kernel<TYPE, Q8, D, WQ>), dim3(n_wg), dim3(kThreads), F::kLds, stream, a);
  return hipGetLastError();
}

template <int TYPE, bool Q8, int D>
hipError_t launch_plan(const PagesPlan& plan, const AttendArgs& a, hipStream_t stream) {
  if constexpr (TYPE == kTypeBf16) {
    if (plan.row_waves == 4) return launch_pages_chunk(D, Q8, plan.row_tiles, a, plan.n_wg, stream);
    return launch_form<TYPE, Q8, D, 1>(a, plan.n_wg, stream);
  } else {
    return plan.row_waves == 4 ? launch_form<TYPE, Q8, D, 4>(a, plan.n_wg, stream)
                               : launch_form<TYPE, Q8, D, 1>(a, plan.n_wg, stream);
  }
}

}  // namespace

PagesPlan pages_plan(int dtype, int d, int n_seq, int n_head, const PagesView& pages, int max_new, const MaskView& mask) {
  constexpr int kComputeUnits = 256;
  const int rows = max_new * (n_head / pages.n_kv_head);
  PagesPlan p{};
  // keys that a row group can see at most
  const long long cap = (long long)pages.width << pages.page_shift;
  long long keys = cap;
  if (mask.window > 0 && mask.causal) {
    const long long seen = (long long)mask.n_sink + mask.window + max_new;
    keys = seen < cap ? seen : cap;
  }
  // Rows of a workgroup.  Keys that 64 or 128 rows share are read once for them and their products fill the matrix cores; 16
  // rows leave more workgroups, whose waves split the keys.  A form is taken for units of more than `over` rows.  us with 16 /
  // 64 / 128 rows to a workgroup, 128 units x 2000 rows of the cache, head_dim 128: bf16, units of 4 rows 29 / 29 / 35, 16 rows 37 /
  // 33 / 39, 32 rows 40 / 38 / 44, 64 rows 53 / 40 / 46, 128 rows 100 / 48 / 50, 256 rows 189 / 78 / 65; e4m3, 32 rows 33 / 45 / 52,
  // 48 rows 38 / 46 / 54, 64 rows 45 / 46 / 54, 80 rows 55 / 54 / 56, 128 rows 76 / 56 / 57, 256 rows 127 / 95 / 70.  With few units
  // the form of 16 rows, which has the shortest start, is ahead for longer: 16 units x 2000, 4 rows 12.5 / 25 / 33, 16 rows 19 /
  // 28 / 36, 32 rows 21 / 33 / 41, e4m3 64 rows 28 / 43 / 51.  A line of `over` is one number between the two: beside it the form
  // that is taken is up to 12 % behind (bf16 16 rows in many units), more often 4 %.  fp32, 16 / 64 rows, head_dim 64: 192 units x
  // 2000 rows, 32 rows 68 / 121, 64 rows 105 / 125, 80 rows 153 / 158, 100 rows 192 / 162, 145 rows 253 / 260 (both forms step with
  // the row groups that they fill), 256 rows 358 / 295; 96 units of 1024 rows x 4000 1232 / 1009.
  // Fewer rows, too, where compute units would be left without work and the keys, in pieces of min_tiles tiles, do not give
  // them any: bf16, 16 units x 6000 rows, 32 rows 27 / 36 / 44, 256 rows 72 / 44 / 48; fp32, where only rows count: 24 units of
  // 145 rows x 585 20 / 44.
  // Lengths are not known here: pieces of keys are counted up to the table's width.  Sequences far shorter than their table get
  // more rows to a workgroup than they would under a table of their own length, and fewer workgroups: 64 tokens of one
  // sequence over 600 rows, 8 KV heads, table for 131072 rows 28 us, for 600 rows 15 us (e4m3 33 and 15); 256 tokens of four
  // over 2000 rows 62 either way.
  struct Rows {
    int waves, tiles, over;
  };
  const bool f32 = dtype == kTypeF32;
  const Rows forms[] = {{1, 1, 0}, {4, 1, f32 ? 64 : pages.type == kTypeE4m3 ? 48 : 16}, {4, 2, 128}};
  const long long units = (long long)n_seq * pages.n_kv_head, all_rows = (long long)n_seq * n_head * max_new;
  long long groups = 0, tiles = 0;
  for (int form = f32 ? 1 : 2; form >= 0; --form) {
    p.row_waves = forms[form].waves;
    p.row_tiles = forms[form].tiles;
    const int tile = f32 || p.row_waves == 4 ? 64 : 128;
    tiles = (keys + tile - 1) / tile + (keys < cap ? 2 : 0);
    p.min_tiles = p.row_waves == 4 ? 16 : all_rows <= 512 ? 1 : f32 ? 16 : 8;
    groups = units * ((rows + p.rows() - 1) / p.rows());
    const long long parts = groups * (!f32 && tiles > p.min_tiles ? tiles / p.min_tiles : 1);
    if (rows > forms[form].over && parts >= kComputeUnits) break;
  }
  // Workgroups that the keys are cut for.  us at targets of 512 / 768 / 1024 / 1536 / 2048: chunks of up to 512 tokens over up to
  // 8192 rows, 32 units, e4m3 228 / 206 / 203 / 220 / 228 (of one length 350 / 373 / 374 / 389 / 393); single tokens over up to 4000
  // rows, 512 units, e4m3 80 / 77 / 82 / 85 / 88 (one length 105 / 113 / 113 / 121 / 125); 16 units x 131072 rows bf16 196 / 225 /
  // 210 / 222 / 232.  min_tiles: what a workgroup has at least, against the cost of its start and of the join: one token of one
  // sequence, 1 / 2 / 16 tiles 10.7 / 12.9 / 12.5; 32 units x 1000 rows, 1 / 2 / 4 / 16 13 / 14 / 17 / 20; but 32 units of 64 tokens
  // x 300 rows uncut 11, cut 18.  No cutting with four row groups to each such workgroup, nor under a window, which bounds what a
  // sequence costs, with one (768 units of single tokens in a window of 2048: 44, cut 48 to 56).
  p.target = (p.row_waves == 4 ? 4 : 2) * kComputeUnits;
  if (tiles <= p.min_tiles || groups >= 4 * p.target || (keys < cap && groups >= p.target)) p.target = 0;
  // every sequence's tiles over `most` are rounded up, once to a group
  const long long cut = groups + p.target, parts = groups * ((tiles + p.min_tiles - 1) / p.min_tiles);
  const long long n_wg = p.target == 0 ? groups : cut < parts ? cut : parts;
  p.n_wg = n_wg <= 0x7fffffff ? (int)n_wg : -1;
  return p;
}

hipError_t launch_pages_attend(int dtype, int d, int n_seq, int n_head, const PagesView& pages, const RowsView& q,
                               const RowsView& out, const ChunkView& chunk, const MaskView& mask, float sm_scale,
                               const PagesPlan& plan, void* ws, hipStream_t stream) {
  AttendArgs a;
  a.c = pages;
  a.q = q;
  a.out = out;
  a.chunk = chunk;
  a.mask = mask;
  a.n_seq = n_seq;
  a.group = n_head / pages.n_kv_head;
  a.rows = plan.rows();
  a.target = plan.target;
  a.min_tiles = plan.min_tiles;
  a.scale_log2e = sm_scale * 1.4426950408889634f;
  a.no_max = no_maximum(a.scale_log2e);
  const size_t part_rows = pages_partial_rows(a.group, chunk.max_new, plan);
  a.part_rows = (int)(part_rows / plan.n_wg);
  a.part = (float*)ws;
  a.stat = a.part + part_rows * d;
  a.cuts = (int2*)(a.stat + part_rows * 2);
  const bool q8 = pages.type == kTypeE4m3;
  hipError_t e;
  if (dtype == kTypeBf16) {
    if (d == 128)
      e = q8 ? launch_plan<kTypeBf16, true, 128>(plan, a, stream) : launch_plan<kTypeBf16, false, 128>(plan, a, stream);
    else e = q8 ? launch_plan<kTypeBf16, true, 64>(plan, a, stream) : launch_plan<kTypeBf16, false, 64>(plan, a, stream);
  } else {
    if (d == 128) e = q8 ? launch_plan<kTypeF32, true, 128>(plan, a, stream) : launch_plan<kTypeF32, false, 128>(plan, a, stream);
    else e = q8 ? launch_plan<kTypeF32, true, 64>(plan, a, stream) : launch_plan<kTypeF32, false, 64>(plan, a, stream);
  }
  if (e != hipSuccess || plan.target == 0) return e;
  const int unit_rows = chunk.max_new * a.group, n_row_group = (unit_rows + a.rows - 1) / a.rows;
  const int join_groups = ((unit_rows < a.rows ? unit_rows : a.rows) + kJoinRows - 1) / kJoinRows;
  const dim3 grid((unsigned)(n_seq * pages.n_kv_head * n_row_group * join_groups));
  auto join = [&](auto type, auto dim) {
    hipLaunchKernelGGL((pages_join_kernel<type(), dim()>), grid, dim3(kThreads), 0, stream, a, n_row_group, join_groups);
  };
  auto of_dim = [&](auto type) {
    if (d == 128) join(type, std::integral_constant<int, 128>{});
    else join(type, std::integral_constant<int, 64>{});
  };
  if (dtype == kTypeBf16) of_dim(std::integral_constant<int, kTypeBf16>{});
  else of_dim(std::integral_constant<int, kTypeF32>{});
  return hipGetLastError();
}

}  // namespace scalekv
