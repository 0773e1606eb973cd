// Attention over pages for many query rows (bf16 arithmetic): the products and the schedule of the pipelined dense
// kernel (attend_pipe.hip: three blocks of 32 keys under way in a wave, an MFMA, a request to the LDS and a step of the
// softmax in turn), with rows fetched from pages, masks, and shared KV heads.
//
// Four waves of 16 RT query rows each share tiles of 64 keys, in two stages.  A wave brings in 16 rows of a tile: they
// lie in one page whatever its size (16 rows or more), so that the page's number and the rows' address are scalars.
// Rows go straight into LDS.  e4m3 rows wait there as codes, a tile ahead, until the wave that has brought them widens
// them into the tile, once for the four waves (exactly).  A wave whose 16 rows some lanes must not read (behind the last
// row, outside window and sinks) fetches zeros for those; pages that do not exist are zeros too.
//
// Running maximum: formed per lane (an eighth of a block's keys), it is joined over the four lanes of a row only where it
// exceeds the row's offset by kRescaleThreshold log2 units in some row of the wave, which after the first blocks is rare;
// the accumulators are rescaled behind the product that is then still to come with the old offset.
//
// What bounds it: the matrix cores and the softmax beside them, as in the dense kernel.  128 units x 4096 tokens x 4420 rows,
// head_dim 128: bf16 1185 to 1220 us (cards differ; 1.0 PFLOP/s; the dense kernel 1046 where this takes 1213), causal 788 us, e4m3
// 1510 us (the codes' widening is on top), head_dim 64 714 us (e4m3 858).  The first twenty passes after an idle chip take up
// to a quarter longer.  The map keeps the matrix pipe busy for 46 % of its cycles, 38 % of those beside vector instructions,
// of which there are 2.6 to an MFMA (e4m3 4.3), and the LDS for 24 %, 1 % of that in bank conflicts; e4m3 36 % and 23 %: the widened
// rows' stores conflict.  2048 tokens of 32 heads in a window of 1024 105 us (0.65 PFLOP/s; e4m3 125): a walk is 18 tiles, one
// for the sinks, and three of them are masked element by element; its start and end weigh (matrix pipe busy 32 %).  The
// lookup by lengths at a workgroup's start costs 0.6 % of the map and 1 us of the window (measured with the lengths as
// constants).  4 ragged sequences of up to 512 tokens over up to 8192 rows, e4m3 200 to 206 us (0.55 PFLOP/s), bf16 170 us: walks
// of 16 tiles and more, their sums through the workspace (75 MB), and 17 us of the join.
#include <type_traits>

#include "pages_attend.h"

namespace scalekv {
namespace {

constexpr int TN = 64;   // keys of a tile
constexpr int kWaves = 4;

// sixteen cached rows of zeros, in the place of what is not there
__device__ __attribute__((aligned(256))) const unsigned char g_zero_rows[16 * 256] = {};

template <int D, bool Q8, int RT>
struct Chunk {
  static constexpr int kRowBytes = 2 * D;              // in LDS
  static constexpr int kTileBytes = TN * kRowBytes;
  static constexpr int kSlabs = D / 32;
  static constexpr int kBlocks = D / 16;
  static constexpr int kChunks = D / 8;
  static constexpr int kRowsPerOp = 64 / kChunks;      // bf16: rows that one transfer of a wave covers
  static constexpr int kOps = 16 / kRowsPerOp;
  static constexpr int kVecs = 16 * D / 16 / 64;       // e4m3: 16-byte vectors of a lane for 16 rows (2, 1)
  static constexpr int kRows = 16 * RT * kWaves;
  static constexpr int kWavesPerSimd = D == 128 ? 2 : 3;
  static constexpr int kLds = 4 * kTileBytes + (Q8 ? 2 * kWaves * 16 * D : 0);  // two stages of K, two of V; codes
  // a wave's part of the LDS behind the tile loop: its sums (add_odd), 16 rows of them with padding, or its output
  static constexpr int kMine = 16 * RT * D * 4 > 16 * (D * 4 + 16) ? 16 * RT * D * 4 : 16 * (D * 4 + 16);
  static_assert(kWaves * kMine <= kLds, "fits in the tiles' place");
};

// 16 bytes a lane from base + voff straight into LDS, at lds_addr + 16 lane (attend_pipe.hip has the reasons for assembly);
// the first with a base of the wave, the second with an address of the lane
template <int IMM>
__device__ __forceinline__ void dma16(const unsigned char* base_uniform, unsigned voff, unsigned lds_addr_uniform) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3"
               :: "s"(lds_addr_uniform), "v"(voff), "s"(base_uniform), "n"(IMM) : "m0", "memory");
}
__device__ __forceinline__ void dma16_lane(const unsigned char* address, unsigned lds_addr_uniform) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :: "s"(lds_addr_uniform), "v"(address) : "m0", "memory");
}

template <int D, bool Q8, int RT>
__global__ __launch_bounds__(64 * kWaves)
__attribute__((amdgpu_waves_per_eu(Chunk<D, Q8, RT>::kWavesPerSimd, Chunk<D, Q8, RT>::kWavesPerSimd)))
void pages_chunk_kernel(AttendArgs a) {
  using G = Chunk<D, Q8, RT>;
  constexpr int kRowBytes = G::kRowBytes, kTileBytes = G::kTileBytes, NSL = G::kSlabs, NCB = G::kBlocks;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const PagesView& c = a.c;

  const int wg = SCALEKV_WG_X;
  const Slice slice = slice_of<TN>(a, wg);
  if (slice.cuts == 0) return;
  const int seq = slice.seq, kv = slice.kv;
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first_row = slice.row_group * G::kRows, wave_row = first_row + wave * (16 * RT);
  const Seen<TN> seen(a, slice, first_row, G::kRows);
  const int per = (seen.n_tile + slice.cuts - 1) / slice.cuts;
  const int t0 = min(slice.cut * per, seen.n_tile), n_tile = min(t0 + per, seen.n_tile) - t0;
  // all rows of the wave see [w_begin, w_end) and the sinks below w_end
  const int w_end = seen.end_of(seen.pos0 + min(wave_row, seen.n_rows - 1) / a.group);
  const int w_begin = seen.begin_of(seen.pos0 + min(wave_row + 16 * RT - 1, seen.n_rows - 1) / a.group);

  // ---- query rows: B operand of the first product, resident
  bf16x8 qf[RT][NSL];
#pragma unroll
  for (int b = 0; b < RT; ++b) {
    const int r = min(wave_row + 16 * b + i, seen.n_rows - 1), t = r / a.group, head = kv * a.group + (r - t * a.group);
    const long long at = (long long)chunk_first(a.chunk, seq) + t;
    const u32x4* src = (const u32x4*)(a.q.p + seq * a.q.seq + head * a.q.head + at * a.q.row);
    const bool there = at >= 0 && at < a.q.n_row;
#pragma unroll
    for (int sl = 0; sl < NSL; ++sl) qf[b][sl] = __builtin_bit_cast(bf16x8, there ? src[4 * sl + g] : u32x4{0, 0, 0, 0});
  }

  // ---- tiles
  auto lds_addr = [](const unsigned char* p) -> unsigned {
    return (unsigned)(size_t)(const __attribute__((address_space(3))) unsigned char*)p;
  };
  unsigned char* const k_lds = smem;
  unsigned char* const v_lds = smem + 2 * kTileBytes;
  unsigned char* const raw_lds = smem + 4 * kTileBytes;  // e4m3: the codes of the next tiles, K's and V's, wave by wave
  bool odd = false;  // this wave has taken values that are not finite out of a tile
  const int32_t* const table = c.table + (long long)seq * c.width;
  const long long kv_ofs = kv * c.head;
  auto key0_of = [&](int t) { return seen.key0(t0 + t); };
  // the page of this wave's rows of tile t; any number outside the pool stands for rows of zeros
  auto ask_page = [&](int t) -> int {
    const int pos = key0_of(t) + 16 * wave;
    return t < n_tile && (seen.plain(t0 + t) || seen.any(pos, 16)) ? table[pos >> c.page_shift] : -1;
  };
  int page_next = -1;  // of the tile whose K rows are requested next (as it was loaded; made a scalar when it is used)
  int page_k = -1;     // of the tile before: its V rows are requested with them
  // this wave's rows of a tensor
  auto rows_at = [&](const unsigned char* pool, int page, int t) -> const unsigned char* {
    const int slot = (key0_of(t) + 16 * wave) & ((1 << c.page_shift) - 1);
    return scalar((unsigned)page < (unsigned)c.n_page ? pool + page * c.page + kv_ofs + slot * (Q8 ? D : kRowBytes)
                                                      : g_zero_rows);
  };
  // bf16: instruction p fills LDS rows 16 wave + kRowsPerOp p ..; the lane that lands in chunk slot s of row r fetches
  // chunk s ^ flip(r)
  const int ld_row = lane / G::kChunks;
  const unsigned ld_k = ld_row * kRowBytes, ld_kchunk = 16 * ((lane % G::kChunks) ^ k_flip_bf16<D>(16 * wave + ld_row));
  const unsigned ld_v = ld_row * kRowBytes + 16 * ((lane % G::kChunks) ^ v_flip_bf16<D>(16 * wave + ld_row));
  constexpr auto k_step = [](int p) -> unsigned { return 16 * k_flip_bf16<D>(G::kRowsPerOp * p); };
  const unsigned k_wave = __builtin_amdgcn_readfirstlane(lds_addr(k_lds + 16 * wave * kRowBytes));
  const unsigned v_wave = __builtin_amdgcn_readfirstlane(lds_addr(v_lds + 16 * wave * kRowBytes));
  auto transfer = [&](const unsigned char* rows, int t, unsigned dst, auto ofs) __attribute__((always_inline)) {
    if (seen.plain(t0 + t) || seen.every(key0_of(t) + 16 * wave, 16)) {
      // (the immediate offset moves the destination along with the source)
      dma16<0>(rows, ofs(0), dst);
      dma16<1024>(rows, ofs(1), dst);
      if constexpr (G::kOps == 4) {
        dma16<2 * 1024>(rows, ofs(2), dst);
        dma16<3 * 1024>(rows, ofs(3), dst);
      }
    } else {
#pragma unroll
      for (int p = 0; p < G::kOps; ++p) {
        const bool there = seen.some(key0_of(t) + 16 * wave + G::kRowsPerOp * p + ld_row);
        dma16_lane((there ? rows : (const unsigned char*)g_zero_rows) + ofs(p) + 1024 * p, dst + 1024 * p);
      }
    }
  };
  // e4m3: the codes of 16 rows, as they lie in the page; a lane widens kVecs vectors of 16 codes, vector p of row
  // kVecRows p + lane / kSrcChunks of those
  constexpr int kSrcChunks = D / 16, kVecRows = 16 / G::kVecs, kRawBytes = 16 * D;
  const int q8_row = lane / kSrcChunks;
  const unsigned raw_k = __builtin_amdgcn_readfirstlane(lds_addr(raw_lds + wave * kRawBytes));
  const unsigned raw_v = raw_k + kWaves * kRawBytes;
  uint8_t k_sc[G::kVecs], v_sc[G::kVecs];
  auto fetch = [&](const unsigned char* pool, const uint8_t* scales, int page, int t, unsigned dst,
                   uint8_t (&sc)[G::kVecs]) __attribute__((always_inline)) {
    const int pos = key0_of(t) + 16 * wave, slot = pos & ((1 << c.page_shift) - 1);
    const unsigned char* rows = rows_at(pool, page, t);
    const unsigned char* scale = scalar((unsigned)page < (unsigned)c.n_page
                                            ? scales + page * c.scale_page + kv * c.scale_head + slot
                                            : g_zero_rows);
    if (seen.plain(t0 + t) || seen.every(pos, 16)) {
#pragma unroll
      for (int p = 0; p < G::kVecs; ++p) sc[p] = scale[kVecRows * p + q8_row];
      dma16<0>(rows, 16 * lane, dst);
      if constexpr (G::kVecs == 2) dma16<1024>(rows, 16 * lane, dst);
    } else {
#pragma unroll
      for (int p = 0; p < G::kVecs; ++p) {
        const bool there = seen.some(pos + kVecRows * p + q8_row);
        // (the scale too: what a row holds that has not been written comes into nothing)
        sc[p] = *(there ? scale + kVecRows * p + q8_row : (const unsigned char*)g_zero_rows);
        dma16_lane((there ? rows : (const unsigned char*)g_zero_rows) + 1024 * p + 16 * lane, dst + 1024 * p);
      }
    }
  };
  // Vector p of them into the tile, in two steps: load() and put()
  u32x4 raw;
  auto load = [&](const unsigned char* codes, int p) { raw = *(const u32x4*)(codes + 1024 * p + 16 * lane); };
  auto put = [&](unsigned char* stage, const uint8_t (&sc)[G::kVecs], int p, bool values, bool edge)
                 __attribute__((always_inline)) {
    // (addresses are formed on the spot: held through the tile loop they are spilled)
    int ld = lane;
    asm volatile("" : "+v"(ld));
    const int row = 16 * wave + kVecRows * p + ld / kSrcChunks;
    u32x4 x[2];
    widen(raw, __uint_as_float((unsigned)sc[p] << 23), x);
    if (values && edge) odd |= __builtin_amdgcn_ballot_w64(take_odd<true>(x[0]) | take_odd<true>(x[1])) != 0;
    const int flip = values ? v_flip_bf16<D>(row) : k_flip_bf16<D>(row);
#pragma unroll
    for (int w = 0; w < 2; ++w) *(u32x4*)(stage + row * kRowBytes + 16 * ((2 * (ld % kSrcChunks) + w) ^ flip)) = x[w];
  };
  unsigned char* const k_codes = raw_lds + wave * kRawBytes;
  unsigned char* const v_codes = raw_lds + (kWaves + wave) * kRawBytes;
  auto issue_k = [&](int t, int page) __attribute__((always_inline)) {
    if constexpr (Q8) fetch(c.k, c.k_scale, page, t, raw_k, k_sc);
    else
      transfer(rows_at(c.k, page, t), t, k_wave + (t & 1) * kTileBytes,
               [&](int p) { return ld_k + (ld_kchunk ^ k_step(p)); });
  };
  auto issue_v = [&](int t, int page) __attribute__((always_inline)) {
    if constexpr (Q8) fetch(c.v, c.v_scale, page, t, raw_v, v_sc);
    else transfer(rows_at(c.v, page, t), t, v_wave + (t & 1) * kTileBytes, [&](int) { return ld_v; });
  };
  auto put_v = [&](int t, int p) __attribute__((always_inline)) {
    put(v_lds + (t & 1) * kTileBytes, v_sc, p, true, !seen.plain(t0 + t) && seen.edge(t0 + t));
  };
  auto put_k = [&](int t, int p) __attribute__((always_inline)) { put(k_lds + (t & 1) * kTileBytes, k_sc, p, false, false); };
  // Between turn(t) and the next: V of tile t + 1 and K of tile t + 2, whose codes have arrived, into the tile; step e of
  // 4 kVecs.  Then the codes behind them are asked for.
  auto widen_step = [&](int t, int e) __attribute__((always_inline)) {
    const int p = e / 2 % G::kVecs;
    const bool values = e / 2 < G::kVecs;
    if (values ? t + 1 >= n_tile : t + 2 >= n_tile) return;
    if (e % 2 == 0) load(values ? v_codes : k_codes, p);
    else if (values) put_v(t + 1, p);
    else put_k(t + 2, p);
  };
  auto ask_codes = [&](int t) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the codes are read, their places may be filled again
    if (t + 2 < n_tile) issue_v(t + 2, page_k);
    const int page = __builtin_amdgcn_readfirstlane(page_next);
    if (t + 3 < n_tile) issue_k(t + 3, page);
    page_k = page;
    page_next = ask_page(t + 4);
    __builtin_amdgcn_sched_barrier(0);
  };
  // bf16: values of an edge tile that are not finite, in the rows that this wave has brought in
  auto sift = [&](int t) {
    unsigned char* const mine = v_lds + (t & 1) * kTileBytes + 16 * wave * kRowBytes + 16 * lane;
    for (int p = 0; p < G::kOps; ++p) {
      u32x4 x = *(const u32x4*)(mine + 1024 * p);
      const bool found = take_odd<true>(x);
      if (found) *(u32x4*)(mine + 1024 * p) = x;
      odd |= __builtin_amdgcn_ballot_w64(found) != 0;
    }
  };

  // ---- operand addresses in the first block of 32 keys; key tile t is 4 rows further on
  unsigned k_adr[NSL], v_adr[NCB];
  {
    const int row = 16 * (i >> 2 & 1) + 8 * (i >> 3) + (i & 3);
#pragma unroll
    for (int sl = 0; sl < NSL; ++sl) k_adr[sl] = lds_addr(k_lds) + row * kRowBytes + 16 * ((4 * sl + g) ^ k_flip_bf16<D>(row));
  }
  {
    const int row = 16 * (g & 1) + 8 * (g >> 1) + (i >> 2);
#pragma unroll
    for (int x = 0; x < NCB; ++x) v_adr[x] = lds_addr(v_lds) + row * kRowBytes + 16 * (2 * x ^ v_flip_bf16<D>(row)) + 8 * (i & 3);
  }
#pragma unroll
  for (int sl = 0; sl < NSL; ++sl) asm volatile("" : "+v"(k_adr[sl]));
#pragma unroll
  for (int x = 0; x < NCB; ++x) asm volatile("" : "+v"(v_adr[x]));

  f32x4 o[RT][NCB];
  float neg[RT], l_run[RT], alpha[RT];  // less the rows' offsets (log2 units), this lane's share of the sums
  bool moved = false;                   // offsets have moved: the accumulators are to be scaled by alpha
#pragma unroll
  for (int b = 0; b < RT; ++b) {
#pragma unroll
    for (int x = 0; x < NCB; ++x) o[b][x] = f32x4{0.f, 0.f, 0.f, 0.f};
    neg[b] = -(a.no_max * a.scale_log2e);
    l_run[b] = 0.f;
    alpha[b] = 1.f;
  }

  typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  constexpr int kHalf = 32 * kRowBytes;
  constexpr int kSlots = 2 * NSL * RT;      // MFMAs of one product over a block
  constexpr int kSteps = 8 * RT / kSlots;   // softmax steps behind each
  constexpr int kKReads = 2 * NSL, kVReads = 2 * NCB;
  constexpr int kBarrierSlot = kSlots / 2 - 1;
  bf16x8 kf[2][NSL];
  s16x4 vf[NCB][2];
  f32x4 sa[RT][2], sb[RT][2];
  u32x4 pa[RT], pb[RT];

  auto read_k = [&](int ofs, int e) { kf[e & 1][e >> 1] = *(lds_bf16x8*)(k_adr[e >> 1] + ofs + 4 * (e & 1) * kRowBytes); };
  auto read_v = [&](int ofs, int e) {
    vf[e >> 1][e & 1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(v_adr[e >> 1] + ofs + 4 * (e & 1) * kRowBytes));
  };
  auto score_mfma = [&](f32x4 (&s)[RT][2], int m) {
    const int sl = m / (2 * RT), t = m / RT % 2, b = m % RT;
    const f32x4 sum = sl ? s[b][t] : f32x4{0.f, 0.f, 0.f, 0.f};
    s[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][sl], qf[b][sl], sum, 0, 0, 0);
  };
  auto value_mfma = [&](const u32x4 (&p)[RT], int m) {
    const int x = m / RT, b = m % RT;
    const bf16x8 vt = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[x][0], vf[x][1], 0, 1, 2, 3, 4, 5, 6, 7));
    o[b][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, p[b]), o[b][x], 0, 0, 0);
  };
  // Step k of 16 RT of a block's softmax: four for each pair of weights.  (The empty statements keep each step in its slot.)
  auto softmax_step = [&](f32x4 (&s)[RT][2], u32x4 (&p)[RT], int k) {
    const int b = k >> 4, x = 2 * (k >> 2 & 3), t = x >> 2, v = x & 3;
    float w0 = s[b][t][v], w1 = s[b][t][v + 1];
    if ((k & 3) == 0) {
      w0 = fmaf(w0, a.scale_log2e, neg[b]);
      w1 = fmaf(w1, a.scale_log2e, neg[b]);
      asm volatile("" : "+v"(w0), "+v"(w1));
    } else if ((k & 3) == 1) {
      w0 = __builtin_amdgcn_exp2f(w0);
      asm volatile("" : "+v"(w0));
    } else if ((k & 3) == 2) {
      w1 = __builtin_amdgcn_exp2f(w1);
      asm volatile("" : "+v"(w1));
    } else {
      // (weights are rounded to bf16 for the matrix cores; the sum adds the rounded ones)
      const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f}, pr = {(__bf16)w0, (__bf16)w1};
      uint32_t word = __builtin_bit_cast(uint32_t, pr);
      l_run[b] = __builtin_amdgcn_fdot2_f32_bf16(pr, ones, l_run[b], false);
      asm volatile("" : "+v"(word), "+v"(l_run[b]));
      p[b][x / 2] = word;
    }
    s[b][t][v] = w0;
    s[b][t][v + 1] = w1;
  };
  // Before the softmax of a block (half h of tile t): hide what its rows do not see, and move the offsets if need be.
  auto prepare = [&](f32x4 (&s)[RT][2], int t, int h) __attribute__((always_inline)) {
    const int key0 = key0_of(t);
    if (!seen.plain(t0 + t) && (key0 + TN > w_end || (seen.window && key0 < w_begin && key0 + TN > seen.sinks))) {
      const int mine = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
      const int pos0 = key0 + 32 * h + 16 * (mine >> 4 & 1) + 8 * (mine >> 5);
#pragma unroll
      for (int b = 0; b < RT; ++b) {
        const int p = seen.pos0 + min(wave_row + 16 * b + (mine & 15), seen.n_rows - 1) / a.group;
        const int end = seen.end_of(p), begin = seen.begin_of(p);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int pos = pos0 + x;
          if (pos >= end || (pos < begin && pos >= seen.sinks)) s[b][x / 4][x % 4] = -INFINITY;
        }
      }
    }
    float mx[RT];
    bool grow = false;
#pragma unroll
    for (int b = 0; b < RT; ++b) {
      mx[b] = s[b][0][0];
#pragma unroll
      for (int x = 1; x < 8; ++x) mx[b] = fmaxf(mx[b], s[b][x / 4][x % 4]);
      grow |= fmaf(mx[b], a.scale_log2e, neg[b]) > kRescaleThreshold;
    }
    moved = __builtin_amdgcn_ballot_w64(grow) != 0;
    if (moved) {
#pragma unroll
      for (int b = 0; b < RT; ++b) {
        const float now = fminf(neg[b], -(xor32_max(xor16_max(mx[b])) * a.scale_log2e));
        alpha[b] = __builtin_amdgcn_exp2f(now - neg[b]);
        neg[b] = now;
        l_run[b] *= alpha[b];
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto rescale = [&]() __attribute__((always_inline)) {
    if (moved) {
      asm volatile("");  // (a branch: the products of all accumulators are not to be formed and thrown away)
#pragma unroll
      for (int b = 0; b < RT; ++b)
#pragma unroll
        for (int x = 0; x < NCB; ++x) o[b][x] *= alpha[b];
    }
  };
  auto slots = [&](auto mfma, auto beside, f32x4 (&s)[RT][2], u32x4 (&p)[RT], int first_step) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < kSlots; ++m) {
      mfma(m);
      beside(m);
#pragma unroll
      for (int r = 0; r < kSteps; ++r) softmax_step(s, p, first_step + m * kSteps + r);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Publishes tile t + 1 of K and tile t of V, and requests the tiles behind them in the place of those that all waves
  // have left.
  auto turn = [&](int t) __attribute__((always_inline)) {
    if constexpr (Q8) {
      __builtin_amdgcn_s_waitcnt(0);  // what this wave has asked for and put is there
      __syncthreads();
    } else {
      __builtin_amdgcn_s_waitcnt(0);
      if (!seen.plain(t0 + t) && seen.edge(t0 + t)) {
        sift(t);
        __builtin_amdgcn_s_waitcnt(0xc07f);
      }
      __syncthreads();
      if (t + 1 < n_tile) issue_v(t + 1, page_k);
      const int page = __builtin_amdgcn_readfirstlane(page_next);
      if (t + 2 < n_tile) issue_k(t + 2, page);
      page_k = page;
      page_next = ask_page(t + 3);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto nothing = [](int) {};
  auto first_half = [&](int t, int st) __attribute__((always_inline)) {
    prepare(sa, t, 0);
    slots([&](int m) { score_mfma(sb, m); },
          [&](int m) {
#pragma unroll
            for (int e = m * kVReads / kSlots; e < (m + 1) * kVReads / kSlots; ++e) read_v((st ^ 1) * kTileBytes + kHalf, e);
          },
          sa, pa, 0);
    slots([&](int m) { value_mfma(pb, m); },
          [&](int m) {
            if (m == kBarrierSlot) turn(t);
            if (m > kBarrierSlot) {
              constexpr int kLeft = kSlots - kBarrierSlot - 1;
              const int x = m - kBarrierSlot - 1;
#pragma unroll
              for (int e = x * kKReads / kLeft; e < (x + 1) * kKReads / kLeft; ++e) read_k((st ^ 1) * kTileBytes, e);
            }
          },
          sa, pa, 8 * RT);
    rescale();
  };
  auto second_half = [&](int t, int st) __attribute__((always_inline)) {
    prepare(sb, t, 1);
    slots([&](int m) { score_mfma(sa, m); },
          [&](int m) {
#pragma unroll
            for (int e = m * kVReads / kSlots; e < (m + 1) * kVReads / kSlots; ++e) read_v(st * kTileBytes, e);
            if constexpr (Q8) {
              // a vector is asked for in one slot and put some slots later
              constexpr int kApart = kSlots / (2 * G::kVecs);
              if (m % kApart == 0) widen_step(t, m / kApart * 2);
              if (m % kApart == kApart - 1) widen_step(t, m / kApart * 2 + 1);
            }
          },
          sb, pb, 0);
    if constexpr (Q8) ask_codes(t);
    slots([&](int m) { value_mfma(pa, m); },
          [&](int m) { if (m < kKReads) read_k((st ^ 1) * kTileBytes + kHalf, m); }, sb, pb, 8 * RT);
    rescale();
  };

  if (n_tile > 0) {
    {
      const int p0 = __builtin_amdgcn_readfirstlane(ask_page(0)), p1 = __builtin_amdgcn_readfirstlane(ask_page(1));
      if constexpr (Q8) {
        const int p2 = __builtin_amdgcn_readfirstlane(ask_page(2));
        issue_k(0, p0);
        issue_v(0, p0);
        __builtin_amdgcn_s_waitcnt(0);
        for (int p = 0; p < G::kVecs; ++p) load(k_codes, p), put_k(0, p);
        for (int p = 0; p < G::kVecs; ++p) load(v_codes, p), put_v(0, p);
        __builtin_amdgcn_s_waitcnt(0xc07f);
        if (n_tile > 1) {
          issue_k(1, p1);
          issue_v(1, p1);
          __builtin_amdgcn_s_waitcnt(0);
          for (int p = 0; p < G::kVecs; ++p) load(k_codes, p), put_k(1, p);
          __builtin_amdgcn_s_waitcnt(0xc07f);
        }
        if (n_tile > 2) issue_k(2, p2);
        page_k = p2;
        page_next = ask_page(3);
      } else {
        issue_k(0, p0);
        issue_v(0, p0);
        if (n_tile > 1) issue_k(1, p1);
        page_k = p1;
        page_next = ask_page(2);
        __builtin_amdgcn_s_waitcnt(0);
      }
    }
    __syncthreads();
    if (wave_row < seen.n_rows) {
#pragma unroll
      for (int e = 0; e < kKReads; ++e) read_k(0, e);
#pragma unroll
      for (int m = 0; m < kSlots; ++m) score_mfma(sa, m);
#pragma unroll
      for (int e = 0; e < kKReads; ++e) read_k(kHalf, e);
#pragma unroll
      for (int m = 0; m < kSlots; ++m) score_mfma(sb, m);
      prepare(sa, 0, 0);
      slots(nothing, nothing, sa, pa, 0);
      turn(0);
      slots(nothing, [&](int m) { if (m < kKReads) read_k(kTileBytes, m); }, sa, pa, 8 * RT);
      // (K of the second tile: its first half; the second half is read beside the first product that takes it)
      int t = 0;
      for (; t + 2 < n_tile; t += 2) {
        second_half(t, 0);
        first_half(t + 1, 1);
        second_half(t + 1, 1);
        first_half(t + 2, 0);
      }
      if (t + 1 < n_tile) {
        second_half(t, 0);
        first_half(t + 1, 1);
        ++t;
      }
      const int ofs = (t & 1) * kTileBytes;
      prepare(sb, t, 1);
      slots(nothing,
            [&](int m) {
#pragma unroll
              for (int e = m * kVReads / kSlots; e < (m + 1) * kVReads / kSlots; ++e) read_v(ofs, e);
            },
            sb, pb, 0);
      slots([&](int m) { value_mfma(pa, m); }, nothing, sb, pb, 8 * RT);
      rescale();
#pragma unroll
      for (int e = 0; e < kVReads; ++e) read_v(ofs + kHalf, e);
#pragma unroll
      for (int m = 0; m < kSlots; ++m) value_mfma(pb, m);
    } else {
      for (int t = 0; t < n_tile; ++t) {  // (a wave without rows only carries its share of the tiles)
        turn(t);
        if constexpr (Q8) {
          for (int e = 0; e < 4 * G::kVecs; ++e) widen_step(t, e);
          ask_codes(t);
        }
      }
    }
  }
  __syncthreads();  // all waves have left the tiles
  bool any_odd = false;
  if (a.mask.causal || seen.window) {  // (without a mask no row sees what another does not)
    if (lane == 0) ((int*)smem)[wave] = odd;
    __syncthreads();
    for (int x = 0; x < kWaves; ++x) any_odd |= ((const int*)smem)[x] != 0;
    __syncthreads();
  }
  if (wave_row >= seen.n_rows) return;
  // (each wave has a part of the LDS to itself from here on, for add_odd() and then for its output)
  unsigned char* const mine = smem + wave * G::kMine;
  if (any_odd) {
    float* const sums = (float*)mine;
#pragma unroll
    for (int b = 0; b < RT; ++b) sums_to_lds<D>(o[b], sums + 16 * b * D);
    add_odd<kTypeBf16, Q8, D, TN, RT>(a, seen, seq, kv, wave_row, t0, t0 + n_tile, 0, TN, neg, sums);
#pragma unroll
    for (int b = 0; b < RT; ++b) sums_from_lds<D>(o[b], sums + 16 * b * D);
  }

  // ---- write
#pragma unroll
  for (int b = 0; b < RT; ++b) l_run[b] = xor32_sum(xor16_sum(l_run[b]));
  if (slice.cuts > 1) {
    // whole rows here too, 16 of them at a time
    constexpr int kSumStride = D * 4 + 16, kLanes = D / 4;
    unsigned char* const sums = mine;
#pragma unroll
    for (int b = 0; b < RT; ++b) {
      const long long row = (long long)wg * a.part_rows + (wave_row - first_row) + 16 * b;
      if (g == 0 && wave_row + 16 * b + i < seen.n_rows) {
        a.stat[2 * (row + i)] = -neg[b];
        a.stat[2 * (row + i) + 1] = l_run[b];
      }
#pragma unroll
      for (int x = 0; x < NCB; ++x) *(f32x4*)(sums + i * kSumStride + 64 * x + 16 * g) = o[b][x];
      own_lds();
#pragma unroll
      for (int p = 0; p < 16 * kLanes / 64; ++p) {
        const int r = (64 / kLanes) * p + lane / kLanes;
        const f32x4 val = *(const f32x4*)(sums + r * kSumStride + 16 * (lane % kLanes));
        if (wave_row + 16 * b + r < seen.n_rows) *(f32x4*)(a.part + (row + r) * D + 4 * (lane % kLanes)) = val;
      }
      own_lds();
    }
    return;
  }
  // whole rows through LDS, padded by 16 bytes against bank conflicts
  constexpr int kOutStride = kRowBytes + 16;
  static_assert(kOutStride <= D * 4, "the output of a wave fits in its part");
#pragma unroll
  for (int b = 0; b < RT; ++b) {
    // a row that sees nothing, or keys of weight zero only, is zero
    const bool empty = l_run[b] == 0.f;
    const float inv = 1.f / l_run[b];
#pragma unroll
    for (int x = 0; x < NCB; ++x) {
      const f32x4 y = empty ? f32x4{0.f, 0.f, 0.f, 0.f} : o[b][x] * inv;
      const bf16x2 lo = {(__bf16)y[0], (__bf16)y[1]}, hi = {(__bf16)y[2], (__bf16)y[3]};
      *(uint2*)(mine + (16 * b + i) * kOutStride + 32 * x + 8 * g) =
          make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
    }
  }
  own_lds();
#pragma unroll
  for (int p = 0; p < 16 * RT / G::kRowsPerOp; ++p) {
    const int r = G::kRowsPerOp * p + lane / G::kChunks;
    const u32x4 val = *(const u32x4*)(mine + r * kOutStride + 16 * (lane % G::kChunks));
    const int nth_row = wave_row + r, t = nth_row / a.group, head = kv * a.group + (nth_row - t * a.group);
    const long long at = (long long)chunk_first(a.chunk, seq) + t;
    if (nth_row < seen.n_rows && at >= 0 && at < a.out.n_row)
      *(u32x4*)(a.out.p + (seq * a.out.seq + head * a.out.head + at * a.out.row) + 16 * (lane % G::kChunks)) = val;
  }
}

template <int D, bool Q8, int RT>
hipError_t launch_form(const AttendArgs& a, int n_wg, hipStream_t stream) {
  using G = Chunk<D, Q8, RT>;
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_dynamic_lds((const void*)pages_chunk_kernel<D, Q8, RT>, G::kLds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((pages_chunk_kernel<D, Q8, RT>), dim3(n_wg), dim3(64 * kWaves), G::kLds, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_chunk(int d, bool q8, int row_tiles, const AttendArgs& a, int n_wg, hipStream_t stream) {
  auto tiles = [&](auto dim, auto quantised) {
    return row_tiles == 2 ? launch_form<dim(), quantised(), 2>(a, n_wg, stream)
                          : launch_form<dim(), quantised(), 1>(a, n_wg, stream);
  };
  auto cache = [&](auto dim) { return q8 ? tiles(dim, std::true_type{}) : tiles(dim, std::false_type{}); };
  return d == 64 ? cache(std::integral_constant<int, 64>{}) : cache(std::integral_constant<int, 128>{});
}

}  // namespace scalekv
