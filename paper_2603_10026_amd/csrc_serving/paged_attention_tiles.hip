// Attention of many new tokens a sequence over a paged cache: a prompt's chunk.
//
// The same cascade as in paged_rows.h.  A workgroup owns 128 packed rows (new tokens times the query heads
// that share a KV head, token by token, so that a causal tile's rows see nearly the same keys) and walks the keys in
// tiles of 64, or one chunk of them; a wavefront owns 32 of the rows as columns of its 32x32x16 products:
//   S^T = K Q^T        A = K tile (LDS), B = Q^T (registers, loaded once)
//   O^T += V^T P^T     A = V^T (LDS transpose reads of the V tile), B = P^T, formed where S^T's accumulators lie
//
// What bounds it is the matrix unit (4 d operations a row and key) and the exponentials beside it.  Tiles go from
// memory straight into LDS, 16 bytes a lane, double-buffered, one barrier a tile, the next tile's loads spread over
// the first product; 8-bit tiles pass through registers, where they become bf16.  A wavefront loads 16 keys of each
// tile, which lie in one page (page % 16 == 0): a scalar address and lane offsets.  Its lanes hold the addresses for
// its next 64 tiles.  Rows are XOR-swizzled in 16-byte slots (no bank conflicts on either kind of read).
//
// The reference m of a row's state follows the maximum only when that has grown by more than kTau (log2 units): (m, l,
// acc) with any common reference gives the same acc / l.  Probabilities are rounded to bf16 for the second product and
// l sums the rounded ones; everything else is fp32.
#include <math.h>

#include <type_traits>

#include "paged_rows.h"

namespace rf {

namespace {

constexpr int kNW = 4, kBK = 64;
constexpr float kTau = 8.0f;

// 16-byte slot swizzles (slot = piece ^ f(row)).
template <int D>
__host__ __device__ constexpr __forceinline__ int fK(int row) {
  return (D == 128) ? (row & 15) : ((row >> 1) & 7);
}
template <int D>
__host__ __device__ constexpr __forceinline__ int fV(int row) {
  return (D == 128) ? (((row & 3) << 2) | ((row >> 2) & 3)) : ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
}

template <int D>
constexpr int tiles_lds_bytes() { return 4 * kBK * D * 2; }  // K, K, V, V

struct TilesScratch {
  ShareScratch share;
  int bad;
  uint32_t noted[8];  // keys edge0 .. edge0 + 255: a tile's rows differ by less than 128 keys
};

// block: of the launch's share of the grid; lds: tiles_lds_bytes(), 1024-byte aligned.
template <int D, bool FP8>
__device__ __forceinline__ void paged_tiles(const PagedArgs& a, unsigned block, unsigned char* lds, TilesScratch* scratch) {
  constexpr int ES = FP8 ? 1 : 2;
  constexpr int KS = D / 16;                       // contraction steps of S^T
  constexpr int DT = D / 32;                       // 32-row tiles of O^T
  constexpr int P = D / 8;                         // 16-byte slots of a bf16 row
  constexpr int ROWB = D * 2;
  constexpr int TILEB = kBK * ROWB;
  constexpr int kRows = kBK / kNW;                 // keys of a tile that a wavefront loads
  constexpr int kLpr = D * ES / 16;                // lanes a row in memory
  constexpr int kRpl = kWave / kLpr;               // rows a load
  constexpr int kLd = kRows / kRpl;                // loads of K, and of V, a tile
  static_assert(kRows == 16, "one page for a wavefront's share of a tile");

  const Paged& p = a.p;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i32 = lane & 31, hh = lane >> 5;

  // Heads vary fastest, so that with 8 KV heads each XCD's L2 holds one head's keys; late tiles, which see the most
  // keys under a causal mask, come first.
  const int unit = __builtin_amdgcn_readfirstlane(block / (unsigned)p.Hkv);
  const int hk = __builtin_amdgcn_readfirstlane(block - unit * p.Hkv);
  Share w;
  const bool found = find_share(p, a.deal, a.n_tiles, unit, &scratch->share, true, &w);
  if (hk == 0 && wave == 0) note_tile(a, unit, found, w);
  if (!found) return;

  const int rows = w.s.n * p.group, r0 = w.tile << kTilesRowsLog2;
  const int shift = w.s.len - w.s.n;  // token i sees keys 0 .. i + shift
  auto last_key = [&](int r) {        // of row r; -1: none
    return a.causal ? max(-1, min(w.s.len - 1, (int)((unsigned)r / (unsigned)p.group) + shift)) : w.s.len - 1;
  };
  const int wave_r0 = r0 + 32 * wave;
  const int wg_last = __builtin_amdgcn_readfirstlane(last_key(min(rows, r0 + 128) - 1));
  const int wg_min_last = __builtin_amdgcn_readfirstlane(last_key(r0));
  const int edge0 = max(0, wg_min_last + 1) & ~(kBK - 1);  // first key of the first tile that not every row sees whole
  if (threadIdx.x < 8) scratch->noted[threadIdx.x] = 0;
  if (threadIdx.x == 0) scratch->bad = 0;
  const int wave_last = wave_r0 < rows ? __builtin_amdgcn_readfirstlane(last_key(min(rows, wave_r0 + 32) - 1)) : -1;
  const int wave_min_last = wave_r0 < rows ? __builtin_amdgcn_readfirstlane(last_key(wave_r0)) : -1;
  const int my_r = min(wave_r0 + i32, rows - 1);
  const int my_last = last_key(my_r);
  // (a chunk's keys are a multiple of 128: whole tiles)
  const int all_tiles = (wg_last + kBK) / kBK;
  const int first = (int)min((int64_t)all_tiles, (int64_t)w.chunk * (w.chunk_keys / kBK));
  const int n_tiles = (int)min((int64_t)all_tiles, (int64_t)first + w.chunk_keys / kBK);

  // ---- addresses: lane t holds the element offset of this wavefront's 16 keys of tile base + t, base % 64 == 0 ----
  uint32_t off_lo = 0, off_hi = 0;
  uint64_t bad = w.s.over ? 1 : 0;
  const int last_group = wg_last & ~15;
  auto refill = [&](int tile) {
    const int key = (int)min((int64_t)(tile + lane) * kBK + wave * kRows, (int64_t)last_group);
    const int at = (unsigned)key / (unsigned)p.page;
    int id = p.pages[(int64_t)w.b * p.table_pitch + at];
    const bool outside = id < 0 || id >= p.n_pages;
    bad |= __builtin_amdgcn_ballot_w64(outside && tile + lane < n_tiles);
    id = outside ? 0 : id;
    const int64_t off = ((int64_t)id * p.page_stride + (int64_t)(key - at * p.page) * p.slot_stride + (int64_t)hk * p.head_stride) * ES;
    off_lo = (uint32_t)off;
    off_hi = (uint32_t)(off >> 32);
  };
  uint64_t tile_off = 0;  // of the tile requested last
  auto seek = [&](int tile) __attribute__((always_inline)) {
    const int at = (tile - first) & 63;
    if (at == 0) refill(tile);
    tile_off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_lo, at) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, at) << 32;
  };

  const uint32_t slot_bytes = (uint32_t)p.slot_stride * ES;
  const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  const uint32_t dma_base = __builtin_amdgcn_readfirstlane(lds_base + wave * kRows * ROWB);
  // This lane's piece of load e: row e * kRpl + lane / kLpr of the 16, its slot the one that the swizzle puts where the
  // lane's 16 bytes go.  The row's share of f is an XOR of lane / kLpr's and a constant's, so that a load's offset comes
  // of one register and a constant.  (8 bit: 16 bytes are two slots, swizzled on their way into LDS.)
  const uint32_t row_off = (lane / kLpr) * slot_bytes;
  const uint32_t k_piece = 16 * ((lane % kLpr) ^ (FP8 ? 0 : fK<D>(lane / kLpr)));
  const uint32_t v_piece = 16 * ((lane % kLpr) ^ (FP8 ? 0 : fV<D>(lane / kLpr)));
  static_assert(FP8 || (fK<D>(kRpl + 3) == (fK<D>(kRpl) ^ fK<D>(3)) && fV<D>(kRpl + 3) == (fV<D>(kRpl) ^ fV<D>(3))), "f(e kRpl + r) = f(e kRpl) ^ f(r)");
  u32x4 held[2][kLd];  // 8 bit: the next tile on its way
  auto issue_one = [&](int buf, int e, int is_v) __attribute__((always_inline)) {
    const unsigned char* base = (is_v ? a.v : a.k) + tile_off + (uint64_t)(e * kRpl) * slot_bytes;
    if constexpr (FP8) {
      held[is_v][e] = *reinterpret_cast<const u32x4*>(base + (k_piece + row_off));
    } else {
      uint32_t piece = is_v ? v_piece : k_piece;
      asm volatile("" : "+v"(piece));  // (opaque, here and below: what is made of it is made here, and not ahead of the
      // loop to be carried through it in registers)
      const uint32_t off = (piece ^ (16 * (is_v ? fV<D>(e * kRpl) : fK<D>(e * kRpl)))) + row_off;
      const uint32_t dst = dma_base + is_v * 2 * TILEB + buf * TILEB + e * 1024;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2"
                   :
                   : "s"(dst), "v"(off), "s"(base)
                   : "memory", "m0");
    }
  };
  auto issue_all = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < kLd; ++e) {
      issue_one(buf, e, 0);
      issue_one(buf, e, 1);
    }
  };
  // 8 bit: what has arrived goes to slot buf as bf16.
  auto put_held = [&](int buf) __attribute__((always_inline)) {
    if constexpr (FP8) {
      int ln = lane;
      asm volatile("" : "+v"(ln));
#pragma unroll
      for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
        for (int e = 0; e < kLd; ++e) {
          const int row = wave * kRows + e * kRpl + ln / kLpr, c = ln % kLpr;
          const int f = is_v ? fV<D>(row) : fK<D>(row);
          unsigned char* at = lds + is_v * 2 * TILEB + buf * TILEB + row * ROWB;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            u32x4 x;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              x[2 * i] = fp8_lo_to_bf16(held[is_v][e][2 * half + i]);
              x[2 * i + 1] = fp8_hi_to_bf16(held[is_v][e][2 * half + i]);
            }
            *reinterpret_cast<u32x4*>(at + (((2 * c + half) ^ f) << 4)) = x;
          }
        }
    }
  };

  if (first < n_tiles) {
    seek(first);
    issue_all(0);
  }

  // ---- LDS read offsets ----
  // K fragment of step kk: row i32 (+ 32 rt), slot (2 kk + hh) ^ fK: step 0's address with kk << 5 XOR-ed in
  uint32_t koff0 = lds_base + i32 * ROWB + ((hh ^ fK<D>(i32)) << 4);
  static_assert(ROWB % 256 == 0 || (KS - 1) << 5 < ROWB, "kk << 5 stays inside the row");
  // transpose reads of V: lane = 32 hh + 16 g2 + 4 j + c reads 8 bytes of key row (16 u + 8 w + 4 hh + j) at head-dim
  // offset 32 t + 16 g2 + 4 c; the 16-lane group gets, in lane 4 c + e, keys j = 0 .. 3 of head-dim 32 t + 16 g2 + 4 c + e
  uint32_t voff0[2];  // [w2], tile t = 0 (tile t: t << 6 XOR-ed in); + u * 16 * ROWB
  {
    const int i16 = lane & 15, g2 = (lane >> 4) & 1;
    const int j = i16 >> 2, c = i16 & 3;
#pragma unroll
    for (int w2 = 0; w2 < 2; ++w2) {
      const int row = 8 * w2 + 4 * hh + j, piece = 2 * g2 + (c >> 1);
      voff0[w2] = lds_base + 2 * TILEB + row * ROWB + (((piece ^ fV<D>(row)) & (P - 1)) << 4) + 8 * (c & 1);
    }
  }

  // ---- Q^T: slot (hh, e) of step kk stands for d = 16 kk + 8 hh + e.  The loop needs a positive scale (the maximum is
  // taken on raw scores): its sign goes into Q, and scale 0 (uniform weights) becomes Q = 0 with scale 1. ----
  u32x4 qf[KS];
  {
    const int i = (unsigned)my_r / (unsigned)p.group, h = hk * p.group + my_r - i * p.group;
    const bf16_t* qp = a.q + (int64_t)(w.s.row0 + i) * a.sq.t + (int64_t)h * a.sq.h + 8 * hh;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = *reinterpret_cast<const u32x4*>(qp + 16 * kk);
  }
  if (a.scale_log2e < 0.f) {
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] ^= 0x80008000u;
  } else if (a.scale_log2e == 0.f) {
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = u32x4{0u, 0u, 0u, 0u};
  }
  const float scale = a.scale_log2e == 0.f ? 1.0f : fabsf(a.scale_log2e);

  float m_ref = -INFINITY, l = 0.f;
  f32x16 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;

  // Scores of a tile: s[rt][r] = raw score (key 32 rt + 8 (r / 4) + 4 hh + r % 4 of the tile, this lane's row).  The
  // fragments are requested as raw instructions and waited for by hand: through the compiler they would wait for the
  // direct-to-LDS loads of the next tile, which go out one by one between the products.
  auto scores = [&](f32x16 (&s)[2], uint32_t slot_off, bool more, int fill) __attribute__((always_inline)) {
    constexpr int kAhead = 4;  // steps whose fragments are on their way (all 8 would hold 32 registers more)
    u32x4 kq[kAhead][2];
    uint32_t kb = koff0 + slot_off;
    asm volatile("" : "+v"(kb));
#define RF_ISSUE_K(KK)                                                                                       \
  {                                                                                                          \
    const uint32_t ka = kb ^ ((KK) << 5);                                                                    \
    asm volatile("ds_read_b128 %0, %1" : "=v"(kq[(KK) % kAhead][0]) : "v"(ka));                              \
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(kq[(KK) % kAhead][1]) : "v"(ka), "n"(32 * ROWB));    \
  }
    RF_ISSUE_K(0)
    RF_ISSUE_K(1)
    RF_ISSUE_K(2)
    RF_ISSUE_K(3)
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[rt][r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kLoads = 2 * kLd;
    constexpr int kEvery = kLoads < KS ? KS / kLoads : 1, kPer = kLoads < KS ? 1 : kLoads / KS;
    static_assert(kLoads * kEvery == KS * kPer, "loads spread evenly over the contraction steps");
    auto st = [&](auto tag) __attribute__((always_inline)) {
      constexpr int kk = decltype(tag)::value;
      u32x4 &k0 = kq[kk % kAhead][0], &k1 = kq[kk % kAhead][1];
      constexpr int kYounger = KS - 1 - kk < kAhead - 1 ? KS - 1 - kk : kAhead - 1;
      asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(k0), "+v"(k1) : "n"(2 * kYounger));
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k0), __builtin_bit_cast(bf16x8, qf[kk]), s[0], 0, 0, 0);
      s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k1), __builtin_bit_cast(bf16x8, qf[kk]), s[1], 0, 0, 0);
      if constexpr (kk + kAhead < KS) RF_ISSUE_K(kk + kAhead)
      if (!FP8 && more && kk % kEvery == 0) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const int e = kk / kEvery * kPer + j;
          issue_one(fill, e >> 1, e & 1);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    st(std::integral_constant<int, 0>{});
    st(std::integral_constant<int, 1>{});
    st(std::integral_constant<int, 2>{});
    st(std::integral_constant<int, 3>{});
    if constexpr (KS > 4) {
      st(std::integral_constant<int, 4>{});
      st(std::integral_constant<int, 5>{});
      st(std::integral_constant<int, 6>{});
      st(std::integral_constant<int, 7>{});
    }
  };
#undef RF_ISSUE_K
  // Running maximum and sum; P^T as operands of the second product.
  auto soften = [&](f32x16 (&s)[2], u32x4 (&pb)[4]) __attribute__((always_inline)) {
    float tmax = -INFINITY;
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, s[rt][r]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(tmax), __float_as_uint(tmax), false, false);
    tmax = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale;
    if (__builtin_amdgcn_ballot_w64(tmax > m_ref + kTau) != 0) {
      const float m_new = fmaxf(m_ref, tmax);
      const float corr = (m_new == -INFINITY) ? 1.0f : fast_exp2(m_ref - m_new);
      m_ref = m_new;
      l *= corr;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] *= corr;
    }
    const float neg_m = (m_ref == -INFINITY) ? 0.f : -m_ref;
    float psum = 0.f, psum1 = 0.f;
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int r2 = 0; r2 < 8; ++r2) {
        const uint32_t pk = pack_bf16(fast_exp2(fmaf(s[rt][2 * r2], scale, neg_m)), fast_exp2(fmaf(s[rt][2 * r2 + 1], scale, neg_m)));
        pb[2 * rt + (r2 >> 2)][r2 & 3] = pk;
        typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
        const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3f803f80u);
        if (rt == 0) psum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones, psum, false);
        else psum1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk), ones, psum1, false);
      }
    l += psum + psum1;
  };

  // One tile.  BUF is a compile-time constant, so that every LDS access is a register plus an immediate offset.
  auto tile_step = [&](int key0, bool more, auto buf_tag) __attribute__((always_inline)) {
    constexpr int BUF = decltype(buf_tag)::value;
    f32x16 s[2];
    scores(s, BUF * TILEB, more, BUF ^ 1);
    u32x2 va[2][DT][2];
    uint32_t vb_[2] = {voff0[0], voff0[1]};
    asm volatile("" : "+v"(vb_[0]), "+v"(vb_[1]));
#define RF_ISSUE_V(STAGE, U)                                                              \
  _Pragma("unroll") for (int t = 0; t < DT; ++t) {                                        \
    _Pragma("unroll") for (int w2 = 0; w2 < 2; ++w2) asm volatile(                        \
        "ds_read_b64_tr_b16 %0, %1 offset:%2"                                             \
        : "=v"(va[STAGE][t][w2])                                                          \
        : "v"(vb_[w2] ^ (t << 6)), "n"(BUF * TILEB + (U) * 16 * ROWB));                   \
  }
    // at most PENDING transpose reads are still in flight; the registers of STAGE are tied to the wait
#define RF_WAIT_V(STAGE, PENDING)                                                         \
  if constexpr (DT == 4)                                                                  \
    asm volatile("s_waitcnt lgkmcnt(%8)"                                                  \
                 : "+v"(va[STAGE][0][0]), "+v"(va[STAGE][0][1]), "+v"(va[STAGE][1][0]),   \
                   "+v"(va[STAGE][1][1]), "+v"(va[STAGE][2][0]), "+v"(va[STAGE][2][1]),   \
                   "+v"(va[STAGE][3][0]), "+v"(va[STAGE][3][1])                           \
                 : "n"(PENDING));                                                         \
  else                                                                                    \
    asm volatile("s_waitcnt lgkmcnt(%4)"                                                  \
                 : "+v"(va[STAGE][0][0]), "+v"(va[STAGE][0][1]), "+v"(va[STAGE][1][0]),   \
                   "+v"(va[STAGE][1][1])                                                  \
                 : "n"(PENDING));
#define RF_PV_STEP(STAGE, U)                                                              \
  _Pragma("unroll") for (int t = 0; t < DT; ++t) {                                        \
    u32x4 x;                                                                              \
    x[0] = va[STAGE][t][0][0]; x[1] = va[STAGE][t][0][1];                                 \
    x[2] = va[STAGE][t][1][0]; x[3] = va[STAGE][t][1][1];                                 \
    acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(                                     \
        __builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, pb[U]), acc[t], 0, 0, 0); \
  }
    RF_ISSUE_V(0, 0)
    RF_ISSUE_V(1, 1)
    if (key0 + kBK - 1 > wave_min_last) {  // uniform: some row does not see all of the tile
#pragma unroll
      for (int rt = 0; rt < 2; ++rt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = key0 + 32 * rt + 8 * (r >> 2) + 4 * hh + (r & 3);
          s[rt][r] = (key <= my_last) ? s[rt][r] : -INFINITY;
        }
    }
    u32x4 pb[4];
    soften(s, pb);
    constexpr int NV = 2 * DT;  // transpose reads a contraction step
    RF_WAIT_V(0, NV)
    RF_PV_STEP(0, 0)
    RF_ISSUE_V(0, 2)
    RF_WAIT_V(1, NV)
    RF_PV_STEP(1, 1)
    RF_ISSUE_V(1, 3)
    RF_WAIT_V(0, NV)
    RF_PV_STEP(0, 2)
    RF_WAIT_V(1, 0)
    RF_PV_STEP(1, 3)
  };

#undef RF_ISSUE_V
#undef RF_WAIT_V
#undef RF_PV_STEP

  // Keys that some rows of the workgroup do not see, or none, have probability 0 there, but 0 times infinity or NaN is
  // not 0.  So, in the tiles that have such keys, V rows that no row sees (slots behind the last token among them) are
  // cleared, and values of the others that are not finite are cleared and their keys noted: once the keys are done, they
  // are added to the rows that see them (a probability is above 0 by definition, so the value itself will do).
  // A wavefront goes over the 16 rows that it has loaded.
  auto clear_unseen = [&](int key0, int buf) __attribute__((always_inline)) {
    int ln = lane;
    asm volatile("" : "+v"(ln));
#pragma unroll
    for (int e = 0; e < kRows * P / kWave; ++e) {
      const int row = wave * kRows + e * (kWave / P) + ln / P, key = key0 + row;
      u32x4* at = reinterpret_cast<u32x4*>(lds + (2 + buf) * TILEB + row * ROWB + 16 * (ln % P));
      u32x4 x = *at;
      uint32_t odd = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t f = not_finite<false>(x[i]);
        odd |= f;
        x[i] = key <= wg_last ? x[i] & ~f : 0u;
      }
      if (key > wg_last || (key > wg_min_last && odd != 0)) *at = x;
      if (key > wg_min_last && key <= wg_last && odd != 0) atomicOr(&scratch->noted[(key - edge0) >> 5], 1u << ((key - edge0) & 31));
    }
  };

  if constexpr (FP8) {
    if (first < n_tiles) put_held(0);
  }
  auto turn = [&](int kt, auto buf_tag) __attribute__((always_inline)) {
    constexpr int BUF = decltype(buf_tag)::value;
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wavefront's share of the tile has landed
    __syncthreads();                     // everyone's has, and everyone is done reading the other slot
    const bool more = kt + 1 < n_tiles;
    const int key0 = kt * kBK;
    if (key0 + kBK - 1 > wg_min_last) {
      clear_unseen(key0, BUF);
      __syncthreads();
    }
    if (more) seek(kt + 1);
    if (FP8 && more) issue_all(BUF ^ 1);  // (inside the branch below they would cost a hundred spilled registers)
    if (key0 > wave_last) {
      if (!FP8 && more) issue_all(BUF ^ 1);
    } else {
      tile_step(key0, more, buf_tag);
    }
    if constexpr (FP8) {
      if (more) put_held(BUF ^ 1);
    }
  };
  for (int kt = first; kt < n_tiles; kt += 2) {
    turn(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < n_tiles) turn(kt + 1, std::integral_constant<int, 1>{});
  }

  for (int i = 0; i < 8 && first < n_tiles; ++i) {
    for (uint32_t noted = __builtin_amdgcn_readfirstlane(scratch->noted[i]); noted != 0; noted &= noted - 1) {
      const int key = edge0 + 32 * i + __builtin_ctz(noted), at = (unsigned)key / (unsigned)p.page;
      int id = p.pages[(int64_t)w.b * p.table_pitch + at];
      id = id < 0 || id >= p.n_pages ? 0 : id;
      const int64_t off = (int64_t)id * p.page_stride + (int64_t)(key - at * p.page) * p.slot_stride + (int64_t)hk * p.head_stride;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t x = cached_bf16<FP8>(a.v, off + 32 * t + 8 * (r >> 2) + 4 * hh + (r & 3));
          const bool take = (key <= my_last) & (not_finite<false>(x) != 0);
          acc[t][r] += take ? from_bf16((bf16_t)x) : 0.f;
        }
    }
  }

  // ---- the state, or O = acc / l: rows through LDS, a wavefront its own 32, so that they leave whole ----
  int lane_ = lane;  // (opaque, as above)
  asm volatile("" : "+v"(lane_));
  l += __shfl_xor(l, 32, 64);
  __syncthreads();  // every wavefront is done with the last tile
  if (bad != 0) scratch->bad = 1;
  __syncthreads();
  if (scratch->bad != 0) l = NAN;  // a page that the cache does not have (a wavefront has looked up a quarter of them)
  if (l != l) m_ref = 0.f;  // (a row of NaN may have no maximum, and is no empty state)
  if (w.chunks > 1) {
    constexpr int kPitch = D + 4, kQuads = D / 4, kHalf = 16;  // 16 rows at a time
    static_assert(kNW * kHalf * kPitch * 4 <= 4 * TILEB, "the rows fit the K/V buffers");
    float* stage = reinterpret_cast<float*>(lds) + wave * (kHalf * kPitch);
    const int64_t row0 = (((int64_t)w.slot * p.Hkv + hk) << kTilesRowsLog2) + 32 * wave;
    if ((lane_ >> 5) == 0 && wave_r0 + (lane_ & 31) < rows) {
      a.part_m[row0 + (lane_ & 31)] = m_ref;
      a.part_l[row0 + (lane_ & 31)] = l;
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (((lane_ & 31) >> 4) == half) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4)
            *reinterpret_cast<f32x4*>(stage + ((lane_ & 31) & 15) * kPitch + 32 * t + 8 * r4 + 4 * (lane_ >> 5)) =
                f32x4{acc[t][4 * r4], acc[t][4 * r4 + 1], acc[t][4 * r4 + 2], acc[t][4 * r4 + 3]};
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < kHalf * kQuads / kWave; ++i) {
        const int row = i * (kWave / kQuads) + lane_ / kQuads, quad = lane_ % kQuads;
        const f32x4 x = *reinterpret_cast<const f32x4*>(stage + row * kPitch + 4 * quad);
        if (wave_r0 + 16 * half + row < rows)
          __builtin_nontemporal_store(x, reinterpret_cast<f32x4*>(a.part_acc + (row0 + 16 * half + row) * D + 4 * quad));
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : a.v_scale / l;
  unsigned char* stage = lds + (wave * 32) * ROWB;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      // acc[t][4 r4 + j] = O[my_r][32 t + 8 r4 + 4 (lane_ >> 5) + j]
      u32x2 x;
      x[0] = pack_bf16(acc[t][4 * r4] * inv, acc[t][4 * r4 + 1] * inv);
      x[1] = pack_bf16(acc[t][4 * r4 + 2] * inv, acc[t][4 * r4 + 3] * inv);
      *reinterpret_cast<u32x2*>(stage + (lane_ & 31) * ROWB + (((4 * t + r4) ^ fK<D>((lane_ & 31))) << 4) + 8 * (lane_ >> 5)) = x;
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  constexpr int kRowsOut = kWave / P;
#pragma unroll
  for (int i = 0; i < 32 / kRowsOut; ++i) {
    const int row = i * kRowsOut + lane_ / P, slot = lane_ % P, r = wave_r0 + row;
    const u32x4 x = *reinterpret_cast<const u32x4*>(stage + row * ROWB + ((slot ^ fK<D>(row)) << 4));
    if (r < rows) {
      const int tok = (unsigned)r / (unsigned)p.group, h = hk * p.group + r - tok * p.group;
      __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(a.o + (int64_t)(w.s.row0 + tok) * a.so.t + (int64_t)h * a.so.h + 8 * slot));
    }
  }
}

template <int D, bool FP8>
__global__ __launch_bounds__(kNW* kWave, 2) void paged_tiles_kernel(const PagedArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[tiles_lds_bytes<D>()];
  __shared__ TilesScratch scratch;
  paged_tiles<D, FP8>(a, blockIdx.x, lds, &scratch);
}

// A batch of both kinds in one launch: sequences of few rows wait for memory while those of many keep the matrix unit
// busy.  The tiles go first, since they last longest (us, in a launch each / this / taking turns eight workgroups at a
// time; 1 sequence of 16 brings new tokens: 32 sequences of 512 over up to 4096 keys, d = 64, 56.5 / 46.1 / 54, 16 of
// 2048 over 8000, d = 128, 314 / 294 / 375, 16 of 64 over 600 19.5 / 13.0 / 13.4).
template <int D, bool FP8>
__global__ __launch_bounds__(kNW* kWave, 2) void paged_both_kernel(const PagedArgs few, const PagedArgs many, unsigned many_blocks) {
  static_assert(kWaves == kNW, "one size of workgroup");
  constexpr int kLds = tiles_lds_bytes<D>() > rows_lds_bytes<D, 1, FP8>() ? tiles_lds_bytes<D>() : rows_lds_bytes<D, 1, FP8>();
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kLds];
  __shared__ TilesScratch scratch;
  if (blockIdx.x < many_blocks) paged_tiles<D, FP8>(many, blockIdx.x, lds, &scratch);
  else paged_rows<D, 1, FP8>(few, blockIdx.x - many_blocks, lds, &scratch.share);
}

}  // namespace

#define RF_BY_TYPE(RF_LAUNCH)                  \
  if (p.d == 128) {                            \
    if (fp8) RF_LAUNCH(128, true);             \
    else RF_LAUNCH(128, false);                \
  } else {                                     \
    if (fp8) RF_LAUNCH(64, true);              \
    else RF_LAUNCH(64, false);                 \
  }                                            \
  return hipGetLastError()

hipError_t launch_paged_tiles(const PagedArgs& a, bool fp8, hipStream_t s) {
  const Paged& p = a.p;
  const int64_t grid = tiles_blocks(a);
  if (grid > UINT32_MAX / (kNW * kWave)) return hipErrorInvalidValue;
#define RF_TILES(DD, F8) hipLaunchKernelGGL((paged_tiles_kernel<DD, F8>), dim3((unsigned)grid), dim3(kNW * kWave), 0, s, a)
  RF_BY_TYPE(RF_TILES);
#undef RF_TILES
}

hipError_t launch_paged_both(const PagedArgs& few, const PagedArgs& many, bool fp8, hipStream_t s) {
  const Paged& p = few.p;
  const int64_t nf = rows_blocks(few), nm = tiles_blocks(many);
  if (nf + nm > UINT32_MAX / (kNW * kWave)) return hipErrorInvalidValue;
#define RF_BOTH(DD, F8)                                                                                          \
  hipLaunchKernelGGL((paged_both_kernel<DD, F8>), dim3((unsigned)(nf + nm)), dim3(kNW * kWave), 0, s, few, many, \
                     (unsigned)nm)
  RF_BY_TYPE(RF_BOTH);
#undef RF_BOTH
}
#undef RF_BY_TYPE

}  // namespace rf
