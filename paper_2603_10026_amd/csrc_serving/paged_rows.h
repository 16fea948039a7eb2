// Attention of a few new tokens a sequence over a paged cache: a decode step, a handful of drafted tokens.
//
//   P = scale q K^T;  m = max_j P;  l = sum_j exp(P - m);  o = sum_j exp(P - m) v[j] / l,   j <= len - n + i
//
// A sequence's new tokens times the query heads that share a KV head are one tile's rows, 16 or 32 of them, so that a
// key and a value are fetched once for all of them; the keys are cut into chunks (find_share) and a workgroup's four
// wavefronts deal the 32-key steps of a chunk among themselves.  Every wavefront carries the running (m, l, acc) of the
// max -> sum-exp -> weighted-sum cascade; the four states are merged through LDS, and a chunk's state goes to the
// workspace (or, of a tile in one chunk, the result to o).
//
// What bounds it is the stream of K and V: 512 bytes a key and KV head (d = 128, bf16) against 32 floating operations
// a byte.  So whole rows are read, 256 bytes by 16 lanes at once, with non-temporal loads, K one step ahead.  K passes
// through a wavefront's own piece of LDS into operand layout, V is transposed in registers, and the scores are computed
// transposed (S^T = K Q^T) so that the probabilities are the second product's operand where they are formed.
//
// A page holds a multiple of 16 slots and a chunk starts at one: the 16 keys of a half step lie in one page, one
// scalar address with 32-bit lane offsets.  The lanes of a wavefront hold the addresses of its next 64 half steps, so
// that the page table is not waited for at every step.
//
// Probabilities are rounded to bf16 for the second product (the matrix unit takes no wider operand at this rate); l
// sums the rounded ones, so that the part of the error that all keys share cancels.  Everything else is fp32.
#pragma once
#include <math.h>

#include "paged_attention.h"

namespace rf {

namespace {

constexpr int kWaves = 4, kStepKeys = 32, kChunkStep = kWaves * kStepKeys;

template <int D, int NR, bool FP8>
constexpr int rows_lds_bytes() {
  const int merge = (kWaves * 16 * (D + 4) + 2 * kWaves * 16) * 4, keys = kWaves * kStepKeys * D * 2;
  return merge > keys ? merge : keys;
}

// block: of the launch's share of the grid; smem: rows_lds_bytes(), 16-byte aligned.
template <int D, int NR, bool FP8>
__device__ __forceinline__ void paged_rows(const PagedArgs& a, unsigned block, unsigned char* smem, ShareScratch* scratch) {
  constexpr int ES = FP8 ? 1 : 2;            // bytes of a cached element
  constexpr int KS = D / 32;                 // contraction steps of S^T
  constexpr int DPL = D / 16;                // values of a V row a lane holds
  constexpr int VW = DPL / 2;                // dwords of them as bf16
  constexpr int VL = DPL * ES / 4;           // dwords of them in memory
  constexpr int kRow = D * ES;               // bytes of a row in memory
  constexpr int kLpr = kRow / 16;            // lanes a K row
  constexpr int kRpl = kWave / kLpr;         // K rows a load
  constexpr int kLoads = kStepKeys / kRpl;   // K loads a step
  constexpr int kLdsRow = D * 2, kSlots = kLdsRow / 16;
  constexpr int kTile = kStepKeys * kLdsRow;
  constexpr int R = 16 * NR;
  constexpr int kPitch = D + 4;

  const Paged& p = a.p;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4;

  // Workgroups are dealt round-robin to the 8 XCDs.  Rows of up to 128 bytes: the KV heads of a share go to one of them,
  // one behind the other, so that its address translation serves neighbouring heads' rows together (32 contexts of 32768
  // in FP8, d = 128, 425 -> 402 us); longer rows gain nothing by it (64 contexts of 4300 in bf16 207 -> 213).
  int unit, hk;
  if constexpr (kRow <= 128) {
    const int turn = __builtin_amdgcn_readfirstlane((block >> 3) / (unsigned)p.Hkv);
    hk = __builtin_amdgcn_readfirstlane((block >> 3) - turn * p.Hkv);
    unit = turn * 8 + (block & 7);
  } else {
    unit = __builtin_amdgcn_readfirstlane(block / (unsigned)p.Hkv);
    hk = __builtin_amdgcn_readfirstlane(block - unit * p.Hkv);
  }
  Share w;
  const bool found = find_share(p, a.deal, a.n_tiles, unit, scratch, false, &w);
  if (hk == 0 && wave == 0) note_tile(a, unit, found, w);
  if (!found) return;

  const int rows = w.s.n * p.group;
  const int r0 = w.tile * R;
  const int shift = w.s.len - w.s.n;  // token i sees keys 0 .. i + shift
  const int i_first = __builtin_amdgcn_readfirstlane(r0 / p.group);
  const int i_last = __builtin_amdgcn_readfirstlane((min(rows, r0 + R) - 1) / p.group);
  const int seen_all = a.causal ? max(0, min(w.s.len, i_first + shift + 1)) : w.s.len;   // keys that every row sees
  const int seen_any = a.causal ? max(0, min(w.s.len, i_last + shift + 1)) : w.s.len;    // ... that any row sees
  const int lo = min((int64_t)seen_any, (int64_t)w.chunk * w.chunk_keys);
  const int hi = min((int64_t)seen_any, (int64_t)lo + w.chunk_keys);

  // this lane's query rows (columns of the transposed score tiles)
  int seen[NR];
  u32x4 qf[NR][KS];
#pragma unroll
  for (int nr = 0; nr < NR; ++nr) {
    const int r = min(r0 + 16 * nr + i16, rows - 1);
    const int i = r / p.group, h = hk * p.group + r - i * p.group;
    seen[nr] = a.causal ? max(0, min(hi, i + shift + 1)) : hi;
    const bf16_t* qp = a.q + (int64_t)(w.s.row0 + i) * a.sq.t + (int64_t)h * a.sq.h + 8 * g;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[nr][kk] = *reinterpret_cast<const u32x4*>(qp + 32 * kk);
  }

  // ---- addresses: lane 2 s + f holds the element offset of half f of this wavefront's step s (of 32) ----
  uint32_t off_lo, off_hi;
  uint64_t bad = w.s.over ? 1 : 0;
  const int last_half = (hi - 1) & ~15;
  auto refill = [&](int step) {
    const int key = min(lo + wave * kStepKeys + (step + (lane >> 1)) * kChunkStep + 16 * (lane & 1), last_half);
    const int at = (unsigned)key / (unsigned)p.page;
    int id = p.pages[(int64_t)w.b * p.table_pitch + at];
    const bool outside = id < 0 || id >= p.n_pages;
    bad |= __builtin_amdgcn_ballot_w64(outside);
    id = outside ? 0 : id;
    const int64_t off = ((int64_t)id * p.page_stride + (int64_t)(key - at * p.page) * p.slot_stride + (int64_t)hk * p.head_stride) * ES;
    off_lo = (uint32_t)off;
    off_hi = (uint32_t)(off >> 32);
  };
  auto half_base = [&](int step, int f) {
    const int at = 2 * (step & 31) + f;
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_lo, at) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, at) << 32);
  };

  // slot e of kreg: key row kRpl e + lane / kLpr of the step; of vreg: key 4 g + e (e < 4), 16 + 4 g + e - 4
  const uint32_t slot_bytes = (uint32_t)p.slot_stride * ES;
  const uint32_t k_lane = (lane / kLpr) * slot_bytes + 16 * (lane % kLpr);
  const uint32_t v_lane = 4 * g * slot_bytes + DPL * ES * i16;
  auto issue_k = [&](const int64_t (&base)[2], u32x4 (&kreg)[kLoads]) {
#pragma unroll
    for (int e = 0; e < kLoads; ++e) {
      const int f = e * kRpl / 16, row = e * kRpl % 16;
      kreg[e] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(a.k + (base[f] + (int64_t)(row * slot_bytes)) + k_lane));
    }
  };
  auto issue_v = [&](const int64_t (&base)[2], uint32_t (&vreg)[8][VL]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned char* at = a.v + (base[e >> 2] + (int64_t)((e & 3) * slot_bytes)) + v_lane;
      if constexpr (VL == 4) {
        const u32x4 t = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
#pragma unroll
        for (int i = 0; i < VL; ++i) vreg[e][i] = t[i];
      } else if constexpr (VL == 2) {
        const u32x2 t = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(at));
#pragma unroll
        for (int i = 0; i < VL; ++i) vreg[e][i] = t[i];
      } else {
        vreg[e][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(at));
      }
    }
  };

  float m2[NR], l[NR];
  f32x4 acc[NR][DPL];  // acc[nr][t][rr] = O[row 16 nr + i16][d = DPL (4 g + rr) + t]
#pragma unroll
  for (int nr = 0; nr < NR; ++nr) {
    m2[nr] = -INFINITY;
    l[nr] = 0.f;
#pragma unroll
    for (int t = 0; t < DPL; ++t) acc[nr][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  unsigned char* ktile = smem + wave * kTile;
  auto k_slot = [&](int row, int piece) { return ktile + row * kLdsRow + ((piece ^ (row & (kSlots - 1))) << 4); };

  // O^T += V^T P^T for the values 2 tp, 2 tp + 1 of each lane's V rows (a 2 x 8 transpose of 16-bit values in registers)
  auto product = [&](const uint32_t (&vr)[8][VL], const u32x4 (&pb)[NR], int tp) __attribute__((always_inline)) {
    u32x4 lo4, hi4;
#pragma unroll
    for (int ep = 0; ep < 4; ++ep) {
      uint32_t x, y;
      if constexpr (FP8) {
        x = (tp & 1) ? fp8_hi_to_bf16(vr[2 * ep][tp >> 1]) : fp8_lo_to_bf16(vr[2 * ep][tp >> 1]);
        y = (tp & 1) ? fp8_hi_to_bf16(vr[2 * ep + 1][tp >> 1]) : fp8_lo_to_bf16(vr[2 * ep + 1][tp >> 1]);
      } else {
        x = vr[2 * ep][tp];
        y = vr[2 * ep + 1][tp];
      }
      lo4[ep] = pair_lo(x, y);
      hi4[ep] = pair_hi(x, y);
    }
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      f32x4 &even = acc[nr][2 * tp], &odd = acc[nr][2 * tp + 1];
      even = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo4), __builtin_bit_cast(bf16x8, pb[nr]), even, 0, 0, 0);
      odd = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi4), __builtin_bit_cast(bf16x8, pb[nr]), odd, 0, 0, 0);
    }
  };

  int64_t base[2];
  int at = 0;
  auto next_bases = [&]() {
    if ((at & 31) == 0) refill(at);
    base[0] = half_base(at, 0);
    base[1] = half_base(at, 1);
    ++at;
  };
  uint64_t odd_keys = 0;  // bit j: key seen_all + j (a tile's rows differ by less than 32 keys)
  u32x4 kreg[kLoads];
  uint32_t vreg[8][VL];
  int key0 = lo + wave * kStepKeys;
  if (key0 < hi) {
    next_bases();
    issue_k(base, kreg);
    issue_v(base, vreg);
  }
  // K of the next step is requested as soon as this step's has gone to LDS, V once this step's has been multiplied.
  for (; key0 < hi; key0 += kChunkStep) {
    const bool more = key0 + kChunkStep < hi;
    // ---- K: registers -> this wavefront's LDS, as bf16 ----
    // (opaque copies of the lane's number here and below: addresses made of them are made here, and not ahead of the loop
    // to be carried through it in registers)
    int ln = lane;
    asm volatile("" : "+v"(ln));
#pragma unroll
    for (int e = 0; e < kLoads; ++e) {
      const int row = e * kRpl + ln / kLpr, c = ln % kLpr;
      if constexpr (FP8) {
        u32x4 w0, w1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w0[2 * i] = fp8_lo_to_bf16(kreg[e][i]);
          w0[2 * i + 1] = fp8_hi_to_bf16(kreg[e][i]);
          w1[2 * i] = fp8_lo_to_bf16(kreg[e][2 + i]);
          w1[2 * i + 1] = fp8_hi_to_bf16(kreg[e][2 + i]);
        }
        *reinterpret_cast<u32x4*>(k_slot(row, 2 * c)) = w0;
        *reinterpret_cast<u32x4*>(k_slot(row, 2 * c + 1)) = w1;
      } else {
        *reinterpret_cast<u32x4*>(k_slot(row, c)) = kreg[e];
      }
    }
    if (more) {
      next_bases();
      issue_k(base, kreg);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

    // ---- S^T = K Q^T, two halves of 16 keys ----
    f32x4 s[NR][2];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) s[nr][0] = s[nr][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KS; ++kk)
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const u32x4 ka = *reinterpret_cast<const u32x4*>(k_slot(16 * f + (ln & 15), 4 * kk + (ln >> 4)));
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
          s[nr][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ka),
                                                             __builtin_bit_cast(bf16x8, qf[nr][kk]), s[nr][f], 0, 0, 0);
      }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();

    // ---- maximum and sum ----
    u32x4 pb[NR];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      float sc[8], tmax = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + 4 * g + ((e < 4) ? e : 12 + e);
        sc[e] = (key < seen[nr]) ? s[nr][e >> 2][e & 3] * a.scale_log2e : -INFINITY;
        tmax = fmaxf(tmax, sc[e]);
      }
      tmax = fmaxf(tmax, __shfl_xor(tmax, 16, 64));
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32, 64));
      const float m_new = fmaxf(m2[nr], tmax);
      const float m_use = (m_new == -INFINITY) ? 0.f : m_new;
      const float corr = fast_exp2(m2[nr] - m_use);
      m2[nr] = m_new;
      float psum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        pb[nr][e] = pack_bf16(fast_exp2(sc[2 * e] - m_use), fast_exp2(sc[2 * e + 1] - m_use));
        psum += bf16_lo(pb[nr][e]);
        psum += bf16_hi(pb[nr][e]);
      }
      l[nr] = l[nr] * corr + psum;
#pragma unroll
      for (int t = 0; t < DPL; ++t) acc[nr][t] *= corr;
    }

    // ---- acc += V^T P^T ----
    if (key0 + kStepKeys > seen_all) {
      // Keys that some rows do not see, or none, have probability 0 there, but 0 times infinity or NaN is not 0.  What no
      // row sees (slots behind the last token among it) is cleared, and values of the others that are not finite are
      // cleared and their keys noted: once the keys are done they are added to the rows that see them (a probability is
      // above 0 by definition, so the value itself will do).
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + 4 * g + ((e < 4) ? e : 12 + e);
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < VL; ++i) {
          const uint32_t f = key >= seen_all ? not_finite<FP8>(vreg[e][i]) : 0u;
          odd |= f;
          vreg[e][i] = key < hi ? vreg[e][i] & ~f : 0u;
        }
        const uint64_t noted = __builtin_amdgcn_ballot_w64(odd != 0 && key < hi);
        if (noted != 0) {
#pragma unroll
          for (int gg = 0; gg < 4; ++gg)
            if ((noted >> (16 * gg) & 0xffff) != 0) odd_keys |= 1ull << (key0 + 4 * gg + ((e < 4) ? e : 12 + e) - seen_all);
        }
      }
    }
#pragma unroll
    for (int tp = 0; tp < VW; ++tp) product(vreg, pb, tp);
    if (more) issue_v(base, vreg);
  }

  for (; odd_keys != 0; odd_keys &= odd_keys - 1) {
    const int key = seen_all + __builtin_ctzll(odd_keys), in = (unsigned)key / (unsigned)p.page;
    int id = p.pages[(int64_t)w.b * p.table_pitch + in];
    id = id < 0 || id >= p.n_pages ? 0 : id;
    const int64_t off = (int64_t)id * p.page_stride + (int64_t)(key - in * p.page) * p.slot_stride + (int64_t)hk * p.head_stride;
#pragma unroll
    for (int rr = 0; rr < 4; ++rr)
#pragma unroll
      for (int t = 0; t < DPL; ++t) {
        const uint32_t x = cached_bf16<FP8>(a.v, off + DPL * (4 * g + rr) + t);
        const float y = not_finite<false>(x) != 0 ? from_bf16((bf16_t)x) : 0.f;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) acc[nr][t][rr] += key < seen[nr] ? y : 0.f;
      }
  }

  // ---- merge of the four wavefronts' states, 16 rows at a time ----
  float* s_acc = reinterpret_cast<float*>(smem);
  float* s_m = s_acc + kWaves * 16 * kPitch;
  float* s_l = s_m + kWaves * 16;
#pragma unroll
  for (int nr = 0; nr < NR; ++nr) {
    float ln = l[nr];
    ln += __shfl_xor(ln, 16, 64);
    ln += __shfl_xor(ln, 32, 64);
    if (bad != 0) {  // a page that the cache does not have: NaN
      m2[nr] = 0.f;
      ln = NAN;
    }
    __syncthreads();  // the K tiles, or the rows before, have been read
    if (g == 0) {
      s_m[wave * 16 + i16] = m2[nr];
      s_l[wave * 16 + i16] = ln;
    }
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
      float* dst = s_acc + (wave * 16 + i16) * kPitch + DPL * (4 * g + rr);
#pragma unroll
      for (int t = 0; t < DPL; t += 4)
        *reinterpret_cast<f32x4*>(dst + t) = f32x4{acc[nr][t][rr], acc[nr][t + 1][rr], acc[nr][t + 2][rr], acc[nr][t + 3][rr]};
    }
    __syncthreads();
    const int here = min(16, rows - r0 - 16 * nr);
    for (int idx = threadIdx.x; idx < here * (D / 4); idx += kWaves * kWave) {
      const int rr = idx / (D / 4), c4 = idx % (D / 4);
      float mg = -INFINITY;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) mg = fmaxf(mg, s_m[i * 16 + rr]);
      const float mg_use = (mg == -INFINITY) ? 0.f : mg;
      float lg = 0.f;
      f32x4 og = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float wgt = fast_exp2(s_m[i * 16 + rr] - mg_use);  // 0 for an empty state
        lg += s_l[i * 16 + rr] * wgt;
        og += *reinterpret_cast<const f32x4*>(s_acc + (i * 16 + rr) * kPitch + 4 * c4) * wgt;
      }
      if (w.chunks > 1) {
        const int64_t at_row = ((int64_t)w.slot * p.Hkv + hk) * R + 16 * nr + rr;
        __builtin_nontemporal_store(og, reinterpret_cast<f32x4*>(a.part_acc + at_row * D + 4 * c4));
        if (c4 == 0) {
          a.part_m[at_row] = lg != lg ? 0.f : mg;  // (a row of NaN may have no maximum, and is no empty state)
          a.part_l[at_row] = lg;
        }
      } else {
        const float inv = lg == 0.f ? 0.f : a.v_scale / lg;
        const int r = r0 + 16 * nr + rr, i = r / p.group, h = hk * p.group + r - i * p.group;
        u32x2 w2;
        w2[0] = pack_bf16(og[0] * inv, og[1] * inv);
        w2[1] = pack_bf16(og[2] * inv, og[3] * inv);
        *reinterpret_cast<u32x2*>(a.o + (int64_t)(w.s.row0 + i) * a.so.t + (int64_t)h * a.so.h + 4 * c4) = w2;
      }
    }
  }
}

}  // namespace

}  // namespace rf
