// The new tokens' way into a paged cache: norm and rotation of queries and keys, keys and values to their slots.
//
//   x' = x g / sqrt(mean x^2 + eps)                                   (per head; with weights only)
//   y[a] = x'[a] cos t - x'[b] sin t,  y[b] = x'[b] cos t + x'[a] sin t   for the pairs (a, b) of the first `rot` values:
//   (j, j + rot / 2), or (2 j, 2 j + 1) if interleaved, t = angle j of the token's position, from the tables
//
// in fp32, rounded once, to bf16 or to the cache's FP8 codes.  A token's position is len - n + i, its place in the cache.
//
// What bounds it is memory: 2 bytes a value in, 2 (1) out, one pass.  A head's values lie in 16 (8) lanes of 8, so the
// sum of squares is a few lane exchanges and the partner of a rotated value is a fixed number of lanes away (its exchange
// through the vector unit instead of LDS: 1 us of 44).  The
// tables' 8 bytes a pair would be twice the values' own traffic if every head read them: a wavefront holds a token's
// angles in registers and goes over several of its heads.
#include "serving_device.h"

namespace rf {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ u32x2 fp8_of(const float* y, float scale) {
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c[i] = y[i] / scale;
    c[i] = c[i] > 448.f ? 448.f : c[i];  // (comparisons: NaN stays)
    c[i] = c[i] < -448.f ? -448.f : c[i];
  }
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i], c[4 * i + 1], 0, false);
    r[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i + 2], c[4 * i + 3], w, true);
  }
  return r;
}

// parts: how many wavefronts share a token's heads; U: turns of a wavefront whose loads are under way at once;
// past: results go past the caches.
template <int D, bool FP8, int U>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(const PagedAppend a, int parts, bool past) {
  constexpr int kLanes = D / 8, kHeads = kWave / kLanes;  // lanes a head, heads a wavefront turns over at once
  const Paged& p = a.p;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((blockIdx.x * kThreads + threadIdx.x) >> 6);
  const int t = __builtin_amdgcn_readfirstlane((unsigned)wave / (unsigned)parts), part = wave - t * parts;
  if (t >= p.T) return;

  const int heads = p.Hq + 2 * p.Hkv, q_end = p.Hq, k_end = p.Hq + p.Hkv;
  const int e0 = 8 * (lane % kLanes), sub = lane / kLanes;
  const int turn = kHeads * parts;
  u32x4 x[U];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * turn + sub;
      const bf16_t* src = h < q_end   ? (const bf16_t*)a.q + (int64_t)t * a.sq.t + (int64_t)h * a.sq.h
                          : h < k_end ? (const bf16_t*)a.k + (int64_t)t * a.sk.t + (int64_t)(h - q_end) * a.sk.h
                                      : (const bf16_t*)a.v + (int64_t)t * a.sv.t + (int64_t)(h - k_end) * a.sv.h;
      x[u] = u32x4{0u, 0u, 0u, 0u};
      if (h < heads) x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + e0));
    }
  };
  // The first values need nothing but the token's number: they are on their way while the arrays say where it belongs.
  load(part * kHeads);

  int b;
  Sequence s;
  int64_t len;
  if (p.B < kWave) {
    // every sequence to a lane: one trip for all that the arrays say
    const int start = p.seq_start[min(lane, p.B)], keys = p.kv_len[min(lane, p.B - 1)];
    b = __builtin_amdgcn_readfirstlane(__popcll(__builtin_amdgcn_ballot_w64(lane <= p.B && start <= t)) - 1);
    if (b < 0 || b >= p.B) return;  // before the first sequence, or behind the last
    s.row0 = min(max(__builtin_amdgcn_readlane(start, b), 0), p.T);
    s.n = min(max(__builtin_amdgcn_readlane(start, b + 1), s.row0), p.T) - s.row0;
    len = __builtin_amdgcn_readlane(keys, b);
  } else {
    b = __builtin_amdgcn_readfirstlane(find_start(p.seq_start, p.B + 1, t));
    if (b < 0 || b >= p.B) return;
    s = load_sequence(p, b);
    len = p.kv_len[b];
  }
  if (t < s.row0 || t >= s.row0 + s.n) return;
  const int64_t pos = len - s.n + (t - s.row0);  // its key's place; negative: it has none

  int64_t slot = -1;
  if (pos >= 0 && pos < capacity_of(p)) {
    const int at = (unsigned)pos / (unsigned)p.page;
    const int id = p.pages[(int64_t)b * p.table_pitch + at];
    if (id >= 0 && id < p.n_pages) slot = (int64_t)id * p.page_stride + (int64_t)((int)pos - at * p.page) * p.slot_stride;
  }

  // ---- angles: y = x c + partner s, with the sign of s ----
  const bool turns = e0 < a.rot;
  float c[8], sn[8];
  int partner = lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c[i] = 1.f;
    sn[i] = 0.f;
  }
  if (turns) {
    const bool known = pos < a.table_rows;
    const int64_t row = pos < 0 || !known ? 0 : pos;
    const float *cr = a.cos + row * a.cos_pitch, *sr = a.sin + row * a.sin_pitch;
    const int half = a.rot / 2;
    if (a.interleaved) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[2 * i] = c[2 * i + 1] = cr[e0 / 2 + i];
        sn[2 * i + 1] = sr[e0 / 2 + i];
        sn[2 * i] = -sn[2 * i + 1];
      }
    } else {
      const bool second = e0 >= half;
      const int j0 = second ? e0 - half : e0;
      partner = second ? lane - half / 8 : lane + half / 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = cr[j0 + i];
        sn[i] = second ? sr[j0 + i] : -sr[j0 + i];
      }
    }
    if (!known) {
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = NAN;  // the tables do not reach this far
    }
  }
  float gq[8], gk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) gq[i] = gk[i] = 1.f;
  if (a.q_norm != nullptr) Elem<bf16_t>::unpack(*reinterpret_cast<const u32x4*>((const bf16_t*)a.q_norm + e0), gq);
  if (a.k_norm != nullptr) Elem<bf16_t>::unpack(*reinterpret_cast<const u32x4*>((const bf16_t*)a.k_norm + e0), gk);

  auto store = [&](auto* at, auto w) {
    if (past) __builtin_nontemporal_store(w, at);
    else *at = w;
  };
  for (int h0 = part * kHeads; h0 < heads; h0 += U * turn) {
    if (h0 != part * kHeads) load(h0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * turn + sub;
      const bool is_q = h < q_end, is_v = h >= k_end;
      float f[8], y[8];
      Elem<bf16_t>::unpack(x[u], f);
      if (is_q ? a.q_norm != nullptr : !is_v && a.k_norm != nullptr) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], ss);
        ss += dpp_f32<kDppQuadXor1>(ss);
        ss += dpp_f32<kDppQuadXor2>(ss);
        ss += dpp_f32<kDppRowHalfMirror>(ss);
        if constexpr (kLanes == 16) ss += dpp_f32<kDppRowMirror>(ss);
        const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= r * (is_q ? gq[i] : gk[i]);
      }
      if (a.rot > 0) {
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = fmaf(f[i], c[i], f[i ^ 1] * sn[i]);
        } else if (D == 128 && a.rot == 128) {
          // (half a row of 16 lanes away: a lane exchange of the vector unit)
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = fmaf(f[i], c[i], dpp_f32<0x128>(f[i]) * sn[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = fmaf(f[i], c[i], __shfl(f[i], partner, 64) * sn[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = is_v || !turns ? f[i] : y[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = f[i];
      }
      if (h >= heads) continue;
      if (is_q) {
        // (a token without a place, which no key answers either, is 0)
        const u32x4 w = pos < 0 ? u32x4{0u, 0u, 0u, 0u} : Elem<bf16_t>::pack(y);
        store(reinterpret_cast<u32x4*>((bf16_t*)a.q_out + (int64_t)t * a.so.t + (int64_t)h * a.so.h + e0), w);
      } else if (slot >= 0) {
        const int64_t at = slot + (int64_t)(is_v ? h - k_end : h - q_end) * p.head_stride + e0;
        unsigned char* cache = (unsigned char*)(is_v ? a.v_cache : a.k_cache);
        if constexpr (FP8) store(reinterpret_cast<u32x2*>(cache + at), fp8_of(y, is_v ? a.v_scale : a.k_scale));
        else store(reinterpret_cast<u32x4*>(cache + 2 * at), is_v ? x[u] : Elem<bf16_t>::pack(y));
      }
    }
  }
}

}  // namespace

// A few tokens: a wavefront for every turn over a token's heads, since the time is the trips to memory one behind the
// other.  Many: three turns under way at once, two rounds of them or one, which leaves a few wavefronts' work to every
// SIMD.  us, U = 3 and 2 to 4 wavefronts a token / U = 1 and one for each turn / one wavefront with U = 2, d = 128,
// 32 + 2 x 8 heads: 48 tokens 4.7 / 3.6 / 9.9, 256 tokens 5.3 / 4.8 / 10.6, 1000 tokens 8.1 / 11 / 14.4, 8500 tokens
// 42.2 / 60 / 46.0.  From 8 MiB on results are written past the caches, which would not keep them: 25000 tokens
// 110 us (5.7 TB/s) and 122 without, 1000 tokens 8.1 and 10.1, but 256 tokens 5.1 and 4.8.  (All bf16 caches and heads of
// 128: where the borders lie for d = 64, whose wavefronts turn over twice the heads, and for 8 bits has not been measured.)
static bool few_tokens(const Paged& p) { return p.T <= 512; }
static int64_t append_parts(const Paged& p) {
  const int64_t T = p.T, heads = p.Hq + 2 * (int64_t)p.Hkv;
  const int per_turn = kWave * 8 / p.d;
  const int64_t turns = (heads + per_turn - 1) / per_turn;
  const int64_t least = (turns + 5) / 6, most = (turns + 2) / 3, wanted = (16384 + T - 1) / T;
  return few_tokens(p) ? turns : wanted < least ? least : wanted < most ? wanted : most;
}
static int64_t append_grid(const Paged& p) {
  return (p.T * append_parts(p) + kThreads / kWave - 1) / (kThreads / kWave);
}

// (a grid holds less than 2^32 threads)
bool paged_append_fits(const Paged& p) { return p.T == 0 || append_grid(p) <= UINT32_MAX / kThreads; }

hipError_t launch_paged_append(const PagedAppend& a, hipStream_t s) {
  const int64_t T = a.p.T, heads = a.p.Hq + 2 * (int64_t)a.p.Hkv, parts = append_parts(a.p), grid = append_grid(a.p);
  const bool few = few_tokens(a.p), past = T * heads * a.p.d * 2 >= (8 << 20);
#define RF_APPEND(DD, F8)                                                                                        \
  if (few) hipLaunchKernelGGL((paged_append_kernel<DD, F8, 1>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, (int)parts, past); \
  else hipLaunchKernelGGL((paged_append_kernel<DD, F8, 3>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, (int)parts, past)
  if (a.p.d == 128) {
    if (a.fp8) {
      RF_APPEND(128, true);
    } else {
      RF_APPEND(128, false);
    }
  } else if (a.p.d == 64) {
    if (a.fp8) {
      RF_APPEND(64, true);
    } else {
      RF_APPEND(64, false);
    }
  } else {
    return hipErrorInvalidValue;
  }
#undef RF_APPEND
  return hipGetLastError();
}

}  // namespace rf
