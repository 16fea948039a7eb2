// Device-side helpers of the serving operators: where a packed token or a workgroup's share of a ragged batch
// lies, from the arrays on the device.
#pragma once
#include "../csrc/rf_device.h"
#include "serving_launch.h"

namespace rf {

// The largest number of keys that a sequence's row of the page table has room for.
__device__ __forceinline__ int capacity_of(const Paged& p) {
  const int64_t c = (int64_t)p.table_len * p.page;
  return c < (INT32_MAX - (1 << 16)) ? (int)c : INT32_MAX - (1 << 16);
}

struct Sequence {
  int row0, n;  // first packed token and how many there are
  int len;      // keys
  bool over;    // more keys than the table has room for
};

// Sequence b, cut to what the tensors hold whatever the arrays say.
__device__ __forceinline__ Sequence load_sequence(const Paged& p, int b) {
  const int s0 = p.seq_start[b], s1 = p.seq_start[b + 1], len = p.kv_len[b], most = capacity_of(p);
  Sequence s;
  s.row0 = min(max(s0, 0), p.T);
  s.n = min(max(s1, s.row0), p.T) - s.row0;
  s.over = len > most;
  s.len = min(max(len, 0), most);
  return s;
}

// The last index i of the ascending starts[0 .. n-1] with starts[i] <= t, -1 if there is none; the whole wavefront
// takes part, 64 probes a step.
__device__ __forceinline__ int find_start(const int32_t* starts, int n, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 64) {
    const int step = (n + 63) >> 6;
    const int at = lane * step;
    const bool ok = at < n && starts[lo + at] <= t;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(ok));
    if (c == 0) return -1;
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  const bool ok = lane < n && starts[lo + lane] <= t;
  return lo + __popcll(__builtin_amdgcn_ballot_w64(ok)) - 1;
}

// Inclusive sum over the lanes up to this one (row shifts within 16 lanes, then the rows' last lanes handed on).
__device__ __forceinline__ int wave_inclusive_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// How a launch of the attention kernels deals out a ragged batch.  The sequences whose packed rows (new tokens times
// query heads that share a KV head) number lo_rows + 1 .. hi_rows belong to the launch, 1 << rows_log2 of them make a
// tile, and a tile's keys are cut into chunks of one length.  That length follows from the keys of the whole batch, so
// that chunks of equal size come out however unequal the sequences are: the host, which does not know the lengths, need
// not.
struct Deal {
  int rows_log2, lo_rows, hi_rows;
  int round;   // shares that the chip takes at once, for one KV head; 0: nothing is cut
  int rounds;  // of the chunks of long contexts
  int slack;   // eighths of a workgroup's share of one round that the longest tile may have more
  __host__ __device__ int target() const { return round * rounds; }
};
constexpr int kLeastChunk = 128;   // keys
constexpr int kLongShare = 2048;   // keys: a workgroup's in one round, from which on contexts are long

struct Share {
  Sequence s;
  int b, tile, chunk, chunks, chunk_keys;
  int slot;        // of this share among those of sequences in several chunks
  int tile_index;  // of its tile among all tiles
  int all_shares, all_tiles;  // of the batch (where there is no such share)
};

// The unit that find_share() counts keys in, as a power of 2: 64 for tables of up to 2^23 keys a sequence, and so much
// larger for longer ones that 32 bits hold the sum over a launch that may cut (at most 2^14 tiles).
__device__ __forceinline__ int unit_log2_of(const Paged& p) {
  const int most = capacity_of(p);
  return most <= 1 << 23 ? 6 : 32 - __clz(most - 1) - 17;
}

// Keys of a chunk, a multiple of 128, or INT32_MAX: from the tiles of the batch, the keys that they have together and
// the longest one's, these in units.
//  - A batch whose longest tile is little more than a workgroup's share of one round is not cut.  (slack: little is an
//    eighth where a chunk's state is small.  A tile of 128 rows leaves 66 KB for a chunk, which the joining launch reads
//    again: 7 eighths.  us at 1 / 4 / 8 eighths, 32 heads over 8, d = 128: 8 sequences of 300 new tokens over 600 to 3000
//    keys 165 / 141 / 137, 2 of 1024 over 800 to 8000 259 / 214 / 213; one of 1024 over 16000, 2 tiles a share,
//    296 / 302 / 316.)
//  - Little work goes in one round: a second one would cost a workgroup's way into the cache (the arrays, the page
//    table, the first keys: three trips to memory) again.  Every sequence's last chunk is half empty on average.
//  - Much goes in several, so that unequal last chunks do not leave the chip idle at the end.
// us of a decode step, 32 heads over 8, d = 128, with chunks for one round / two / four: 64 contexts of 400 to 8192
// 229 / 210 / 203; one of 32768 34 / 40 / 43; 8 of 2000 19 / 20 / 21.
__device__ __forceinline__ int chunk_keys_of(const Deal& d, unsigned tiles, unsigned units, unsigned longest, int unit_log2) {
  if (d.round == 0) return INT32_MAX;
  const unsigned even = (units + d.round - 1) / (unsigned)d.round;
  if (longest <= even + even * d.slack / 8) return INT32_MAX;
  unsigned share;
  if (even <= (unsigned)(kLongShare >> unit_log2)) {
    const unsigned left = tiles < (unsigned)d.round ? d.round - tiles / 2 : d.round;
    share = (units + left - 1) / left;
  } else {
    share = (units + d.target() - 1) / (unsigned)d.target();
  }
  return (int)min((((uint64_t)share << unit_log2) + 127) & ~(uint64_t)127, (uint64_t)(INT32_MAX - 127));
}

__device__ __forceinline__ unsigned chunks_of(int len, int chunk_keys) {
  return len <= chunk_keys ? 1u : ((unsigned)len + (unsigned)chunk_keys - 1) / (unsigned)chunk_keys;
}

__device__ __forceinline__ int tiles_of(const Paged& p, const Deal& d, const Sequence& s) {
  const int rows = s.n * p.group;
  return rows > d.lo_rows && rows <= d.hi_rows ? ((rows - 1) >> d.rows_log2) + 1 : 0;
}

// What find_share needs of LDS.
struct ShareScratch {
  int totals[4][4];
  Share share;
  int found;
};

// Share number `unit` of the batch; false past the last one.  Shares are counted sequence by sequence, tile by tile.
// There are at most target + tiles of them, and at most 2 target with more than one chunk to their tile: such a tile has
// over chunk_keys keys, so ceil(keys / chunk_keys) is below twice keys / chunk_keys, and the sum of all keys / chunk_keys
// is at most target.  All of this holds for sequences that do not overlap; where the arrays say nonsense and more tiles
// come of it than the host has counted (n_tiles), the batch has no shares.  Called by whole workgroups of 256 threads.
// last_first: shares of batches of up to 64 sequences are numbered from the last one on.
__device__ __forceinline__ bool find_share(const Paged& p, const Deal& d, int n_tiles, int unit, ShareScratch* scratch,
                                           bool last_first, Share* out) {
  const int lane = threadIdx.x & 63;
  const int unit_log2 = unit_log2_of(p);
  auto units_of = [&](const Sequence& x) { return ((unsigned)x.len + (1u << unit_log2) - 1) >> unit_log2; };
  if (p.B <= kWave) {
    // a sequence to a lane, in every wavefront
    Sequence s{0, 0, 0, false};
    if (lane < p.B) s = load_sequence(p, lane);
    const int tiles = tiles_of(p, d, s);
    // (no sequence has more tiles than n_tiles, which a grid's size keeps below 2^24: the sum does not wrap)
    const int tiles_upto = wave_inclusive_scan(tiles), all_tiles = __builtin_amdgcn_readlane(tiles_upto, 63);
    if (all_tiles > n_tiles) {
      out->all_shares = out->all_tiles = 0;
      return false;
    }
    int chunk_keys = INT32_MAX;
    if (d.round > 0) {
      const unsigned units = __builtin_amdgcn_readlane(wave_inclusive_scan(tiles * units_of(s)), 63);
      const unsigned longest = (unsigned)wave_max(tiles > 0 ? (float)units_of(s) : 0.f);
      chunk_keys = __builtin_amdgcn_readfirstlane(chunk_keys_of(d, all_tiles, units, longest, unit_log2));
    }
    const int chunks = chunks_of(s.len, chunk_keys);
    const int upto = wave_inclusive_scan(tiles * chunks), slots_upto = wave_inclusive_scan(chunks > 1 ? tiles * chunks : 0);
    const int all_shares = __builtin_amdgcn_readlane(upto, 63);
    if (last_first && unit < all_shares) unit = all_shares - 1 - unit;
    const uint64_t past = __builtin_amdgcn_ballot_w64(upto > unit);
    if (past == 0) {
      out->all_shares = all_shares;
      out->all_tiles = all_tiles;
      return false;
    }
    const int f = __ffsll((unsigned long long)past) - 1;
    auto get = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
    out->chunks = get(chunks);
    const int units = get(tiles) * out->chunks, at = unit - (get(upto) - units);
    out->tile = out->chunks == 1 ? at : __builtin_amdgcn_readfirstlane((unsigned)at / (unsigned)out->chunks);
    out->chunk = at - out->tile * out->chunks;
    out->slot = get(slots_upto) - units + at;
    out->tile_index = get(tiles_upto) - get(tiles) + out->tile;
    out->b = f;
    out->chunk_keys = chunk_keys;
    out->s = Sequence{get(s.row0), get(s.n), get(s.len), get((int)s.over) != 0};
    return true;
  }
  // four sequences to a thread, 1024 at a time
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int kEach = 4, kBlock = 4 * kWave * kEach;
  Sequence s[kEach];
  int tiles[kEach];
  auto load = [&](int b0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int b = b0 + threadIdx.x * kEach + i;
      s[i] = Sequence{0, 0, 0, false};
      if (b < p.B) s[i] = load_sequence(p, b);
      tiles[i] = tiles_of(p, d, s[i]);
    }
  };
  load(0);
  if (threadIdx.x == 0) scratch->found = 0;
  unsigned units = 0, longest = 0;
  float all = 0.f;
  for (int b0 = 0;;) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      units += tiles[i] * units_of(s[i]);
      longest = max(longest, tiles[i] > 0 ? units_of(s[i]) : 0);
      all += (float)tiles[i];
    }
    b0 += kBlock;
    if (b0 >= p.B) break;
    load(b0);
  }
  units = wave_inclusive_scan(units);
  all = wave_sum(all);
  longest = (unsigned)wave_max((float)longest);
  if (lane == 63) {
    scratch->totals[0][wave] = units;
    scratch->totals[1][wave] = (int)fminf(all, 1e9f);
    scratch->totals[2][wave] = longest;
  }
  __syncthreads();
  units = longest = 0;
  all = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    units += scratch->totals[0][i];
    all += (float)scratch->totals[1][i];
    longest = max(longest, (unsigned)scratch->totals[2][i]);
  }
  if (__builtin_amdgcn_readfirstlane(all > (float)n_tiles)) {
    out->all_shares = out->all_tiles = 0;
    return false;
  }
  const int chunk_keys = __builtin_amdgcn_readfirstlane(chunk_keys_of(d, (unsigned)all, units, longest, unit_log2));
  if (p.B > kBlock) load(0);
  int base = 0, slot_base = 0, tile_base = 0;
  for (int b0 = 0;;) {
    int mine = 0, slots = 0, here = 0, chunks[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      chunks[i] = chunks_of(s[i].len, chunk_keys);
      mine += tiles[i] * chunks[i];
      slots += chunks[i] > 1 ? tiles[i] * chunks[i] : 0;
      here += tiles[i];
    }
    const int upto = wave_inclusive_scan(mine), slots_upto = wave_inclusive_scan(slots), here_upto = wave_inclusive_scan(here);
    __syncthreads();  // the totals before have been read
    if (lane == 63) {
      scratch->totals[0][wave] = upto;
      scratch->totals[1][wave] = slots_upto;
      scratch->totals[2][wave] = here_upto;
    }
    __syncthreads();
    int from = base + upto - mine, slot = slot_base + slots_upto - slots, tile = tile_base + here_upto - here;
    for (int i = 0; i < 4; ++i) {
      if (i < wave) {
        from += scratch->totals[0][i];
        slot += scratch->totals[1][i];
        tile += scratch->totals[2][i];
      }
      base += scratch->totals[0][i];
      slot_base += scratch->totals[1][i];
      tile_base += scratch->totals[2][i];
    }
    if (unit >= from && unit < from + mine) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int units = tiles[i] * chunks[i];
        if (unit >= from && unit < from + units) {
          Share w;
          w.s = s[i];
          w.b = b0 + threadIdx.x * kEach + i;
          w.tile = (unsigned)(unit - from) / (unsigned)chunks[i];
          w.chunk = unit - from - w.tile * chunks[i];
          w.chunks = chunks[i];
          w.chunk_keys = chunk_keys;
          w.slot = slot + unit - from;
          w.tile_index = tile + w.tile;
          w.all_shares = w.all_tiles = 0;
          scratch->share = w;
          scratch->found = 1;
        }
        from += units;
        slot += chunks[i] > 1 ? units : 0;
        tile += tiles[i];
      }
    }
    __syncthreads();
    if (scratch->found != 0) {
      const Share w = scratch->share;
      auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
      out->s = Sequence{uniform(w.s.row0), uniform(w.s.n), uniform(w.s.len), uniform((int)w.s.over) != 0};
      out->b = uniform(w.b);
      out->tile = uniform(w.tile);
      out->chunk = uniform(w.chunk);
      out->chunks = uniform(w.chunks);
      out->chunk_keys = uniform(w.chunk_keys);
      out->slot = uniform(w.slot);
      out->tile_index = uniform(w.tile_index);
      return true;
    }
    b0 += kBlock;
    if (b0 >= p.B) {
      out->all_shares = __builtin_amdgcn_readfirstlane(base);
      out->all_tiles = __builtin_amdgcn_readfirstlane(tile_base);
      return false;
    }
    load(b0);
  }
}

// A 4-byte word of FP8 E4M3 codes as bf16 (exact): codes 0, 1 / codes 2, 3.
__device__ __forceinline__ uint32_t fp8_lo_to_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}
__device__ __forceinline__ uint32_t fp8_hi_to_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
}

// All bits of the packed values (bf16, or FP8 E4M3) that are infinities or NaN: an exponent of all ones; all but the sign
// set.
template <bool FP8>
__device__ __forceinline__ uint32_t not_finite(uint32_t x) {
  if constexpr (FP8) return ((((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
  return ((((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
}

// Element `at` of a cache as bf16.
template <bool FP8>
__device__ __forceinline__ uint32_t cached_bf16(const unsigned char* cache, int64_t at) {
  if constexpr (FP8) return fp8_lo_to_bf16(cache[at]) & 0xffffu;
  return reinterpret_cast<const bf16_t*>(cache)[at];
}

}  // namespace rf
