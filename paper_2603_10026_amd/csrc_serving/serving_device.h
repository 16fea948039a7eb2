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
// query heads that share a KV head) number lo_rows + 1 .. hi_rows belong to the launch, 1 << rows_log2 of them make a tile,
// and a tile's keys are cut into chunks of one length.  That length follows from the keys of the whole batch, so that
// about `target` chunks of equal size come out however unequal the sequences are: the host, which does not know the
// lengths, need not.  (target 0: one chunk a tile.)
struct Deal {
  int rows_log2, lo_rows, hi_rows;
  int target, least;  // least: keys of the smallest chunk, a multiple of 128
};

struct Share {
  Sequence s;
  int b, tile, chunk, chunks, chunk_keys;
  int slot;        // of this share among those of sequences in several chunks
  int tile_index;  // of its tile among all tiles
  int all_shares, all_tiles;  // of the batch (where there is no such share)
};

// Share number `unit` of the batch; false past the last one.  Shares
// are counted sequence by sequence, tile by tile.  There are at most target + tiles of them, and at most 2 target with
// more than one chunk to their tile: such a tile has over chunk_keys keys, so ceil(keys / chunk_keys) is below twice
// keys / chunk_keys, and the sum of all keys / chunk_keys is at most target.
__device__ __forceinline__ bool find_share(const Paged& p, const Deal& d, int unit, Share* out) {
  const int lane = threadIdx.x & 63;
  auto load = [&](int b0, int* tiles) {
    Sequence s{0, 0, 0, false};
    *tiles = 0;
    if (b0 + lane < p.B) {
      s = load_sequence(p, b0 + lane);
      const int rows = s.n * p.group;
      if (rows > d.lo_rows && rows <= d.hi_rows) *tiles = ((rows - 1) >> d.rows_log2) + 1;
    }
    return s;
  };
  int tiles;
  Sequence s = load(0, &tiles);
  int chunk_keys = INT32_MAX;
  if (d.target > 0) {
    float keys = (float)tiles * (float)s.len;
    for (int b0 = 64; b0 < p.B; b0 += 64) {
      int t;
      const Sequence x = load(b0, &t);
      keys += (float)t * (float)x.len;
    }
    // (1.0001: at least what the sum in 32 bits may have lost)
    const float share = fminf(ceilf(wave_sum(keys) / (float)d.target * 1.0001f), 2e9f);
    chunk_keys = max(d.least, ((int)share + 127) & ~127);
  }
  int base = 0, slot_base = 0, tile_base = 0;
  for (int b0 = 0;;) {
    const int chunks = s.len <= chunk_keys ? 1 : (int)(((unsigned)s.len + chunk_keys - 1) / (unsigned)chunk_keys);
    const int upto = wave_inclusive_scan(tiles * chunks);
    const int slots_upto = wave_inclusive_scan(chunks > 1 ? tiles * chunks : 0);
    const int tiles_upto = wave_inclusive_scan(tiles);
    const uint64_t past = __builtin_amdgcn_ballot_w64(base + upto > unit);
    if (past != 0) {
      const int f = __ffsll((unsigned long long)past) - 1;
      auto get = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
      out->chunks = get(chunks);
      const int units = get(tiles) * out->chunks;
      const int at = unit - (base + get(upto) - units);
      out->tile = out->chunks == 1 ? at : __builtin_amdgcn_readfirstlane(at / out->chunks);
      out->chunk = at - out->tile * out->chunks;
      out->slot = slot_base + get(slots_upto) - units + at;
      out->tile_index = tile_base + get(tiles_upto) - get(tiles) + out->tile;
      out->b = b0 + f;
      out->chunk_keys = __builtin_amdgcn_readfirstlane(chunk_keys);
      out->s.row0 = get(s.row0);
      out->s.n = get(s.n);
      out->s.len = get(s.len);
      out->s.over = get((int)s.over) != 0;
      return true;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
    slot_base += __builtin_amdgcn_readlane(slots_upto, 63);
    tile_base += __builtin_amdgcn_readlane(tiles_upto, 63);
    b0 += 64;
    if (b0 >= p.B) {
      out->all_shares = base;
      out->all_tiles = tile_base;
      return false;
    }
    s = load(b0, &tiles);
  }
}

// A 4-byte word of FP8 E4M3 codes as bf16 (exact): codes 0, 1 / codes 2, 3.
__device__ __forceinline__ uint32_t fp8_lo_to_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
}
__device__ __forceinline__ uint32_t fp8_hi_to_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
}

// Nonzero where one of two packed bf16 values is an infinity or NaN (its exponent all ones).
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// Element `at` of a cache as bf16.
template <bool FP8>
__device__ __forceinline__ uint32_t cached_bf16(const unsigned char* cache, int64_t at) {
  if constexpr (FP8) return fp8_lo_to_bf16(cache[at]) & 0xffffu;
  return reinterpret_cast<const bf16_t*>(cache)[at];
}

}  // namespace rf
