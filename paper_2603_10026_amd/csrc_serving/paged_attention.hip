// Attention over a paged cache: which kernel takes which sequences, and the launch that joins the chunks of those whose
// keys were cut (the level-k fused expression of the attention cascade, as in the merge of partial states):
//   m = max_c m_c;  l = sum_c l_c 2^(m_c - m);  o = v_scale sum_c acc_c 2^(m_c - m) / l
#include "paged_attention.h"

namespace rf {

namespace {

constexpr int kJoinThreads = 256, kJoinWaves = kJoinThreads / kWave;

struct JoinArgs {
  PagedArgs part[2];
  int blocks[2];    // of each part
  int per_tile[2];  // workgroups of a tile and KV head
};

// D / 4 lanes hold a row's values.  Tiles of few rows, which may have many chunks: a wavefront takes a row and deals its
// chunks among the 64 / (D / 4) groups of lanes.  Tiles of many rows, of few chunks: a row to each group.
template <int D>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(const JoinArgs j) {
  constexpr int kQuads = D / 4, kGroups = kWave / kQuads, U = 8;
  const bool many = blockIdx.x >= j.blocks[0];
  const PagedArgs& a = many ? j.part[1] : j.part[0];
  const int block = blockIdx.x - (many ? j.blocks[0] : 0), parts = many ? j.per_tile[1] : j.per_tile[0];
  const Paged& p = a.p;
  const int lg = a.deal.rows_log2;
  const int lane = threadIdx.x & 63, grp = lane / kQuads, c4 = lane % kQuads;
  const int tile = __builtin_amdgcn_readfirstlane((unsigned)block / (unsigned)(parts * p.Hkv));
  const int rest = block - tile * parts * p.Hkv;
  const int hk = __builtin_amdgcn_readfirstlane((unsigned)rest / (unsigned)parts);
  const JoinTile t = a.tiles[tile];
  if (t.chunks == 1) return;
  const int64_t pitch = (int64_t)p.Hkv << lg;  // rows of the workspace from one chunk to the next
  const int each = many ? kGroups : 1, stride = many ? 1 : kGroups;
  const int wave = __builtin_amdgcn_readfirstlane((rest - hk * parts) * kJoinWaves + (threadIdx.x >> 6));
  for (int r0 = wave * each; r0 < t.rows; r0 += parts * kJoinWaves * each) {
    const int rr = many ? min(r0 + grp, t.rows - 1) : r0;
    const int64_t row = t.slot * pitch + ((int64_t)hk << lg) + rr;
    float m = -INFINITY, l = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = many ? 0 : grp; c0 < t.chunks; c0 += U * stride) {
      float mc[U], lc[U];
      f32x4 ac[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = row + min(c0 + u * stride, t.chunks - 1) * pitch;
        mc[u] = a.part_m[at];
        lc[u] = a.part_l[at];
        ac[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(a.part_acc + at * D + 4 * c4));
      }
      float m_new = m;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        mc[u] = c0 + u * stride < t.chunks ? mc[u] : -INFINITY;
        m_new = fmaxf(m_new, mc[u]);
      }
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float corr = fast_exp2(m - m_use);
      l *= corr;
      sum *= corr;
      m = m_new;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool none = mc[u] == -INFINITY;  // an empty state, whose sums may hold anything
        const float w = fast_exp2(mc[u] - m_use);
        l += none ? 0.f : lc[u] * w;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += none ? 0.f : ac[u][i] * w;
      }
    }
    if (!many) {
#pragma unroll
      for (int d = kQuads; d < kWave; d <<= 1) {
        const float mo = __shfl_xor(m, d, 64), m_new = fmaxf(m, mo), m_use = m_new == -INFINITY ? 0.f : m_new;
        const float w = fast_exp2(m - m_use), wo = fast_exp2(mo - m_use);
        l = l * w + __shfl_xor(l, d, 64) * wo;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = sum[i] * w + __shfl_xor(sum[i], d, 64) * wo;
        m = m_new;
      }
    }
    if (many ? r0 + grp >= t.rows : grp != 0) continue;
    const float inv = l == 0.f ? 0.f : a.v_scale / l;
    const int r = t.row + rr, i = (unsigned)r / (unsigned)p.group, h = hk * p.group + r - i * p.group;
    u32x2 w2;
    w2[0] = pack_bf16(sum[0] * inv, sum[1] * inv);
    w2[1] = pack_bf16(sum[2] * inv, sum[3] * inv);
    *reinterpret_cast<u32x2*>(a.o + (int64_t)i * a.so.t + (int64_t)h * a.so.h + 4 * c4) = w2;
  }
}

// Tiles that a launch may meet at most: every sequence adds less than one to its rows' whole tiles.
int64_t most_tiles(const Paged& p, int rows_log2) {
  return (((int64_t)p.T * p.group) >> rows_log2) + (p.B < p.T ? p.B : p.T);
}

// The launches of a call: [0] of few rows, [1] of many; none where tiles is 0.
struct Plan {
  Deal deal[2];
  int64_t tiles[2];
};

constexpr int kRoundsRows = 4, kRoundsTiles = 2, kSlackRows = 1, kSlackTiles = 7;  // see chunk_keys_of()

// Two workgroups to each of the 256 compute units; one, where the two kinds share the chip.  That is what the kernels for
// d = 128 hold (by registers; three for 16 rows of an 8-bit cache).  Those for d = 64 hold three (tiles, and 32 rows) to
// five (16 rows, 8 bit): what shares for so many would gain there has not been measured.
int round_of(const Paged& p, int64_t tiles, bool alone, int rows_log2, int slack) {
  const int workgroups = alone ? 512 : 256;
  // no sequence is long enough, or there are so many workgroups that one long sequence more or less does not matter
  if ((int64_t)p.table_len * p.page <= kLeastChunk || tiles * p.Hkv > 32 * 512 || p.Hkv > workgroups) return 0;
  const int round = workgroups / p.Hkv;
  // one sequence of so many tiles that none is over its share: whatever its length, nothing to join
  if (p.B == 1 && ((((int64_t)p.T * p.group - 1) >> rows_log2) + 1) * (8 + slack) >= 8 * (int64_t)round) return 0;
  return round;
}

Plan plan_of(const Paged& p, int64_t max_q, bool cut) {
  const int64_t longest = max_q < p.T ? max_q : p.T;
  const int64_t rows = longest * p.group;
  Plan w{};
  // Few rows: up to 32, where no sequence has more; up to 16 beside longer ones.  Only where all sequences are as long
  // as the longest one is there nothing for one of the two.
  const bool few_only = rows <= 32;
  const bool many_only = !few_only && p.T == longest * p.B;
  const int few_log2 = few_only && rows > 16 ? 5 : 4;
  if (!many_only) {
    w.tiles[0] = few_only ? most_tiles(p, few_log2) : p.B < p.T ? p.B : p.T;
    w.deal[0] = Deal{few_log2, 0, few_only ? INT32_MAX : 16, cut ? round_of(p, w.tiles[0], few_only, few_log2, kSlackRows) : 0,
                     kRoundsRows, kSlackRows};
  }
  if (!few_only) {
    w.tiles[1] = most_tiles(p, kTilesRowsLog2);
    w.deal[1] = Deal{kTilesRowsLog2, many_only ? 0 : 16, INT32_MAX,
                     cut ? round_of(p, w.tiles[1], many_only, kTilesRowsLog2, kSlackTiles) : 0, kRoundsTiles, kSlackTiles};
  }
  return w;
}

// Chunks of all tiles, if each had as many as the page table has room for.
int64_t most_chunks(const Plan& w, const Paged& p, int i) {
  return w.tiles[i] * (((int64_t)p.table_len * p.page + kLeastChunk - 1) / kLeastChunk);
}
// Shares that there may be, and rows of the workspace: see find_share().
int64_t units_of(const Plan& w, const Paged& p, int i) {
  if (w.deal[i].round == 0) return w.tiles[i];
  const int64_t shares = w.tiles[i] + w.deal[i].target(), most = most_chunks(w, p, i);
  return shares < most ? shares : most;
}
int64_t slots_of(const Plan& w, const Paged& p, int i) {
  const int64_t chunks = 2 * (int64_t)w.deal[i].target(), most = most_chunks(w, p, i);
  return ((chunks < most ? chunks : most) * p.Hkv) << w.deal[i].rows_log2;
}
int64_t part_bytes(const Plan& w, const Paged& p, int i) {
  return w.tiles[i] > 0 && w.deal[i].round > 0 ? slots_of(w, p, i) * (p.d + 2) * 4 + w.tiles[i] * (int64_t)sizeof(JoinTile) : 0;
}

}  // namespace

// (a grid holds less than 2^32 threads)
bool paged_attention_fits(const Paged& p, int64_t max_q) {
  const Plan w = plan_of(p, max_q, true);
  return (w.tiles[0] + w.deal[0].target() + 8 + w.tiles[1] + w.deal[1].target()) * p.Hkv <= UINT32_MAX / 256;
}

size_t paged_attention_bytes(const Paged& p, int64_t max_q) {
  const Plan w = plan_of(p, max_q, true);
  return (size_t)(part_bytes(w, p, 0) + part_bytes(w, p, 1));
}

hipError_t launch_paged_attention(const PagedAttention& x, void* workspace, hipStream_t s) {
  const Paged& p = x.p;
  const Plan w = plan_of(p, x.max_q, workspace != nullptr);
  JoinArgs j{};
  char* at = (char*)workspace;
  for (int i = 0; i < 2; ++i) {
    PagedArgs& a = j.part[i];
    a.p = p;
    a.deal = w.deal[i];
    a.q = (const bf16_t*)x.q;
    a.k = (const unsigned char*)x.k_cache;
    a.v = (const unsigned char*)x.v_cache;
    a.o = (bf16_t*)x.o;
    a.sq = x.sq;
    a.so = x.so;
    a.scale_log2e = x.scale_log2e;
    a.v_scale = x.v_scale;
    a.causal = x.causal;
    if (w.tiles[i] == 0) continue;
    a.n_tiles = (int)w.tiles[i];
    a.n_units = (int)units_of(w, p, i);
    if (w.deal[i].round > 0) {
      const int64_t slots = slots_of(w, p, i);
      a.part_acc = (float*)at;
      a.part_m = a.part_acc + slots * p.d;
      a.part_l = a.part_m + slots;
      a.tiles = (JoinTile*)(a.part_l + slots);
      at += part_bytes(w, p, i);
      // (a wavefront's rows in one turn, where max_q is right and there are no more than a tile has)
      const int64_t rows = (int64_t)(x.max_q < p.T ? x.max_q : p.T) * p.group, R = 1 << w.deal[i].rows_log2;
      const int64_t most = rows < 1 ? 1 : rows < R ? rows : R, turn = kJoinWaves * (i == 0 ? 1 : 4 * kWave / p.d);
      j.per_tile[i] = (int)((most + turn - 1) / turn);
      j.blocks[i] = (int)(w.tiles[i] * p.Hkv * j.per_tile[i]);
    }
  }
  const hipError_t e = w.tiles[1] == 0   ? launch_paged_rows(j.part[0], x.fp8, s)
                       : w.tiles[0] == 0 ? launch_paged_tiles(j.part[1], x.fp8, s)
                                         : launch_paged_both(j.part[0], j.part[1], x.fp8, s);
  if (e != hipSuccess) return e;
  const int blocks = j.blocks[0] + j.blocks[1];
  if (blocks == 0) return hipSuccess;
  if (p.d == 128) hipLaunchKernelGGL((paged_join_kernel<128>), dim3(blocks), dim3(kJoinThreads), 0, s, j);
  else hipLaunchKernelGGL((paged_join_kernel<64>), dim3(blocks), dim3(kJoinThreads), 0, s, j);
  return hipGetLastError();
}

}  // namespace rf
