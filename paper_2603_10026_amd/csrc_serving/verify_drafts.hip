// Verification of drafted tokens.  A sequence's rows r = 0 .. n hold the target's probabilities p_r, the draft's q_r
// and the drafted token x_r (the last row has none):
//   a = the first r < n with u_r q_r(x_r) >= p_r(x_r), or n;   x_0 .. x_{a-1} are accepted
//   w(t) = max(0, p_a(t) - q_a(t))  (a = n: p_a(t);  where w is 0 all over: p_a(t));  W = sum_t w(t)
//   the token behind them is the first t with w(0) + .. + w(t) > u W
// which draws from the target's distribution whatever the draft's was.
//
// The products, the differences and the sums are taken in 64 bits: u q and p are compared exactly, and a border between
// two tokens is off by 2^-52 of the whole and not by an fp32 rounding of it (a vocabulary has some hundred thousand borders,
// fp32 sums that are off by 1e-7 would move one draw in a hundred).
//
// What bounds it is one row of p and of q for each sequence.  A row is cut into slices: the first launch finds a
// (every workgroup for itself: two gathered values a draft, three dependent trips to memory) and sums its slice, the
// second finds the slice that the draw falls into and then the token inside it.  Without a workspace one workgroup goes
// over all slices of a sequence.  A slice is summed by 256 threads in one order in either form, so that a draw at a border,
// which the rounding of the sums decides, gives the same token.
#include "serving_device.h"

namespace rf {

namespace {

constexpr int kSumThreads = 256, kDrawThreads = 1024;
constexpr int kSlices = 64;       // at most, of a row: a lane each
constexpr int kMostWaves = kDrawThreads / kWave;

// Sum over each kSumThreads of the workgroup's threads, in every one of them.
__device__ __forceinline__ double group_sum(double v, double* s_red) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
  __syncthreads();  // what was there has been read
  if ((threadIdx.x & 63) == 0) s_red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  const int first = threadIdx.x / kSumThreads * (kSumThreads / kWave);
#pragma unroll
  for (int i = 0; i < kSumThreads / kWave; ++i) v += s_red[first + i];
  return v;
}

// Inclusive sum over the lanes up to this one.
__device__ __forceinline__ double scan(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(v, d, 64);
    if (lane >= d) v += o;
  }
  return v;
}

template <typename T>
struct Row {
  const T *p, *q;  // q null: 0, but 1 at the drafted token
  int64_t token;   // that one (-1: none)
  int64_t V;
  // w(t) for t = t0 .. t0 + kPerVec - 1; 0 past the end
  __device__ __forceinline__ void weights(int64_t t0, double* w) const {
    constexpr int N = Elem<T>::kPerVec;
    float a[N], b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = b[i] = 0.f;
    if (t0 + N <= V) {
      const u32x4 pv = *reinterpret_cast<const u32x4_any*>(p + t0);
      Elem<T>::unpack(pv, a);
      if (q != nullptr) {
        const u32x4 qv = *reinterpret_cast<const u32x4_any*>(q + t0);
        Elem<T>::unpack(qv, b);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (t0 + i < V) {
          a[i] = Elem<T>::load(p + t0 + i);
          if (q != nullptr) b[i] = Elem<T>::load(q + t0 + i);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double d = (double)a[i] - (double)(t0 + i == token ? 1.f : b[i]);
      w[i] = d < 0 ? 0.0 : d;  // (NaN stays)
    }
  }
  // Sum of w(lo .. hi - 1), of a slice to each kSumThreads of the workgroup's threads.
  __device__ __forceinline__ double slice_sum(int64_t lo, int64_t hi, double* s_red) const {
    constexpr int N = Elem<T>::kPerVec;
    double sum = 0;
#pragma unroll 2
    for (int64_t t = lo + threadIdx.x % kSumThreads * N; t < hi; t += kSumThreads * N) {
      double w[N];
      weights(t, w);
#pragma unroll
      for (int i = 0; i < N; ++i) sum += w[i];
    }
    return group_sum(sum, s_red);
  }
  // The first t of lo .. hi - 1 of weight above 0 whose running sum is over x; the last one of weight above 0 if none is
  // (the border was lost to the order of the sums), -1 without such a one.  By kDrawThreads threads.
  __device__ __forceinline__ int64_t find(int64_t lo, int64_t hi, double x, double* s_red, int* s_at) const {
    constexpr int N = Elem<T>::kPerVec;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double before = 0;
    int64_t last = -1;
    for (int64_t t0 = lo; t0 < hi; t0 += kDrawThreads * N) {
      const int64_t t = t0 + threadIdx.x * N;
      double w[N], sum = 0;
      int mine = -1;
      if (t < hi) {
        weights(t, w);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          sum += w[i];
          if (w[i] > 0) mine = i;
        }
      }
      const double upto = scan(sum);
      if (lane == 63) s_red[wave] = upto;
      const uint64_t some = __builtin_amdgcn_ballot_w64(mine >= 0);
      const int back = some != 0 ? 63 - __clzll((unsigned long long)some) : -1;  // the last lane with some weight
      if (lane == max(back, 0)) s_at[kMostWaves + wave] = back < 0 ? -1 : (int)threadIdx.x * N + mine;
      if (lane == 0) s_at[wave] = -1;
      __syncthreads();
      double base = before;
      for (int i = 0; i < wave; ++i) base += s_red[i];
      // the wavefront that the border lies in, and there the first lane with weight that is past it
      if (base <= x && base + s_red[wave] > x) {
        const uint64_t over = some & __builtin_amdgcn_ballot_w64(base + upto > x);
        const int front = over != 0 ? __ffsll((unsigned long long)over) - 1 : back;
        if (lane == front) {
          double run = base + (upto - sum);
          int at = mine;
          for (int i = N - 1; i >= 0; --i) {
            double r = run;
#pragma unroll
            for (int j = 0; j < N; ++j) r += j <= i ? w[j] : 0.0;
            bool weighs = false;
#pragma unroll
            for (int j = 0; j < N; ++j) weighs |= j == i && w[j] > 0;
            if (weighs && r > x) at = i;
          }
          s_at[wave] = threadIdx.x * N + at;
        }
      }
      __syncthreads();
      for (int i = 0; i < kMostWaves; ++i)
        if (s_at[i] >= 0) return t0 + s_at[i];
      for (int i = 0; i < kMostWaves; ++i) {
        if (s_at[kMostWaves + i] >= 0) last = t0 + s_at[kMostWaves + i];
        before += s_red[i];
      }
      __syncthreads();
    }
    return last;
  }
};

struct Place {
  int row0, n, accepted;  // rows of the sequence; drafts: n - 1
};

__device__ __forceinline__ Place rows_of(const VerifyDrafts& a, int b) {
  Place w;
  const int s0 = a.seq_start[b], s1 = a.seq_start[b + 1];
  w.row0 = min(max(s0, 0), a.R);
  w.n = min(max(s1, w.row0), a.R) - w.row0;
  w.accepted = max(0, w.n - 1);
  return w;
}

// The sequence's rows and how many of its drafts are accepted: 64 drafts at a time, by every wavefront.
template <typename T>
__device__ __forceinline__ Place place_of(const VerifyDrafts& a, int b) {
  Place w = rows_of(a, b);
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < w.n - 1; i0 += 64) {
    const int i = i0 + lane;
    bool refused = false;
    if (i < w.n - 1) {
      const int64_t r = w.row0 + i;
      const int x = a.tokens[r];
      refused = true;
      if (x >= 0 && x < a.V) {
        const float p = Elem<T>::load((const T*)a.target + r * a.target_pitch + x);
        const float q = a.draft != nullptr ? Elem<T>::load((const T*)a.draft + r * a.draft_pitch + x) : 1.0f;
        refused = !((double)a.u_accept[r] * (double)q < (double)p);
      }
    }
    const uint64_t no = __builtin_amdgcn_ballot_w64(refused);
    if (no != 0) {
      w.accepted = i0 + __ffsll((unsigned long long)no) - 1;
      break;
    }
  }
  return w;
}

template <typename T>
__device__ __forceinline__ Row<T> row_of(const VerifyDrafts& a, const Place& w, bool whole) {
  const int64_t r = w.row0 + w.accepted;
  const bool refused = !whole && w.accepted < w.n - 1;
  Row<T> row;
  row.p = (const T*)a.target + r * a.target_pitch;
  row.q = refused && a.draft != nullptr ? (const T*)a.draft + r * a.draft_pitch : nullptr;
  row.token = refused && a.draft == nullptr ? a.tokens[r] : -1;
  row.V = a.V;
  return row;
}

// Values of a slice: whole turns of a summing workgroup, so that every slice starts at the same place of a vector.  A
// workgroup makes three trips to memory before its first value, so that it should have some thousand values, but not
// many thousands (us, both launches, fp32, slices of 8192 / 4096 / 2048 values: 64 x 131072 20.9 / 18.3 / 18.4, 128 x
// 131072 29.6 / 26.5 / -; bf16, 128 x 50001 13.4 / 12.1 / 13.0); where few workgroups come of it, half as many.
inline int64_t slice_values(int64_t B, int64_t V, int per_turn) {
  int64_t v = B * ((V + 4095) / 4096) >= 256 ? 4096 : 2048;
  const int64_t least = (V + kSlices - 1) / kSlices;
  v = least > v ? least : v;
  return (v + per_turn - 1) / per_turn * per_turn;
}

// sums: [B][slices], then how many drafts each sequence has accepted, [B] of 32 bits.
template <typename T>
__global__ __launch_bounds__(kSumThreads) void verify_sums_kernel(const VerifyDrafts a, double* sums, int slices, int64_t values) {
  __shared__ double s_red[kSumThreads / kWave];
  const int b = (unsigned)blockIdx.x / (unsigned)slices, s = blockIdx.x - b * slices;
  const Place w = place_of<T>(a, b);
  if (w.n == 0) return;
  const Row<T> row = row_of<T>(a, w, false);
  const int64_t lo = s * values;
  const double sum = row.slice_sum(lo, min(a.V, lo + values), s_red);
  if (threadIdx.x == 0) {
    sums[(int64_t)b * slices + s] = sum;
    if (s == 0) reinterpret_cast<int32_t*>(sums + (int64_t)a.B * slices)[b] = w.accepted;
  }
}

// sums null: all is found here.
template <typename T>
__global__ __launch_bounds__(kDrawThreads) void verify_draw_kernel(const VerifyDrafts a, const double* sums, int slices, int64_t values) {
  __shared__ double s_red[kMostWaves], s_sums[kSlices];
  __shared__ int s_at[2 * kMostWaves];
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const double drawn = (double)a.u_sample[b];
  Place w;
  double mine = 0;  // a slice's sum, to each lane
  if (sums != nullptr) {
    mine = lane < slices ? sums[(int64_t)b * slices + lane] : 0.0;
    const int accepted = reinterpret_cast<const int32_t*>(sums + (int64_t)a.B * slices)[b];
    w = rows_of(a, b);
    w.accepted = w.n > 0 ? accepted : 0;
  } else {
    w = place_of<T>(a, b);
  }
  if (threadIdx.x == 0) a.accepted[b] = w.accepted;
  if (w.n == 0) return;
  Row<T> row = row_of<T>(a, w, false);
  double upto, total;
  for (int turn = 0;; ++turn) {
    if (sums == nullptr || turn != 0) {
      for (int s0 = 0; s0 < slices; s0 += kDrawThreads / kSumThreads) {
        const int s = s0 + threadIdx.x / kSumThreads;  // (past the last slice: no values)
        const int64_t lo = s * values;
        const double v = row.slice_sum(lo, min(a.V, lo + values), s_red);
        if (threadIdx.x % kSumThreads == 0 && s < slices) s_sums[s] = v;
      }
      __syncthreads();
      mine = lane < slices ? s_sums[lane] : 0.0;
    }
    upto = scan(mine);
    total = __shfl(upto, 63, 64);
    if (total != 0 || w.accepted == w.n - 1 || turn != 0) break;
    row = row_of<T>(a, w, true);  // nothing is left of the target: its own probabilities
  }
  int64_t token = -1;
  if (total > 0 && total <= 1.7976931348623157e308) {
    const double x = fmax(drawn * total, 0.0);
    const uint64_t some = __builtin_amdgcn_ballot_w64(mine > 0), over = some & __builtin_amdgcn_ballot_w64(upto > x);
    // (x at or past the total: the last slice that has any)
    const int s = over != 0 ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll((unsigned long long)some);
    const double before = s > 0 ? __shfl(upto, max(s - 1, 0), 64) : 0.0;
    const int64_t lo = s * values;
    token = row.find(lo, min(a.V, lo + values), x - before, s_red, s_at);
  }
  for (int i = threadIdx.x; i < w.n; i += kDrawThreads)
    a.out[w.row0 + i] = i < w.accepted ? a.tokens[w.row0 + i] : i == w.accepted ? (int32_t)token : -1;
}

int num_slices(int64_t V, int64_t values) { return (int)((V + values - 1) / values); }

}  // namespace

// (a grid holds less than 2^32 threads)
bool verify_drafts_fits(int64_t B) { return B <= UINT32_MAX / kDrawThreads; }

size_t verify_drafts_bytes(int64_t B, int64_t V) {
  const int slices = num_slices(V, slice_values(B, V, kSumThreads * 4));  // (rows of 4-byte values have as many slices or more)
  return slices > 1 && B * slices <= UINT32_MAX / kSumThreads ? ((size_t)B * slices * sizeof(double) + (size_t)B * sizeof(int32_t) + 15) & ~(size_t)15 : 0;
}

hipError_t launch_verify_drafts(const VerifyDrafts& a, void* workspace, hipStream_t s) {
  const int64_t values = slice_values(a.B, a.V, kSumThreads * (a.bf16 ? 8 : 4));
  const int slices = num_slices(a.V, values);
  double* sums = slices > 1 ? (double*)workspace : nullptr;
#define RF_VERIFY(T)                                                                                                    \
  if (sums != nullptr)                                                                                                  \
    hipLaunchKernelGGL((verify_sums_kernel<T>), dim3((unsigned)(a.B * slices)), dim3(kSumThreads), 0, s, a, sums, slices, values); \
  hipLaunchKernelGGL((verify_draw_kernel<T>), dim3((unsigned)a.B), dim3(kDrawThreads), 0, s, a, sums, slices, values)
  if (a.bf16) {
    RF_VERIFY(bf16_t);
  } else {
    RF_VERIFY(float);
  }
#undef RF_VERIFY
  return hipGetLastError();
}

}  // namespace rf
