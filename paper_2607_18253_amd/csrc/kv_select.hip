// kv_select.hip -- which rows of a context stay within a budget.
//
// Of a sequence's n rows and a kv head, the first F and the last L stay, and of those between the
// ones of the largest weights, of equal ones the lowest positions; all in ascending order.  A weight
// is taken as a 32-bit number that orders as it does (-0 as 0, NaN above all).  The smallest number
// to stay is found digit by digit from the top: counts of a digit's values among the numbers that
// agree with it so far, in LDS, and a prefix sum over them from the largest value down.  The digits
// are 10, 11 and 11 bits, those of a context that is cut over workgroups 9, 8, 8 and 7: the first one is sign
// and exponent at least, since of weights that lie close together a shorter one is the same for most, and
// their counts would wait for one another.  The positions then come out in one more pass, by
// prefix sums over ballots.
//
// Bound by latency: a few dependent steps between barriers for some 10 KB of weights, 24 us for 2040 contexts
// of 1.3k rows on the mean (waves wait 57 % of their time, LDS is busy in 8 % of the cycles; read again for
// every digit 67); and a context that is cut takes five launches, 33 us for 8 of 130k rows (349 with a
// workgroup each).
#include "../../include/lar.h"
#include "kv_cut.h"

namespace lar {
namespace {

// A number that orders as the weight does.
__device__ __forceinline__ uint32_t order(float w) {
  const uint32_t b = __float_as_uint(w + 0.0f);  // -0 + 0 = 0
  return w != w ? 0xffffffffu : b >> 31 ? ~b : b | 0x80000000u;
}

// A sequence and kv head: its context, its budget, its weights.
struct Context {
  const KvSelectArgs& A;
  int n, end, head;      // end: first row of the last ones
  const int32_t* table;
  int32_t* rows;
  bool lost = false;
  __device__ __forceinline__ Context(const KvSelectArgs& a, int x) : Context(a, x / a.g.hkv, x % a.g.hkv) {}
  __device__ __forceinline__ Context(const KvSelectArgs& a, int seq, int h) : A(a), head(h) {
    n = A.spans[seq].ctx;
    end = n - A.last;
    table = A.table + (int64_t)seq * A.cols;
    rows = A.rows + ((int64_t)seq * A.g.hkv + head) * A.budget;
  }
  __device__ __forceinline__ int32_t page(int j) const { return table[j >> A.g.sh]; }
  __device__ __forceinline__ uint32_t weight(int32_t page, int j) {
    const bool in = (uint32_t)page < A.n_blocks;  // else page 0's: no branch between the loads
    lost |= !in;
    const uint32_t row = (in ? (uint32_t)page : 0u) * ((uint32_t)A.g.hkv << A.g.sh) + ((uint32_t)head << A.g.sh);
    const float w = A.weights[row + (uint32_t)(j & ((1 << A.g.sh) - 1))];
    return in ? order(w) : 0u;
  }
  __device__ __forceinline__ bool between(int j) const { return j >= A.first && j < end; }
};

// All rows of a context within its budget: entries from i on, every step-th.  A budget may end at 2^31 - 1.
__device__ __forceinline__ void fill(const KvSelectArgs& A, const Context& c, uint32_t i, uint32_t step) {
  for (; i < (uint32_t)A.budget; i += step) c.rows[i] = i < (uint32_t)c.n ? (int)i : -1;
}

// Inclusive prefix sum over a wave.
__device__ __forceinline__ int wave_sums(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}

// The value of a digit at which `want` is reached, counting from the largest one down, and how many
// of that value itself are wanted then.  count[v]: of value BINS - 1 - v.  All threads get them.
template <int BINS, int THREADS>
__device__ __forceinline__ void reach(const int* count, int* part, int* found, int& want, uint32_t& digit) {
  constexpr int kEach = (BINS + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int c[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int v = tid * kEach + i;
    c[i] = v < BINS ? count[v] : 0;
    sum += c[i];
  }
  int upto = wave_sums(sum);
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  for (int w = 0; w < THREADS / 64; ++w) upto += w < wave ? part[w] : 0;
  int before = upto - sum;
  if (before < want && want <= upto) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (before < want && want <= before + c[i]) {
        found[0] = BINS - 1 - (tid * kEach + i);
        found[1] = want - before;
      }
      before += c[i];
    }
  }
  __syncthreads();
  digit = (uint32_t)found[0];
  want = found[1];
}

// One workgroup for each sequence and kv head, R numbers for a thread in registers; contexts of
// more rows are read again in every pass.
template <int THREADS, int R>
__global__ __launch_bounds__(THREADS, 4) void k_kv_select(KvSelectArgs A) {
  constexpr int kBins = 2048, kWaves = THREADS / 64, kRows = THREADS * R;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ int count[kBins];
  __shared__ int part[kWaves], found[2];
  __shared__ int2 sums[R * kWaves];  // above the least, and equal to it
  if (*A.plan.now != A.plan.id) {
    if (tid == 0) *A.err = kKvOtherPlan;
    return;
  }
  Context c(A, blockIdx.x);
  if (c.n <= A.budget) {
    fill(A, c, tid, THREADS);
    return;
  }
  uint32_t x[R];
  const auto load = [&](int j0) {  // past the context the last row's, without a branch of threads
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (j0 + r * THREADS >= c.n) break;  // the same for all threads, here and below
      x[r] = (uint32_t)c.page(min(j0 + r * THREADS + tid, c.n - 1));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (j0 + r * THREADS >= c.n) break;
      x[r] = c.weight((int32_t)x[r], min(j0 + r * THREADS + tid, c.n - 1));
    }
  };
  load(0);
  int want = A.budget - A.first - A.last;  // rows of those between
  const bool some = want > 0;
  uint32_t least = 0;
  if (some) {
#pragma unroll 1
    for (int shift = 22; shift >= 0; shift -= 11) {
      for (int i = tid; i < kBins; i += THREADS) count[i] = 0;
      __syncthreads();
      for (int j0 = 0; j0 < c.n; j0 += kRows) {
        if (c.n > kRows) load(j0);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (j0 + r * THREADS >= c.n) break;
          const int j = j0 + r * THREADS + tid;
          const bool on = c.between(j) && (shift == 22 || (x[r] ^ least) >> (shift + 11) == 0);
          if (on) atomicAdd(&count[kBins - 1 - (x[r] >> shift & (kBins - 1))], 1);
        }
      }
      __syncthreads();
      uint32_t digit;
      reach<kBins, THREADS>(count, part, found, want, digit);
      least |= digit << shift;
    }
  }
  // rows above the least, and of the equal ones the first `want`
  int out = 0, equal = 0;
  for (int j0 = 0; j0 < c.n; j0 += kRows) {
    if (c.n > kRows) load(j0);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (j0 + r * THREADS >= c.n) break;
      const int j = j0 + r * THREADS + tid;
      const bool mid = c.between(j);
      const int a = __popcll(__ballot(j < c.n && (!mid || (some && x[r] > least))));
      const int e = __popcll(__ballot(mid && some && x[r] == least));
      if (lane == 0) sums[r * kWaves + wave] = make_int2(a, e);
    }
    __syncthreads();
    if (wave == 0) {  // to what is before each
      int a = out, e = equal;
      for (int i0 = 0; i0 < R * kWaves && j0 + i0 / kWaves * THREADS < c.n; i0 += 64) {
        const int i = i0 + lane;
        const int2 s = i < R * kWaves && j0 + i / kWaves * THREADS < c.n ? sums[i] : make_int2(0, 0);
        const int2 u = make_int2(wave_sums(s.x), wave_sums(s.y));
        if (i < R * kWaves) sums[i] = make_int2(a + u.x - s.x, e + u.y - s.y);
        a += __builtin_amdgcn_readlane(u.x, 63);
        e += __builtin_amdgcn_readlane(u.y, 63);
      }
      if (lane == 0) {
        found[0] = a;
        found[1] = e;
      }
    }
    __syncthreads();
    out = found[0];
    equal = found[1];
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (j0 + r * THREADS >= c.n) break;
      const int j = j0 + r * THREADS + tid;
      const bool mid = c.between(j), above = j < c.n && (!mid || (some && x[r] > least));
      const bool same = mid && some && x[r] == least;
      const uint64_t ma = __ballot(above), ms = __ballot(same);
      const int2 s = sums[r * kWaves + wave];
      const int a = s.x + __popcll(ma & below), e = s.y + __popcll(ms & below);
      if (above || (same && e < want)) c.rows[a + (e < want ? e : want)] = j;
    }
  }
  if (c.lost) *A.err = kKvLostPage;
}

// ------------------------------------------------------------------ long contexts
// Each context is cut into stretches of kStretch rows with a workgroup each; a launch for each digit
// writes a stretch's counts, and starts with the digit before it from the sum of all stretches'.
constexpr int kStretch = kSelectStretch, kCut = 256, kEach = kStretch / kCut;
constexpr int kDigits = kSelectDigits, kBins = kSelectBins;
constexpr int shift_of(int d) { return d == 0 ? 23 : d == 1 ? 15 : d == 2 ? 7 : 0; }
constexpr int bins_of(int d) { return d == 0 ? 512 : d == 3 ? 128 : 256; }

// A workgroup's stretch, and what it has in the working memory.
struct Cut : KvCut {
  const KvSelectArgs& A;
  __device__ __forceinline__ explicit Cut(const KvSelectArgs& a) : KvCut(kv_cut(a.spans, a.n_seq, a.g.hkv, blockIdx.x)), A(a) {}
  // the least number so far and what is wanted of those that agree with it, before digit d
  __device__ __forceinline__ int* state(int d) const {
    return A.work + ((int64_t)seq * A.g.hkv + head) * (2 * kDigits) + 2 * d;
  }
  // rows of the stretch above the digits so far
  __device__ __forceinline__ int* above() const {
    return A.work + (int64_t)A.n_seq * A.g.hkv * (2 * kDigits) + first;
  }
  // counts of a stretch, aligned to 16 bytes
  __device__ __forceinline__ int* counts(int d, int k) const {
    return A.work + (int64_t)A.n_seq * A.g.hkv * (2 * kDigits) + (A.cuts + 3) / 4 * 4 + ((first + k) * kDigits + d) * kBins;
  }
  // its rows' numbers, from the first pass on: they need not be gathered again
  __device__ __forceinline__ uint32_t* numbers() const { return A.numbers + (first + k) * kStretch; }
};

// Takes digit D of the least number from all stretches' counts: a thread has four bins of some stretches,
// eight loads on their way at a time.  `prior`: its counts of those before this one.
template <int D>
__device__ __forceinline__ void settle(const Cut& w, int* count, int* part, int* found, int& want, uint32_t& least,
                                       uint32_t& digit, int (&prior)[4]) {
  constexpr int kQuads = bins_of(D) / 4, kSide = kCut / kQuads;
  const int quad = threadIdx.x % kQuads;
  for (int i = threadIdx.x; i < bins_of(D); i += kCut) count[i] = 0;
  int sum[4] = {0, 0, 0, 0};
  for (int k0 = threadIdx.x / kQuads; k0 < w.cuts; k0 += 8 * kSide) {
    int4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = make_int4(0, 0, 0, 0);
      if (k0 + i * kSide < w.cuts) x[i] = *(const int4*)(w.counts(D, k0 + i * kSide) + 4 * quad);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int n[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        sum[b] += n[b];
        prior[b] += k0 + i * kSide < w.k ? n[b] : 0;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int b = 0; b < 4; ++b) atomicAdd(&count[4 * quad + b], sum[b]);
  __syncthreads();
  reach<bins_of(D), kCut>(count, part, found, want, digit);
  least |= digit << shift_of(D);
}

template <int DIGIT>
__global__ __launch_bounds__(kCut) void k_kv_select_count(KvSelectArgs A) {
  const int tid = threadIdx.x;
  __shared__ int count[kBins], part[kCut / 64], found[2], more;
  if (*A.plan.now != A.plan.id) {
    if (tid == 0) *A.err = kKvOtherPlan;
    return;
  }
  const Cut w(A);
  const int k = w.k;
  Context c(A, w.seq, w.head);
  int want = A.budget - A.first - A.last;
  if (c.n <= A.budget || want == 0) return;
  uint32_t v[kEach];
#pragma unroll
  for (int r = 0; r < kEach; ++r) {
    if (DIGIT == 0)
      v[r] = (uint32_t)c.page(min(k * kStretch + r * kCut + tid, c.n - 1));
    else
      v[r] = w.numbers()[r * kCut + tid];
  }
  if (DIGIT == 0)
#pragma unroll
    for (int r = 0; r < kEach; ++r) v[r] = c.weight((int32_t)v[r], min(k * kStretch + r * kCut + tid, c.n - 1));
  if (DIGIT == 0)
#pragma unroll
    for (int r = 0; r < kEach; ++r) w.numbers()[r * kCut + tid] = v[r];
  uint32_t least = 0;
  if constexpr (DIGIT > 0) {
    constexpr int kPast = DIGIT - 1;
    uint32_t digit;
    if (DIGIT > 1) {
      least = (uint32_t)w.state(kPast)[0];
      want = w.state(kPast)[1];
    }
    // this stretch's own, asked for before the digit is known
    constexpr int kOwn = (bins_of(kPast) + kCut - 1) / kCut;
    int own[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) own[i] = w.counts(kPast, k)[tid + i * kCut];
    const int above = DIGIT > 1 ? w.above()[k] : 0;
    if (tid == 0) more = 0;
    int prior[4] = {};
    settle<kPast>(w, count, part, found, want, least, digit, prior);
    if (k == 0 && tid == 0) {
      w.state(DIGIT)[0] = (int)least;
      w.state(DIGIT)[1] = want;
    }
    int sum = 0;  // of this stretch's rows with larger values of it
#pragma unroll
    for (int i = 0; i < kOwn; ++i) sum += tid + i * kCut < bins_of(kPast) - 1 - (int)digit ? own[i] : 0;
    if (sum) atomicAdd(&more, sum);
    __syncthreads();
    if (tid == 0) w.above()[k] = above + more;
  }
  constexpr int kShift = shift_of(DIGIT), kValues = bins_of(DIGIT);
  for (int i = tid; i < kValues; i += kCut) count[i] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kEach; ++r) {
    const int j = k * kStretch + r * kCut + tid;
    if (c.between(j) && (DIGIT == 0 || (v[r] ^ least) >> shift_of(DIGIT ? DIGIT - 1 : 0) == 0))
      atomicAdd(&count[kValues - 1 - (int)(v[r] >> kShift & (kValues - 1))], 1);
  }
  __syncthreads();
  for (int i = tid; i < kValues; i += kCut) w.counts(DIGIT, k)[i] = count[i];
  if (c.lost) *A.err = kKvLostPage;
}

// The positions, after all digits.
__global__ __launch_bounds__(kCut) void k_kv_select_write(KvSelectArgs A) {
  constexpr int kWaves = kCut / 64, D = kDigits - 1;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ int count[kBins], part[kWaves], found[2], before[2];
  __shared__ int2 sums[kEach * kWaves];
  if (*A.plan.now != A.plan.id) {
    if (tid == 0) *A.err = kKvOtherPlan;
    return;
  }
  const Cut w(A);
  const int k = w.k;
  Context c(A, w.seq, w.head);
  if (c.n <= A.budget) {
    fill(A, c, k * kCut + tid, w.cuts * kCut);
    return;
  }
  int want = A.budget - A.first - A.last;
  const bool some = want > 0;
  const int j0 = k * kStretch;
  uint32_t v[kEach];
#pragma unroll
  for (int r = 0; r < kEach; ++r) {
    v[r] = some ? w.numbers()[r * kCut + tid] : 0;
  }
  uint32_t least = 0, digit = 0;
  if (tid < 2) before[tid] = 0;
  if (some) {
    least = (uint32_t)w.state(D)[0];
    want = w.state(D)[1];
    const int past = tid < k ? w.above()[tid] : 0;
    int prior[4] = {};
    settle<D>(w, count, part, found, want, least, digit, prior);
    // rows above the least, and equal ones, of the stretches before this one
    const int bin = bins_of(D) - 1 - (int)digit;
    int a = past, e = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int at = 4 * (tid % (bins_of(D) / 4)) + b;
      a += at < bin ? prior[b] : 0;
      e += at == bin ? prior[b] : 0;
    }
    static_assert(kSelectCuts <= kCut);
    if (a) atomicAdd(&before[0], a);
    if (e) atomicAdd(&before[1], e);
  }
  __syncthreads();
  // the first and last rows before this stretch
  int out = before[0] + min(j0, A.first) + max(0, j0 - c.end), equal = before[1];
  uint32_t is = 0;  // bits: above, and equal
#pragma unroll
  for (int r = 0; r < kEach; ++r) {
    const int j = j0 + r * kCut + tid;
    const bool mid = c.between(j);
    const bool above = j < c.n && (!mid || (some && v[r] > least)), same = mid && some && v[r] == least;
    is |= (above ? 1u : 0u) << r | (same ? 1u : 0u) << (16 + r);
    const int a = __popcll(__ballot(above)), e = __popcll(__ballot(same));
    if (lane == 0) sums[r * kWaves + wave] = make_int2(a, e);
  }
  __syncthreads();
  if (wave == 0) {
    static_assert(kEach * kWaves == 64);
    const int2 s = sums[lane];
    sums[lane] = make_int2(out + wave_sums(s.x) - s.x, equal + wave_sums(s.y) - s.y);
  }
  __syncthreads();
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int r = 0; r < kEach; ++r) {
    const bool above = is >> r & 1, same = is >> (16 + r) & 1;
    const uint64_t ma = __ballot(above), ms = __ballot(same);
    const int2 s = sums[r * kWaves + wave];
    const int a = s.x + __popcll(ma & below), e = s.y + __popcll(ms & below);
    if (above || (same && e < want)) c.rows[a + (e < want ? e : want)] = j0 + r * kCut + tid;
  }
}

}  // namespace

hipError_t launch_kv_select(const KvSelectArgs& a, hipStream_t stream) {
  const int n = a.n_seq * a.g.hkv, threads = kv_select_threads(n, a.longest);
  if (a.work) {
    k_kv_select_count<0><<<a.cuts, kCut, 0, stream>>>(a);
    k_kv_select_count<1><<<a.cuts, kCut, 0, stream>>>(a);
    k_kv_select_count<2><<<a.cuts, kCut, 0, stream>>>(a);
    k_kv_select_count<3><<<a.cuts, kCut, 0, stream>>>(a);
    k_kv_select_write<<<a.cuts, kCut, 0, stream>>>(a);
  } else if (threads == 1024) {
    k_kv_select<1024, 32><<<n, 1024, 0, stream>>>(a);
  } else if (threads == 512) {
    k_kv_select<512, 32><<<n, 512, 0, stream>>>(a);
  } else {
    k_kv_select<256, 8><<<n, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace lar
