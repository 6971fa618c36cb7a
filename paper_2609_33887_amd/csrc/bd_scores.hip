// Token scores of logit rows: log probability of a given token, entropy of the
// row's softmax and its k most probable tokens, in one pass over the logits.
//
// With M the row's largest logit, d = x - M and R = sum over all but one largest
// of e^d: log p_t = (x_t - M) - log1p(R) and H = log1p(R) - sum e^d d / (1 + R),
// whose terms never cancel, so a token of probability near 1 keeps its digits.
//
// A wave walks its part of the row 512 logits at a time and keeps the values
// above a threshold, a lower bound of the k-th largest so far, in a list in LDS;
// everything else goes into two sums, A = sum 2^y and S = sum 2^y y for
// y = (x - ref) log2(e).  The list holds the largest values, which therefore never
// enter the sums: R is formed without subtracting the largest term again.  The
// threshold comes from the first 512 logits (the k-th largest of the 64 lanes'
// maxima) and rises whenever the list passes 64 entries: then its k largest stay
// and the rest is added to the sums.
//
// Bound by the reading of the logits where rows are many (2011 rows of 152064 in bf16,
// 0.61 GB in 132 us, 4.6 TB/s; a copy moves 5.2); few rows are cut into segments and
// are a chain of threshold, steps, sorting and join (96 rows in fp32, 58 MB, 26 us).
//
// An entry is one 64-bit number, the value's ordered bits over the complement of
// its index: larger means earlier in the result, and no two are equal.
#include "bd_internal.h"

#include <math.h>

namespace bd {

constexpr int SC_NT = 256, SC_WAVES = SC_NT / 64;
constexpr int SC_STEP = 512;                   // logits of a wave's step, 8 a lane
constexpr int SC_FULL = 64;                    // a list longer than this is cut to k
constexpr int SC_CAP = SC_FULL + SC_STEP;      // a whole step fits above it
constexpr float SC_L2E = 1.44269504088896340736f, SC_LN2 = 0.69314718055994530942f;
constexpr float SC_BIG = 0x1p125f;             // differences of values below this do not overflow

// A (row, segment)'s result: sums, their reference and its largest values in order.
struct ScPart {
  float A, S, ref;
  int n;
};

// Unsigned key in the order of the values (no NaN); equal zeros have one key.
__device__ __forceinline__ uint32_t sc_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sc_value(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint64_t sc_entry(float x, int id) { return ((uint64_t)sc_key(x) << 32) | (uint32_t)~id; }
__device__ __forceinline__ float sc_x(uint64_t e) { return sc_value((uint32_t)(e >> 32)); }
__device__ __forceinline__ int sc_id(uint64_t e) { return ~(int)(uint32_t)e; }
// The difference first: equal logits give 0 whatever their size (a row may hold nothing
// but its type's lowest value), and digits are lost only where the difference has few.
__device__ __forceinline__ float sc_y(float x, float ref) { return (x - ref) * SC_L2E; }
// e * y with 0 * -inf = 0: what has no weight adds nothing
__device__ __forceinline__ float mul_zero(float e, float y) { return e == 0.f ? 0.f : e * y; }
// (A, S) relative to a reference that lies d below (d <= 0: above) the one they have
__device__ __forceinline__ void sc_rebase(float& A, float& S, float d) {
  const float f = __builtin_amdgcn_exp2f(d);
  S = mul_zero(f, fmaf(A, d, S));
  A *= f;
}

__device__ __forceinline__ float sc_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}
__device__ __forceinline__ float sc_max(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

// 8 logits from p on, whatever its alignment, and their values
template <typename T> struct ScRaw { uint32_t w[2 * sizeof(T)]; };
template <typename T>
__device__ __forceinline__ ScRaw<T> sc_load(const T* p) {
  ScRaw<T> r;
  __builtin_memcpy(r.w, p, sizeof r.w);
  return r;
}
__device__ __forceinline__ void sc_values(const ScRaw<float>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.w[i]);
}
__device__ __forceinline__ void sc_values(const ScRaw<bf16_t>& r, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(r.w[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ float sc_load1(const float* p) { return *p; }
__device__ __forceinline__ float sc_load1(const bf16_t* p) { return __uint_as_float((uint32_t)*p << 16); }

struct ScWave {
  float tau, ref, A, S;         // A, S: this lane's
  int cnt;
  __device__ __forceinline__ void add(float x) {
    // (the bound, which a NaN passes, keeps 2^-inf * -inf from being one)
    const float y = __builtin_elementwise_maximum(sc_y(x, ref), -300.f), e = __builtin_amdgcn_exp2f(y);
    A += e;
    S = fmaf(e, y, S);
  }
  // Whether add_plain may be used, and a value that weighs nothing in the sums.
  __device__ __forceinline__ bool plain() const { return fabsf(ref) < SC_BIG; }
  __device__ __forceinline__ float none() const { return plain() ? -2.f * SC_BIG : -INFINITY; }
  __device__ __forceinline__ void add_plain(float x) {        // |x| < SC_BIG, or NaN
    const float y = sc_y(x, ref), e = __builtin_amdgcn_exp2f(y);
    A += e;
    S = fmaf(e, y, S);
  }
  // The list's k largest stay, the rest goes into the sums.  A bit search for a bound
  // that exactly k entries reach; it ends where the count is k, mostly after the
  // first bits in which the values differ.
  template <int PER>
  __device__ __forceinline__ void cut(uint64_t* list, int k, int lane) {
    uint64_t e[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) e[i] = i * 64 + lane < cnt ? list[i * 64 + lane] : 0u;   // no value has key 0
    uint64_t t = 0;
#pragma unroll 1
    for (int b = 63; b >= 0; --b) {
      const uint64_t tr = t | (1ull << b);
      int n = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) n += __popcll(__ballot(e[i] >= tr));
      if (n >= k) t = tr;
      if (n == k) break;
    }
    // what is summed from here on lies at or below the threshold: below 2^64
    tau = sc_x(t);
    const float up = sc_y(tau, ref);
    if (up > 64.f && tau < INFINITY) {
      sc_rebase(A, S, -up);
      ref = tau;
    }
    int at = 0;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool stay = e[i] >= t;
      const uint64_t m = __ballot(stay);
      if (stay) list[at + __popcll(m & ((1ull << lane) - 1ull))] = e[i];
      else if (e[i]) add(sc_x(e[i]));
      at += __popcll(m);
    }
    cnt = at;
  }
  __device__ __forceinline__ void compact(uint64_t* list, int k, int lane) {
    __builtin_amdgcn_wave_barrier();
    if (cnt > k) {
      if (cnt <= 128) cut<2>(list, k, lane);
      else cut<SC_CAP / 64>(list, k, lane);
    }
    __builtin_amdgcn_wave_barrier();
  }
};

// The logit of the row's given token (NaN if there is none).
template <typename T>
__device__ __forceinline__ float sc_token(const ScoreArgs& a, int row, const T* x, bool have) {
  if (!a.logprob) return 0.f;
  const int t = a.tokens[row];
  if (!have || t < 0 || t >= a.V) return NAN;
  return t == a.suppress ? -INFINITY : sc_load1(x + t);
}

// The outputs of a row from its list (sorted, n <= 32 entries) and its sums; one wave.
__device__ __forceinline__ void sc_finish(const ScoreArgs& a, int row, const uint64_t* top, int n, float A, float S, float ref,
                                          float token, int lane) {
  const bool in = lane < n;
  const uint64_t mine = in ? top[lane] : 0u;
  const float M = n ? sc_x(top[0]) : -INFINITY, d = sc_x(mine) - M;
  float R = 0.f, W = 0.f;
  if (in && lane > 0) {
    const float y = d * SC_L2E;
    R = __builtin_amdgcn_exp2f(y);
    W = mul_zero(R, y);
  }
  R = sc_sum(R);
  W = sc_sum(W);
  if (n) sc_rebase(A, S, -sc_y(M, ref));
  R += A;
  W += S;
  float lz = log1pf(R), ent = lz - SC_LN2 * W / (1.f + R);
  if (n == 0 && A == A) {                                     // nothing above -inf
    lz = INFINITY;
    ent = 0.f;
  } else if (n == 0 || M == INFINITY) {
    lz = ent = NAN;
  }
  if (lane == 0) {
    if (a.entropy) a.entropy[row] = ent;
    if (a.logprob) a.logprob[row] = n == 0 ? (lz == INFINITY && token == token ? -INFINITY : NAN) : (token - M) - lz;
  }
  if (lane < a.k) {
    if (a.top_id) a.top_id[(size_t)row * a.k + lane] = in ? sc_id(mine) : -1;
    if (a.top_logprob) a.top_logprob[(size_t)row * a.k + lane] = in ? d - lz : lz != lz ? lz : -INFINITY;
  }
}

// Sorts the m entries of `all` into out (the k first); the others go into the sums of
// the calling threads.  Entries of 0 are none.
__device__ __forceinline__ void sc_sort(const uint64_t* all, int m, int k, uint64_t* out, float ref, float& A, float& S,
                                        int tid) {
  for (int i = tid; i < m; i += SC_NT) {
    const uint64_t e = all[i];
    if (!e) continue;
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < m; ++j) rank += all[j] > e;
    if (rank < k) {
      out[rank] = e;
    } else {
      const float y = sc_y(sc_x(e), ref), w = __builtin_amdgcn_exp2f(y);
      A += w;
      S += mul_zero(w, y);
    }
  }
}

// Sums of the workgroup's threads in a fixed order; all threads get them.
__device__ __forceinline__ void sc_block_sum(float& A, float& S, float (*red)[2], int tid) {
  A = sc_sum(A);
  S = sc_sum(S);
  __syncthreads();
  if ((tid & 63) == 0) {
    red[tid >> 6][0] = A;
    red[tid >> 6][1] = S;
  }
  __syncthreads();
  A = S = 0.f;
#pragma unroll
  for (int w = 0; w < SC_WAVES; ++w) {
    A += red[w][0];
    S += red[w][1];
  }
}

template <typename T>
__global__ __launch_bounds__(SC_NT) __attribute__((amdgpu_waves_per_eu(8, 8)))
void k_scores(ScoreArgs a, int segs, int seg_len) {
  __shared__ uint64_t list[SC_WAVES][SC_CAP];
  __shared__ uint64_t all[SC_WAVES * SCORE_MAX_K], top[SCORE_MAX_K];
  __shared__ float red[SC_WAVES][2];
  __shared__ float wref[SC_WAVES];
  __shared__ int wcnt[SC_WAVES];
  const int row = blockIdx.x / segs, seg = blockIdx.x % segs;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int src = a.row_index ? a.row_index[row] : row;
  const bool have = (unsigned)src < (unsigned)a.logit_rows;
  const T* x = (const T*)a.logits + (have ? (int64_t)src * a.ld : 0);
  const int lo = seg * seg_len, hi = have ? min(a.V, lo + seg_len) : lo;
  const float token = segs == 1 ? sc_token<T>(a, row, x, have) : 0.f;
  uint64_t* mine = list[wave];
  ScWave st;
  st.tau = -INFINITY;
  st.ref = st.A = st.S = 0.f;
  st.cnt = 0;
  bool first = true;
  constexpr int STRIDE = SC_WAVES * SC_STEP;
  int b = lo + wave * SC_STEP;
  ScRaw<T> raw{};
  if (b + SC_STEP <= hi) raw = sc_load(x + b + lane * 8);
  for (; b < hi; b += STRIDE) {
    const int i0 = b + lane * 8;
    float v[8];
    if (b + SC_STEP <= hi) {
      sc_values(raw, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = i0 + j < hi ? sc_load1(x + i0 + j) : -INFINITY;
    }
    if (b + STRIDE + SC_STEP <= hi) raw = sc_load(x + i0 + STRIDE);   // in flight meanwhile
    if ((unsigned)(a.suppress - b) < (unsigned)SC_STEP) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (i0 + j == a.suppress) v[j] = -INFINITY;
    }
    float mx = v[0], mn = v[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) {
      mx = fmaxf(mx, v[j]);
      mn = fminf(mn, v[j]);
    }
    if (first && __any(mx > -INFINITY)) {
      // threshold: just below the k-th largest of the lanes' maxima, to 16 bits
      first = false;
      const uint32_t key = mx == mx ? sc_key(mx) : 0u;
      uint32_t t = 0;
#pragma unroll 1
      for (int bit = 31; bit >= 16; --bit)
        if (__popcll(__ballot(key >= (t | (1u << bit)))) >= a.k) t |= 1u << bit;
      const float top_v = sc_max(mx == mx ? mx : -INFINITY);
      st.ref = fabsf(top_v) < INFINITY ? top_v : 0.f;
      // strictly below: the values equal to it belong to the list
      // (below 0 comes the smallest negative: -0 is 0)
      const uint32_t low = sc_key(-INFINITY);
      st.tau = t > low + 1u ? sc_value(t - (t == 0x80000000u ? 2u : 1u)) : -INFINITY;
    }
    if (__any(mx > st.tau)) {
      const float none = st.none();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = v[j] > st.tau;
        const uint64_t m = __ballot(in);
        if (m) {
          if (in) mine[st.cnt + __popcll(m & ((1ull << lane) - 1ull))] = sc_entry(v[j], i0 + j);
          v[j] = in ? none : v[j];
          st.cnt += __popcll(m);
        }
      }
    }
    if (st.plain() && __all(mn > -SC_BIG)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) st.add_plain(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) st.add(v[j]);
    }
    if (st.cnt > SC_FULL) st.compact(mine, a.k, lane);
  }
  st.compact(mine, a.k, lane);
  // ---- the waves' lists and sums, relative to one reference
  const float most = sc_max(lane < st.cnt && sc_x(mine[lane]) < INFINITY ? sc_x(mine[lane]) : -INFINITY);
  if (lane == 0) {
    // none: the sums are 0, or NaN; entries that leave the list here lie at or below the reference
    wref[wave] = st.cnt ? fmaxf(st.ref, most) : -INFINITY;
    wcnt[wave] = st.cnt;
  }
  __syncthreads();
  float ref = -INFINITY;
  int n = 0, at = 0;
#pragma unroll
  for (int w = 0; w < SC_WAVES; ++w) {
    ref = fmaxf(ref, wref[w]);
    if (w < wave) at += wcnt[w];
    n += wcnt[w];
  }
  if (ref == -INFINITY) ref = 0.f;
  float A = st.A, S = st.S;
  if (st.cnt) sc_rebase(A, S, sc_y(st.ref, ref));
  if (lane < st.cnt) all[at + lane] = mine[lane];
  __syncthreads();
  sc_sort(all, n, a.k, top, ref, A, S, tid);
  n = min(n, a.k);
  sc_block_sum(A, S, red, tid);
  if (!have) A = NAN;
  if (segs == 1) {
    if (wave == 0) sc_finish(a, row, top, n, A, S, ref, token, lane);
  } else {
    char* w = (char*)a.ws + (size_t)blockIdx.x * (sizeof(ScPart) + (size_t)a.k * sizeof(uint64_t));
    if (tid == 0) *(ScPart*)w = ScPart{A, S, n ? ref : -INFINITY, n};
    if (tid < n) ((uint64_t*)(w + sizeof(ScPart)))[tid] = top[tid];
  }
}

// Joins a row's segments.  It waits for memory more than it computes, so everything is
// asked for before anything is used.
constexpr int SC_MAX_SEGS = 16;
template <typename T>
__global__ __launch_bounds__(SC_NT) void k_scores_merge(ScoreArgs a, int segs) {
  constexpr int PER = SC_MAX_SEGS * SCORE_MAX_K / SC_NT;
  __shared__ uint64_t all[SC_MAX_SEGS * SCORE_MAX_K], top[SCORE_MAX_K];
  __shared__ float red[SC_WAVES][2];
  __shared__ ScPart head[SC_MAX_SEGS];
  const int row = blockIdx.x, tid = threadIdx.x;
  const size_t part = sizeof(ScPart) + (size_t)a.k * sizeof(uint64_t);
  const char* w = (const char*)a.ws + (size_t)row * segs * part;
  const int m = segs * a.k;
  uint64_t e[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int z = min(i * SC_NT + tid, m - 1);                // (places behind a segment's entries hold anything)
    e[i] = ((const uint64_t*)(w + z / a.k * part + sizeof(ScPart)))[z % a.k];
  }
  const int src = a.row_index ? a.row_index[row] : row;
  const bool have = (unsigned)src < (unsigned)a.logit_rows;
  const float token = sc_token<T>(a, row, (const T*)a.logits + (have ? (int64_t)src * a.ld : 0), have);
  if (tid < segs) head[tid] = *(const ScPart*)(w + tid * part);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int z = i * SC_NT + tid;
    if (z < m) all[z] = z % a.k < head[z / a.k].n ? e[i] : 0u;
  }
  float ref = -INFINITY;
  int n = 0;
#pragma unroll 4
  for (int s = 0; s < segs; ++s) {
    ref = fmaxf(ref, head[s].ref);
    n += head[s].n;
  }
  if (ref == -INFINITY) ref = 0.f;
  float A = 0.f, S = 0.f;
  if (tid < segs) {
    A = head[tid].A;                                          // 0 or NaN where a segment has no entry
    S = head[tid].S;
    if (head[tid].n) sc_rebase(A, S, sc_y(head[tid].ref, ref));
  }
  __syncthreads();
  sc_sort(all, m, a.k, top, ref, A, S, tid);
  sc_block_sum(A, S, red, tid);
  if (tid < 64) sc_finish(a, row, top, min(n, a.k), A, S, ref, token, tid);
}

// Segments of a row: about 1024 workgroups in all, four a CU, which read as fast as
// more do, while every segment costs its own threshold, sorting and part of the join
// (us of replayed calls on the same 152064 logits a row, 1 / 2 / 4 / 8 / 16 segments: 2011
// rows bf16 145 / 163 / 196 / 254 / 377, 400 rows 66 / 61 / 61 / 70 / 96, 96 rows fp32 65 /
// 44 / 32 / 27 / 27, one row 52 / 36 / 25 / 20 / 16; among calls on other rows the first
// takes the 132 above); a wave keeps two steps of its own (24 rows of 32768: 4 segments
// 14.2, 8 13.0).
static int score_segs(int rows, int V) {
  const int most = (V + 2 * SC_WAVES * SC_STEP - 1) / (2 * SC_WAVES * SC_STEP);
  int s = (int)((1024 + (int64_t)rows / 2) / rows);
  s = s < most ? s : most;
  s = s < SC_MAX_SEGS ? s : SC_MAX_SEGS;
  return s < 1 ? 1 : s;
}

size_t score_ws_bytes(int rows, int V, int k) {
  const int s = score_segs(rows, V);
  return s == 1 ? 0 : (size_t)rows * s * (sizeof(ScPart) + (size_t)k * sizeof(uint64_t));
}

hipError_t launch_token_scores(const ScoreArgs& a, bool bf16, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  if (a.k < 1 || a.k > SCORE_MAX_K || a.V < 1) return hipErrorInvalidValue;
  const int segs = score_segs(a.rows, a.V);
  if (segs > 1 && (!a.ws || a.ws_bytes < score_ws_bytes(a.rows, a.V, a.k))) return hipErrorInvalidValue;
  // whole steps a segment
  int len = (a.V + segs - 1) / segs;
  len = (len + SC_WAVES * SC_STEP - 1) / (SC_WAVES * SC_STEP) * (SC_WAVES * SC_STEP);
  const int64_t grid = (int64_t)a.rows * segs;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
#define BD_SCORES(T_)                                                    \
  do {                                                                   \
    k_scores<T_><<<(int)grid, SC_NT, 0, st>>>(a, segs, len);             \
    if (segs > 1) k_scores_merge<T_><<<a.rows, SC_NT, 0, st>>>(a, segs); \
  } while (0)
  if (bf16) BD_SCORES(bf16_t);
  else BD_SCORES(float);
#undef BD_SCORES
  return hipGetLastError();
}

}  // namespace bd
