// Paged KV cache in 8 bits: block tables and slot maps, the store and read of
// its pages.
//
// A page holds T tokens (a multiple of 32) of every kv head.  Codes are OCP fp8
// E4M3; (page, kv head) has one power-of-two scale for K and one for V.  The
// bytes of a (page, head) are tiles of 32 tokens in the order the attention's
// matrix fragments take them, so that a wave reads a tile in whole 1 KiB loads
// of 16 bytes a lane, with no LDS pass and no transposition:
//   K tile [hd / 32][dim % 32 / 16][token][dim % 16]
//   V tile [hd / 32][token / 4 % 2][dim % 32][token / 16][token / 8 % 2][token % 4]
// Lane (h = lane / 32, c = lane % 32) of a K load holds dims 32 y + 16 h .. + 15
// of token c: two 8-deep MFMA operands.  Of a V load it holds dim 32 d + c of
// tokens 16 x + 8 i + 4 h + j (x, i < 2, j < 4): the tokens whose scores the same
// lane half holds after the score product, in its register order.
#include "bd_kv.h"

namespace bd {

// ---------------------------------------------------------------- block tables
// Prefix sums over the requests of the pages given back, the pages taken and the new
// rows.  The stack of free pages is read and written through these sums, so every page
// has its place whatever thread moves it: workgroup 0 pushes and pops; the others write
// the slot map and find a popped page themselves, in the stack as it was (its places
// below the old height are not written) or, where it is one of the pages given back,
// in the table of the request that gave it (whose entries stay).  So one launch does
// all, each workgroup with sums of its own.  It is latency, a chain of loads and
// barriers: 7.3 us for 256 requests and up to 24576 rows (5.7 and 3.6 in two launches).
//
// Requests may want far more than there is: a request's pages are fewer than 2^25, so
// a wave's fit 32 bits, and the waves' sums are taken in 64.  Where the totals pass the
// test, all sums fit 32 bits (the rows' too, which wrap where they do not).
constexpr int PG_NT = 1024;
__global__ __launch_bounds__(PG_NT) void k_kv_pages(PageArgs a) {
  extern __shared__ int lds[];                 // [3][n + 1]: pages back, pages taken, rows
  __shared__ uint32_t tmp[PG_NT / 64][3];
  int* rel = lds;
  int* take = lds + a.n + 1;
  int* row = lds + 2 * (a.n + 1);
  const int tid = threadIdx.x, cap = a.max_pages * a.T;
  int64_t cr = 0, ct = 0;
  uint32_t cw = 0;
  for (int s0 = 0; s0 < a.n; s0 += PG_NT) {
    const int s = s0 + tid;
    uint32_t d[3] = {0, 0, 0}, inc[3];
    if (s < a.n) {
      const int have = min(max(a.have[s], 0), cap), want = min(max(a.want[s], 0), cap);
      const int hp = pages_of(have, a.T), wp = pages_of(want, a.T);
      d[0] = max(hp - wp, 0);
      d[1] = max(wp - hp, 0);
      d[2] = max(want - have, 0);
    }
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int j = 0; j < 3; ++j) inc[j] = d[j];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1)
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        const uint32_t o = __shfl_up(inc[j], off);
        if (lane >= off) inc[j] += o;
      }
    __syncthreads();                           // the sums before are read
    if (lane == 63)
#pragma unroll
      for (int j = 0; j < 3; ++j) tmp[wave][j] = inc[j];
    __syncthreads();
    uint32_t before[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < PG_NT / 64; ++i) {
#pragma unroll
      for (int j = 0; j < 3; ++j) before[j] += i < wave ? tmp[i][j] : 0u;
    }
    if (s < a.n) {
      rel[s] = (int)((uint32_t)cr + before[0] + inc[0] - d[0]);
      take[s] = (int)((uint32_t)ct + before[1] + inc[1] - d[1]);
      row[s] = (int)(cw + before[2] + inc[2] - d[2]);
    }
#pragma unroll
    for (int i = 0; i < PG_NT / 64; ++i) {
      cr += tmp[i][0];
      ct += tmp[i][1];
      cw += tmp[i][2];
    }
  }
  const int nf = min(max(*a.free_count, 0), a.n_pages);
  // too few pages, or more of them than the pool has: nothing is done
  const int64_t miss = nf + cr > a.n_pages ? a.n_pages - nf - cr : ct > nf + cr ? ct - nf - cr : 0;
  const int lack = miss > INT32_MAX ? INT32_MAX : miss < -INT32_MAX ? -INT32_MAX : (int)miss;
  if (tid == 0) {
    rel[a.n] = (int)cr;
    take[a.n] = (int)ct;
    row[a.n] = (int)cw;
  }
  __syncthreads();                             // the sums stand, and every thread has read the count
  // page of column col of request s as it will be
  auto page = [&](int s, int col) {
    const int hp = pages_of(min(max(a.have[s], 0), cap), a.T);
    if (col < hp) return a.table[(size_t)s * a.max_pages + col];
    const int top = nf + (int)cr - 1 - (take[s] + col - hp);
    if (top < nf) return a.free_pages[top];
    const int from = find_segment(rel, a.n, top - nf);
    const int wp = pages_of(min(max(a.want[from], 0), cap), a.T);
    return a.table[(size_t)from * a.max_pages + wp + top - nf - rel[from]];
  };
  if (blockIdx.x > 0 || gridDim.x == 1) {      // the slot map
    const int wgs = gridDim.x == 1 ? 1 : gridDim.x - 1, wg = gridDim.x == 1 ? 0 : blockIdx.x - 1;
    const int lim = lack ? 0 : min((int)cw, a.rows_cap);
    for (int r = wg * PG_NT + tid; r < lim; r += wgs * PG_NT) {
      const int s = find_segment(row, a.n, r);
      const int pos = min(max(a.have[s], 0), cap) + r - row[s];
      a.row_seq[r] = s;
      a.row_pos[r] = pos;
      a.slot[r] = (int64_t)page(s, pos / a.T) * a.T + pos % a.T;
    }
    if (gridDim.x > 1) return;
    __syncthreads();                           // the pages as they were are read
  }
  if (tid == 0) {
    a.info[0] = lack ? nf : (int)(nf + cr - ct);
    a.info[1] = lack ? 0 : (int)cw;
    a.info[2] = lack;
    a.info[3] = lack ? 0 : (int)ct;
  }
  for (int s = tid; s <= a.n; s += PG_NT) a.row_start[s] = lack ? 0 : row[s];
  if (lack) return;
  for (int i = tid; i < cr; i += PG_NT) {
    const int s = find_segment(rel, a.n, i);
    const int wp = pages_of(min(max(a.want[s], 0), cap), a.T);
    a.free_pages[nf + i] = a.table[(size_t)s * a.max_pages + wp + i - rel[s]];
  }
  for (int i = tid; i < ct; i += PG_NT) {
    const int s = find_segment(take, a.n, i);
    const int col = pages_of(min(max(a.have[s], 0), cap), a.T) + i - take[s];
    a.table[(size_t)s * a.max_pages + col] = page(s, col);
  }
}

// One workgroup alone where the caller's count is the info buffer, which it overwrites
// while others would read it.
hipError_t launch_kv_pages(const PageArgs& a, hipStream_t st) {
  if (a.n < 1 || a.n > KV_MAX_SEQS) return hipErrorInvalidValue;
  const int wgs = a.info == a.free_count ? 0 : (int)(((int64_t)a.rows_cap + PG_NT - 1) / PG_NT);
  k_kv_pages<<<1 + (wgs < 512 ? wgs : 512), PG_NT, 3 * (size_t)(a.n + 1) * sizeof(int), st>>>(a);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void k_kv_fresh(int32_t* free_pages, int n_pages, int32_t* free_count, int32_t* have,
                                                  int32_t* want, int n, int tokens) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n_pages) free_pages[i] = i;
  if (i < n) {
    have[i] = 0;
    want[i] = tokens;
  }
  if (i == 0) *free_count = n_pages;
}

hipError_t launch_kv_fresh(int32_t* free_pages, int n_pages, int32_t* free_count, int32_t* have, int32_t* want, int n,
                           int tokens, hipStream_t st) {
  const int most = n_pages > n ? n_pages : n;
  k_kv_fresh<<<(most + 255) / 256, 256, 0, st>>>(free_pages, n_pages, free_count, have, want, n, tokens);
  return hipGetLastError();
}

// ---------------------------------------------------------------- store, read
// The page that work item `item` stands for: items are the pages that the
// requests' rows touch, request by request.  False where there is none.
struct PageItem {
  int seq, page, row, t0, t1;    // table column's page, first row, tokens [t0, t1) of the page
};
template <int NT>
__device__ __forceinline__ bool page_item(const KvPages& c, const KvRows& a, int item, PageItem* out) {
  __shared__ int tmp[NT / 64];
  __shared__ int got[5];
  const int cap = a.max_pages * c.T;
  int base = 0;
  for (int s0 = 0; s0 < a.n; s0 += NT) {
    const int s = s0 + (int)threadIdx.x;
    SeqRows r{0, 0, 0};
    int np = 0;
    if (s < a.n) {
      r = seq_rows(a, s, cap);
      np = r.cnt > 0 ? (r.pos + r.cnt - 1) / c.T - r.pos / c.T + 1 : 0;
    }
    int total;
    const int inc = block_scan<NT>(np, tmp, &total) + base;
    if (item < base + total) {                 // the same for all threads
      if (np > 0 && item < inc && item >= inc - np) {
        const int k = item - (inc - np), col = r.pos / c.T + k;
        const int p0 = col * c.T;
        got[0] = s;
        got[1] = a.table[(size_t)s * a.max_pages + col];
        got[3] = max(r.pos - p0, 0);
        got[4] = min(r.pos + r.cnt - p0, c.T);
        got[2] = r.row + p0 + got[3] - r.pos;
      }
      __syncthreads();
      out->seq = got[0];
      out->page = got[1];
      out->row = got[2];
      out->t0 = got[3];
      out->t1 = got[4];
      return (unsigned)out->page < (unsigned)c.n_pages;
    }
    base += total;
  }
  return false;
}

// Exponent E of the scale 2^E of values up to amax: the smallest with
// amax / 2^E <= 448 = 0.875 2^9, kept in [-126, 119] (a normal float, and 448 2^E
// one too); the lowest where amax is 0.
__device__ __forceinline__ int scale_exp(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 126 - 9 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, -126), 119);
}
// |x|, 0 for infinities and NaN
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.4028234663852886e38f ? a : 0.f;
}
// Two codes: y to the nearest E4M3 value (ties to even), infinities to the
// largest, NaN to the NaN code.
__device__ __forceinline__ uint32_t codes2(float y0, float y1) {
  const float a = fminf(fmaxf(y0, -448.f), 448.f), b = fminf(fmaxf(y1, -448.f), 448.f);
  uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
  if (y0 != y0) c = (c & 0xFF00u) | 0x7Fu;
  if (y1 != y1) c = (c & 0x00FFu) | 0x7F00u;
  return c;
}
__device__ __forceinline__ float value1(uint32_t code) { return __builtin_amdgcn_cvt_f32_fp8((int)code, 0); }
// Four codes rounded again after a factor f <= 1 (NaN stays NaN).
__device__ __forceinline__ uint32_t recode4(uint32_t w, float f) {
  const float a = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * f, b = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * f;
  const float c = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * f, d = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * f;
  return codes2(a, b) | (codes2(c, d) << 16);
}

// Byte of (token t, dim e) in a (page, head)'s K and V.
__device__ __forceinline__ int k_byte(int t, int e, int hd) {
  return t / KT * KT * hd + ((e >> 5) * 64 + ((e >> 4) & 1) * 32 + t % KT) * 16 + (e & 15);
}
// V: 16-byte word of (tile, dim, token / 4 % 2); byte of token t in it.
__device__ __forceinline__ int v_word(int tile, int e, int h, int hd) {
  return tile * KT * hd + ((e >> 5) * 64 + h * 32 + (e & 31)) * 16;
}
__device__ __forceinline__ int v_byte(int t, int e, int hd) {
  return v_word(t / KT, e, (t >> 2) & 1, hd) + ((t >> 4) & 1) * 8 + ((t >> 3) & 1) * 4 + (t & 3);
}
__device__ __forceinline__ int v_token(int h, int b) { return (b >> 3) * 16 + ((b >> 2) & 1) * 8 + h * 4 + (b & 3); }

// A workgroup stores one (page, kv head), half of its threads K and half V (the
// workgroup is told its page once for both): the largest magnitude of the new
// rows gives the exponent (not below the page's own while it keeps tokens in front of
// them), then the rows are coded.  Kept codes are rounded again if the exponent rises;
// a page whose first token is new is cleared behind the new rows.  A thread takes 16
// values that make one 16-byte word of codes, and holds its first words' values from
// the search to the coding, so that rows of pages up to 64 tokens are read once.
//
// Bound by the chain request -> table -> rows -> exponent -> codes: one token of 64
// requests takes 6.7 us, and with many pages six workgroups a CU do not hide all of it
// (16 prompts of 512 to 1024 tokens, 16 heads of 64 in fp32, 123 MB in 39 us, 3.2 TB/s;
// with rows read twice and a workgroup a head for both K and V in turn: 44).
constexpr int ST_NT = 256, ST_HALF = ST_NT / 2;
constexpr int ST_HELD = 2;                     // words of a thread held
template <typename TT>
__global__ __launch_bounds__(ST_NT) void k_kv_store(KvPages c, KvRows a, const TT* __restrict__ K, const TT* __restrict__ V,
                                                    int64_t ldk, int64_t ldv) {
  __shared__ float red[ST_NT / 64];
  const bool is_v = __builtin_amdgcn_readfirstlane(threadIdx.x / ST_HALF);
  const int head = blockIdx.x % c.Hkv, hd = c.hd, tid = threadIdx.x % ST_HALF;
  PageItem it;
  if (!page_item<ST_NT>(c, a, blockIdx.x / c.Hkv, &it)) return;
  const int cnt = it.t1 - it.t0;
  const int64_t ld = is_v ? ldv : ldk;
  const TT* src = (is_v ? V : K) + (int64_t)it.row * ld + head * hd;      // row of token t0
  const size_t ph = (size_t)it.page * c.Hkv + head;
  uint8_t* codes = (is_v ? c.v : c.k) + ph * c.T * hd;
  float* scale = (is_v ? c.vs : c.ks) + ph;
  const bool kept = it.t0 > 0;
  const int old = kept ? scale_exponent(*scale) : -126;
  // Word i of the new rows.  K: 16 dims of a token; eight tokens side by side, so that
  // a wave reads whole rows' parts and writes runs of 128 bytes.  V: 16 tokens of a dim
  // (the halves of a tile's), over the tiles that hold new tokens; or, of a few tokens
  // behind kept ones, single codes: a token's dims side by side, whose bytes are stored
  // alone (one token of 64 requests: 6.9 us against 8.3 with whole words).
  const int ksh = hd == 128 ? 3 : 2, hsh = ksh + 4;
  const bool few = is_v && kept && cnt * hd <= 16 * ST_HALF;
  const int tile0 = it.t0 / KT, tiles = (it.t1 + KT - 1) / KT - tile0;
  const int words = few ? ST_HALF : is_v ? tiles * 2 * hd : (cnt + 7) / 8 * 8 << ksh;
  auto load = [&](int i, float* x) {
    if (few) {
#pragma unroll
      for (int b = 0; b < 16; ++b) {
        const int u = b * ST_HALF + i;
        x[b] = u < cnt << hsh ? load1(src + (int64_t)(u >> hsh) * ld + (u & (hd - 1))) : 0.f;
      }
    } else if (is_v) {
      const int e = i & (hd - 1), h = (i >> hsh) & 1, t = (tile0 + (i >> (hsh + 1))) * KT - it.t0;
#pragma unroll
      for (int b = 0; b < 16; ++b) {
        const int u = t + v_token(h, b);
        x[b] = u >= 0 && u < cnt ? load1(src + (int64_t)u * ld + e) : 0.f;
      }
    } else {
      const int t = (i >> (3 + ksh)) * 8 + (i & 7), e = ((i >> 3) & ((1 << ksh) - 1)) * 16;
#pragma unroll
      for (int b = 0; b < 16; ++b) x[b] = 0.f;
      if (t < cnt) {
        load8(src + (int64_t)t * ld + e, x);
        load8(src + (int64_t)t * ld + e + 8, x + 8);
      }
    }
  };
  float held[ST_HELD][16], top = 0.f;
#pragma unroll
  for (int j = 0; j < ST_HELD; ++j)
    if (j * ST_HALF + tid < words) load(j * ST_HALF + tid, held[j]);
#pragma unroll
  for (int j = 0; j < ST_HELD; ++j)
    if (j * ST_HALF + tid < words) {
#pragma unroll
      for (int b = 0; b < 16; ++b) top = fmaxf(top, finite_abs(held[j][b]));
    }
  for (int i = ST_HELD * ST_HALF + tid; i < words; i += ST_HALF) {
    float x[16];
    load(i, x);
#pragma unroll
    for (int b = 0; b < 16; ++b) top = fmaxf(top, finite_abs(x[b]));
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  if ((tid & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();                             // (and every thread has read the scale)
  top = fmaxf(red[is_v ? 2 : 0], red[is_v ? 3 : 1]);
  const int ex = max(scale_exp(top), old);
  const int rise = kept ? min(ex - old, 60) : 0;
  if (tid == 0) *scale = pow2i(ex);
  const float f = pow2i(-ex), fo = pow2i(-rise);
  // K's tokens before the new ones and V's tiles before theirs (single codes: also those
  // of the tile they go into): rounded again
  if (rise) {
    const int before = is_v ? (few ? tile0 + tiles : tile0) * 2 * hd : it.t0 << ksh;
    for (int i = tid; i < before; i += ST_HALF) {
      u32x4* w = (u32x4*)(codes + (is_v ? (size_t)i * 16 : (size_t)k_byte(i >> ksh, (i & ((1 << ksh) - 1)) * 16, hd)));
      u32x4 o = *w;
      const int t = (i >> (hsh + 1)) * KT;                    // V: the word's tile
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t q = recode4(o[j], fo);
        if (!is_v || t < tile0 * KT) {
          o[j] = q;
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const uint32_t m = 0xFFu << (8 * b);
            if (t + v_token((i >> 5) & 1, 4 * j + b) < it.t0) o[j] = (o[j] & ~m) | (q & m);
          }
        }
      }
      *w = o;
    }
  }
  __syncthreads();                             // before bytes of the same words are stored
  auto store = [&](int i, const float* x) {
    if (few) {
#pragma unroll
      for (int b = 0; b < 16; ++b) {
        const int u = b * ST_HALF + i;
        if (u < cnt << hsh) codes[v_byte(it.t0 + (u >> hsh), u & (hd - 1), hd)] = (uint8_t)codes2(x[b] * f, 0.f);
      }
      return;
    }
    u32x4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      o[j] = codes2(x[4 * j] * f, x[4 * j + 1] * f) | (codes2(x[4 * j + 2] * f, x[4 * j + 3] * f) << 16);
    if (is_v) {
      const int e = i & (hd - 1), h = (i >> hsh) & 1, tile = tile0 + (i >> (hsh + 1));
      u32x4* w = (u32x4*)(codes + v_word(tile, e, h, hd));
      if (kept) {
        // bytes of tokens before the new ones (rounded again) and behind (as they were)
        const u32x4 was = *w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t q = rise ? recode4(was[j], fo) : was[j];
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int t = tile * KT + v_token(h, 4 * j + b);
            const uint32_t m = 0xFFu << (8 * b);
            if (t < it.t0) o[j] = (o[j] & ~m) | (q & m);
            else if (t >= it.t1) o[j] = (o[j] & ~m) | (was[j] & m);
          }
        }
      }
      *w = o;
    } else {
      const int t = (i >> (3 + ksh)) * 8 + (i & 7), e = ((i >> 3) & ((1 << ksh) - 1)) * 16;
      if (t < cnt) *(u32x4*)(codes + k_byte(it.t0 + t, e, hd)) = o;
    }
  };
#pragma unroll
  for (int j = 0; j < ST_HELD; ++j)
    if (j * ST_HALF + tid < words) store(j * ST_HALF + tid, held[j]);
  for (int i = ST_HELD * ST_HALF + tid; i < words; i += ST_HALF) {
    float x[16];
    load(i, x);
    store(i, x);
  }
  // a new page behind the new rows: zeros
  if (!kept) {
    const int t1 = is_v ? (tile0 + tiles) * KT : it.t1, rest = (c.T - t1) << ksh;
    for (int i = tid; i < rest; i += ST_HALF) {
      const int t = t1 + (i >> ksh), e = (i & ((1 << ksh) - 1)) * 16;
      *(u32x4*)(codes + (is_v ? (size_t)t1 * hd + (size_t)i * 16 : (size_t)k_byte(t, e, hd))) = u32x4{0u, 0u, 0u, 0u};
    }
  }
}

static int page_items_cap(const KvPages& c, const KvRows& a) {
  const int64_t i = (int64_t)a.rows / c.T + 2 * (int64_t)a.n;
  return (int)(i < a.rows ? i : a.rows);
}

hipError_t launch_kv_store(const KvPages& c, const KvRows& a, bool bf16, const void* K, const void* V, int64_t ldk,
                           int64_t ldv, hipStream_t st) {
  const int64_t wgs = (int64_t)page_items_cap(c, a) * c.Hkv;
  if (wgs == 0) return hipSuccess;
  if (wgs > INT32_MAX) return hipErrorInvalidValue;
  if (bf16)
    k_kv_store<bf16_t><<<(int)wgs, ST_NT, 0, st>>>(c, a, (const bf16_t*)K, (const bf16_t*)V, ldk, ldv);
  else
    k_kv_store<float><<<(int)wgs, ST_NT, 0, st>>>(c, a, (const float*)K, (const float*)V, ldk, ldv);
  return hipGetLastError();
}

__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(bf16_t* p, float x) {
  uint32_t u = __float_as_uint(x);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) { *p = 0x7FC0; return; }
  u += 0x7FFFu + ((u >> 16) & 1u);
  *p = (bf16_t)(u >> 16);
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *(floatx4*)p = floatx4{x[0], x[1], x[2], x[3]};
  *(floatx4*)(p + 4) = floatx4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16_t* p, const float* x) {
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2_k){x[2 * i], x[2 * i + 1]}, bf16x2_k));
  *(u32x4*)p = o;
}

// Rows back from the pages, one (page, kv head) a workgroup as above; a row whose
// page id is none of the pool's reads as zeros.  Bound by the writing of the rows: the
// prompts above in 23 us, 5.4 TB/s.
template <typename TT>
__global__ __launch_bounds__(ST_NT) void k_kv_read(KvPages c, KvRows a, TT* __restrict__ K, TT* __restrict__ V, int64_t ldk,
                                                   int64_t ldv) {
  const bool is_v = __builtin_amdgcn_readfirstlane(threadIdx.x / ST_HALF);
  const int head = blockIdx.x % c.Hkv, hd = c.hd, tid = threadIdx.x % ST_HALF;
  PageItem it{0, 0, 0, 0, 0};
  const bool live = page_item<ST_NT>(c, a, blockIdx.x / c.Hkv, &it);
  const int cnt = it.t1 - it.t0;
  const size_t ph = live ? (size_t)it.page * c.Hkv + head : 0;
  const float sc = live ? (is_v ? c.vs : c.ks)[ph] : 0.f;
  const uint8_t* codes = (is_v ? c.v : c.k) + ph * c.T * hd;
  const int64_t ld = is_v ? ldv : ldk;
  TT* dst = (is_v ? V : K) + (int64_t)it.row * ld + head * hd;
  const int esh = hd == 128 ? 7 : 6;
  if (is_v && cnt <= 4) {                      // few tokens: single codes (one of 64 requests 3.3 us against 4.0, eight 6.7 against 6.4)
    for (int i = tid; i < cnt << esh; i += ST_HALF) {
      const int t = i >> esh, e = i & (hd - 1);
      store1(dst + (int64_t)t * ld + e, live ? value1(codes[v_byte(it.t0 + t, e, hd)]) * sc : 0.f);
    }
  } else if (is_v) {
    // words of 16 codes, two of a thread's asked for before the first is used
    const int tile0 = it.t0 / KT, words = ((it.t1 + KT - 1) / KT - tile0) * hd * 2;
    for (int i0 = tid; i0 < words; i0 += 2 * ST_HALF) {
      u32x4 w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = min(i0 + j * ST_HALF, words - 1);
        w[j] = u32x4{0u, 0u, 0u, 0u};
        if (live) w[j] = *(const u32x4*)(codes + v_word(tile0 + (i >> (esh + 1)), i & (hd - 1), (i >> esh) & 1, hd));
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = i0 + j * ST_HALF, e = i & (hd - 1), t0 = (tile0 + (i >> (esh + 1))) * KT - it.t0;
        if (i >= words) break;
#pragma unroll
        for (int b = 0; b < 16; ++b) {
          const int t = t0 + v_token((i >> esh) & 1, b);
          if (t >= 0 && t < cnt) store1(dst + (int64_t)t * ld + e, value1((w[j][b >> 2] >> (8 * (b & 3))) & 0xFFu) * sc);
        }
      }
    }
  } else {
    // eight dims of a token, so that a wave writes whole runs; four asked for at once
    const int words = cnt << (esh - 3);
    for (int i0 = tid; i0 < words; i0 += 4 * ST_HALF) {
      u32x2 w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = min(i0 + j * ST_HALF, words - 1);
        w[j] = u32x2{0u, 0u};
        if (live) w[j] = *(const u32x2*)(codes + k_byte(it.t0 + (i >> (esh - 3)), i * 8 & (hd - 1), hd));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j * ST_HALF;
        if (i >= words) break;
        float x[8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          x[4 * b] = __builtin_amdgcn_cvt_f32_fp8((int)w[j][b], 0) * sc;
          x[4 * b + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[j][b], 1) * sc;
          x[4 * b + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[j][b], 2) * sc;
          x[4 * b + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[j][b], 3) * sc;
        }
        store8(dst + (int64_t)(i >> (esh - 3)) * ld + (i * 8 & (hd - 1)), x);
      }
    }
  }
}

hipError_t launch_kv_read(const KvPages& c, const KvRows& a, bool bf16, void* K, void* V, int64_t ldk, int64_t ldv,
                          hipStream_t st) {
  const int64_t wgs = (int64_t)page_items_cap(c, a) * c.Hkv;
  if (wgs == 0) return hipSuccess;
  if (wgs > INT32_MAX) return hipErrorInvalidValue;
  if (bf16)
    k_kv_read<bf16_t><<<(int)wgs, ST_NT, 0, st>>>(c, a, (bf16_t*)K, (bf16_t*)V, ldk, ldv);
  else
    k_kv_read<float><<<(int)wgs, ST_NT, 0, st>>>(c, a, (float*)K, (float*)V, ldk, ldv);
  return hipGetLastError();
}

}  // namespace bd
