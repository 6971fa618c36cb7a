// Block-causal attention over the paged 8-bit cache.
//
// A query at position p of request s sees the keys j < kv_len with
// j / B <= p / B (B = 0: all of them); o = sum_j softmax_j(scale q.k_j) v_j with
// k_j, v_j the code values times their page's scale.  The queries of one
// (request, kv head) are its rows x the G q-heads that share the kv head, in
// that order; a wave takes 32 of them on MFMA 32x32x16, S^T = K Q^T and
// O^T += V^T P^T, so that a lane owns one query and half of a tile's keys and
// the softmax state stays in the lane.
//
// Numbers.  Codes become bf16 (K) or fp16 (V) exactly; the scales never touch
// them: a tile lies in one page, K's scale multiplies its scores and V's
// exponent goes into the weights, w = 2^(t + E_v - r) for the score t in log2
// units and a running reference r, next to p = 2^(t - m) for the sum l.  Both
// references are whole numbers, so that what leads from one to another is an exact
// power of two, and lag (they move when a tile exceeds them by 2^8, or w 2^15).
// The products take w as two fp16 parts: 22 bits, or 2^-33 of the row's largest w
// where that is more (one part, 11 bits, moved one bf16 output in thirty to its
// neighbour, 8e-4 of the outputs' norm against 5e-5; 8 windows of 128 rows over
// 8320 keys took 103 us and take 129).  Queries are one, two or three bf16 planes
// (bf16, the models' pairs, fp32: exact).  Sums are fp32.
//
// What bounds it.  Single tokens read every code once: 48 requests of very unequal
// lengths, 0.80 GB in 166 us, 4.8 TB/s (a copy moves 5.2).  With 100 queries or
// more a (request, kv head) it is the sum of matrix and vector instructions, which do
// not overlap: a stage forms all its scores, then the weights, then the outputs.  A
// bf16 wave's tile takes 24 matrix instructions of 32 cycles and 199 vector ones, 64 of
// them conversions of the codes: 8 windows of 128 rows over 8320 keys, 70 GFLOP in
// 129 us, 0.54 PFLOP/s (a library product of 8192^3 makes 1.2), 130 such tiles a SIMD
// in 242,000 cycles, of which vector instructions are issued in 52 % and the matrix
// units busy in 41 %.  (The scaled fp8 matrix instruction would take K's codes as they
// are, but its sums of 64 products are off by 1.5e-4 of their magnitudes.)  Calls over
// few, unlike units take as long as the longest.  Short calls are a chain of loads:
// plan, table, tiles, 10 us for one token over 33 keys.
#include "bd_kv.h"

namespace bd {

constexpr int A_HELD = 256;        // requests whose rows and lengths are held in LDS

template <int MODE> struct AttnMode;
template <> struct AttnMode<KVQ_BF16> { typedef bf16_t T; static constexpr int NQ = 1; };
template <> struct AttnMode<KVQ_F32> { typedef float T; static constexpr int NQ = 3; };
template <> struct AttnMode<KVQ_PAIR> { typedef bf16_t T; static constexpr int NQ = 2; };

__device__ __forceinline__ floatx16_k zero16() {
  return floatx16_k{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}
__device__ __forceinline__ bf16x8 fp8x8_bf16(uint32_t a, uint32_t b) {
  const bf16x2_k p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
  const bf16x2_k q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  const bf16x2_k r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
  const bf16x2_k s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
__device__ __forceinline__ f16x8 fp8x8_f16(uint32_t a, uint32_t b) {
  const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
  const f16x2 q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
  const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
  const f16x2 s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  return f16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
// Bytes 0xff where a code is NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t t = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
  return (t >> 7) * 0xFFu;
}

// Query planes: 8 values as bf16, the remainders as bf16 again.
template <int NQ>
__device__ __forceinline__ void split_planes(const float* x, bf16x8* q) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i];
#pragma unroll
  for (int p = 0; p < NQ; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __bf16 b = (__bf16)y[i];
      q[p][i] = b;
      y[i] -= (float)b;
    }
}

// Four outputs.
template <int MODE>
__device__ __forceinline__ void attn_store4(typename AttnMode<MODE>::T* o, size_t plane, float a, float b, float c, float d) {
  if constexpr (MODE == KVQ_F32) {
    *(floatx4*)o = floatx4{a, b, c, d};
  } else {
    const uint32_t h0 = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2_k){a, b}, bf16x2_k));
    const uint32_t h1 = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2_k){c, d}, bf16x2_k));
    *(u32x2*)o = u32x2{h0, h1};
    if constexpr (MODE == KVQ_PAIR) {
      const float e0 = a - __uint_as_float(h0 << 16), e1 = b - __uint_as_float(h0 & 0xFFFF0000u);
      const float e2 = c - __uint_as_float(h1 << 16), e3 = d - __uint_as_float(h1 & 0xFFFF0000u);
      *(u32x2*)(o + plane) = u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2_k){e0, e1}, bf16x2_k)),
                                   __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2_k){e2, e3}, bf16x2_k))};
    }
  }
}

// x / d for 0 <= x < 2^31 and 1 / d rounded to nearest: (x + 1/2) / d is at least
// 1 / 2d from a whole number, far more than the product's error.
__device__ __forceinline__ int div_by(int x, double inv) { return (int)(((double)x + 0.5) * inv); }

// What a request brings: its rows, keys, query tiles and key tiles.
struct AttnSeq {
  int row, cnt, pos, len, nqt, kt;
};
// Keys that a query at position p sees.
__device__ __forceinline__ int key_end(int p, const KvAttnArgs& g, int len) {
  if (p < 0) return 0;
  return g.B ? (int)min((unsigned)(div_by(p, g.inv_B) + 1) * (unsigned)g.B, (unsigned)len) : len;
}
template <int AQ>
__device__ __forceinline__ AttnSeq attn_seq(const KvAttnArgs& g, const KvPages& c, int G, int s) {
  AttnSeq r;
  r.row = g.a.row_start[s];
  r.pos = g.a.pos0[s];
  int n = g.a.row_cnt ? g.a.row_cnt[s] : g.a.row_start[s + 1] - r.row;
  if (r.row < 0) n = 0;
  n = min(n, g.a.rows - r.row);
  r.cnt = max(n, 0);
  const int len = g.kv_len ? g.kv_len[s] : r.pos + r.cnt;
  r.len = min(max(len, 0), g.a.max_pages * c.T);
  r.nqt = (G * r.cnt + AQ - 1) / AQ;
  r.kt = max((key_end(r.pos + max(r.cnt, 1) - 1, g, r.len) + KT - 1) / KT, 1);   // rows without keys are work too: zeros
  return r;
}

// A unit of work is a (request, kv head, query tile).  Where its keys are dealt to
// several workgroups, first .. first + n - 1, each leaves a partial result: the
// first in its place 1, the others (whose range starts inside the unit) in place 0.
// A workgroup's range holds the first part of one such unit at most, the last it takes.
struct AttnUnit {
  int row, nq;               // the request's first row and its queries of a kv head
  int kv, qt, n;             // n = 0: no unit is cut at the end of this range
};
struct AttnWs {
  int* count;                // ranges
  AttnUnit* unit;            // [workgroups]
  float* lse;                // [workgroups][2][AQ]
  float* o;                  // [workgroups][2][AQ][hd]
};
__host__ __device__ inline size_t attn_up(size_t x) { return (x + 255) & ~(size_t)255; }
__host__ __device__ inline AttnWs attn_ws(void* ws, int wgs, int AQ) {
  AttnWs w;
  char* p = (char*)ws;
  w.count = (int*)p;
  p += 256;
  w.unit = (AttnUnit*)p;
  p += attn_up((size_t)wgs * sizeof(AttnUnit));
  w.lse = (float*)p;
  p += attn_up((size_t)wgs * 2 * AQ * sizeof(float));
  w.o = (float*)p;
  return w;
}

// Workgroups that the card runs at once (two of four waves a CU, or one of eight),
// over which the keys of fewer units are dealt (us of a replayed call: 8 windows of 128
// rows over 8320 keys 136, over 256 of four waves 145); the fewest key tiles dealt to one
// (single tokens with 2 / 4 / 8 tiles a wave: one over 4096 keys 16 / 19 / 24, over 32768
// 34 / 26 / 29, eight over up to 4096 24 / 26 / 36; a window of 96 rows over 4096 28 / 23 /
// 27); and the tiles' time that a join costs, its partials' way through memory and the
// ranges that begin and end inside units (24 windows of up to 1440 keys 48, cut at half
// the price 54).
__host__ __device__ constexpr int attn_slots(int KW) { return KW == 8 ? 256 : 512; }
// Waves over the keys for each number of query groups.
__host__ __device__ constexpr int attn_kw(int QW) { return QW == 1 ? 8 : QW == 2 ? 2 : 1; }
__host__ __device__ constexpr int attn_min_chunk(int KW) { return 4 * KW; }
__host__ __device__ constexpr int attn_join_cost(int KW) { return 12 + 6 * KW; }

typedef __attribute__((address_space(3))) void kva_lds_t;
typedef const __attribute__((address_space(4))) int32_t* kva_ints;     // read through the scalar cache
// Fourth word of a raw buffer resource (gfx9 family): 32-bit data, no stride.
constexpr int KVA_DWORD3 = 0x00020000;

// One stage: BT tiles of keys for each of the KW waves of a query group, K then V (two
// where one wave has a query group and registers for them, heads of 64 or bf16 queries:
// 136 against 139 us for 8 windows over 8320 keys, fp32 prompts of heads of 64 49 against
// 51, but those windows in fp32 201 against 174),
// and for every wave its tiles' scales, each in 64 words alike.
template <int HD, int QW, int KW, int BT>
struct KvStage {
  uint8_t b[KW][BT][2 * KT * HD];
  float sc[QW * KW][BT][2][64];
};

// A workgroup of QW x KW waves: QW groups of 32 queries, the key tiles of every
// stage dealt to KW waves of each group.  Tiles stream into LDS by asynchronous
// loads, one or two stages ahead of the one consumed.
//
// The work comes from the lengths on the device; every workgroup forms it for
// itself.  Either a workgroup takes whole units (neighbours read the same keys), or,
// where there are few of them over long keys, the units' key tiles are laid end to
// end and cut into equal ranges, one a workgroup: no range is longer than another,
// however unlike the requests' lengths are.
template <int HD, int MODE, int QW, int KW, int BT>
__global__ __launch_bounds__(64 * QW * KW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_kv_attn(KvPages c, KvAttnArgs g, int slots) {
  typedef typename AttnMode<MODE>::T T;
  constexpr int NQ = AttnMode<MODE>::NQ, NY = HD / 32, NT = 64 * QW * KW, AQ = 32 * QW;
  constexpr int LPW = 2 * NY / QW;             // 1 KiB loads a wave issues for a tile
  constexpr int LPS = BT * (LPW + 2);          // loads of a stage, its scales among them
  constexpr int D = KW == 8 && HD == 128 ? 2 : 3;   // stages of the ring: 136 KB, else 108 KB at most
  static_assert(LPW * QW == 2 * NY && LPS < 64, "whole loads");
  constexpr int A_SLOTS = attn_slots(KW);
  typedef KvStage<HD, QW, KW, BT> Stage;
  extern __shared__ int pre[];                 // [n]: units, or key tiles, of the requests before; then the requests held
  AttnSeq* held = (AttnSeq*)(pre + g.a.n);
  __shared__ __attribute__((aligned(1024))) Stage st0, st1, st2;
  __shared__ int tmp[NT / 64];
  __shared__ float fw[NT / 64];
  __shared__ int iw[NT / 64][2];
  __shared__ float xs[KW][QW][3][64];
  // (151 KB of 160 in the largest form, with 10 of the most requests)
  static_assert(D * sizeof(Stage) + sizeof(xs) + sizeof(tmp) + sizeof(fw) + sizeof(iw) + KV_ATTN_SEQS * sizeof(int) +
                A_HELD * sizeof(AttnSeq) <= 160 * 1024, "the local memory of a CU");
  const int G = g.H / c.Hkv, n = g.a.n, tid = threadIdx.x;
  // ---- plan
  AttnSeq mine{};
  if (tid < n) mine = attn_seq<AQ>(g, c, G, tid);
  int chunk = 0;                               // key tiles a workgroup takes; 0: whole units
  int units = 0;
  if (g.ws) {
    float w = (float)mine.nqt * (float)mine.kt, work = 0.f;
    int t = mine.nqt, longest = mine.nqt ? mine.kt : 0;
    for (int s = tid + NT; s < n; s += NT) {
      const AttnSeq r = attn_seq<AQ>(g, c, G, s);
      t += r.nqt;
      w += (float)r.nqt * (float)r.kt;
      longest = max(longest, r.nqt ? r.kt : 0);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      w += __shfl_xor(w, off);
      t += __shfl_xor(t, off);
      longest = max(longest, __shfl_xor(longest, off));
    }
    if ((tid & 63) == 0) {
      fw[tid >> 6] = w;
      iw[tid >> 6][0] = t;
      iw[tid >> 6][1] = longest;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) {
      work += fw[i];
      units += iw[i][0];
      longest = max(longest, iw[i][1]);
    }
    units *= c.Hkv;
    // (a share is no longer than the longest request, and the tiles' sum stays in 32 bits)
    work *= (float)c.Hkv;
    const int share = units < A_SLOTS ? (int)ceilf(work * (1.0f / A_SLOTS)) + 1 : 0;
    if (units < A_SLOTS && work < 0x1p30f && longest > share + attn_join_cost(KW)) chunk = max(share, attn_min_chunk(KW));
    chunk = __builtin_amdgcn_readfirstlane(chunk);
  }
  int total = 0;
  for (int s0 = 0; s0 < n; s0 += NT) {
    const int s = s0 + tid;
    int k = 0, all;
    if (s < n) {
      if (s0) mine = attn_seq<AQ>(g, c, G, s);
      k = mine.nqt * c.Hkv * (chunk ? mine.kt : 1);
      if (s < A_HELD) held[s] = mine;
    }
    const int inc = block_scan<NT>(k, tmp, &all);
    if (s < n) pre[s] = total + inc - k;
    total += all;
  }
  __syncthreads();
  total = __builtin_amdgcn_readfirstlane(total);
  AttnWs ws{};
  if (g.ws) {
    ws = attn_ws(g.ws, slots, AQ);
    // never more ranges than the workspace holds (the sum above was taken in fp32)
    if (chunk && (int64_t)chunk * slots < total) chunk = (total + slots - 1) / slots;
  }
  const int places = chunk ? (total + chunk - 1) / chunk : total;
  if (g.ws && blockIdx.x == 0 && tid == 0) *ws.count = chunk ? places : 0;

  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qw = wave % QW, kw = wave / QW;
  const int h = lane >> 5, q_lane = lane & 31;
  const int tpp = c.T / KT;
  const size_t page_bytes = (size_t)c.T * HD;
  // The workgroup's places in the work: whole units id, id + grid, ..; or the tiles
  // [w chunk, + chunk).  Consecutive places go to one XCD.
  const int per = (places + 7) / 8;
  int id = blockIdx.x;
  int at = 0, end = 0;                                        // what is left of the workgroup's range
  int wg = 0;                                                 // its number
  for (;;) {
    if (at >= end) {                                          // the next place
      do {
        if (id >= 8 * per) return;
        wg = (id & 7) * per + (id >> 3);
        id += gridDim.x;
      } while (wg >= places);
      at = chunk ? wg * chunk : wg;
      end = chunk ? min(at + chunk, total) : at + 1;
      if (chunk && tid == 0) ws.unit[wg].n = 0;
    }
    // ---- the unit, or its part
    const int s = __builtin_amdgcn_readfirstlane(find_segment(pre, n, at));
    AttnSeq r = s < A_HELD ? held[s] : attn_seq<AQ>(g, c, G, s);
    r.row = __builtin_amdgcn_readfirstlane(r.row);
    r.cnt = __builtin_amdgcn_readfirstlane(r.cnt);
    r.pos = __builtin_amdgcn_readfirstlane(r.pos);
    r.len = __builtin_amdgcn_readfirstlane(r.len);
    r.nqt = __builtin_amdgcn_readfirstlane(r.nqt);
    r.kt = __builtin_amdgcn_readfirstlane(r.kt);
    const int in = at - pre[s];
    // unit of the request: in / kt tiles of kt each
    const int v = __builtin_amdgcn_readfirstlane(chunk ? (int)(((double)in + 0.5) / (double)r.kt) : in);
    const int t_lo = __builtin_amdgcn_readfirstlane(chunk ? in - v * r.kt : 0);
    const int t_end = chunk ? min(t_lo + (end - at), r.kt) : r.kt;
    const bool whole = t_lo == 0 && t_end == r.kt;
    at += chunk ? t_end - t_lo : 1;
    const int kv = __builtin_amdgcn_readfirstlane((int)(((double)v + 0.5) / (double)r.nqt)), qt = v - kv * r.nqt;
    const int QG = G * r.cnt, q0 = qt * AQ + qw * 32;
    const int q_in = min(q0 + q_lane, QG - 1);                // lanes past the last query repeat it
    const bool qvalid = q0 + q_lane < QG;
    const int qr = div_by(q_in, g.inv_G), hq = kv * G + q_in - qr * G;
    const int qend = key_end(r.pos + qr, g, r.len);
    // the wave's smallest and largest bound, and the workgroup's largest
    const int qend_lo = key_end(r.pos + div_by(min(q0, QG - 1), g.inv_G), g, r.len);
    const int qend_hi = q0 < QG ? key_end(r.pos + div_by(min(q0 + 31, QG - 1), g.inv_G), g, r.len) : 0;
    const int wend = key_end(r.pos + div_by(min(qt * AQ + AQ - 1, QG - 1), g.inv_G), g, r.len);
    const int t_hi = min((wend + KT - 1) / KT, t_end);
    const int ns = t_hi > t_lo ? (t_hi - t_lo + KW * BT - 1) / (KW * BT) : 0;
    const __amdgpu_buffer_rsrc_t rks = __builtin_amdgcn_make_buffer_rsrc((void*)c.ks, 0, -1, KVA_DWORD3);
    const __amdgpu_buffer_rsrc_t rvs = __builtin_amdgcn_make_buffer_rsrc((void*)c.vs, 0, -1, KVA_DWORD3);
    const kva_ints table = (kva_ints)(g.a.table + (size_t)s * g.a.max_pages);

    // Loads of a stage, 16 bytes a lane: the wave's share of its tiles and the tiles'
    // scales.  A page id was read a tile ahead (`pid`; the next one is read here), so
    // the loads wait for nothing.  tl: the tiles, or NONE where there are no keys: past
    // the last tile, or with a page id that is none of the pool's (page 0 is loaded).
    constexpr int NONE = 1 << 25;                             // a tile behind every key
    struct Tiles {
      int t[BT];
    };
    int ft = t_lo + kw * BT, fcol = ft / tpp, foff = ft % tpp, pid = -1;   // the tile to load, its table column, its place in the page
    const int jump = KW * BT - BT + 1;                        // from a stage's last tile to the next one's first
    auto fetch = [&](Stage& sg) {
      Tiles tl;
#pragma unroll
      for (int b = 0; b < BT; ++b) {
        const bool live = (unsigned)pid < (unsigned)c.n_pages;
        const size_t ph = (size_t)(live ? pid : 0) * c.Hkv + kv;
        const size_t off = ph * page_bytes + (size_t)foff * (KT * HD);
        tl.t[b] = live ? ft : NONE;
        const int step = b + 1 < BT ? 1 : jump;
        ft += step;
        foff += step;
        while (foff >= tpp) {
          foff -= tpp;
          ++fcol;
        }
        pid = -1;
        if (ft < t_hi) pid = table[fcol];
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(c.k + off), 0, -1, KVA_DWORD3);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(c.v + off), 0, -1, KVA_DWORD3);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rks, (kva_lds_t*)sg.sc[wave][b][0], 4, 0, (uint32_t)ph * 4u, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rvs, (kva_lds_t*)sg.sc[wave][b][1], 4, 0, (uint32_t)ph * 4u, 0, 0);
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
          const int p = qw * LPW + i;                          // parts 0 .. NY - 1: K, then V
          __builtin_amdgcn_raw_ptr_buffer_load_lds(p < NY ? rk : rv, (kva_lds_t*)(sg.b[kw][b] + p * 1024), 16, lane * 16,
                                                   (p % NY) * 1024, 0, 0);
        }
      }
      return tl;
    };

    floatx16_k oacc[NY];
    float m_run = -INFINITY, r_run = -INFINITY, l_part = 0.f;
#pragma unroll
    for (int d = 0; d < NY; ++d) oacc[d] = zero16();
    bf16x8 qf[2 * NY][NQ];
    auto queries = [&]() {
      const size_t qo = (size_t)(r.row + qr) * g.ldq + (size_t)hq * HD + h * 16;
#pragma unroll
      for (int y = 0; y < NY; ++y)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const T* p = (const T*)g.q + qo + y * 32 + e * 8;
          if constexpr (MODE == KVQ_F32) {
            float x[8];
            load8(p, x);
            split_planes<NQ>(x, qf[2 * y + e]);
          } else {
            qf[2 * y + e][0] = __builtin_bit_cast(bf16x8, *(const u32x4*)p);
            if constexpr (MODE == KVQ_PAIR) qf[2 * y + e][1] = __builtin_bit_cast(bf16x8, *(const u32x4*)(p + g.q_plane));
          }
        }
    };

    auto compute = [&](const Stage& sg, const Tiles& tl) {
      if (tl.t[0] * KT >= qend_hi && (BT == 1 || tl.t[BT - 1] * KT >= qend_hi)) return;   // uniform over the wave
      u32x4 vb[BT][NY];
      floatx16_k a[BT];
      float sc[BT], ev[BT];
      bool part = false, odd = false;
#pragma unroll
      for (int b = 0; b < BT; ++b) {
        const uint8_t* kp = sg.b[kw][b] + lane * 16;
        u32x4 kb[NY];
#pragma unroll
        for (int y = 0; y < NY; ++y) kb[y] = *(const u32x4*)(kp + y * 1024);
        const float sk = sg.sc[wave][b][0][lane], sv = sg.sc[wave][b][1][lane];
#pragma unroll
        for (int y = 0; y < NY; ++y) vb[b][y] = *(const u32x4*)(kp + (NY + y) * 1024);
        a[b] = zero16();
#pragma unroll
        for (int y = 0; y < NY; ++y)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const bf16x8 kf = fp8x8_bf16(kb[y][2 * e], kb[y][2 * e + 1]);
#pragma unroll
            for (int p = NQ - 1; p >= 0; --p)
              a[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[2 * y + e][p], a[b], 0, 0, 0);
          }
        // one factor for the tile, unless it leaves the positive normal floats (below)
        sc[b] = g.scale_log2 * sk;
        odd |= __any(__builtin_amdgcn_classf(sc[b], 0x2FF));
        ev[b] = (float)scale_exponent(sv);
        part |= tl.t[b] * KT + KT > qend_lo;                   // some query does not see all of the tile
      }
      bool bad = false;
      if (part || odd) {
        // keys of the smallest scales, or a scale argument far from 1: the argument goes to
        // the scores at once (as a branch of its own this check took 4 % of a long call)
        if (odd) {
#pragma unroll
          for (int b = 0; b < BT; ++b) {
            const bool out = __builtin_amdgcn_classf(sc[b], 0x2FF);
            a[b] *= out ? g.scale_log2 : 1.f;
            sc[b] = out ? fmaxf(sg.sc[wave][b][0][lane], 0x1p-126f) : sc[b];
          }
        }
#pragma unroll
        for (int b = 0; b < BT; ++b) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (tl.t[b] * KT + 8 * (i >> 2) + 4 * h + (i & 3) >= qend) a[b][i] = -INFINITY;
          // A NaN value times the zero weight of a query that does not see it is NaN:
          // such codes become zeros here and mark the outputs of those that see them
          // below.  (A tile that every query sees needs no care.)
#pragma unroll
          for (int d = 0; d < NY; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t nb = nan_bytes(vb[b][d][j]);
              bad |= nb != 0;
              vb[b][d][j] &= ~nb;
            }
        }
      }
      float tm[BT];
      bool rise = false;
#pragma unroll
      for (int b = 0; b < BT; ++b) {
        tm[b] = a[b][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) tm[b] = fmaxf(tm[b], a[b][i]);
        tm[b] *= sc[b];                                        // of the lane's keys: half of the query's
        rise |= tm[b] > m_run + 8.f || tm[b] + ev[b] > r_run + 15.f;
      }
      if (__any(rise)) {
        float mn = m_run, rn = r_run;
#pragma unroll
        for (int b = 0; b < BT; ++b) {
          const float t = fmaxf(tm[b], __shfl_xor(tm[b], 32));
          mn = fmaxf(mn, ceilf(t));
          rn = fmaxf(rn, ceilf(t) + (ev[b] - 9.f));
        }
        const float al = __builtin_amdgcn_exp2f(mn == -INFINITY ? 0.f : m_run - mn);
        const float ao = __builtin_amdgcn_exp2f(rn == -INFINITY ? 0.f : r_run - rn);
        m_run = mn;
        r_run = rn;
        l_part *= al;
#pragma unroll
        for (int d = 0; d < NY; ++d) oacc[d] *= ao;
      }
      const float m_ref = m_run == -INFINITY ? 0.f : m_run, r_ref = r_run == -INFINITY ? 0.f : r_run;
      // Weights straight from the exponent, w = 2^(t + E_v - r), as two fp16 parts; the
      // sum's terms are p = w 2^-lf, lf = E_v + m - r.  From lf = 100 on w 2^-100 stands for
      // p (below 2^-85, where l is 1/2 at least).  Below lf = -60, of a page whose V scale is
      // nothing beside the reference's, w is 0 in fp16: p is summed here and the key left out.
      const float ahead = m_ref - r_ref;
      bool far = false;
#pragma unroll
      for (int b = 0; b < BT; ++b) far |= ev[b] + ahead < -60.f;
      if (__any(far)) {
#pragma unroll
        for (int b = 0; b < BT; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool out = ev[b] + ahead < -60.f;
            l_part += out ? __builtin_amdgcn_exp2f(fmaf(a[b][i], sc[b], -m_ref)) : 0.f;
            a[b][i] = out ? -INFINITY : a[b][i];
          }
      }
      // (w - hi as a product with a number that the compiler does not know is one mixed
      // instruction; as a difference it is a conversion more)
      float minus1 = -1.f;
      asm("" : "+s"(minus1));
      f16x8 pf[BT][2][2];
#pragma unroll
      for (int b = 0; b < BT; ++b) {
        float ws = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            const float w0 = __builtin_amdgcn_exp2f(fmaf(a[b][8 * x + j], sc[b], ev[b] - r_ref));
            const float w1 = __builtin_amdgcn_exp2f(fmaf(a[b][8 * x + j + 1], sc[b], ev[b] - r_ref));
            ws += w0;
            ws += w1;
            const f16x2 hi = __builtin_convertvector((floatx2_k){w0, w1}, f16x2);
            const f16x2 lo = __builtin_convertvector((floatx2_k){fmaf((float)hi[0], minus1, w0), fmaf((float)hi[1], minus1, w1)}, f16x2);
            pf[b][x][0][j] = hi[0];
            pf[b][x][0][j + 1] = hi[1];
            pf[b][x][1][j] = lo[0];
            pf[b][x][1][j + 1] = lo[1];
          }
        l_part = fmaf(ws, __builtin_amdgcn_exp2f(-fminf(fmaxf(ev[b] + ahead, -60.f), 100.f)), l_part);
      }
#pragma unroll
      for (int b = 0; b < BT; ++b)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int d = 0; d < NY; ++d) {
            const f16x8 vf = fp8x8_f16(vb[b][d][2 * x], vb[b][d][2 * x + 1]);
#pragma unroll
            for (int p = 1; p >= 0; --p)
              oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pf[b][x][p], oacc[d], 0, 0, 0);
          }
      if ((part || odd) && __any(bad)) {
#pragma unroll 1
        for (int b = 0; b < BT; ++b) {
          const int k0 = (b ? tl.t[BT - 1] : tl.t[0]) * KT;
#pragma unroll
          for (int d = 0; d < NY; ++d) {
            const u32x4 vn = *(const u32x4*)(sg.b[kw][b] + lane * 16 + (NY + d) * 1024);
            floatx16_k hit = zero16();
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              f16x8 see;
#pragma unroll
              for (int j = 0; j < 8; ++j)
                see[j] = k0 + 16 * x + 8 * (j >> 2) + 4 * h + (j & 3) < qend ? (_Float16)1.0f : (_Float16)0.0f;
              hit = __builtin_amdgcn_mfma_f32_32x32x16_f16(fp8x8_f16(nan_bytes(vn[2 * x]) & 0x38383838u, nan_bytes(vn[2 * x + 1]) & 0x38383838u),
                                                           see, hit, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) oacc[d][i] = hit[i] > 0.f ? NAN : oacc[d][i];
          }
        }
      }
    };
    // Stage k is consumed when its loads have landed; with three stages those of the
    // one after it may still be in flight.  The ring is filled unconditionally (past
    // the last stage it is loaded again): a load under a branch would leave the
    // compiler unsure of what is in flight.  With QW > 1 the barrier tells that
    // everyone's part has landed and that the slot filled next is read.
    constexpr int AHEAD = (D - 2) * LPS;                      // loads in flight behind the stage that is waited for
#define BD_KVA_STEP(CUR, TC, NXT, TN, K)                                              \
    __builtin_amdgcn_s_waitcnt((AHEAD & 15) | ((AHEAD >> 4) << 14) | (7 << 4) | (0 << 8)); \
    if constexpr (QW > 1) __builtin_amdgcn_s_barrier();                               \
    TN = fetch(NXT);                                                                  \
    compute(CUR, TC);                                                                 \
    if ((K) + 1 >= ns) break;
    __syncthreads();                                          // the last unit's parts are read
    if (ns > 0) {
      if (ft < t_hi) pid = table[fcol];
      if constexpr (D == 3) {
        Tiles ta = fetch(st0), tb = fetch(st1), tc;
        queries();
        for (int k = 0;; k += 3) {
          BD_KVA_STEP(st0, ta, st2, tc, k)
          BD_KVA_STEP(st1, tb, st0, ta, k + 1)
          BD_KVA_STEP(st2, tc, st1, tb, k + 2)
        }
      } else {
        Tiles ta = fetch(st0), tb;
        queries();
        for (int k = 0;; k += 2) {
          BD_KVA_STEP(st0, ta, st1, tb, k)
          BD_KVA_STEP(st1, tb, st0, ta, k + 1)
        }
      }
      __builtin_amdgcn_s_waitcnt(0x0070);                     // nothing in flight into the ring
    }
#undef BD_KVA_STEP
    // ---- The KW waves' parts, in wave order: wave j of a group joins and writes the
    // j-th share of the output's registers, R of them, which the others leave in the
    // ring for it.
    constexpr int R = HD / 2 / KW;
    constexpr int PER = sizeof(Stage) / (R * 64 * sizeof(float));       // shares a stage holds
    static_assert(QW * KW * (KW - 1) <= PER * D && R % 4 == 0, "the shares fit the ring");
    auto place = [&](int j, int k) {                          // share j of wave k (k != j)
      const int p = (qw * KW + j) * (KW - 1) + (k < j ? k : k - 1);
      float* base = p < PER ? (float*)&st0 : (float*)&st1;
      if constexpr (D == 3) base = p < 2 * PER ? base : (float*)&st2;
      return base + (p % PER) * (R * 64) + lane;
    };
    if constexpr (KW > 1) __syncthreads();
#pragma unroll
    for (int j = 0; j < KW; ++j)
      if (KW > 1 && kw != j) {
        float* w = place(j, kw);
#pragma unroll
        for (int i = 0; i < R; ++i) w[i * 64] = oacc[(j * R + i) / 16][(j * R + i) % 16];
      }
    float mx = m_run, rx = r_run, l = l_part + __shfl_xor(l_part, 32);
    if constexpr (KW > 1) {
      xs[kw][qw][0][lane] = m_run;
      xs[kw][qw][1][lane] = r_run;
      xs[kw][qw][2][lane] = l;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        mx = fmaxf(mx, xs[k][qw][0][lane]);
        rx = fmaxf(rx, xs[k][qw][1][lane]);
      }
    }
    const float m_ref = mx == -INFINITY ? 0.f : mx, r_ref = rx == -INFINITY ? 0.f : rx;
    if constexpr (KW > 1) {
      l = 0.f;
#pragma unroll
      for (int k = 0; k < KW; ++k) l += xs[k][qw][2][lane] * __builtin_amdgcn_exp2f(xs[k][qw][0][lane] - m_ref);
    }
    // o = O 2^(r - m) / l; a query that sees nothing gives zeros.  2^(r - m) may lie below
    // the normal floats while o does not (r - m is the V scale's exponent less 9 to 15).
    const float norm = mx != -INFINITY ? 1.0f / l : l != l ? l : 0.f;
    const int up = (int)fminf(fmaxf(r_ref - m_ref, -400.f), 400.f);
    const size_t slot = ((size_t)wg * 2 + (t_lo == 0 ? 1 : 0)) * AQ + qw * 32 + q_lane;
#pragma unroll
    for (int j = 0; j < KW; ++j)
      if (kw == j) {
        float x[R];
        const float f0 = __builtin_amdgcn_exp2f(r_run - r_ref);
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = 0.f;
#pragma unroll
        for (int k = 0; k < KW; ++k) {
          if (k == j) {
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = fmaf(f0, oacc[(j * R + i) / 16][(j * R + i) % 16], x[i]);
          } else {
            const float f = __builtin_amdgcn_exp2f(xs[k][qw][1][lane] - r_ref);
            const float* w = place(j, k);
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = fmaf(f, w[i * 64], x[i]);
          }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = __builtin_amdgcn_ldexpf(x[i] * norm, up);
        // register 16 d + 4 m + i (i < 4): dim 32 d + 8 m + 4 h + i of the lane's query
#pragma unroll
        for (int i = 0; i < R; i += 4) {
          const int reg = j * R + i, dim = reg / 16 * 32 + reg % 16 / 4 * 8 + 4 * h;
          if (whole) {
            if (qvalid)
              attn_store4<MODE>((T*)g.out + (size_t)(r.row + qr) * g.ldo + (size_t)hq * HD + dim, g.o_plane, x[i], x[i + 1], x[i + 2], x[i + 3]);
          } else {
            *(floatx4*)(ws.o + slot * HD + dim) = floatx4{x[i], x[i + 1], x[i + 2], x[i + 3]};
          }
        }
      }
    if (!whole && kw == 0 && h == 0) ws.lse[slot] = l != l ? l : mx == -INFINITY ? -INFINITY : mx + __builtin_amdgcn_logf(l);
    if (!whole && t_lo == 0 && tid == 0) {
      const int last = pre[s] + (v + 1) * r.kt - 1;           // the unit's last tile
      ws.unit[wg] = AttnUnit{r.row, QG, kv, qt, last / chunk - wg + 1};
    }
  }
}

// Joins the parts of a unit: weights 2^(lse - max lse), in the order of the keys.
// All it does is wait for memory, so four parts' sums and rows are asked for at once
// and the maximum runs along (32 queries a workgroup, the sums read first: 12.1 us
// against 9.4 for 128 queries of 16 long keys' parts).
template <int HD, int MODE, int AQ>
__global__ __launch_bounds__(256) void k_kv_attn_join(KvPages c, KvAttnArgs g, int slots) {
  typedef typename AttnMode<MODE>::T T;
  constexpr int TPI = HD / 4, Q = 256 / TPI, P = 4;          // threads a query, queries a workgroup, parts at once
  const AttnWs ws = attn_ws(g.ws, slots, AQ);
  const int t = blockIdx.x / (AQ / Q), q = (blockIdx.x % (AQ / Q)) * Q + threadIdx.x / TPI, e = threadIdx.x % TPI * 4;
  const AttnUnit w = ws.unit[t];
  if (t >= *ws.count || w.n == 0) return;
  const int G = g.H / c.Hkv, qi = w.qt * AQ + q;
  if (qi >= w.nq) return;
  const int qr = div_by(qi, g.inv_G), hq = w.kv * G + qi - qr * G;
  float mx = -INFINITY, L = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < w.n; k0 += P) {
    float ls[P], m = mx;
    floatx4 o[P];
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const int kk = min(k0 + k, w.n - 1);
      const size_t slot = ((size_t)(t + kk) * 2 + (kk == 0 ? 1 : 0)) * AQ + q;
      ls[k] = ws.lse[slot];
      o[k] = *(const floatx4*)(ws.o + slot * HD + e);
    }
#pragma unroll
    for (int k = 0; k < P; ++k) m = fmaxf(m, ls[k]);
    const float ref = m == -INFINITY ? 0.f : m, f0 = __builtin_amdgcn_exp2f(mx - ref);
    mx = m;
    L *= f0;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] *= f0;
#pragma unroll
    for (int k = 0; k < P; ++k)
      if (k0 + k < w.n) {
        const float f = __builtin_amdgcn_exp2f(ls[k] - ref);
        L += f;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = fmaf(f, o[k][j], a[j]);
      }
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  T* o = (T*)g.out + (size_t)(w.row + qr) * g.ldo + (size_t)hq * HD + e;
  attn_store4<MODE>(o, g.o_plane, a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv);
}

// Units of the rows at most: as many whole query tiles and one more a request, and
// not more than rows.
static int64_t attn_units_cap(int H, int Hkv, int n, int rows, int AQ) {
  const int64_t G = H / Hkv;
  const int64_t t = Hkv * ((G * rows) / AQ + n), by_row = (int64_t)Hkv * rows * ((G + AQ - 1) / AQ);
  return t < by_row ? t : by_row;
}

// Ranges that the keys (tables that span `keys` positions) may be cut into; 0 where
// they never are: the query tiles of the rows fill the card, or no table is long
// enough for a join to pay.
static int attn_ranges(int H, int Hkv, int n, int rows, int64_t keys, int QW) {
  const int AQ = 32 * QW, KW = attn_kw(QW);
  const int64_t G = H / Hkv, kt = (keys + KT - 1) / KT;
  if (Hkv * ((G * rows + AQ - 1) / AQ) >= attn_slots(KW) || kt <= attn_join_cost(KW)) return 0;
  const int64_t most = attn_units_cap(H, Hkv, n, rows, AQ) * kt / attn_min_chunk(KW) + 1;
  return (int)(most < attn_slots(KW) ? most : attn_slots(KW));
}
static size_t attn_form_bytes(int hd, int ranges, int AQ) {
  const size_t r = ranges;
  return r ? 256 + attn_up(r * sizeof(AttnUnit)) + attn_up(r * 2 * AQ * 4) + r * 2 * AQ * hd * 4 : 0;
}

// Groups of 32 queries a workgroup.  One group with its keys dealt to eight waves
// reads every key tile for 32 queries only but is done soonest, and needs no join while
// its units find a CU each: taken for 32 queries a (request, kv head) and where there
// are at most 256 such units (us with 1 / 2 / 4 groups, q-heads in fours, 1440 keys:
// one window of 96 rows 19 / 23 / 26, four 21 / 34 / 38, twelve 55 / 48 / 53).  Two groups
// with two waves each halve the time of the longest unit: for 64 queries, where all fit
// the card at once, and with heads of 128 and tables of 1024 keys or more up to 1280 units
// (32 ragged windows 78 / 66 / 69, 48 of them 116 / 72 / 80, 16 prompts of 512 in 2048
// units 95 / 40 / 39, but 24 windows of 128 keys 48 / 20 / 18; of heads of 64 four groups
// lose less: 6 prompts of 1023 in 920 units 87 / 43 / 41).  Unless the tables span so many
// keys that the workgroups are busy for long: four groups take two tiles a stage, the
// fastest loop (twelve windows over 8192 keys 187 / 158 / 146).
static int attn_qw(int H, int Hkv, int hd, int n, int rows, int max_rows, int64_t keys) {
  const int64_t G = H / Hkv, q = G * (max_rows > 0 ? max_rows : (rows + n - 1) / n), kt = (keys + KT - 1) / KT;
  auto units = [&](int Q) {
    const int64_t each = (q + Q - 1) / Q * n, all = G * rows / Q + n;
    return Hkv * (each < all ? each : all);
  };
  if (q <= 32 || units(32) <= 256) return 1;
  if (q <= 64 || (units(64) <= (hd == 128 && kt >= 32 ? 1280 : 512) && units(128) * kt <= 56 * 512)) return 2;
  return 4;
}

size_t kv_attn_ws_bytes(int H, int Hkv, int hd, int n, int rows, int max_rows, int64_t keys) {
  const int qw = attn_qw(H, Hkv, hd, n, rows, max_rows, keys);
  return attn_form_bytes(hd, attn_ranges(H, Hkv, n, rows, keys, qw), 32 * qw);
}

hipError_t launch_kv_attention(const KvPages& c, const KvAttnArgs& g, int mode, hipStream_t st) {
  if ((c.hd != 64 && c.hd != 128) || g.a.n < 1 || g.a.n > KV_ATTN_SEQS) return hipErrorInvalidValue;
  if (g.a.rows == 0) return hipSuccess;
  KvAttnArgs a = g;
  a.inv_B = g.B ? 1.0 / g.B : 0.0;
  a.inv_G = (double)c.Hkv / g.H;
  const int64_t keys = (int64_t)g.a.max_pages * c.T;
  const int qw = attn_qw(g.H, c.Hkv, c.hd, g.a.n, g.a.rows, g.max_rows, keys), AQ = 32 * qw;
  const int slots = attn_ranges(g.H, c.Hkv, g.a.n, g.a.rows, keys, qw);
  if (a.ws && g.ws_bytes < attn_form_bytes(c.hd, slots, AQ)) return hipErrorInvalidValue;
  if (!slots) a.ws = nullptr;
  const int64_t units = attn_units_cap(g.H, c.Hkv, g.a.n, g.a.rows, AQ), most = a.ws && units < slots ? slots : units;
  const int grid = most < 2048 ? (int)((most + 7) / 8 * 8) : 2048;
  const size_t lds = (size_t)g.a.n * sizeof(int) + (size_t)(g.a.n < A_HELD ? g.a.n : A_HELD) * sizeof(AttnSeq);
#define BD_KVA2(HD_, MODE_, QW_, KW_)                                                                                        \
  do {                                                                                                                       \
    k_kv_attn<HD_, MODE_, QW_, KW_, (KW_ == 1 && (HD_ == 64 || MODE_ == KVQ_BF16)) ? 2 : 1>                                  \
        <<<grid, 64 * QW_ * KW_, lds, st>>>(c, a, slots);                                                                    \
    if (a.ws) k_kv_attn_join<HD_, MODE_, 32 * QW_><<<slots * QW_ * (HD_ / 32), 256, 0, st>>>(c, a, slots);                                        \
  } while (0)
#define BD_KVA(HD_, MODE_)                       \
  do {                                           \
    if (qw == 1) BD_KVA2(HD_, MODE_, 1, 8);      \
    else if (qw == 2) BD_KVA2(HD_, MODE_, 2, 2); \
    else BD_KVA2(HD_, MODE_, 4, 1);              \
  } while (0)
  if (c.hd == 128) {
    if (mode == KVQ_BF16) BD_KVA(128, KVQ_BF16);
    else if (mode == KVQ_F32) BD_KVA(128, KVQ_F32);
    else BD_KVA(128, KVQ_PAIR);
  } else {
    if (mode == KVQ_BF16) BD_KVA(64, KVQ_BF16);
    else if (mode == KVQ_F32) BD_KVA(64, KVQ_F32);
    else BD_KVA(64, KVQ_PAIR);
  }
#undef BD_KVA
#undef BD_KVA2
  return hipGetLastError();
}

}  // namespace bd
