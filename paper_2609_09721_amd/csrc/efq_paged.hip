// Rotary positions, a paged key/value cache and softmax attention over it, for
// AMD Instinct MI355X (gfx950, CDNA4).
//
// Kernels:
//   rope_kernel        rotary positions with one or several axes (HBM bound).
//   kv_append_kernel   new keys (turned on the way) and values into the pages,
//                      bf16 or MXFP8 (HBM bound; latency for a few tokens).
//   paged_step_kernel  attention of one or a few tokens per sequence: every wave
//                      streams keys and values of its own (HBM bound).
//   paged_chunk_kernel attention of many tokens per sequence: waves of 32 rows
//                      share key/value tiles in LDS (matrix-core bound).
//   paged_merge_kernel joins the parts of a row that ran split over its keys.
//
// This file is the library's one translation unit: it takes the attention
// forward, its quantisers and the host helpers in from efq_attn.hip.
#include "efq_attn.hip"

namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Round two fp32 to a pair of bf16, to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  const f32x2 x = {lo, hi};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(x, bf16x2));
}
constexpr unsigned kOnes = 0x3f803f80u;    // a pair of ones
__device__ __forceinline__ float bf16_lo(unsigned u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(unsigned u) { return __uint_as_float(u & 0xffff0000u); }

// fp32 2^(byte - 127) of an E8M0 byte, as the conversions take it (0 stands
// for 2^-127 there).
__device__ __forceinline__ float e8m0_scale(unsigned byte) { return __uint_as_float(byte << 23); }

// Four E4M3 codes times their scale as bf16, exact (4 significant bits).
__device__ __forceinline__ uint2 e4m3_bf16x4(unsigned codes, float scale) {
  return make_uint2(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true)));
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Lanes l, l + 16, l + 32, l + 48 of a wave: the largest, the sum.
__device__ __forceinline__ float max_of_groups(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmax_swapped(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmax_swapped(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_groups(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Lanes l and l + 32.
__device__ __forceinline__ float max_of_halves(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmax_swapped(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_of_halves(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ------------------------------------------------------- rotary positions
// (x, y) -> (x cos a - y sin a, y cos a + x sin a), a = pos * inv_freq.  The angle's
// turns, and the sine and cosine of what is left of the last one, are formed in
// fp64 and rounded once: fp32 would lose all of the angle's fraction at far positions
// (a position of 2^20 leaves it 4 bits after the point), and an fp32 sine of the
// rest, off by up to 2^-23, rounds some turned values to the other of two bf16 (and
// with them to another E4M3) where the exact turn does not.  One sine and cosine per
// token and pair serve every head: a workgroup forms them once, in LDS, so the passes
// over the heads are loads, six operations a pair and stores; in fp64 they cost 0 to
// 2 % of a call (8192 tokens of 40 heads 31.0 and 31.1 us).
struct RotArgs {
  const float* inv_freq;
  const int32_t* axis;
  const int32_t* pos;
  long tokens;      // distance between the axes of pos
  int pairs, axes, interleaved;
};

__device__ __forceinline__ float2 rot_of(const RotArgs& r, long token, int pair, bool inverse) {
  const int ax = r.axis ? r.axis[pair] : 0;
  const int pos = (unsigned)ax < (unsigned)r.axes ? r.pos[ax * r.tokens + token] : 0;
  const double turns = (double)pos * (double)r.inv_freq[pair] * 0.15915494309189533577;
  double s, c;
  sincospi(2.0 * (turns - rint(turns)), &s, &c);
  return make_float2((float)c, (float)(inverse ? -s : s));
}

struct RopeArgs {
  const char* x;
  char* y;
  long x_token, x_head, y_token, y_head;   // bytes
  int tokens, heads, chunks;               // chunks: items of a head
  int tt;                                  // tokens of a workgroup
  int dt, dh, dc;                          // one step of the workgroups of a token, in tokens, heads, chunks
  int inverse;
  RotArgs rot;
};

// What is read once asks the caches not to keep it: one token over 131000 keys
// (32/8 heads, D 128, bf16) 99.9 -> 87.5 us (5.37 -> 6.13 TB/s), 300 tokens over
// 1000 keys each 141 -> 131 us.
__device__ __forceinline__ u32x4 stream16(const char* p) { return __builtin_nontemporal_load((const u32x4*)p); }
// So do writes that the last-level cache (256 MB) would not hold until they are
// read, or whose reader works long on each: 32760 tokens of 24 heads of 128 turned in
// fp32 (403 MB) 139 -> 131 us, but 60000 of 8 (246 MB) 73 -> 81; 16000 tokens
// (32/8 heads, D 128) appended to bf16 pages 87 -> 79, 11400 to MXFP8 ones 62 -> 58.
constexpr long kLastLevel = 256 << 20;
template <bool STREAM, typename T>         // (at compile time: a branch would be merged into one plain store)
__device__ __forceinline__ void put(char* p, T x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, (T*)p);
  else *(T*)p = x;
}

// The values of 16-byte pieces.
template <bool F32>
struct Piece {
  static constexpr int E = F32 ? 4 : 8;
  u32x4 w;
  __device__ __forceinline__ float get(int i) const {
    if constexpr (F32) return __uint_as_float(w[i]);
    else return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
  }
  __device__ __forceinline__ void set2(int i, float u, float v) {    // values i and i + 1, i even
    if constexpr (F32) w[i] = __float_as_uint(u), w[i + 1] = __float_as_uint(v);
    else w[i / 2] = pack_bf16(u, v);
  }
};
// A piece of neighbouring pairs.
template <bool F32>
__device__ __forceinline__ void turn_beside(Piece<F32>& p, const float2* cs) {
#pragma unroll
  for (int j = 0; j < Piece<F32>::E / 2; ++j) {
    const float2 c = cs[j];
    const float u = p.get(2 * j), v = p.get(2 * j + 1);
    p.set2(2 * j, __builtin_fmaf(u, c.x, -(v * c.y)), __builtin_fmaf(v, c.x, u * c.y));
  }
}
// Two pieces, the first and second values of the same pairs.
template <bool F32>
__device__ __forceinline__ void turn_halves(Piece<F32>& lo, Piece<F32>& hi, const float2* cs) {
#pragma unroll
  for (int j = 0; j < Piece<F32>::E; j += 2) {
    const float2 c = cs[j], d = cs[j + 1];
    const float u = lo.get(j), v = hi.get(j), x = lo.get(j + 1), y = hi.get(j + 1);
    lo.set2(j, __builtin_fmaf(u, c.x, -(v * c.y)), __builtin_fmaf(x, d.x, -(y * d.y)));
    hi.set2(j, __builtin_fmaf(v, c.x, u * c.y), __builtin_fmaf(y, d.x, x * d.y));
  }
}

constexpr int kMostShared = 8;     // most tokens of a workgroup

// An item is a 16-byte piece of a head (neighbouring pairs) or the two pieces of
// the same pairs (halves), so that the lanes of a load lie side by side; pieces
// behind the pairs pass through.  Every value is read once, past the caches.  A
// thread has several items on their way at once, found by stepping (token, head,
// chunk) on, since a division an item would cost as much as the turn.
template <bool F32, bool INTERLEAVED, bool STREAM>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  extern __shared__ float2 rot[];          // [tt][pairs]
  const long t0 = (long)blockIdx.x * a.tt;
  const int nt = (int)min((long)a.tt, a.tokens - t0);
  const int pairs = a.rot.pairs;
  for (int i = threadIdx.x; i < nt * pairs; i += 256)
    rot[i] = rot_of(a.rot, t0 + i / pairs, i % pairs, a.inverse);
  __syncthreads();
  constexpr int E = Piece<F32>::E, U = INTERLEAVED ? 4 : 2;
  const int per = a.heads * a.chunks, first = blockIdx.y * 256 + threadIdx.x;
  const int turned = INTERLEAVED ? 2 * pairs / E : pairs / E;
  int t = first / per, h = first % per / a.chunks, c = first % a.chunks;
  while (t < nt) {
    Piece<F32> lo[U], hi[INTERLEAVED ? 1 : U];
    int vt[U], vh[U], vc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      vt[u] = t, vh[u] = h, vc[u] = c;
      c += a.dc, h += a.dh, t += a.dt;
      if (c >= a.chunks) c -= a.chunks, ++h;
      if (h >= a.heads) h -= a.heads, ++t;
    }
    // bytes of an item's pieces in its head; behind the pairs (halves) two side by side
    auto at_lo = [&](int u) { return 16 * (INTERLEAVED || vc[u] < turned ? vc[u] : 2 * vc[u]); };
    auto at_hi = [&](int u) { return 16 * (vc[u] < turned ? vc[u] + turned : 2 * vc[u] + 1); };
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (vt[u] < nt) {
        const char* x = a.x + (t0 + vt[u]) * a.x_token + vh[u] * a.x_head;
        lo[u].w = stream16(x + at_lo(u));
        if constexpr (!INTERLEAVED) hi[u].w = stream16(x + at_hi(u));
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (vt[u] < nt) {
        char* y = a.y + (t0 + vt[u]) * a.y_token + vh[u] * a.y_head;
        const float2* cs = rot + vt[u] * pairs + vc[u] * (INTERLEAVED ? E / 2 : E);
        if constexpr (INTERLEAVED) {
          if (vc[u] < turned) turn_beside(lo[u], cs);
        } else {
          if (vc[u] < turned) turn_halves(lo[u], hi[u], cs);
          put<STREAM>(y + at_hi(u), hi[u].w);
        }
        put<STREAM>(y + at_lo(u), lo[u].w);
      }
  }
}

// ------------------------------------------------------------ paged batch
constexpr int kMostKeys = 1 << 30;         // of a sequence: key indexes stay in 32 bits
constexpr int kMostTokens = 1 << 26;       // of a call
constexpr long kMostGroups = 0xffffffffL / 256;   // of a launch: its threads are counted in 32 bits
struct Batch {
  const int32_t *q_start, *seq_k, *table;
  int seqs, tokens, width, pages, shift;   // page_size = 1 << shift
  __device__ __forceinline__ int start(int i) const { return min(max(q_start[i], 0), tokens); }
  __device__ __forceinline__ long room() const { return min((long)width << shift, (long)kMostKeys); }
  // keys of sequence i that its table has slots for
  __device__ __forceinline__ int keys(int i) const { return (int)min((long)max(seq_k[i], 0), room()); }
  // Key of token t of sequence i, from its length and its end as they are given: one
  // that was cut would put a token that the table has no slot for on an older key's.
  __device__ __forceinline__ long key_of(int i, int t) const { return (long)seq_k[i] - q_start[i + 1] + t; }
};

// The last sequence i with at(i, start(i)) <= x, -1 for none, where at rises;
// first and end get start(i) and start(i + 1).  A wave looks at 64 sequences at
// a time: two loads and a ballot for up to 64.
template <typename F>
__device__ __forceinline__ int last_at_most(const Batch& b, long x, F&& at, int& first, int& end) {
  int found = -1;
  first = end = 0;
  for (int i0 = 0; i0 < b.seqs; i0 += 64) {
    const int i = i0 + ((int)threadIdx.x & 63), j = min(i, b.seqs - 1);
    const int s = b.start(j), e = b.start(j + 1);
    const unsigned long long m = __builtin_amdgcn_ballot_w64(i < b.seqs && at(j, s) <= x);
    if (m) {
      const int l = 63 - __builtin_clzll(m);
      found = i0 + l;
      first = __builtin_amdgcn_readlane(s, l);
      end = __builtin_amdgcn_readlane(e, l);
    }
    if (m != ~0ull) break;
  }
  return uniform(found);
}

// ----------------------------------------------------------------- append
struct AppendArgs {
  const char *k, *v, *q;
  char *qo, *kc, *vc;
  uint8_t *ks, *vs;
  long k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head;   // bytes
  Batch b;
  int heads, heads_q, tt, rotate;
  int log_tt;
  RotArgs rot;
};

// Eight consecutive values (chunk c) of a turned row; for halves, o holds the
// chunk of their partners.
__device__ __forceinline__ u32x4 turn8(u32x4 w, u32x4 o, int c, const RotArgs& r, const float2* cs) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[2 * j] = bf16_lo(w[j]), v[2 * j + 1] = bf16_hi(w[j]);
  if (r.interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 z = cs[4 * c + j];
      const float x = v[2 * j], y = v[2 * j + 1];
      w[j] = pack_bf16(__builtin_fmaf(x, z.x, -(y * z.y)), __builtin_fmaf(y, z.x, x * z.y));
    }
    return w;
  }
  const bool low = 8 * c < r.pairs;
  const float2* z = cs + (low ? 8 * c : 8 * c - r.pairs);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float y = (j & 1) ? bf16_hi(o[j / 2]) : bf16_lo(o[j / 2]);
    v[j] = low ? __builtin_fmaf(v[j], z[j].x, -(y * z[j].y)) : __builtin_fmaf(v[j], z[j].x, y * z[j].y);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
  return w;
}

// One thread holds 8 consecutive values of a row, D / 8 threads a row, so a
// 32-value block of MXFP8 is four neighbouring lanes, as in mxfp8_block, and the
// other halves of a turned row's pairs are in its lanes.  A workgroup's tokens
// are walked through head by head, since a page holds a head's tokens side by
// side: 11400 tokens (32/8 heads, D 128) into MXFP8 pages 78 -> 60 us.
// In place (q_out = q) a row's loads precede its stores: the row belongs to one
// instruction of one wave.
// With several tokens to a workgroup (MANY) a thread has four rows on their way
// at once and loads and stores past the caches; few tokens, whose rows were written
// just before, are taken from them: 2000 tokens into bf16 pages 12.8 us, 17.6 as
// many.  16000 tokens (393 MB) 79 us, 5.0 TB/s, 11400 into MXFP8 pages (258 MB) 58
// us, 4.4: the writes are scattered, a head's tokens at a time.
template <int D, bool F8, bool MANY>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  extern __shared__ float2 rot[];          // [tt][pairs]
  __shared__ long slot[kMostShared];       // row of head 0 in the cache, -1: none
  constexpr int C = D / 8, U = MANY ? 4 : 1;
  const long t0 = (long)blockIdx.x * a.tt;
  const int nt = (int)min((long)a.tt, a.b.tokens - t0);
  const int wave = threadIdx.x >> 6;
  for (int t = wave; t < nt; t += 4) {
    const int tok = (int)t0 + t;
    int first, end;
    const int i = last_at_most(a.b, tok, [](int, int start) { return (long)start; }, first, end);
    long s = -2;                           // padding: nothing of the token is written
    if (i >= 0 && tok < end) {
      s = -1;
      const long at = a.b.key_of(i, tok);
      if (at >= 0 && at < a.b.room()) {
        const int page = a.b.table[(long)i * a.b.width + (at >> a.b.shift)];
        if ((unsigned)page < (unsigned)a.b.pages)
          s = (((long)page * a.heads) << a.b.shift) + (at & ((1 << a.b.shift) - 1));
      }
    }
    if ((threadIdx.x & 63) == 0) slot[t] = s;
  }
  const int pairs = a.rotate ? a.rot.pairs : 0;
  for (int i = threadIdx.x; i < nt * pairs; i += 256)
    rot[i] = rot_of(a.rot, t0 + i / pairs, i % pairs, false);
  __syncthreads();
  const int total = (2 * a.heads + a.heads_q) << a.log_tt, c = threadIdx.x % C;
  const bool turned = 8 * c < 2 * pairs;
  const int partner = (threadIdx.x & 63) - c + (8 * c < pairs ? c + pairs / 8 : c - pairs / 8);   // a lane
  for (int i = (blockIdx.y * 256 + threadIdx.x) / C; i < total; i += U * (256 / C) * gridDim.y) {
    u32x4 w[U];
    int vt[U], vr[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = i + u * (256 / C) * gridDim.y;
      vt[u] = j < total ? j & (a.tt - 1) : a.tt, vr[u] = j >> a.log_tt;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (vt[u] < nt) {
        const bool is_q = vr[u] >= 2 * a.heads, is_v = !is_q && vr[u] >= a.heads;
        const long tok = t0 + vt[u];
        const char* row = is_q ? a.q + tok * a.q_token + (vr[u] - 2 * a.heads) * a.q_head
                        : is_v ? a.v + tok * a.v_token + (vr[u] - a.heads) * a.v_head
                               : a.k + tok * a.k_token + vr[u] * a.k_head;
        w[u] = MANY ? stream16(row + 16 * c) : *(const u32x4*)(row + 16 * c);
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (vt[u] >= nt) continue;           // whole rows, here and below
      const long s = slot[vt[u]];
      const bool is_q = vr[u] >= 2 * a.heads, is_v = !is_q && vr[u] >= a.heads;
      if (is_q ? s == -2 : s < 0) continue;
      u32x4 x = w[u];
      if (pairs && !is_v) {
        u32x4 o = x;
        if (!a.rot.interleaved)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] = (unsigned)__shfl((int)x[j], partner);
        if (turned) x = turn8(x, o, c, a.rot, rot + vt[u] * pairs);
      }
      if (is_q) {
        put<MANY>(a.qo + (t0 + vt[u]) * a.o_token + (vr[u] - 2 * a.heads) * a.o_head + 16 * c, x);
        continue;
      }
      const long to = s + ((long)(is_v ? vr[u] - a.heads : vr[u]) << a.b.shift);
      if constexpr (!F8) {
        put<MANY>((is_v ? a.vc : a.kc) + to * (2 * D) + 16 * c, x);
      } else {
        unsigned am = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) am = max(am, max(x[j] & 0x7fffu, (x[j] >> 16) & 0x7fffu));
        am = max(am, (unsigned)__shfl_xor((int)am, 1));
        am = max(am, (unsigned)__shfl_xor((int)am, 2));
        const int e = (int)(am >> 7), k = e == 0 ? -127 : max(e - 135, -127);
        typedef __attribute__((ext_vector_type(2))) short s16x2;
        auto y = [&](float f) { return __builtin_amdgcn_fmed3f(ldexpf(f, -k), -448.0f, 448.0f); };
        unsigned p[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          s16x2 z = {0, 0};
          z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, y(bf16_lo(x[2 * j])), y(bf16_hi(x[2 * j])), 1.0f, false);
          z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, y(bf16_lo(x[2 * j + 1])), y(bf16_hi(x[2 * j + 1])), 1.0f, true);
          p[j] = __builtin_bit_cast(unsigned, z);
        }
        put<MANY>((is_v ? a.vc : a.kc) + to * D + 8 * c, u32x2{p[0], p[1]});
        if ((c & 3) == 0) (is_v ? a.vs : a.ks)[to * (D / 32) + c / 4] = (uint8_t)(k + 127);
      }
    }
  }
}

// -------------------------------------------------------- paged attention
// Rows: the new tokens of one sequence times the G query heads that share a
// key/value head, row r = token r / G, head h G + r % G.  A workgroup takes
// BM of them at a time.  In the step kernel, where the host knows of no sequence
// with more than BM rows, slot n of the grid is sequence n, whose workgroup goes
// on to further BM rows if there are any.  Otherwise slot n belongs to the last
// sequence i with floor((q_start[i] - q_start[0]) G / BM) + i <= n, so that a
// sequence has at least ceil(new G / BM) slots whatever the lengths, and the
// grid, which the host knows without reading them, is ceil(tokens G / BM) +
// seqs - 1; slots without rows leave at once.
//
// Both kernels compute scores transposed, S^T = K Q^T, so a lane owns one row
// (column of the product), and O^T += V^T P^T with P^T taken from the score
// registers as they lie: the keys of a matrix instruction may come in any
// order if both operands have the same one.  V^T comes out of row-major LDS by
// the transposing read (ds_read_b64_tr_b16: 16 lanes give 4 rows x 16 columns,
// each gets one column's 4 values).  The running maximum is kept in log2 units
// (score scale log2 e), in which alpha and the probabilities are one fma and
// one exp2.  The row sum is that of the fp32 probabilities.  The step kernel's product
// takes each as a bf16 and, as a second one, what that rounding left (2^-16 of each in
// all); the chunk kernel's, which the matrix core bounds, as one bf16 (at most 2^-8
// of each, independent of one another), and divides O by the sum of these, so that a
// row that one key dominates is still exact.
struct PagedArgs {
  const char* q;
  char* out;
  float* lse;
  const char *kc, *vc;
  const uint8_t *ks, *vs;
  long q_token, q_head, o_token, o_head;   // bytes
  Batch b;
  float sl2;                               // scale log2 e
  int Hq, Hkv, G, causal, out_f32;
  int nsplit, chunk;                       // most splits of a row, keys of one
  int direct;                              // a slot is a sequence
  long rows;                               // tokens * Hq
  float* part_o;                           // [nsplit][rows][D]
  float2* part_ml;                         // [nsplit][rows]: maximum (log2 units), sum
};

struct Slot {
  int seq, row0, rows, q0, new_, keys;     // first row, rows of the slot; first token, new tokens, keys
  int key0;                                // key of the first token
};

// The slot but for its keys, which the caller loads beside what else it knows to
// ask for by then.
template <int BM>
__device__ __forceinline__ bool find_slot(const PagedArgs& a, int n, Slot& s) {
  int end;
  if (a.direct) {
    s.seq = n;
    s.q0 = a.b.start(n);
    end = a.b.start(n + 1);
    s.row0 = 0;
  } else {
    const int origin = a.b.start(0);
    auto at = [&](int i, int start) { return (long)max(start - origin, 0) * a.G / BM + i; };
    s.seq = last_at_most(a.b, n, at, s.q0, end);
    if (s.seq < 0) return false;
    s.row0 = (int)(n - at(s.seq, s.q0)) * BM;
  }
  s.new_ = max(end - s.q0, 0);
  s.rows = min(BM, s.new_ * a.G - s.row0);
  return s.rows > 0;
}
// On to the sequence's next rows.
template <int BM>
__device__ __forceinline__ bool next_rows(const PagedArgs& a, Slot& s) {
  s.row0 += BM;
  s.rows = min(BM, s.new_ * a.G - s.row0);
  return a.direct && s.rows > 0;
}

// The slot's keys.  (Tokens past the table see what it holds.  A length that no
// sequence has, past kMostKeys, is the table's.)
__device__ __forceinline__ void find_keys(const PagedArgs& a, Slot& s) {
  s.keys = a.b.keys(s.seq);
  long at = a.b.key_of(s.seq, s.q0);
  if (a.b.seq_k[s.seq] > kMostKeys) at = (long)s.keys - s.new_;
  s.key0 = (int)min(max(at, -(long)kMostKeys), (long)kMostKeys);
}
// Keys that row r of the slot sees.
__device__ __forceinline__ int seen(const PagedArgs& a, const Slot& s, int r) {
  return a.causal ? min(max(s.key0 + (s.row0 + r) / a.G + 1, 0), s.keys) : s.keys;
}

__device__ __forceinline__ int splits_of(const PagedArgs& a, int keys) {
  return max(1, min(a.nsplit, (int)(((long)keys + a.chunk - 1) / a.chunk)));
}

// Final values of four consecutive columns.
__device__ __forceinline__ void put4(char* at, int f32, f32x4 o) {
  if (f32) *(f32x4*)at = o;
  else *(uint2*)at = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
}

// ---- one or a few tokens
// Four waves of a workgroup take every fourth tile (32 keys) of a split's keys,
// each with its own running maximum, sum and O^T, joined at the end through LDS.
// The second product runs twice, on the probabilities' bf16 and on the rest of each,
// since the matrix core has time to spare: fp32 outputs are off by 1e-6 to 2e-6,
// with the bf16 alone by 0.0003 to 0.0011, at 0 to 3 % of a call's time (6 % where it
// works most: 16 sequences of 16 tokens over 4000 MXFP8 keys 40.3 to 42.8 us).
// Nothing is shared while streaming, so there is no barrier in the loop; a wave
// has one tile on its way while it works on the one before, 16 KB of bf16 at
// D 128, 128 KB a CU with its two workgroups.  16 RT rows: K in matrix-operand
// order straight into registers, V through LDS for its transposition.
//
// One token over 131000 keys (32/8 heads, D 128, bf16; 537 MB) takes 84 to 86 us, 6.2
// to 6.4 TB/s, in caches that are a process's first allocations, and 97 to 110 us, 4.9
// to 5.5 TB/s, in memory that was handed out before; a kernel that streams the same
// bytes in order reaches 6.7 TB/s in both.  17 sequences of 5000 to 20000 keys (797
// MB) 138 us, 5.8 TB/s.
constexpr int kStepWaves = 4;
constexpr int kStepHalves = 2;     // 16-key halves of a wave's tile

template <int D, int RT>
struct StepLds {
  static constexpr int kV = 16 * kStepHalves * D * 2;                // V tile of a wave
  static constexpr int kO = 16 * RT * (D + 4) * 4;                   // O of a wave
  static constexpr int kWave = kV > kO ? kV : kO;
  static constexpr int kTotal = kStepWaves * (kWave + 16 * RT * 8);  // and maximum, sum
};

// Where chunk c (8 columns) of V row r lies: a 16-lane group reads 4 rows x 32
// bytes, two groups 8 rows, which the swizzle spreads over all banks.
template <int D>
__device__ __forceinline__ int step_v_at(int r, int c) {
  const int f = D == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1;
  return r * (2 * D) + ((c ^ f) << 4);
}

// One tile in registers.  A lane has row lane % 16 of every 16-key half of K:
// 16-byte pieces g, g + 4, .. of it (g = lane / 16), so that a load takes 64
// consecutive bytes of 16 rows; V by whole rows.
template <int D, bool F8>
struct StepTile {
  static constexpr int KS = D / 32;                       // k-steps of 32 columns
  static constexpr int KN = F8 ? D / 64 : D / 32;         // 16-byte pieces of a K row's lane
  static constexpr int VN = kStepHalves * (F8 ? D / 64 : D / 32);  // 16-byte pieces of V a lane
  static constexpr int VROWS = F8 ? 1024 / D : 512 / D;   // V rows of one load
  u32x4 k[kStepHalves][KN], v[VN];
  unsigned ksc[F8 ? kStepHalves : 1], vsc[F8 ? VN : 1];   // a K row's scales, a V piece's scale
  __device__ __forceinline__ void load_k(const PagedArgs& a, const long* row, int lane) {
    const unsigned r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int hf = 0; hf < kStepHalves; ++hf) {
      const char* p = a.kc + row[hf] * (F8 ? D : 2 * D);
      const unsigned off = r * (F8 ? D : 2 * D) + 16 * g;
#pragma unroll
      for (int n = 0; n < KN; ++n) k[hf][n] = stream16(p + (off + 64 * n));
      if constexpr (F8) {
        const uint8_t* e = a.ks + row[hf] * (D / 32);
        if constexpr (D == 128) ksc[hf] = *(const unsigned*)(e + 4 * r);
        else ksc[hf] = *(const unsigned short*)(e + 2 * r);
      }
    }
  }
  __device__ __forceinline__ void load_v(const PagedArgs& a, const long* row, int lane) {
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      const int hf = n * VROWS / 16;
      const unsigned r = n * VROWS % 16 + lane * VROWS / 64;
      const unsigned c = lane % (64 / VROWS);
      if constexpr (F8) {
        v[n] = stream16(a.vc + row[hf] * D + (r * D + 16 * c));
        vsc[n] = (a.vs + row[hf] * (D / 32))[r * (D / 32) + c / 2];
      } else {
        v[n] = stream16(a.vc + row[hf] * (2 * D) + (r * (2 * D) + 16 * c));
      }
    }
  }
  // K operand of 16-key half hf and k-step s: the columns of step_q_col
  __device__ __forceinline__ bf16x8 k_op(int hf, int s, int g) const {
    if constexpr (F8) {
      // piece s / 2 has codes 64 (s / 2) + 16 g ..: block 2 (s / 2) + g / 2
      const float sc = e8m0_scale((ksc[hf] >> (16 * (s / 2) + 8 * (g >> 1))) & 255u);
      const uint2 x = e4m3_bf16x4(k[hf][s / 2][2 * (s & 1)], sc), y = e4m3_bf16x4(k[hf][s / 2][2 * (s & 1) + 1], sc);
      return __builtin_bit_cast(bf16x8, u32x4{x.x, x.y, y.x, y.y});
    } else {
      return __builtin_bit_cast(bf16x8, k[hf][s]);
    }
  }
  // rows from `live` on, and those of a page that is none, become zero
  __device__ __forceinline__ void put_v(uint8_t* lds, int lane, bool cut, int live, unsigned bad) {
#pragma unroll
    for (int n = 0; n < VN; ++n) {
      const int r = n * VROWS + lane * VROWS / 64, c = lane % (64 / VROWS);
      const bool none = cut && (r >= live || (bad >> (n * VROWS / 16) & 1));
      if (none) v[n] = u32x4{0u, 0u, 0u, 0u};
      if constexpr (F8) {
        const float sc = e8m0_scale(none ? 0u : vsc[n]);
        const uint2 x = e4m3_bf16x4(v[n][0], sc), y = e4m3_bf16x4(v[n][1], sc);
        const uint2 z = e4m3_bf16x4(v[n][2], sc), w = e4m3_bf16x4(v[n][3], sc);
        *(u32x4*)(lds + step_v_at<D>(r, 2 * c)) = u32x4{x.x, x.y, y.x, y.y};
        *(u32x4*)(lds + step_v_at<D>(r, 2 * c + 1)) = u32x4{z.x, z.y, w.x, w.y};
      } else {
        *(u32x4*)(lds + step_v_at<D>(r, c)) = v[n];
      }
    }
  }
};

// First of the 8 columns of a head that lane group g holds in k-step s.
template <int D, bool F8>
__device__ __forceinline__ int step_q_col(int g, int s) {
  return F8 ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
}

// One slot's rows, split sp of their keys.
template <int D, bool F8, int RT>
__device__ __forceinline__ void step_rows(const PagedArgs& a, Slot& s, int h, int sp, uint8_t* lds) {
  typedef StepLds<D, RT> L;
  constexpr int KS = D / 32, SLABS = D / 16, KEYS = 16 * kStepHalves, ROUND = kStepWaves * KEYS, AHEAD = 64 / kStepHalves;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));           // nothing of it is kept from one round of rows to the next
  const int wave = uniform(threadIdx.x >> 6);
  const int g = lane >> 4, col = lane & 15;

  // The wave's tiles begin at k0 + KEYS wave + ROUND it; lane kStepHalves (it %
  // AHEAD) + half holds the page of that tile's half, for AHEAD tiles at a time.
  // The first ones, and Q, are asked for beside the sequence's length.
  const int k0 = (int)min((long)sp * a.chunk, (long)kMostKeys);
  const int32_t* table = a.b.table + (long)s.seq * a.b.width;
  auto pages_from = [&](int it) {
    const long key = (long)k0 + KEYS * wave + (long)ROUND * (it + lane / kStepHalves) + 16 * (lane % kStepHalves);
    const long at = key >> a.b.shift;
    return at < a.b.width ? table[at] : 0;
  };
  int ids = pages_from(0);
  bf16x8 q[RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = s.row0 + min(16 * rt + col, s.rows - 1);
    const char* p = a.q + (long)(s.q0 + row / a.G) * a.q_token + (h * a.G + row % a.G) * a.q_head;
#pragma unroll
    for (int i = 0; i < KS; ++i) q[rt][i] = *(const bf16x8*)(p + 2 * step_q_col<D, F8>(g, i));
  }
  find_keys(a, s);
  const int ns = splits_of(a, s.keys);
  if (sp >= ns) return;
  const int last = seen(a, s, s.rows - 1);
  const int k1 = max(k0, sp == ns - 1 ? last : min(last, k0 + a.chunk));
  const int free_of_mask = min(k1, seen(a, s, 0));     // keys below are seen by every row
  int vis[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) vis[rt] = min(k1, seen(a, s, min(16 * rt + col, s.rows - 1)));
  f32x4 o[RT][SLABS];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -INFINITY;
    l[rt] = 0.0f;
#pragma unroll
    for (int i = 0; i < SLABS; ++i) o[rt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  uint8_t* vt = lds + wave * L::kWave;

  const int ntiles = (k1 - k0 - KEYS * wave + ROUND - 1) / ROUND;
  const unsigned in_page = (1u << a.b.shift) - 1;
  // cache rows of a tile's halves; a bit for each half whose page is none.
  // Halves behind the last key stay within their sequence's pages, or page 0.
  auto rows_of = [&](int it, long* row) {
    unsigned bad = 0;
#pragma unroll
    for (int hf = 0; hf < kStepHalves; ++hf) {
      const int id = __builtin_amdgcn_readlane(ids, kStepHalves * (it % AHEAD) + hf);
      const unsigned key = k0 + KEYS * wave + ROUND * it + 16 * hf;
      const bool none = (unsigned)id >= (unsigned)a.b.pages;
      if (none) bad |= 1u << hf;
      row[hf] = (((long)(none ? 0 : id) * a.Hkv + h) << a.b.shift) + (key & in_page);
    }
    return bad;
  };
  if (ntiles > 0) {
    StepTile<D, F8> t;
    long row[kStepHalves];
    unsigned bad = rows_of(0, row);
    t.load_k(a, row, lane);
    t.load_v(a, row, lane);
    for (int it = 0; it < ntiles; ++it) {
      const int key0 = k0 + KEYS * wave + ROUND * it;
      const unsigned now_bad = bad;
      f32x4 sc[RT][kStepHalves];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int hf = 0; hf < kStepHalves; ++hf) sc[rt][hf] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int hf = 0; hf < kStepHalves; ++hf)
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          const bf16x8 kop = t.k_op(hf, i, g);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            sc[rt][hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop, q[rt][i], sc[rt][hf], 0, 0, 0);
        }
      const bool cut = key0 + KEYS > k1 || now_bad;
      t.put_v(vt, lane, cut, k1 - key0, now_bad);
      if (it + 1 < ntiles) {
        if ((it + 1) % AHEAD == 0) ids = pages_from(it + 1);
        bad = rows_of(it + 1, row);
        t.load_k(a, row, lane);
        t.load_v(a, row, lane);
      }
      asm volatile("" ::: "memory");       // the tile is written before it is read; LDS keeps a wave's order
      const bool mask = cut || key0 + KEYS > free_of_mask;
      bf16x8 p[RT][kStepHalves / 2], rest[RT][kStepHalves / 2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        if (mask) {
#pragma unroll
          for (int hf = 0; hf < kStepHalves; ++hf)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (key0 + 16 * hf + 4 * g + j >= vis[rt] || (now_bad >> hf & 1)) sc[rt][hf][j] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int hf = 0; hf < kStepHalves; ++hf) {
          mx = max3f(mx, sc[rt][hf][0], sc[rt][hf][1]);
          mx = max3f(mx, sc[rt][hf][2], sc[rt][hf][3]);
        }
        mx = max_of_groups(mx) * a.sl2;
        if (__builtin_amdgcn_ballot_w64(mx > m[rt])) {
          const float mn = __builtin_fmaxf(m[rt], mx);
          const float alpha = __builtin_amdgcn_exp2f(m[rt] - (mn == -INFINITY ? 0.0f : mn));
          m[rt] = mn;
          l[rt] *= alpha;
#pragma unroll
          for (int i = 0; i < SLABS; ++i) o[rt][i] *= alpha;
        }
        const float ref = m[rt] == -INFINITY ? 0.0f : m[rt];
#pragma unroll
        for (int pr = 0; pr < kStepHalves / 2; ++pr) {
          u32x4 w, left;
          float sum = 0.0f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x4& x = sc[rt][2 * pr + j / 2];
            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * (j & 1)], a.sl2, -ref));
            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[2 * (j & 1) + 1], a.sl2, -ref));
            sum += e0 + e1;
            w[j] = pack_bf16(e0, e1);
            left[j] = pack_bf16(e0 - bf16_lo(w[j]), e1 - bf16_hi(w[j]));
          }
          l[rt] += sum;
          p[rt][pr] = __builtin_bit_cast(bf16x8, w);
          rest[rt][pr] = __builtin_bit_cast(bf16x8, left);
        }
      }
#pragma unroll
      for (int pr = 0; pr < kStepHalves / 2; ++pr)
#pragma unroll
        for (int i = 0; i < SLABS; ++i) {
          const int r = 32 * pr + 4 * g + (col >> 2), c = 2 * i + ((col >> 1) & 1), b = 8 * (col & 1);
          const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + step_v_at<D>(r, c) + b));
          const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + step_v_at<D>(r + 16, c) + b));
          const bf16x8 vop = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            o[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, rest[rt][pr], o[rt][i], 0, 0, 0);
            o[rt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop, p[rt][pr], o[rt][i], 0, 0, 0);
          }
        }
      asm volatile("" ::: "memory");
    }
  }

  // Join the four waves: O, maximum and sum of each through LDS.
  __syncthreads();
  float* ow = (float*)vt;
  float2* ml = (float2*)(lds + kStepWaves * L::kWave);    // [wave][16 RT]
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = sum_of_groups(l[rt]);
    if (g == 0) ml[wave * 16 * RT + 16 * rt + col] = make_float2(m[rt], l[rt]);
#pragma unroll
    for (int i = 0; i < SLABS; ++i) *(f32x4*)(ow + (16 * rt + col) * (D + 4) + 16 * i + 4 * g) = o[rt][i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < s.rows * (D / 4); i += 64 * kStepWaves) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    float M = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) M = __builtin_fmaxf(M, ml[w * 16 * RT + r].x);
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    if (M != -INFINITY)
#pragma unroll
      for (int w = 0; w < kStepWaves; ++w) {
        const float2 z = ml[w * 16 * RT + r];
        const float e = __builtin_amdgcn_exp2f(z.x - M);
        sum += e * z.y;
        x += e * *(const f32x4*)((const float*)(lds + w * L::kWave) + r * (D + 4) + c);
      }
    const int row = s.row0 + r, tok = s.q0 + row / a.G, hq = h * a.G + row % a.G;
    const long at = (long)tok * a.Hq + hq;
    if (ns == 1) {
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      put4(a.out + tok * a.o_token + hq * a.o_head + c * (a.out_f32 ? 4 : 2), a.out_f32, x * inv);
      if (c == 0 && a.lse)
        a.lse[at] = sum > 0.0f ? (M + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
    } else {
      *(f32x4*)(a.part_o + ((long)sp * a.rows + at) * D + c) = x;
      if (c == 0) a.part_ml[(long)sp * a.rows + at] = make_float2(M, sum);
    }
  }
}

template <int D, bool F8, int RT>
__global__ __launch_bounds__(64 * kStepWaves, 2) void paged_step_kernel(PagedArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  const int h = blockIdx.x % a.Hkv;
  Slot s;
  if (!find_slot<16 * RT>(a, (int)(blockIdx.x / a.Hkv), s)) return;
  do {
    step_rows<D, F8, RT>(a, s, h, (int)blockIdx.y, lds);
    __syncthreads();
  } while (next_rows<16 * RT>(a, s));
}

// ---- many tokens
// Waves of 32 rows share 64-key tiles of K and V in LDS, in rings of three or
// four.  A SIMD overlaps its matrix core and its vector unit when one of its two
// waves does only matrix work and the other only vector work, not when both do
// some of each; so at D 128 eight waves form two groups that swap phases at a
// barrier: while one group runs M (P V of tile j, scores of tile j + 1: 32 matrix
// instructions), the other runs V (exponentials of a tile).  At D 64 a phase is
// too short for that (a barrier costs a tenth of it) and rows are short enough
// for three workgroups of four waves a CU, which overlap by themselves.
//
// 2048 tokens behind 14000 keys (32/8 heads, D 128, bf16; 504 GFLOP) take 445 to 461
// us by the box, 1094 to 1133 TFLOP/s; 4096 behind 28000, MXFP8, 1713 to 1764 us, 1143
// to 1177.  The matrix core is busy 63 % of the cycles and the chip lowers its clock
// for the power: 1.66 to 1.72 GHz in twenty calls in a row, which then take 475 to 492
// us (on keys and values of one constant it runs at 2.23).  D 64, 7 sequences of up to 1500 tokens
// behind 3001 (16/4 heads): 82 to 85 us, 674 to 701 TFLOP/s.  There neither unit is
// full (vector 0.45, matrix 0.33 of the cycles): 800 workgroups of 15 to 63 tiles go
// to 768 places in the order of their slots, so the fullest CU has 137 tiles or more
// where an even share is 111.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<N, I + 1>(f);
  }
}

template <int D, bool F8, int NW>
struct ChunkLds {
  static constexpr int kTile = kBc * D * 2;     // bytes of 64 rows of K or V
  static constexpr int kRing = F8 || NW == 4 ? 3 : 4;   // tiles of each
  static constexpr int kTotal = 2 * kRing * kTile;
};

// Swizzles of 16-byte chunk c of row r.  K: 16 rows at one column chunk. V: the
// transposing read takes 4 rows x 64 bytes in 32 lanes.
template <int D>
__device__ __forceinline__ int chunk_k_swz(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D>
__device__ __forceinline__ int chunk_v_swz(int r) { return D == 128 ? ((r & 3) << 2) ^ (r & 2) : ((r >> 1) & 1) << 2; }

// One 1 KB direct-to-LDS load through a buffer resource (address, bytes): lane
// i's 16 bytes at voff land at LDS address `to` + 16 i, zeros where voff is past
// the resource's bytes.  In assembly, since the compiler would wait for all such
// loads before the next transposing read; it has no register output, and the
// kernel's own waits count it.  Waits that the compiler places for its loads
// count it too, and so only wait longer.
__device__ __forceinline__ void load_lds_1k(u32x4 rsrc, unsigned to, int voff) {
  // (five wait states from a vector instruction that writes a scalar register to
  // a memory instruction that reads it, one from the write of m0.  The compiler
  // reserves m0: it keeps nothing there over instructions, so there is nothing to
  // clobber, and these kernels have no other instruction that reads it)
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(to), "v"(voff), "s"(rsrc) : "memory");
}
// 16 bytes, one byte at `from` + voff, zero where voff is past `bytes`.
__device__ __forceinline__ u32x4 raw_load16(const char* from, unsigned bytes, int voff) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(from, bytes), voff, 0, 0));
}
__device__ __forceinline__ unsigned raw_load1(const char* from, unsigned bytes, int voff) {
  return (unsigned char)__builtin_amdgcn_raw_buffer_load_b8(make_rsrc(from, bytes), voff, 0, 0);
}

// A kernel's lambdas that hold its registers by reference have to be inlined.
#define EFQ_INLINE __attribute__((always_inline))

// What brings the K and V tiles of one slot into LDS.  A wave brings the same 8
// or 16 rows of every tile, which lie in one page.  Where they lie is worked out
// for 64 tiles at once, lane t for tile t of a group, so that a step only reads
// it out of the lane.
template <int D, bool F8, int NW>
struct ChunkFeed {
  static constexpr int RB = F8 ? D : 2 * D;                 // bytes of a row
  static constexpr int ROWS = kBc / NW;                     // rows of a wave
  static constexpr int PER = ROWS * RB / 1024;              // its 1 KB loads of K, and of V
  static_assert(PER * 1024 == ROWS * RB && 16 % ROWS == 0, "a wave's rows are whole loads in one page");
  static constexpr int RI = ROWS / PER;                     // rows of a load
  // Of the group's tiles: address of K and V (MXFP8: cache row, in k), bytes of
  // the wave's rows that are keys (MXFP8: rows), a bit for each 16-key quarter
  // whose page is none (and 4 bits up, of the group before).
  unsigned klo, khi, vlo, vhi, n, none;
  unsigned v_lo, v_hi, v_n;                                 // of the tile before: V follows K by a tile
  u32x4 kc[F8 ? PER : 1], vc[F8 ? PER : 1];                 // MXFP8: codes and scales on their way
  unsigned ke[F8 ? PER : 1], ve[F8 ? PER : 1];
  int off[2];                                               // the lane's place in a load of K, of V

  __device__ __forceinline__ void init(int wave, int lane) {
    const int r = wave * ROWS + lane * RI / 64, c = lane % (64 / RI);
    off[0] = F8 ? 16 * lane : (lane * RI / 64) * RB + ((c ^ chunk_k_swz<D>(r)) << 4);
    off[1] = F8 ? 16 * lane : (lane * RI / 64) * RB + ((c ^ chunk_v_swz<D>(r)) << 4);
  }
  // the place in load n against load 0's: further rows, and the swizzle's bits
  // that they set
  template <int N, int V>
  __device__ __forceinline__ int place() const {
    const int swz = V ? chunk_v_swz<D>(N * RI) : chunk_k_swz<D>(N * RI);
    return (off[V] ^ (F8 ? 0 : swz << 4)) + N * 1024;
  }

  // (the group's pages are waited for: a microsecond in the 64 tiles' hundred)
  __device__ __forceinline__ void take_pages(const PagedArgs& a, const int32_t* table, int h, int k0, int k1, int tile0,
                                             int wave, int lane) {
    none <<= 4;
    int id = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long at = (long)k0 + (long)kBc * (tile0 + lane) + 16 * i;
      const int page = at < k1 ? table[at >> a.b.shift] : 0;
      if ((unsigned)page >= (unsigned)a.b.pages) none |= 1u << i;
      if (wave * ROWS / 16 == i) id = page;
    }
    const bool ok = (unsigned)id < (unsigned)a.b.pages;
    const long key = (long)k0 + (long)kBc * (tile0 + lane) + wave * ROWS;
    const long row = (((long)(ok ? id : 0) * a.Hkv + h) << a.b.shift) + ((unsigned)key & ((1u << a.b.shift) - 1));
    const int live = ok ? (int)min(max((long)k1 - key, 0L), (long)ROWS) : 0;
    if constexpr (F8) {
      klo = (unsigned)row, khi = (unsigned)(row >> 32), n = live;
    } else {
      const unsigned long long k = (unsigned long long)(a.kc + row * RB), v = (unsigned long long)(a.vc + row * RB);
      klo = (unsigned)k, khi = (unsigned)(k >> 32) & 0xffffu, vlo = (unsigned)v, vhi = (unsigned)(v >> 32) & 0xffffu;
      n = live * RB;
    }
  }
  // K of tile t is next, V of the tile before it
  __device__ __forceinline__ void next_tile(int t, unsigned& lo, unsigned& hi, unsigned& bytes) {
    lo = __builtin_amdgcn_readlane(klo, t & 63);
    hi = __builtin_amdgcn_readlane(khi, t & 63);
    bytes = __builtin_amdgcn_readlane(n, t & 63);
  }
  __device__ __forceinline__ void keep_v(int t, unsigned lo, unsigned hi, unsigned bytes) {
    v_lo = F8 ? lo : __builtin_amdgcn_readlane(vlo, t & 63);
    v_hi = F8 ? hi : __builtin_amdgcn_readlane(vhi, t & 63);
    v_n = bytes;
  }
  template <int N, int V>
  __device__ __forceinline__ void ask(const PagedArgs& a, unsigned lo, unsigned hi, unsigned bytes, unsigned to, int lane) {
    if constexpr (!F8) {
      load_lds_1k(u32x4{lo, hi, bytes, 0x00020000u}, to + N * 1024, place<N, V>());
    } else {
      const unsigned long long row = (unsigned long long)hi << 32 | lo;
      u32x4& c = V ? vc[N] : kc[N];
      unsigned& e = V ? ve[N] : ke[N];
      c = raw_load16((V ? a.vc : a.kc) + row * RB, bytes * RB, place<N, V>());
      e = raw_load1((const char*)((V ? a.vs : a.ks) + row * (D / 32)), bytes * (D / 32),
                    (lane * RI / 64 + N * RI) * (D / 32) + lane % (64 / RI) / 2);
    }
  }
  // MXFP8: what has come, as bf16, into the tile
  template <int N, int V>
  __device__ __forceinline__ void land(uint8_t* to, int wave, int lane) {
    const int r = wave * ROWS + N * RI + lane * RI / 64, c = lane % (64 / RI);
    const int swz = V ? chunk_v_swz<D>(r) : chunk_k_swz<D>(r);
    const u32x4& x = V ? vc[N] : kc[N];
    const float sc = e8m0_scale(V ? ve[N] : ke[N]);
    const uint2 e = e4m3_bf16x4(x[0], sc), f = e4m3_bf16x4(x[1], sc);
    const uint2 y = e4m3_bf16x4(x[2], sc), z = e4m3_bf16x4(x[3], sc);
    *(u32x4*)(to + r * 2 * D + (((2 * c) ^ swz) << 4)) = u32x4{e.x, e.y, f.x, f.y};
    *(u32x4*)(to + r * 2 * D + (((2 * c + 1) ^ swz) << 4)) = u32x4{y.x, y.y, z.x, z.y};
  }
};

// The running reference of a row need not be its maximum: it moves only when a
// lane's probabilities of a tile sum up to more than this, so almost never
// after the first tile, and until then no maximum is taken and nothing rescaled.
// The sums stay below 2^42 (2^16 a tile and lane), times the values.  With the
// maximum as the reference a dominant key's probability would be 1 and exact; here
// it is rounded like any other, so O is divided by the sum of the rounded ones, in
// which a dominant key's rounding cancels (the matrix core sums them, from the
// product's own operand), while log-sum-exp and the weights of a row's parts keep
// the unrounded sum.  Relative error of O in fp32, by the unrounded sum / the rounded
// one / with the maximum as the reference: 2048 tokens behind 14000 (D 128, bf16)
// 0.00164 / 0.00150 / 0.00099, 4096 behind 28000 (MXFP8) 0.00162 / 0.00119 / 0.00068,
// up to 1500 behind 3001 (D 64) 0.00163 / 0.00125 / 0.00078; it costs 2 to 4 % of a
// call (431 to 445 us, 1670 to 1715, 81 to 83), the maximum 30 to 50 %.  A limit of 64
// without it: 0.00142, 0.00124 and 0.00138 for 441, 1686 and 85 us, and up to 9 % on
// short rows (300 tokens 16.6 to 18.2 us).
constexpr float kMostSum = 65536.0f;

// One slot's rows, split sp of their keys.
template <int D, bool F8, int NW>
__device__ __forceinline__ void chunk_rows(const PagedArgs& a, Slot& s, int h, int sp, uint8_t* lds) {
  constexpr int KK = D / 16, DT = D / 32, kTile = ChunkLds<D, F8, NW>::kTile, NB = ChunkLds<D, F8, NW>::kRing;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;
  find_keys(a, s);
  const int ns = splits_of(a, s.keys);
  if (sp >= ns) return;
  const int last = seen(a, s, s.rows - 1);
  const int k0 = uniform((int)min((long)sp * a.chunk, (long)s.keys));
  const int k1 = uniform(max(k0, sp == ns - 1 ? last : min(last, k0 + a.chunk)));
  const int ntiles = (k1 - k0 + kBc - 1) / kBc;

  const int r0 = 32 * wave, r = r0 + col;
  const int row = s.row0 + min(r, s.rows - 1), tok = s.q0 + row / a.G, hq = h * a.G + row % a.G;
  bf16x8 q[KK];
  {
    const char* p = a.q + (long)tok * a.q_token + hq * a.q_head;
#pragma unroll
    for (int i = 0; i < KK; ++i) q[i] = *(const bf16x8*)(p + 32 * i + 16 * half);
  }
  const int vis = min(k1, seen(a, s, min(r, s.rows - 1)));
  const int free_of_mask = uniform(min(k1, seen(a, s, min(r0, s.rows - 1))));   // keys below are seen by the wave's rows
  // tiles that some row of the wave sees
  const int mine = uniform(r0 < s.rows ? (min(k1, seen(a, s, min(r0 + 31, s.rows - 1))) - k0 + kBc - 1) / kBc : 0);
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
  float m = -INFINITY, l = 0.0f, ref = 0.0f;                // ref: m, or 0 while no key was seen

  // LDS addresses of the operands in place 0 of the rings: K column chunk i, V
  // head-dim tile i; and of what the wave brings
  const unsigned lds0 = lds_addr(lds);
  unsigned ka[KK], va[DT];
#pragma unroll
  for (int i = 0; i < KK; ++i) ka[i] = lds0 + col * 2 * D + (((2 * i + half) ^ chunk_k_swz<D>(col)) << 4);
  {
    const int vr = 4 * half + ((lane & 15) >> 2);
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      const int c = 4 * i + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
      va[i] = lds0 + NB * kTile + vr * 2 * D + ((c ^ chunk_v_swz<D>(vr)) << 4) + 8 * (lane & 1);
    }
  }

  // Step j brings K tile t = j + NB and V tile t - 1, a load (of K, then of V)
  // at a time.  Past the last tile the loads go on, of no bytes, so that a wait
  // counts the same loads in every step.  t is in ring place SLOT, j too.
  typedef ChunkFeed<D, F8, NW> Feed;
  Feed feed;
  feed.init(wave, lane);
  feed.none = feed.v_n = feed.v_lo = feed.v_hi = 0u;
  const int32_t* table = a.b.table + (long)s.seq * a.b.width;
  const unsigned brings = lds0 + wave * (Feed::PER * 1024);
  unsigned f_lo, f_hi, f_n;                                 // K's place in the step's fetch
  auto turn_page = [&](int t) EFQ_INLINE {
    if ((t & 63) == 0) feed.take_pages(a, table, h, k0, k1, t, wave, lane);
  };
  auto fetch_one = [&](auto slot, auto piece, int t) EFQ_INLINE {
    constexpr int SLOT = decltype(slot)::value, I = decltype(piece)::value;
    if constexpr (I == 0) feed.next_tile(t, f_lo, f_hi, f_n);
    if constexpr (I < Feed::PER) {
      feed.template ask<I, 0>(a, f_lo, f_hi, f_n, brings + SLOT * kTile, lane);
    } else {
      feed.template ask<I - Feed::PER, 1>(a, feed.v_lo, feed.v_hi, feed.v_n, brings + (NB + (SLOT + NB - 1) % NB) * kTile, lane);
      if constexpr (I == 2 * Feed::PER - 1) feed.keep_v(t, f_lo, f_hi, f_n);
    }
  };
  auto fetch = [&](auto slot, int t) EFQ_INLINE {
    static_for<2 * Feed::PER>([&](auto i) EFQ_INLINE { fetch_one(slot, i, t); });
  };
  auto land = [&](auto slot) EFQ_INLINE {                   // the K tile of place SLOT, the V tile of the one before
    constexpr int SLOT = decltype(slot)::value;
    if constexpr (F8) {
      static_for<Feed::PER>([&](auto i) EFQ_INLINE {
        feed.template land<decltype(i)::value, 0>(lds + SLOT * kTile, wave, lane);
        feed.template land<decltype(i)::value, 1>(lds + (NB + (SLOT + NB - 1) % NB) * kTile, wave, lane);
      });
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  };

  f32x16 sc[2];
  bf16x8 p[4];
  // The sums of rounded probabilities, the same in all four: the 16-wide product
  // takes a P operand's lanes l + 16 for k 8 to 15, 24 to 31 of column l % 16, so rows
  // 0 to 3 and 8 to 11 of its result, which lanes 0 to 15 and 32 to 47 get, sum the
  // other k, and the rest those.
  f32x4 lr = {0.0f, 0.0f, 0.0f, 0.0f};
  const unsigned own = ((lane >> 4) & 1) == ((lane >> 2) & 1) ? kOnes : 0u;
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{own, own, own, own});
  // M(j) is NV products of V tile j with its probabilities, then NK of K tile
  // j + 1 with Q, in pairs whose second operand is read first, so that one wait
  // serves both.  Operands are read kAhead products before they are used (an LDS
  // read takes as long as about four), the first ones at the end of the vector
  // phase before.  A wave issues an instruction in five cycles at best and a
  // product takes 32: what stands between two products is counted.
  constexpr int NV = 4 * DT, NK = 2 * KK, kAhead = 4;
  bf16x8 op[NV + NK];
  auto read_op = [&](auto slot, auto n) EFQ_INLINE {        // slot: of tile j
    constexpr int SLOT = decltype(slot)::value, N = decltype(n)::value;
    if constexpr (N < NV) {
      const lds_cptr at = lds_at(va[N % DT]) + SLOT * kTile + (N / DT) * 32 * D;
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * D));
      op[N] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    } else if constexpr (N < NV + NK) {
      constexpr int I = N - NV;
      op[N] = *(__attribute__((address_space(3))) const bf16x8*)(lds_at(ka[I / 2]) + (SLOT + 1) % NB * kTile + (I % 2) * 64 * D);
    }
  };
  auto product = [&](auto n) EFQ_INLINE {
    constexpr int N = decltype(n)::value;
    if constexpr (N < NV) {
      o[N % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[N], p[N / DT], o[N % DT], 0, 0, 0);
    } else {
      constexpr int I = N - NV, W = I % 2;
      if constexpr (I < 2) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[W][i] = 0.0f;
      }
      sc[W] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[N], q[I / 2], sc[W], 0, 0, 0);
    }
  };
  auto phase_m = [&](auto slot, int j) EFQ_INLINE {
    if (j >= mine) return fetch(slot, j + NB);
    __builtin_amdgcn_s_setprio(1);
    static_for<(NV + NK) / 2>([&](auto n) EFQ_INLINE {
      constexpr int N = 2 * decltype(n)::value, kEvery = (NV + NK) / (2 * Feed::PER);
      product(std::integral_constant<int, N + 1>{});
      read_op(slot, std::integral_constant<int, N + kAhead>{});
      __builtin_amdgcn_sched_barrier(0);
      product(std::integral_constant<int, N>{});
      read_op(slot, std::integral_constant<int, N + kAhead + 1>{});
      if constexpr (N < NV && N % DT == 0) lr = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, p[N / DT], lr, 0, 0, 0);
      // the step's loads, in the products' shadow
      if constexpr (N % kEvery == kEvery / 2) fetch_one(slot, std::integral_constant<int, N / kEvery>{}, j + NB);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto phase_v = [&](auto slot, int j) EFQ_INLINE {         // probabilities of tile j, in place SLOT
    if (j >= mine) return;
    __builtin_amdgcn_s_setprio(0);
    const int key0 = k0 + kBc * j;
    // (the feed's group is that of tile j + NB - 1)
    const unsigned none = (unsigned)__builtin_amdgcn_readlane(feed.none, j & 63) >> ((j & 63) > 64 - NB ? 4 : 0) & 15u;
    if (none || key0 + kBc > free_of_mask) {
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int kw = 32 * w + 8 * (i >> 2) + 4 * half + (i & 3);
          if (key0 + kw >= vis || (none >> (2 * w + (i >> 3)) & 1)) sc[w][i] = -INFINITY;
        }
    }
    u32x4 pw[4];
    float sum;
    auto probabilities = [&]() EFQ_INLINE {
      float part[4];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        part[ks] = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x16& x = sc[ks / 2];
          const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[8 * (ks & 1) + 2 * i], a.sl2, -ref));
          const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[8 * (ks & 1) + 2 * i + 1], a.sl2, -ref));
          part[ks] += e0;
          part[ks] += e1;
          pw[ks][i] = pack_bf16(e0, e1);
        }
      }
      sum = (part[0] + part[1]) + (part[2] + part[3]);
    };
    probabilities();
    if (__builtin_amdgcn_ballot_w64(!(sum <= kMostSum) || m == -INFINITY)) {
      const float mx = max_of_halves(__builtin_fmaxf(max16(sc[0]), max16(sc[1]))) * a.sl2;
      const float mn = __builtin_fmaxf(m, mx);
      const float alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
      m = mn;
      ref = mn == -INFINITY ? 0.0f : mn;
      l *= alpha;
      lr *= alpha;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= alpha;
      probabilities();
    }
    l += sum;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) p[ks] = __builtin_bit_cast(bf16x8, pw[ks]);
    static_for<kAhead>([&](auto n) EFQ_INLINE { read_op(slot, n); });
  };

  // The second group runs a phase behind the first.  bf16, step j: K tile
  // j + NB and V tile j + NB - 1 are asked for in M(j), into the places of tiles
  // j and j - 1, which both groups have read by then; before the barrier behind
  // M(j) a wave waits for its part of K tile j + 3 and V tile j + 2: the first
  // group begins to read K tile j + 2 and V tile j + 1 in the phase after.  (One
  // group, NB = 3: for K tile j + 2 and V tile j + 1.)  MXFP8 (NB = 3): K tile
  // j + 3 and V tile j + 2 come into registers in M(j) and are written in V(j + 1).
  constexpr int kLoads = 2 * Feed::PER;                     // of a wave in a step
  constexpr bool PAIR = NW == 8;
  constexpr int kKept = (PAIR ? NB - 3 : NB - 2) * kLoads;  // of them on their way at a wait
  if (ntiles > 0) {
    turn_page(0);
    static_for<NB>([&](auto t) EFQ_INLINE {                 // (V of tile -1: no bytes)
      fetch(t, decltype(t)::value);
      land(t);
    });
    if constexpr (!F8) wait_vmem_le(kKept);
    wg_barrier();
    if (mine > 0) {
      static_for<NK>([&](auto n) EFQ_INLINE {
        constexpr int N = NV + decltype(n)::value;
        read_op(std::integral_constant<int, NB - 1>{}, std::integral_constant<int, N>{});
        product(std::integral_constant<int, N>{});
      });
    }
    phase_v(std::integral_constant<int, 0>{}, 0);
    wg_barrier();                                           // K tile 0 is read before its place is filled again
    const bool second = PAIR && wave >= NW / 2;
    if (second) wg_barrier();
    for (int j0 = 0; j0 < ntiles; j0 += NB)
      static_for<NB>([&](auto slot) EFQ_INLINE {
        constexpr int SLOT = decltype(slot)::value;
        const int j = j0 + SLOT;
        if (j < ntiles) {
          turn_page(j + NB);
          phase_m(slot, j);
          if constexpr (!F8) wait_vmem_le(kKept);
          wg_barrier();
          if (j + 1 < ntiles) phase_v(std::integral_constant<int, (SLOT + 1) % NB>{}, j + 1);
          land(slot);
          if constexpr (PAIR) wg_barrier();
        }
      });
    if (PAIR && !second) wg_barrier();
    if constexpr (!F8) wait_vmem();                         // nothing is on its way to LDS when it is given up
  }
  l = sum_of_halves(l);
  if (r >= s.rows) return;
  const long at = (long)tok * a.Hq + hq;
  if (ns == 1) {
    const float inv = l > 0.0f ? 1.0f / lr[0] : 0.0f;
    char* p = a.out + tok * a.o_token + hq * a.o_head;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 x = {o[i][4 * j] * inv, o[i][4 * j + 1] * inv, o[i][4 * j + 2] * inv, o[i][4 * j + 3] * inv};
        put4(p + (32 * i + 8 * j + 4 * half) * (a.out_f32 ? 4 : 2), a.out_f32, x);
      }
    if (half == 0 && a.lse) a.lse[at] = l > 0.0f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  } else {
    float* p = a.part_o + ((long)sp * a.rows + at) * D;
    const float weight = l > 0.0f ? l / lr[0] : 0.0f;      // to that of the unrounded sum
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(f32x4*)(p + 32 * i + 8 * j + 4 * half) =
            f32x4{o[i][4 * j] * weight, o[i][4 * j + 1] * weight, o[i][4 * j + 2] * weight, o[i][4 * j + 3] * weight};
    if (half == 0) a.part_ml[(long)sp * a.rows + at] = make_float2(m, l);
  }
}

template <int D, bool F8, int NW>
__global__ __launch_bounds__(64 * NW, NW == 4 && !F8 ? 3 : 2) void paged_chunk_kernel(PagedArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  const int h = blockIdx.x % a.Hkv;
  Slot s;
  // the last slots see the most keys: first
  if (!find_slot<32 * NW>(a, (int)(gridDim.x / a.Hkv) - 1 - (int)(blockIdx.x / a.Hkv), s)) return;
  chunk_rows<D, F8, NW>(a, s, h, (int)blockIdx.y, lds);
}

// W waves (1 or 4) per row that ran split: the parts, weighted to the common
// maximum, every W-th part by one wave, then the waves in order.  A short
// kernel is its chain of dependent loads, so the maxima are asked for before
// the sequence's length is known, and four parts' sums at a time.
template <int D>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs a, int W) {
  constexpr int C = D / 64;
  __shared__ float shared[4][C * 64 + 1];
  const int wave = uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const long at = W == 4 ? (long)blockIdx.x : (long)blockIdx.x * 4 + wave;
  if (at >= a.rows) return;                  // whole workgroups where waves share a row
  const float early = lane < a.nsplit ? a.part_ml[lane * a.rows + at].x : -INFINITY;
  const int tok = (int)(at / a.Hq), hq = (int)(at % a.Hq);
  int first, end;
  const int i = last_at_most(a.b, tok, [](int, int start) { return (long)start; }, first, end);
  if (i < 0 || tok >= end) return;
  const int ns = splits_of(a, a.b.keys(i));
  if (ns == 1) return;
  float M = lane < ns ? early : -INFINITY;
  for (int s = lane + 64; s < ns; s += 64) M = __builtin_fmaxf(M, a.part_ml[s * a.rows + at].x);
  M = max_of_groups(M);
#pragma unroll
  for (int w = 8; w > 0; w >>= 1) M = __builtin_fmaxf(M, __shfl_xor(M, w));
  const float ref = M == -INFINITY ? 0.0f : M;
  const int w0 = W == 4 ? wave : 0;
  float sum = 0.0f, x[C] = {};
  for (int s0 = w0; s0 < ns; s0 += 4 * W) {
    float e[4], v[4][C];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + u * W;
      const long from = min(s, ns - 1) * a.rows + at;
      const float2 z = a.part_ml[from];
      e[u] = s < ns ? __builtin_amdgcn_exp2f(z.x - ref) : 0.0f;     // 0 for a part that saw no key
      sum += e[u] * z.y;
#pragma unroll
      for (int c = 0; c < C; ++c) v[u][c] = a.part_o[from * D + C * lane + c];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int c = 0; c < C; ++c) x[c] = __builtin_fmaf(e[u], v[u][c], x[c]);
  }
  if (W == 4) {
#pragma unroll
    for (int c = 0; c < C; ++c) shared[wave][C * lane + c] = x[c];
    if (lane == 0) shared[wave][C * 64] = sum;
    __syncthreads();
    if (wave > 0) return;
    sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) x[c] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      sum += shared[w][C * 64];
#pragma unroll
      for (int c = 0; c < C; ++c) x[c] += shared[w][C * lane + c];
    }
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  char* out = a.out + tok * a.o_token + hq * a.o_head;
  if constexpr (C == 2) {
    if (a.out_f32) *(f32x2*)(out + 8 * lane) = f32x2{x[0] * inv, x[1] * inv};
    else *(unsigned*)(out + 4 * lane) = pack_bf16(x[0] * inv, x[1] * inv);
  } else {
    if (a.out_f32) *(float*)(out + 4 * lane) = x[0] * inv;
    else *(__bf16*)(out + 2 * lane) = (__bf16)(x[0] * inv);
  }
  if (lane == 0 && a.lse) a.lse[at] = sum > 0.0f ? (M + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

// ================================================================ host side
int check_rows(const efq_rows* r, const char* name, int es) {
  if (!r || !r->data) return fail(EFQ_EINVAL, "%s is NULL", name);
  if (!aligned16(r->data)) return fail(EFQ_EINVAL, "%s must be 16-byte aligned", name);
  const int64_t most = (int64_t)1 << 32;   // times 2^26 tokens and 4 bytes stays in 64 bits
  if (r->token < 0 || r->head < 0 || r->token > most || r->head > most)
    return fail(EFQ_EINVAL, "%s: strides must be in [0, 2^32]", name);
  if (r->token * es % 16 || r->head * es % 16)
    return fail(EFQ_EINVAL, "%s: strides must be multiples of 16 bytes", name);
  return EFQ_OK;
}
// Rows that are written: no two heads or tokens may lie on each other, and where
// they begin with those of `in` they are those, row for row.
int check_out_rows(const efq_rows* r, const char* name, int es, int tokens, int heads, int head_dim,
                   const efq_rows* in = nullptr) {
  const int rc = check_rows(r, name, es);
  if (rc) return rc;
  if ((heads > 1 && r->head < head_dim) || (tokens > 1 && r->token < head_dim) ||
      (heads > 1 && tokens > 1 && r->token < r->head * (heads - 1) + head_dim &&
       r->head < r->token * (tokens - 1) + head_dim))
    return fail(EFQ_EINVAL, "%s: rows overlap", name);
  if (in && in->data == r->data && ((tokens > 1 && in->token != r->token) || (heads > 1 && in->head != r->head)))
    return fail(EFQ_EINVAL, "%s: in place, but with other strides", name);
  return EFQ_OK;
}

int check_rotary(const efq_rotary* r, int head_dim) {
  if (!r->inv_freq || !r->pos) return fail(EFQ_EINVAL, "rotary: null pointer");
  if (r->axes < 1) return fail(EFQ_EINVAL, "rotary: axes must be >= 1");
  if (r->pairs < 1 || 2 * (int64_t)r->pairs > head_dim)
    return fail(EFQ_EINVAL, "rotary: %d pairs in a head of %d", r->pairs, head_dim);
  if (r->pairs % 8) return fail(EFQ_EUNSUPPORTED, "rotary: pairs must be a multiple of 8");
  return EFQ_OK;
}
RotArgs rot_args(const efq_rotary* r, int tokens) {
  return RotArgs{r->inv_freq, r->axis, r->pos, tokens, r->pairs, r->axes, r->interleaved != 0};
}

int check_cache(const efq_cache* c) {
  if (!c) return fail(EFQ_EINVAL, "cache is NULL");
  if (c->pages < 1 || c->heads_kv < 1) return fail(EFQ_EINVAL, "cache: pages and heads_kv must be >= 1");
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(EFQ_EUNSUPPORTED, "cache: head_dim %d unsupported (64 or 128)", c->head_dim);
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return fail(EFQ_EUNSUPPORTED, "cache: page_size %d unsupported (16, 32, 64, 128 or 256)", c->page_size);
  if (c->format != EFQ_CACHE_BF16 && c->format != EFQ_CACHE_MXFP8)
    return fail(EFQ_EINVAL, "cache: unknown format %d", c->format);
  if (!c->k || !c->v || (c->format == EFQ_CACHE_MXFP8 && (!c->k_scale || !c->v_scale)))
    return fail(EFQ_EINVAL, "cache: null pointer");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(EFQ_EINVAL, "cache: k and v must be 16-byte aligned");
  if (c->format == EFQ_CACHE_MXFP8 && (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3))
    return fail(EFQ_EINVAL, "cache: scales must be 4-byte aligned");
  return EFQ_OK;
}
int check_batch(const efq_batch* b) {
  if (!b) return fail(EFQ_EINVAL, "batch is NULL");
  if (b->seqs < 1 || b->table_width < 1 || b->tokens < 0 || b->max_q < 0 || b->max_k < 0)
    return fail(EFQ_EINVAL, "batch: seqs and table_width must be >= 1, the rest >= 0");
  if (b->seqs > (1 << 20) || b->tokens > kMostTokens)
    return fail(EFQ_EUNSUPPORTED, "batch: more than 2^20 sequences or 2^26 tokens");
  if (!b->q_start || !b->seq_k || !b->page_table) return fail(EFQ_EINVAL, "batch: null pointer");
  return EFQ_OK;
}
Batch batch_args(const efq_batch* b, const efq_cache* c) {
  return Batch{b->q_start, b->seq_k, b->page_table, b->seqs, b->tokens, b->table_width, c->pages,
               __builtin_ctz((unsigned)c->page_size)};
}

// Tokens of a workgroup (a power of two) and workgroups of a token in the kernels
// that walk over tokens: few tokens are spread over the chip a workgroup per 256
// threads' work, many share one workgroup as long as eight are left for a CU, and
// no more than `enough` work needs: short workgroups keep a CU's reads and writes
// mixed.  rope, enough 768 pieces of 16 bytes (an item of halves is two): 32760
// tokens of 768 pieces (fp32) at 1 / 2 / 4 / 8 tokens 139 / 149 / 156 / 163 us, 8192 of 640 (bf16)
// 30.7 / 30.6 / 32.2, 20000 of 128 23.8 / 19.2 / 16.8 / 18.0.  Append, whose pages hold
// a head's tokens side by side: 11400 tokens (32/8 heads, D 128) into MXFP8 pages at
// 1 / 2 / 4 / 8 tokens 71 / 64 / 61 / 65 us.  More tokens than a launch has workgroups
// for share them, up to kMostShared.
void token_grid(int tokens, int threads_per_token, int enough, int& tt, int& parts) {
  static_assert((kMostTokens + kMostShared - 1) / kMostShared <= kMostGroups, "the most tokens fit a launch");
  for (tt = 4; tt > 1 && (tokens < tt * 8 * kCUs || tt / 2 * threads_per_token >= enough); tt /= 2) {}
  while (((long)tokens + tt - 1) / tt > kMostGroups) tt *= 2;
  parts = tt > 1 || tokens > 4 * kCUs ? 1 : (threads_per_token + 255) / 256;
}

template <bool F32, bool INTERLEAVED>
hipError_t launch_rope(const RopeArgs& a, dim3 grid, int lds, bool stream_out, hipStream_t st) {
  if (stream_out) hipLaunchKernelGGL((rope_kernel<F32, INTERLEAVED, true>), grid, dim3(256), lds, st, a);
  else hipLaunchKernelGGL((rope_kernel<F32, INTERLEAVED, false>), grid, dim3(256), lds, st, a);
  return hipGetLastError();
}
template <int D, bool F8, bool MANY>
hipError_t launch_append(const AppendArgs& a, dim3 grid, int lds, hipStream_t st) {
  hipLaunchKernelGGL((kv_append_kernel<D, F8, MANY>), grid, dim3(256), lds, st, a);
  return hipGetLastError();
}

// How a call's rows are cut: the kernel, its rows per workgroup, and the
// splits over the keys with the scratch they take.
struct PagedPlan {
  int rt;              // 1, 2: step kernel with 16 rt rows; 0: chunk kernel
  int bm, nsplit, chunk;
  bool direct;         // a slot is a sequence
  long slots;
  size_t bytes;
};
PagedPlan paged_plan(const efq_cache* c, const efq_batch* b, int heads_q) {
  PagedPlan p;
  const int G = heads_q / c->heads_kv;
  const long most_q = b->max_q ? b->max_q : std::max<long>(1, (long)b->tokens - b->seqs + 1);
  const long rows = most_q * G;
  // The chunk kernel's waves share what they read, the step kernel's rows all
  // pass through every wave.  32 rows: 16 sequences x 8 tokens over 4000 keys
  // (32/8 heads, D 128, bf16) step 41 us, chunk 47; 64 rows: x 16 tokens 61 and
  // 49, MXFP8 43 and 49 (one sequence over 20000 keys 29 and 27); D 64, 16 tokens over
  // 20000 keys 17.0 and 18.2.
  const bool low = c->format == EFQ_CACHE_MXFP8, narrow = c->head_dim == 64;
  p.rt = rows <= 16 ? 1 : rows <= (low || narrow ? 64 : 32) ? 2 : 0;
  p.bm = p.rt ? 16 * p.rt : narrow ? 128 : 256;
  p.direct = p.rt && rows <= p.bm;
  p.slots = p.direct ? b->seqs : ((long)b->tokens * G + p.bm - 1) / p.bm + b->seqs - 1;
  const long keys = std::min({(long)b->table_width * c->page_size, (long)kMostKeys, b->max_k ? (long)b->max_k : (long)kMostKeys});
  long n = 1;
  if (p.rt) {
    // Splits of the longest sequence.  A CU reads no faster with two workgroups than
    // with one, and the whole chip's as fast as HBM gives, so what counts is that
    // each CU has as much as every other.  One workgroup for (nearly) every CU, where
    // the items come out so: one sequence of 131000 keys (32/8 heads, D 128, bf16) in
    // 16 / 32 / 64 / 256 pieces 130 / 84 / 88 / 98 us, 8 of 16000 in 2 / 4 / 8 / 16
    // 108 / 66 / 69 / 70, 3 of 30000 in 8 / 10 / 16 59 / 52 / 62, 8 x 5 tokens over 6000
    // in 2 / 4 / 8 47 / 32 / 36.  Single tokens over MXFP8 pages want two, one converts
    // while the other waits: 8 of 16000 in 4 / 8 / 16 47 / 43 / 44.  Else two, and pieces small
    // enough to end together, down to 448 KB of keys and values, which stream in about
    // ten times what it takes to start a workgroup, while the unsplit call has fewer
    // than eight rounds of workgroups (17 sequences of 5000 to 20000 keys in pieces
    // of 6700 / 2900 / 1540 / 830 keys: 164 / 171 / 145 / 138 us).  The join costs
    // a launch, so short sequences stay whole (one of 500 keys in one piece 8.3 us,
    // in two 12.9; 8 of 600 12.0 and 12.9, of 800 15.6 and in four 12.8; 8 tokens
    // over 600 keys 13.2 and 13.0, over 800 15.6 and 13.1; D 64, 1000 keys 8.2 and
    // 12.0), and pieces have 192 keys at least.
    const long items = std::max<long>(1, p.slots * c->heads_kv);
    const long key_bytes = 2 * (low ? c->head_dim + c->head_dim / 32 : 2 * c->head_dim);
    const long even = kCUs / items, idle = kCUs - even * items;
    if (b->seqs == 1) {
      n = (kCUs + items - 1) / items;
    } else if (!(low && p.rt == 1) && even >= 2 && idle <= (even >= 4 ? kCUs / 8 : 0)) {
      n = even;
    } else {
      n = std::max((2 * kCUs + items - 1) / items, std::min(keys * key_bytes / (448 << 10), 16 * kCUs / items));
    }
    n = keys < (narrow ? 1024 : p.rt == 2 ? 640 : 768) ? 1 : std::max<long>(1, std::min(n, keys / 192));
  } else {
    // As many pieces (of at least 256 keys) as leave the chip one round of
    // workgroups, by the average of the sequences' rows; rounded up where lengths
    // differ, since short sequences fill fewer.  64 tokens over 20000 keys (32/8
    // heads, D 128, bf16: 8 workgroups unsplit) in 8 / 16 / 32 pieces 67 / 48 / 45
    // us, 700 tokens over 20000 (88) in 1 / 2 / 3 / 4 pieces 394 / 251 / 329 / 275.
    const long items = b->seqs * (((long)b->tokens * G / b->seqs + p.bm - 1) / p.bm) * c->heads_kv;
    n = std::max<long>(1, std::min((kCUs + (b->seqs > 1 ? items / 2 : 0)) / std::max<long>(1, items), keys / 256));
  }
  p.chunk = (int)(((keys + n - 1) / n + 127) / 128 * 128);
  p.nsplit = (int)std::max<long>(1, (keys + p.chunk - 1) / p.chunk);
  p.bytes = p.nsplit == 1 ? 0 : round256((size_t)p.nsplit * b->tokens * heads_q * 8) +
                                    (size_t)p.nsplit * b->tokens * heads_q * c->head_dim * 4;
  if (p.bytes > ((size_t)512 << 20)) {
    p.bytes = 0;
    p.nsplit = 1;
  }
  if (p.nsplit == 1) p.chunk = 0x7fffff00;
  return p;
}

// More dynamic LDS than the default limit for one kernel, raised once per
// device (check_device has bounded the device index); ID tells kernels apart.
template <int ID>
hipError_t raise_lds_of(const void* kernel, int lds) {
  static std::once_flag once[kMaxDevices];
  static hipError_t set_err[kMaxDevices];
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  std::call_once(once[dev], [=]() {
    set_err[dev] = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  });
  return set_err[dev];
}

template <int D, bool F8, int RT>
hipError_t launch_step(const PagedArgs& a, dim3 grid, hipStream_t st) {
  constexpr int lds = StepLds<D, RT>::kTotal;
  const hipError_t e = raise_lds_of<(D * 2 + F8) * 8 + RT>((const void*)paged_step_kernel<D, F8, RT>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_step_kernel<D, F8, RT>), grid, dim3(64 * kStepWaves), lds, st, a);
  return hipGetLastError();
}
template <int D, bool F8, int NW>
hipError_t launch_chunk(const PagedArgs& a, dim3 grid, hipStream_t st) {
  constexpr int lds = ChunkLds<D, F8, NW>::kTotal;
  const hipError_t e = raise_lds_of<(D * 2 + F8) * 8>((const void*)paged_chunk_kernel<D, F8, NW>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_chunk_kernel<D, F8, NW>), grid, dim3(64 * NW), lds, st, a);
  return hipGetLastError();
}
template <int D, bool F8>
hipError_t launch_paged(const PagedArgs& a, const PagedPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)(p.slots * a.Hkv), (unsigned)a.nsplit);
  const hipError_t e = p.rt == 1 ? launch_step<D, F8, 1>(a, grid, st)
                     : p.rt == 2 ? launch_step<D, F8, 2>(a, grid, st)
                                 : launch_chunk<D, F8, D == 64 ? 4 : 8>(a, grid, st);
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int W = a.nsplit > 4 ? 4 : 1;
  hipLaunchKernelGGL(paged_merge_kernel<D>, dim3((unsigned)(W == 4 ? a.rows : (a.rows + 3) / 4)), dim3(256), 0, st, a, W);
  return hipGetLastError();
}

}  // namespace

// ================================================================== C ABI
extern "C" {

int efq_rope(const efq_rows* x, const efq_rows* y, int tokens, int heads, int head_dim, int dtype,
             const efq_rotary* rot, int inverse, efq_stream_t stream) {
  if (tokens < 0 || heads < 1 || head_dim < 1) return fail(EFQ_EINVAL, "tokens must be >= 0, heads and head_dim >= 1");
  if (head_dim % 16 || head_dim > 512)
    return fail(EFQ_EUNSUPPORTED, "head_dim %d unsupported (a multiple of 16 up to 512)", head_dim);
  if (heads > (1 << 16) || tokens > kMostTokens)
    return fail(EFQ_EUNSUPPORTED, "more than 2^16 heads or 2^26 tokens");
  if (dtype != EFQ_BF16 && dtype != EFQ_F32) return fail(EFQ_EINVAL, "unknown dtype %d", dtype);
  if (!rot) return fail(EFQ_EINVAL, "rotary is NULL");
  if (tokens == 0) return EFQ_OK;
  const int es = dtype == EFQ_F32 ? 4 : 2;
  int rc;
  if ((rc = check_rotary(rot, head_dim)) || (rc = check_rows(x, "x", es)) ||
      (rc = check_out_rows(y, "y", es, tokens, heads, head_dim, x)))
    return rc;
  if ((rc = check_device())) return rc;
  RopeArgs a;
  a.x = (const char*)x->data;
  a.y = (char*)y->data;
  a.x_token = x->token * es, a.x_head = x->head * es, a.y_token = y->token * es, a.y_head = y->head * es;
  a.tokens = tokens, a.heads = heads, a.chunks = head_dim * es / (rot->interleaved ? 16 : 32), a.inverse = inverse != 0;
  a.rot = rot_args(rot, tokens);
  int parts;
  token_grid(tokens, heads * a.chunks, rot->interleaved ? 768 : 384, a.tt, parts);
  const int step = 256 * parts, per = heads * a.chunks;
  a.dt = step / per, a.dh = step % per / a.chunks, a.dc = step % a.chunks;
  const dim3 grid((unsigned)(((long)tokens + a.tt - 1) / a.tt), (unsigned)parts);
  const int lds = a.tt * rot->pairs * (int)sizeof(float2);
  hipStream_t st = (hipStream_t)stream;
  const bool stream_out = (long)tokens * heads * head_dim * es > kLastLevel;
  hipError_t e;
  if (es == 4) e = rot->interleaved ? launch_rope<true, true>(a, grid, lds, stream_out, st) : launch_rope<true, false>(a, grid, lds, stream_out, st);
  else e = rot->interleaved ? launch_rope<false, true>(a, grid, lds, stream_out, st) : launch_rope<false, false>(a, grid, lds, stream_out, st);
  if (e != hipSuccess) return fail(EFQ_EHIP, "rope launch: %s", hipGetErrorString(e));
  return EFQ_OK;
}

int efq_kv_append(const efq_rows* k, const efq_rows* v, const efq_cache* cache, const efq_batch* batch,
                  const efq_rotary* rot, const efq_rows* q, int heads_q, const efq_rows* q_out,
                  efq_stream_t stream) {
  int rc;
  if ((rc = check_cache(cache)) || (rc = check_batch(batch))) return rc;
  const int D = cache->head_dim;
  if (q ? heads_q < 1 || heads_q > (1 << 16) : heads_q != 0)
    return fail(EFQ_EINVAL, "heads_q must be in [1, 65536] with q and 0 without");
  if (cache->heads_kv > (1 << 16)) return fail(EFQ_EUNSUPPORTED, "more than 65536 heads");
  if (batch->tokens == 0) return EFQ_OK;
  if ((rc = check_rows(k, "k", 2)) || (rc = check_rows(v, "v", 2))) return rc;
  if (rot && (rc = check_rotary(rot, D))) return rc;
  if (q && ((rc = check_rows(q, "q", 2)) || (rc = check_out_rows(q_out, "q_out", 2, batch->tokens, heads_q, D, q)))) return rc;
  if ((rc = check_device())) return rc;
  AppendArgs a;
  memset(&a, 0, sizeof a);
  a.k = (const char*)k->data, a.k_token = 2 * k->token, a.k_head = 2 * k->head;
  a.v = (const char*)v->data, a.v_token = 2 * v->token, a.v_head = 2 * v->head;
  if (q) {
    a.q = (const char*)q->data, a.q_token = 2 * q->token, a.q_head = 2 * q->head;
    a.qo = (char*)q_out->data, a.o_token = 2 * q_out->token, a.o_head = 2 * q_out->head;
  }
  a.kc = (char*)cache->k, a.vc = (char*)cache->v;
  a.ks = (uint8_t*)cache->k_scale, a.vs = (uint8_t*)cache->v_scale;
  a.b = batch_args(batch, cache);
  a.heads = cache->heads_kv, a.heads_q = heads_q;
  if (rot) a.rotate = 1, a.rot = rot_args(rot, batch->tokens);
  int parts;
  const int rows = 2 * a.heads + heads_q;
  token_grid(batch->tokens, rows * (D / 8), 1 << 30, a.tt, parts);
  a.log_tt = __builtin_ctz((unsigned)a.tt);
  const dim3 grid((unsigned)(((long)batch->tokens + a.tt - 1) / a.tt), (unsigned)parts);
  const int lds = rot ? a.tt * rot->pairs * (int)sizeof(float2) : 0;
  hipStream_t st = (hipStream_t)stream;
  const bool f8 = cache->format == EFQ_CACHE_MXFP8;
  hipError_t e;
  if (a.tt > 1) e = D == 128 ? (f8 ? launch_append<128, true, true>(a, grid, lds, st) : launch_append<128, false, true>(a, grid, lds, st))
                             : (f8 ? launch_append<64, true, true>(a, grid, lds, st) : launch_append<64, false, true>(a, grid, lds, st));
  else e = D == 128 ? (f8 ? launch_append<128, true, false>(a, grid, lds, st) : launch_append<128, false, false>(a, grid, lds, st))
                    : (f8 ? launch_append<64, true, false>(a, grid, lds, st) : launch_append<64, false, false>(a, grid, lds, st));
  if (e != hipSuccess) return fail(EFQ_EHIP, "append launch: %s", hipGetErrorString(e));
  return EFQ_OK;
}

static int check_paged(const efq_cache* cache, const efq_batch* batch, int heads_q) {
  int rc;
  if ((rc = check_cache(cache)) || (rc = check_batch(batch))) return rc;
  if (heads_q < 1 || heads_q > (1 << 16) || heads_q % cache->heads_kv)
    return fail(EFQ_EINVAL, "heads_q %d not a positive multiple of heads_kv %d (up to 65536)", heads_q, cache->heads_kv);
  const long G = heads_q / cache->heads_kv;
  if (((long)batch->tokens * G / 16 + batch->seqs) * cache->heads_kv >= (1L << 22) || (long)batch->tokens * heads_q >= (1L << 25))
    return fail(EFQ_EUNSUPPORTED, "batch: too many tokens for one call");
  return EFQ_OK;
}

size_t efq_attn_paged_workspace_bytes(const efq_cache* cache, const efq_batch* batch, int heads_q) {
  if (check_paged(cache, batch, heads_q) != EFQ_OK || batch->tokens == 0) return 0;
  return paged_plan(cache, batch, heads_q).bytes;
}

int efq_attn_paged(const efq_rows* q, int heads_q, const efq_cache* cache, const efq_batch* batch,
                   float scale, int causal, const efq_rows* out, int out_dtype, float* lse, void* ws,
                   size_t ws_bytes, efq_stream_t stream) {
  int rc;
  if ((rc = check_paged(cache, batch, heads_q)) || (rc = check_scale(scale))) return rc;
  if (out_dtype != EFQ_BF16 && out_dtype != EFQ_F32) return fail(EFQ_EINVAL, "unknown dtype %d", out_dtype);
  if (batch->tokens == 0) return EFQ_OK;
  const int D = cache->head_dim;
  if ((rc = check_rows(q, "q", 2)) ||
      (rc = check_out_rows(out, "out", out_dtype == EFQ_F32 ? 4 : 2, batch->tokens, heads_q, D, q)))
    return rc;
  if (out_dtype == EFQ_F32 && out->data == q->data) return fail(EFQ_EINVAL, "out: fp32 rows in the place of q's");
  if ((uintptr_t)lse & 3) return fail(EFQ_EINVAL, "lse must be 4-byte aligned");
  if (ws_bytes != 0 && !ws) return fail(EFQ_EWORKSPACE, "workspace is NULL");
  if (ws && !aligned16(ws)) return fail(EFQ_EINVAL, "workspace must be 16-byte aligned");
  if ((rc = check_device())) return rc;
  PagedPlan p = paged_plan(cache, batch, heads_q);
  PagedArgs a;
  const int es = out_dtype == EFQ_F32 ? 4 : 2;
  a.q = (const char*)q->data, a.q_token = 2 * q->token, a.q_head = 2 * q->head;
  a.out = (char*)out->data, a.o_token = es * out->token, a.o_head = es * out->head;
  a.lse = lse;
  a.kc = (const char*)cache->k, a.vc = (const char*)cache->v;
  a.ks = (const uint8_t*)cache->k_scale, a.vs = (const uint8_t*)cache->v_scale;
  a.b = batch_args(batch, cache);
  a.sl2 = scale * kInvLn2;
  a.Hq = heads_q, a.Hkv = cache->heads_kv, a.G = heads_q / cache->heads_kv;
  a.causal = causal != 0, a.out_f32 = out_dtype == EFQ_F32;
  a.rows = (long)batch->tokens * heads_q;
  if (ws_bytes < p.bytes) p.nsplit = 1, p.chunk = 0x7fffff00;
  a.nsplit = p.nsplit, a.chunk = p.chunk, a.direct = p.direct;
  a.part_ml = (float2*)ws;
  a.part_o = (float*)((uint8_t*)ws + round256((size_t)p.nsplit * a.rows * 8));
  hipStream_t st = (hipStream_t)stream;
  const bool f8 = cache->format == EFQ_CACHE_MXFP8;
  const hipError_t e = D == 128 ? (f8 ? launch_paged<128, true>(a, p, st) : launch_paged<128, false>(a, p, st))
                                : (f8 ? launch_paged<64, true>(a, p, st) : launch_paged<64, false>(a, p, st));
  if (e != hipSuccess) return fail(EFQ_EHIP, "paged attention launch: %s", hipGetErrorString(e));
  return EFQ_OK;
}

}  // extern "C"
