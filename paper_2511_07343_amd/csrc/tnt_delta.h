// The gated delta rule (linear test-time memory): argument block, launchers and
// the device helpers that its kernels share.  Internal to the library.
//
// Per (sequence, head), with the state S [dk][dv], c the running sum of the log
// decays g inside a chunk of 64 tokens and D[i][j] = e^(c_i - c_j) for i >= j:
//     kk = strict lower part of D * (K K^T)
//     E  = V - e^c (K S)                       what the entering state gets wrong
//     W  = (I + kk diag(lr))^-1 E              every token's own error
//     O  = scale (e^c (Q S) + (D * Q K^T) (lr W))
//     S' = e^(c_64) S + K^T (e^(c_64 - c) lr W)
// Every exponent is a difference of a later and an earlier sum, so nothing
// overflows however strong the decay (g > 0 grows the state as the recurrence does).  Log decays are clamped at -80.
//
// Precision.  States, gate gradients and everything on the way to them are
// fp32, and are to be as exact as fp32 sums: an fp32 operand of an MFMA product
// is split into three bf16 terms (8 + 8 + 8 bits, exactly), a bf16 input is one exact
// term, and a product is the sum of the term products down to 2^-24 (3 MFMAs
// with one bf16 input, 6 without).  That is 16/3 (16/6) of the rate of the fp32
// MFMA.  One bf16 term would round every entry of a state by up to 2^-8 at every
// chunk; measured with three, in the 2-norm: states 5e-8 to 1.3e-7 off, fp32 outputs and
// gradients 1.2e-7 to 2.5e-7, dg 3.5e-7 to 6.3e-7 (a loop in fp32: 1e-7 to 4e-7).
#pragma once

#include "tnt_regtile.h"

namespace tnt {

constexpr int DC = 64;              // tokens a chunk
constexpr float DELTA_GMIN = -80.f;  // log decays below act as this

struct Str { int64_t b, h, l; };  // element strides of [B][heads][L](..)

struct DeltaArgs {
  const void *q, *k, *v, *dO;
  const float *g, *lr, *S0, *dfin;
  void *o, *dq, *dk, *dv;
  float *fin, *dg, *dlr, *dS0;
  Str sq, sk, sv, so, sg, sl, sdO, sdq, sdk, sdv, sdg, sdl;
  int B, H, Hk, per, L, d_k, d_v;  // per = H / Hk
  int DK, dvt;                     // padded key size; 16-column tiles of the values
  int pitch;                       // floats a row of the values' arrays: 32, 64 or 128
  int nseq;                        // sequences
  int nc;                          // chunks a row (not packed)
  int slots;                       // chunk slots (packed: an upper bound)
  const int* seq_start;            // packed: [nseq + 1], else null
  float scale;
  // workspace
  int* first;    // packed: first slot of every sequence [nseq + 1]
  int4* table;   // packed: (sequence, first token, tokens, -) of every slot
  float2* cum;   // [slots][H][64]  c as a pair of floats
  // [slots][H][64] each.  Forward: e^c, e^(c_64 - c) lr; backward, in the same place:
  // scale e^c, e^(c_64 - c) and -e^c lr
  float *ec, *eu, *el;
  float* ge;     // [slots][H]  e^(c_64)
  __bf16* KF;    // [slots][Hk] fragments of K (rows: tokens)
  __bf16* KT;    // [slots][Hk] fragments of K^T (rows: dk)
  __bf16* QT;    // [slots][Hk] fragments of Q^T, backward
  __bf16* TF;    // [slots][H] fragments of the inverse, three terms
  float* W;      // [slots][H][64][pitch]
  float* S;      // [slots][H][DK][pitch]  states entering every chunk
  float* dS;     // [slots][H][DK][pitch]  adjoints of the states leaving every chunk
  float* dU;     // [slots][H][64][pitch]  P^T dO
  float* dR;     // [slots][H][64][pitch]
};

struct DeltaStepArgs {
  const void *q, *k, *v;
  const float *g, *lr;
  const int* slot;
  float* state;
  void* o;
  Str sq, sk, sv, so, sg, sl;
  int B, H, per, T, d_k, d_v, nslots;
  float scale;
};

hipError_t launch_delta_plan(const DeltaArgs& a, hipStream_t st);
hipError_t launch_delta_prep(const DeltaArgs& a, bool bf16, bool bwd, hipStream_t st);
hipError_t launch_delta_chain(const DeltaArgs& a, bool bf16, hipStream_t st);
hipError_t launch_delta_out(const DeltaArgs& a, bool bf16, hipStream_t st);
hipError_t launch_delta_dlocal(const DeltaArgs& a, bool bf16, hipStream_t st);
hipError_t launch_delta_bchain(const DeltaArgs& a, bool bf16, hipStream_t st);
hipError_t launch_delta_grads(const DeltaArgs& a, bool bf16, hipStream_t st);
hipError_t launch_delta_step(const DeltaStepArgs& a, bool bf16, hipStream_t st);

// bf16 elements of the fragments of one chunk: K or Q (either way round), the inverse
inline size_t delta_kfrag(int DK, bool bf16) { return (size_t)DC * DK * (bf16 ? 1 : 3); }
constexpr size_t DELTA_TFRAG = 6 * 3 * 512;

#ifdef __HIPCC__
// An operand of the 16x16x32 MFMA as a sum of NP bf16 terms.
template <int NP> struct Fr { bf16x8 p[NP]; };
template <typename E> constexpr int terms_of() { return sizeof(E) == 2 ? 1 : 3; }

// fp32 = h + m + l, exactly: the value rounded to 8 bits, the next 8 bits of the rest by a mask,
// and what is left.  The rest has either sign, so the products that are left out, m l and
// smaller, have too: below 2^-24 each, they cancel over a sum.  (h by a mask as well leaves
// them all the product's sign, -0.7 2^-24 of a sum of positive terms.  The training call of
// 16 heads of 32768 tokens at dk 128 takes 4.78 ms so and 4.88 here; shorter ones and smaller
// heads are within 1 %.)  Past 3.39e38 h is infinite.
// The upper halves of two words, a's below b's:
__device__ __forceinline__ uint32_t upper2(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float upper(float a) { return __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
template <int N> __device__ __forceinline__ void split_n(const float (&x)[N], uint32_t (&t)[3][N / 2]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{x[j], x[j + 1]}), b2));
    const float r0 = x[j] - __uint_as_float(h << 16), r1 = x[j + 1] - __uint_as_float(h & 0xffff0000u);
    t[0][j / 2] = h;
    t[1][j / 2] = upper2(r0, r1);
    t[2][j / 2] = upper2(r0 - upper(r0), r1 - upper(r1));
  }
}
__device__ __forceinline__ Fr<3> split8(const float (&x)[8]) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  uint32_t t[3][4];
  split_n(x, t);
  Fr<3> f;
#pragma unroll
  for (int p = 0; p < 3; ++p) f.p[p] = __builtin_bit_cast(bf16x8, (u4{t[p][0], t[p][1], t[p][2], t[p][3]}));
  return f;
}
// four values of a tile (rows 4q..4q+3 of a column) into the three planes of a
// fragment array at `dst` (elements; planes 512 apart)
__device__ __forceinline__ void terms4_store(const uint32_t (&t)[3][2], __bf16* dst) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int p = 0; p < 3; ++p) *reinterpret_cast<u2*>(dst + 512 * p) = u2{t[p][0], t[p][1]};
}
__device__ __forceinline__ void split4_store(const float (&x)[4], __bf16* dst) {
  uint32_t t[3][2];
  split_n(x, t);
  terms4_store(t, dst);
}
// the r-th of them by itself
__device__ __forceinline__ void terms4_put(const uint32_t (&t)[3][2], int r, __bf16* dst) {
#pragma unroll
  for (int p = 0; p < 3; ++p) reinterpret_cast<uint16_t*>(dst)[512 * p] = (uint16_t)(t[p][r >> 1] >> (16 * (r & 1)));
}

// acc += A B, terms down to 2^-24 of the product, the smallest first
template <int NA, int NB>
__device__ __forceinline__ void mma_terms(f4& acc, const Fr<NA>& a, const Fr<NB>& b) {
#pragma unroll
  for (int s = (NA > 1 || NB > 1) ? 2 : 0; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (i + j == s) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[j], acc, 0, 0, 0);
}

// The same for N independent accumulators, each term of all of them before the next: a
// product waits for the one before it on its own accumulator only every N.
template <int N, int NA, int NB>
__device__ __forceinline__ void mma_terms_n(f4 (&acc)[N], const Fr<NA> (&a)[N], const Fr<NB>& b) {
#pragma unroll
  for (int s = (NA > 1 || NB > 1) ? 2 : 0; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (i + j == s)
#pragma unroll
          for (int n = 0; n < N; ++n)
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[n].p[i], b.p[j], acc[n], 0, 0, 0);
}

// Operands over 16 contraction indices (4q + (0..3)): one accumulator tile as it stands.
template <int NP> struct Hf { bf16x4 p[NP]; };
__device__ __forceinline__ f4 mma16(const bf16x4& a, const bf16x4& b, const f4& c) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s4, a), __builtin_bit_cast(s4, b), c, 0, 0, 0);
}
template <int N, int NA, int NB>
__device__ __forceinline__ void mma_terms_n(f4 (&acc)[N], const Hf<NA> (&a)[N], const Hf<NB>& b) {
#pragma unroll
  for (int s = (NA > 1 || NB > 1) ? 2 : 0; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (i + j == s)
#pragma unroll
          for (int n = 0; n < N; ++n) acc[n] = mma16(a[n].p[i], b.p[j], acc[n]);
}
// one or two state tiles of a wave as the operand over their rows
template <int SR> struct StateOp;
template <> struct StateOp<2> {
  template <int NP> using A = Fr<NP>;
  __device__ __forceinline__ static Fr<3> of(const f4 (&S)[2]) {
    const float x[8] = {S[0][0], S[0][1], S[0][2], S[0][3], S[1][0], S[1][1], S[1][2], S[1][3]};
    return split8(x);
  }
  // the fragment of row tile rt over the wave's rows; KS steps of 32 a row
  template <int NP> __device__ __forceinline__ static Fr<NP> load(const __bf16* F, int rt, int KS, int w, int lane) {
    Fr<NP> f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
      f.p[i] = *reinterpret_cast<const bf16x8*>(F + (size_t)(rt * KS + w) * 512 * NP + 512 * i + 8 * lane);
    return f;
  }
};
template <> struct StateOp<1> {
  template <int NP> using A = Hf<NP>;
  __device__ __forceinline__ static Hf<3> of(const f4 (&S)[1]) {
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    const float x[4] = {S[0][0], S[0][1], S[0][2], S[0][3]};
    uint32_t t[3][2];
    split_n(x, t);
    Hf<3> f;
#pragma unroll
    for (int p = 0; p < 3; ++p) f.p[p] = __builtin_bit_cast(bf16x4, (u2{t[p][0], t[p][1]}));
    return f;
  }
  template <int NP> __device__ __forceinline__ static Hf<NP> load(const __bf16* F, int rt, int KS, int w, int lane) {
    Hf<NP> f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
      f.p[i] = *reinterpret_cast<const bf16x4*>(F + (size_t)(rt * KS + (w >> 1)) * 512 * NP + 512 * i + 8 * lane +
                                                4 * (w & 1));
    return f;
  }
};
// waves of a chain, state tiles and token row tiles of each
template <int DK> struct ChainShape {
  static constexpr int NW = DK == 32 ? 2 : 4, SR = DK == 128 ? 2 : 1, RT = 4 / NW;
};

// two such sets with operands of their own
template <int N, int NA, int NB>
__device__ __forceinline__ void mma_terms_2(f4 (&acc)[N], const Fr<NA> (&a)[N], const Fr<NB>& b, f4 (&acc2)[N],
                                            const Fr<NA> (&a2)[N], const Fr<NB>& b2) {
#pragma unroll
  for (int s = (NA > 1 || NB > 1) ? 2 : 0; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if (i + j == s)
#pragma unroll
          for (int n = 0; n < N; ++n) {
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[n].p[i], b.p[j], acc[n], 0, 0, 0);
            acc2[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a2[n].p[i], b2.p[j], acc2[n], 0, 0, 0);
          }
}

// Contraction indices of a lane's 8 elements in a step of 32: k0 + 4q + (0..3) and
// k0 + 16 + 4q + (0..3), q = lane / 16: the order in which two stacked accumulator
// tiles hold their rows, so that tiles serve as operands without a move.
__device__ __forceinline__ Fr<1> frag_of(const bf16x4& a, const bf16x4& b) {
  Fr<1> f;
  f.p[0] = join(a, b);
  return f;
}
__device__ __forceinline__ Fr<3> frag_of(const f4& a, const f4& b) {
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return split8(x);
}
template <typename E> struct V4;
template <> struct V4<__bf16> { typedef bf16x4 t; };
template <> struct V4<float> { typedef f4 t; };
template <typename E> __device__ __forceinline__ typename V4<E>::t zero_v4() {
  typename V4<E>::t z;
  z[0] = z[1] = z[2] = z[3] = (E)0.f;
  return z;
}
// elements k0 + 4q.. and k0 + 16 + 4q.. of a row of `d` (a multiple of 8) elements, zero
// past it.  The loads are not conditional (a lane past the end reads the row's last
// elements): a load under a branch is waited for where the branch joins.
template <typename E> struct Raw { typename V4<E>::t x, y; };
template <typename E>
__device__ __forceinline__ Raw<E> row_raw(const E* base, uint32_t row_at, int k0, int q, int d) {
  Raw<E> r;
  const int ka = k0 + 4 * q;
  r.x = *reinterpret_cast<const typename V4<E>::t*>(base + (row_at + (uint32_t)min(ka, d - 4)));
  r.y = *reinterpret_cast<const typename V4<E>::t*>(base + (row_at + (uint32_t)min(ka + 16, d - 4)));
  return r;
}
template <typename E>
__device__ __forceinline__ Fr<terms_of<E>()> raw_frag(Raw<E> r, int k0, int q, int d) {
  const int ka = k0 + 4 * q;
  const typename V4<E>::t z = zero_v4<E>();
  return frag_of(ka < d ? r.x : z, ka + 16 < d ? r.y : z);
}
template <typename E>
__device__ __forceinline__ Fr<terms_of<E>()> row_frag(const E* base, uint32_t row_at, int k0, int q, int d) {
  return raw_frag<E>(row_raw<E>(base, row_at, k0, q, d), k0, q, d);
}
template <int NP>
__device__ __forceinline__ Fr<NP> load_frag(const __bf16* p, int lane) {
  Fr<NP> f;
#pragma unroll
  for (int i = 0; i < NP; ++i) f.p[i] = *reinterpret_cast<const bf16x8*>(p + 512 * i + 8 * lane);
  return f;
}
template <int NP>
__device__ __forceinline__ void store_frag(__bf16* p, int lane, const Fr<NP>& f) {
#pragma unroll
  for (int i = 0; i < NP; ++i) *reinterpret_cast<bf16x8*>(p + 512 * i + 8 * lane) = f.p[i];
}
// A load at a byte offset from a wave-uniform base: one offset register a lane.
template <typename T> __device__ __forceinline__ T load_at(const void* base, uint32_t bytes) {
  return *reinterpret_cast<const T*>((const char*)base + bytes);
}
// 8 elements `step` apart in LDS (a column of a staged tile), as a fragment
template <typename E>
__device__ __forceinline__ Fr<terms_of<E>()> col_frag(const E* p, int step) {
  typename V4<E>::t x, y;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = p[j * step];
    y[j] = p[(16 + j) * step];
  }
  return frag_of(x, y);
}

// One chunk: its sequence, first token (in its batch row), tokens; false: an unused slot.
struct Chunk { int seq, b, t0, n; };
__device__ __forceinline__ bool chunk_of(const DeltaArgs& a, int slot, Chunk& c) {
  if (a.seq_start) {
    if (slot >= a.first[a.nseq]) return false;
    const int4 t = a.table[slot];
    c.seq = t.x; c.b = 0; c.t0 = t.y; c.n = t.z;
  } else {
    c.seq = c.b = slot / a.nc;
    c.t0 = (slot - c.b * a.nc) * DC;
    c.n = min(DC, a.L - c.t0);
  }
  return true;
}
// slots [s0, s1) of a sequence
__device__ __forceinline__ void slots_of(const DeltaArgs& a, int seq, int& s0, int& s1) {
  if (a.seq_start) {
    s0 = a.first[seq];
    s1 = a.first[seq + 1];
  } else {
    s0 = seq * a.nc;
    s1 = s0 + a.nc;
  }
}

// A sequence's chunks: slots [s0, s1), first token in batch row b, tokens.
struct Walk { int s0, s1, b, t0, len; };
__device__ __forceinline__ Walk walk_of(const DeltaArgs& a, int seq) {
  Walk k;
  slots_of(a, seq, k.s0, k.s1);
  k.b = a.seq_start ? 0 : seq;
  k.t0 = 0;
  k.len = a.L;
  if (a.seq_start && k.s0 < k.s1) {
    const int4 f = a.table[k.s0], l = a.table[k.s1 - 1];
    k.t0 = f.y;
    k.len = l.y + l.z - f.y;
  }
  return k;
}

// (sequence, head) unit and 16-column tile of a chain's workgroup.  Consecutive block
// numbers go to consecutive XCDs: the tiles of a unit, which read the same keys and the
// same triangular factors, are given numbers that agree modulo 8.  false: nothing to do.
__device__ __forceinline__ bool chain_unit(const DeltaArgs& a, int& seq, int& h, int& ct) {
  const unsigned x = blockIdx.x & 7, y = blockIdx.x >> 3;
  ct = y % a.dvt;
  const int u = (y / a.dvt) * 8 + x;
  seq = u / a.H;
  h = u - seq * a.H;
  return seq < a.nseq;
}

// Row tiles of the 64 tokens that wave w of the forward's chain takes between the chains' two
// contractions.  Tiles 0, 1 of a lower triangular factor have one step of 32, tiles 2, 3
// two; two waves take one of each.
template <int NW> __device__ __forceinline__ int chain_tile(int w, int i) {
  return NW == 4 ? w : i ? 3 - w : w;
}

// T's rows of one wave (RT tiles) times the chunk's 64 rows in LDS planes: chains of three
// products, in turn; tiles 0, 1 take step 0 alone.
template <int NW>
__device__ __forceinline__ void tri_product_lds(f4 (&x)[4 / NW], const Fr<3> (&t)[4 / NW][2], const __bf16* planes,
                                            int w, int lane) {
  constexpr int RT = 4 / NW;
  const Fr<3> b[2] = {load_frag<3>(planes, lane), load_frag<3>(planes + 1536, lane)};
  f4 lo[RT][2], hi[RT][2];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int s = 0; s < 2; ++s) lo[i][s] = hi[i][s] = f4{0.f, 0.f, 0.f, 0.f};
  auto need = [&](int i, int s) {
    const int rt = chain_tile<NW>(w, i);
    return s == 0 || rt >= 2;
  };
  constexpr int TI[6] = {2, 1, 0, 1, 0, 0}, TJ[6] = {0, 1, 2, 0, 1, 0};
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (need(i, s)) {
          lo[i][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i][s].p[TI[k]], b[s].p[TJ[k]], lo[i][s], 0, 0, 0);
          hi[i][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i][s].p[TI[3 + k]], b[s].p[TJ[3 + k]], hi[i][s], 0, 0, 0);
        }
#pragma unroll
  for (int i = 0; i < RT; ++i) x[i] = (lo[i][0] + lo[i][1]) + (hi[i][0] + hi[i][1]);
}

// X = F^T Y for a lower triangular F [64][64] (the six fragments of F^T that are not zero:
// tiles 0, 1 over both steps, tiles 2, 3 over step 1) and Y's 64 rows of a column tile in
// registers: six chains of six products, in turn.
__device__ __forceinline__ void tri_product_t(f4 (&x)[4], const Fr<3> (&t)[6], const Fr<3> (&y)[2]) {
  constexpr int TI[6] = {2, 1, 0, 1, 0, 0}, TJ[6] = {0, 1, 2, 0, 1, 0};
  f4 p[6];
#pragma unroll
  for (int f = 0; f < 6; ++f) p[f] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 6; ++k)
#pragma unroll
    for (int f = 0; f < 6; ++f) {
      const int s = f < 4 ? f & 1 : 1;
      p[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[f].p[TI[k]], y[s].p[TJ[k]], p[f], 0, 0, 0);
    }
  x[0] = p[0] + p[1];
  x[1] = p[2] + p[3];
  x[2] = p[4];
  x[3] = p[5];
}

// Column `col` of a chunk's 64 rows as the lane's accumulator tiles hold them (row
// 16 t + 4q + r in element 4 t + r); rows past the n there are repeat the last.
template <typename E>
__device__ __forceinline__ void load_column(E (&x)[16], const E* p, uint32_t l, int col, int n, int q) {
  if (n == DC) {  // rows at uniform distances: scalar addresses and one offset a lane
    const uint32_t at = (uint32_t)(4 * q) * l + (uint32_t)col;
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = (p + (size_t)(16 * (e >> 2) + (e & 3)) * l)[at];
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = p[(uint32_t)min(16 * (e >> 2) + 4 * q + (e & 3), n - 1) * l + (uint32_t)col];
  }
}

// A block barrier that orders LDS alone: loads and stores of global memory stay in
// flight across it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// e^(x + y) of a difference of two such pairs.  Where a lies before b it may be infinite:
// such places are masked by a choice, never by a factor of zero.
__device__ __forceinline__ float exp_diff(const float2& a, const float2& b) {
  return expf((a.x - b.x) + (a.y - b.y));
}
__device__ __forceinline__ float exp_pair(const float2& a) { return expf(a.x + a.y); }

// sum over the 16 lanes of a row group / over the four row groups
__device__ __forceinline__ float sum16(float x) {
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) x += __shfl_xor(x, m, 64);
  return x;
}
__device__ __forceinline__ float sum_groups(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
#endif
}  // namespace tnt
