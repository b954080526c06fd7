// The gated delta rule, forward: chunk plan of packed sequences, the inverse of every
// chunk, the chain of states, the outputs.  See tnt_delta.h for the mathematics.
#include "tnt_delta.h"

namespace tnt {
namespace {

constexpr int AP = 68;  // floats a row of the 64x64 matrices in LDS (16-byte rows)

// ---------------------------------------------------------------------------------
// Packed sequences: seq_start [nseq + 1] on the device -> the first chunk slot of every
// sequence and the table of slots.  One workgroup, a thread a sequence: a scan of the chunk
// counts, then each thread writes its sequence's slots in turn.  A launch, and 64 ns a chunk of
// the longest sequence, whose chain takes over 1 us of each.  Starts are clamped into [0, L]
// and made non-decreasing, so that no list of starts leads outside the tensors.
// ---------------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void delta_plan_kernel(const int* start, int nseq, int L, int slots,
                                                          int* first, int4* table) {
  __shared__ int wsum[16], wmax[16];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int carry = 0, carry_max = 0;  // chunks so far; largest start so far
  // a sequence's clamped start: the running maximum of the starts up to it
  for (int base = 0; base < nseq; base += 1024) {
    const int i = base + tid;
    int s = i <= nseq ? min(max(start[min(i, nseq)], 0), L) : 0;
    int e = i < nseq ? min(max(start[i + 1], 0), L) : 0;
    int m = s;  // inclusive running maximum over the block
    for (int k = 1; k < 64; k <<= 1) {
      const int o = __shfl_up(m, k, 64);
      if (lane >= k) m = max(m, o);
    }
    if (lane == 63) wmax[w] = m;
    __syncthreads();
    int before = carry_max;
    for (int k = 0; k < w; ++k) before = max(before, wmax[k]);
    int all = carry_max;
    for (int k = 0; k < 16; ++k) all = max(all, wmax[k]);
    m = max(m, before);
    const int n = i < nseq ? max(0, e - m) : 0;
    const int c = (n + DC - 1) / DC;
    int x = c;
    for (int k = 1; k < 64; k <<= 1) {
      const int o = __shfl_up(x, k, 64);
      if (lane >= k) x += o;
    }
    if (lane == 63) wsum[w] = x;
    __syncthreads();
    int off = carry, total = carry;
    for (int k = 0; k < 16; ++k) {
      if (k < w) off += wsum[k];
      total += wsum[k];
    }
    if (i < nseq) {
      const int f = off + x - c;
      first[i] = f;
      for (int j = 0; j < c && f + j < slots; ++j)
        table[f + j] = int4{i, m + DC * j, min(DC, n - DC * j), 0};
    }
    carry = total;
    carry_max = all;
    __syncthreads();
  }
  if (tid == 0) first[nseq] = min(carry, slots);
}

// ---------------------------------------------------------------------------------
// Per chunk and head: the running sum of the log decays, and the inverse of the unit
// lower triangular I + kk diag(lr) (forward: columns scaled; backward: I + diag(lr) kk,
// whose transpose the adjoint needs).  The leading head of a group also writes the
// chunk's keys (backward: and queries) as MFMA fragments, rows and transposed, so that
// the chains load whole fragments, 16 bytes a lane.
//
// The inverse in fp32: the four diagonal 16x16 blocks by forward substitution (one wave,
// a group of 16 lanes a block, a lane a column), then two levels of
// [T1 0; -T2 A T1 T2] with fp32 MFMAs.  Substitution and block products stay accurate
// where keys repeat (powers of A, the series form, would grow like binomials).
// ---------------------------------------------------------------------------------
__device__ __forceinline__ f4 mma16_f32(const float* A, const f4& b, f4 acc, int q) {
  // A: the lane's row, 16 contraction elements; b: tile rows 4q + r
  const f4 x = *reinterpret_cast<const f4*>(A + 4 * q);
#pragma unroll
  for (int r = 0; r < 4; ++r) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[r], b[r], acc, 0, 0, 0);
  return acc;
}
__device__ __forceinline__ f4 tile_rows(const float* T, int row0, int col0, int q, int c) {
  f4 b;
#pragma unroll
  for (int r = 0; r < 4; ++r) b[r] = T[(row0 + 4 * q + r) * AP + col0 + c];
  return b;
}

template <typename E, int DK, bool BWD>
__global__ __launch_bounds__(256) void delta_prep_kernel(DeltaArgs a) {
  constexpr int NP = terms_of<E>(), KS = DK / 32, PK = DK + 8;
  __shared__ __attribute__((aligned(16))) E Kl[DC * PK];
  __shared__ __attribute__((aligned(16))) float Al[DC * AP], Tl[DC * AP];
  __shared__ float2 cl[DC];
  __shared__ float ll[DC];
  Chunk ch;
  const int slot = blockIdx.x / a.H, h = blockIdx.x - slot * a.H;
  if (!chunk_of(a, slot, ch)) return;
  const int hk = h / a.per, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int q = lane >> 4, c = lane & 15;
  typedef typename V4<E>::t v4;
  const E* kp = (const E*)a.k + ch.b * a.sk.b + hk * a.sk.h + ch.t0 * a.sk.l;
  for (int i = tid; i < DC * (DK / 4); i += 256) {
    const int row = i / (DK / 4), col = 4 * (i - row * (DK / 4));
    v4 x = zero_v4<E>();
    if (row < ch.n && col < a.d_k) x = *reinterpret_cast<const v4*>(kp + row * a.sk.l + col);
    *reinterpret_cast<v4*>(Kl + row * PK + col) = x;
  }
  for (int i = tid; i < DC * AP; i += 256) Tl[i] = 0.f;
  if (w == 0) {
    const int64_t t = ch.t0 + lane;
    const bool in = lane < ch.n;
    const float gr = in ? a.g[ch.b * a.sg.b + h * a.sg.h + t * a.sg.l] : 0.f;
    ll[lane] = in ? a.lr[ch.b * a.sl.b + h * a.sl.h + t * a.sl.l] : 0.f;
    double s = gr < DELTA_GMIN ? DELTA_GMIN : gr;
    for (int m = 1; m < 64; m <<= 1) {
      const double o = __shfl_up(s, m, 64);
      if (lane >= m) s += o;
    }
    float2 cc;
    cc.x = (float)s;
    cc.y = (float)(s - (double)cc.x);
    cl[lane] = cc;
    const size_t at = ((size_t)slot * a.H + h) * DC + lane;
    a.cum[at] = cc;
    float2 e;
    e.x = __shfl(cc.x, 63, 64);
    e.y = __shfl(cc.y, 63, 64);
    const float ec = exp_pair(cc), ee = exp_diff(e, cc), lr = ll[lane];
    if (lane == 0) a.ge[(size_t)slot * a.H + h] = exp_pair(e);
    if (BWD) {
      a.ec[at] = a.scale * ec;
      a.eu[at] = ee;
      a.el[at] = -ec * lr;
    } else {
      a.ec[at] = ec;
      a.eu[at] = ee * lr;
    }
  }
  __syncthreads();
  // kk, scaled: tile (w, j), j <= w
  {
    f4 acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = zero4();
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const Fr<NP> fa = row_frag<E>(Kl, (16 * w + c) * PK, 32 * s, q, DK);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j <= w) mma_terms(acc[j], fa, row_frag<E>(Kl, (16 * j + c) * PK, 32 * s, q, DK));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j <= w) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * w + 4 * q + r, col = 16 * j + c;
          float x = 0.f;
          const float d = acc[j][r] * exp_diff(cl[row], cl[col]) * ll[BWD ? row : col];
          if (row > col) x = d;
          Al[row * AP + col] = x;
        }
      }
  }
  // fragments of the keys and queries
  if (h == hk * a.per) {
    const size_t at = ((size_t)slot * a.Hk + hk) * DC * DK * NP;
    for (int f = w; f < 4 * KS; f += 4) {
      const int rt = f / KS, s = f - rt * KS;
      store_frag<NP>(a.KF + at + (size_t)f * 512 * NP, lane,
                     row_frag<E>(Kl, (16 * rt + c) * PK, 32 * s, q, DK));
    }
    for (int f = w; f < DK / 8; f += 4) {
      const int dt = f >> 1, s = f & 1;
      store_frag<NP>(a.KT + at + (size_t)f * 512 * NP, lane,
                     col_frag<E>(Kl + (32 * s + 4 * q) * PK + 16 * dt + c, PK));
    }
    if (BWD) {
      __syncthreads();  // every thread of the block takes this branch
      const E* qp = (const E*)a.q + ch.b * a.sq.b + hk * a.sq.h + ch.t0 * a.sq.l;
      for (int i = tid; i < DC * (DK / 4); i += 256) {
        const int row = i / (DK / 4), col = 4 * (i - row * (DK / 4));
        v4 x = zero_v4<E>();
        if (row < ch.n && col < a.d_k) x = *reinterpret_cast<const v4*>(qp + row * a.sq.l + col);
        *reinterpret_cast<v4*>(Kl + row * PK + col) = x;
      }
      __syncthreads();
      for (int f = w; f < DK / 8; f += 4) {
        const int dt = f >> 1, s = f & 1;
        store_frag<NP>(a.QT + at + (size_t)f * 512 * NP, lane,
                       col_frag<E>(Kl + (32 * s + 4 * q) * PK + 16 * dt + c, PK));
      }
    }
  }
  __syncthreads();
  if (w == 0) {  // diagonal blocks: block q, column c
    const float* Ab = Al + (16 * q) * AP + 16 * q;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = i == c ? 1.f : 0.f;
#pragma unroll
      for (int j = 0; j < i; ++j) s -= Ab[i * AP + j] * x[j];
      x[i] = s;
      Tl[(16 * q + i) * AP + 16 * q + c] = s;
    }
  }
  __syncthreads();
  if (w < 2) {  // blocks (1, 0) and (3, 2)
    const int i0 = 32 * w + 16, j0 = 32 * w;
    f4 y = mma16_f32(Al + (i0 + c) * AP + j0, tile_rows(Tl, j0, j0, q, c), zero4(), q);
    f4 z = mma16_f32(Tl + (i0 + c) * AP + i0, y, zero4(), q);
#pragma unroll
    for (int r = 0; r < 4; ++r) Tl[(i0 + 4 * q + r) * AP + j0 + c] = -z[r];
  }
  __syncthreads();
  if (w < 2) {  // rows 32..63, block column w
    f4 y[2];
#pragma unroll
    for (int bi = 0; bi < 2; ++bi) {
      y[bi] = zero4();
      for (int bk = w; bk < 2; ++bk)
        y[bi] = mma16_f32(Al + (32 + 16 * bi + c) * AP + 16 * bk, tile_rows(Tl, 16 * bk, 16 * w, q, c),
                          y[bi], q);
    }
#pragma unroll
    for (int bi = 0; bi < 2; ++bi) {
      f4 z = zero4();
#pragma unroll
      for (int bk = 0; bk <= bi; ++bk)
        z = mma16_f32(Tl + (32 + 16 * bi + c) * AP + 32 + 16 * bk, y[bk], z, q);
#pragma unroll
      for (int r = 0; r < 4; ++r) Tl[(32 + 16 * bi + 4 * q + r) * AP + 16 * w + c] = -z[r];
    }
  }
  __syncthreads();
  // fragments of T (rows i, steps ks <= i / 2) or of T^T (steps ks >= i / 2)
  __bf16* tf = a.TF + ((size_t)slot * a.H + h) * DELTA_TFRAG;
  for (int f = w; f < 6; f += 4) {
    if (!BWD) {
      const int i = f < 2 ? f : 2 + ((f - 2) >> 1), s = f < 2 ? 0 : (f & 1);
      const float* p = Tl + (16 * i + c) * AP + 32 * s + 4 * q;
      store_frag<3>(tf + f * 1536, lane, frag_of(*(const f4*)p, *(const f4*)(p + 16)));
    } else {
      const int i = f < 4 ? f >> 1 : f - 2, s = f < 4 ? (f & 1) : 1;
      store_frag<3>(tf + f * 1536, lane, col_frag<float>(Tl + (32 * s + 4 * q) * AP + 16 * i + c, AP));
    }
  }
}

// ---------------------------------------------------------------------------------
// The chain of states.  One workgroup walks the chunks of a (sequence, head) for 16
// columns of the values: the state's rows lie across its waves as fp32 tiles, for the whole
// sequence (four waves of one or two tiles; at dk 32 two of one).  Per chunk: partial K S of
// each wave's rows, summed through LDS; E and W = T E by row tiles; the update of each
// wave's rows.  Three barriers, on LDS alone; the next chunk's fragments are requested a
// chunk ahead, always (the last chunk requests itself again: were the request conditional,
// the waits for this chunk's fragments would have to assume it absent and so include it).
// 1.5 us a chunk at dk 64 (32 x 4 column tiles), 2.0 us at 128 (16 x 8), one workgroup a CU:
// at 128 a wave issues in 32 % of its cycles, waits for the issue of an instruction after
// another in 47 % and for LDS, barriers and memory in 20 %.  Two workgroups on a CU take 1.7
// times as long a chunk each (1408 column tiles of 23 chunks; 20, 62 and 18 %): the dependent
// instructions of a wave bound it, and two waves of a SIMD are in each other's way in issuing.
// The matrix units are at work in 6 % of a launch's cycles on half the CUs, 11 % on all.
// Rows past a chunk's end repeat its last token's values and write nothing (their lr is
// 0), columns past d_v the last column's: the backward's arrays are zero there.
// ---------------------------------------------------------------------------------
template <typename E, int DK> struct ChainLoad {
  static constexpr int NP = terms_of<E>(), NW = ChainShape<DK>::NW, RT = ChainShape<DK>::RT, SR = ChainShape<DK>::SR;
  typename StateOp<SR>::template A<NP> kf[4];
  Fr<NP> kt[SR][2];
  Fr<3> t[RT][2];
  E v[RT][4];  // as loaded: converted where it is used
  f4 ec[RT], eu[RT];
  float ge;
};

template <typename E, int DK>
__device__ __forceinline__ void chain_load(const DeltaArgs& a, ChainLoad<E, DK>& x, const Walk& k, int slot,
                                           int h, int w, int lane, int col) {
  typedef ChainLoad<E, DK> X;
  constexpr int NP = X::NP, KS = DK / 32;
  const int q = lane >> 4, past = (slot - k.s0) * DC;
  const size_t kat = ((size_t)slot * a.Hk + h / a.per) * DC * DK * NP;
  const size_t hat = (size_t)slot * a.H + h;
  const int n = min(DC, k.len - past);
#pragma unroll
  for (int rt = 0; rt < 4; ++rt) x.kf[rt] = StateOp<X::SR>::template load<NP>(a.KF + kat, rt, KS, w, lane);
#pragma unroll
  for (int t = 0; t < X::SR; ++t)
#pragma unroll
    for (int s = 0; s < 2; ++s)
      x.kt[t][s] = load_frag<NP>(a.KT + kat + (size_t)((X::SR * w + t) * 2 + s) * 512 * NP, lane);
  const __bf16* tf = a.TF + hat * DELTA_TFRAG;
  x.ge = a.ge[hat];
  const E* vb = (const E*)a.v + k.b * a.sv.b + h * a.sv.h + (int64_t)(k.t0 + past) * a.sv.l;
  const uint32_t vl = (uint32_t)a.sv.l, vc = (uint32_t)min(col, a.d_v - 1);
#pragma unroll
  for (int i = 0; i < X::RT; ++i) {
    const int rt = chain_tile<X::NW>(w, i);
    x.t[i][0] = load_frag<3>(tf + (rt < 2 ? rt : 2 * rt - 2) * 1536, lane);
    x.t[i][1] = load_frag<3>(tf + (rt < 2 ? rt : 2 * rt - 1) * 1536, lane);  // rt < 2: not used
    x.ec[i] = *reinterpret_cast<const f4*>(a.ec + hat * DC + 16 * rt + 4 * q);
    x.eu[i] = *reinterpret_cast<const f4*>(a.eu + hat * DC + 16 * rt + 4 * q);
#pragma unroll
    for (int r = 0; r < 4; ++r) x.v[i][r] = vb[(uint32_t)min(16 * rt + 4 * q + r, n - 1) * vl + vc];
  }
}

// where row tile t's four values of a column lie in a fragment array of 64 rows
__device__ __forceinline__ int half_at(int t, int lane) { return (t >> 1) * 1536 + lane * 8 + 4 * (t & 1); }

template <typename E, int DK, int PV>
__global__ __launch_bounds__(64 * ChainShape<DK>::NW, sizeof(E) == 2 && DK > 32 ? 2 : 1)
void delta_chain_kernel(DeltaArgs a) {
  typedef ChainLoad<E, DK> X;
  constexpr int NW = X::NW, RT = X::RT, SR = X::SR;
  __shared__ __attribute__((aligned(16))) f4 part[NW * 256];
  __shared__ __attribute__((aligned(16))) __bf16 Ep[3072], Up[3072];
  int seq, h, ct;
  if (!chain_unit(a, seq, h, ct)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id_uniform();
  const int q = lane >> 4, col = 16 * ct + (lane & 15);
  constexpr int pitch = PV;
  f4 S[SR];
#pragma unroll
  for (int t = 0; t < SR; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * (SR * w + t) + 4 * q + r;
      S[t][r] = a.S0 && row < a.d_k && col < a.d_v
                    ? a.S0[((size_t)seq * a.H + h) * a.d_k * a.d_v + row * a.d_v + col] : 0.f;
    }
  const Walk k = walk_of(a, seq);
  auto chunk = [&](X& cur, X& nxt, int slot) {
    chain_load<E, DK>(a, nxt, k, min(slot + 1, k.s1 - 1), h, w, lane, col);
    const size_t hat = (size_t)slot * a.H + h;
    float* sp = a.S + (hat * DK + 16 * SR * w) * pitch + (uint32_t)(4 * q * pitch + col);
#pragma unroll
    for (int t = 0; t < SR; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) sp[(uint32_t)((16 * t + r) * pitch)] = S[t][r];
    // K S
    const auto sf = StateOp<SR>::of(S);
    f4 ks[4] = {zero4(), zero4(), zero4(), zero4()};
    mma_terms_n(ks, cur.kf, sf);
#pragma unroll
    for (int rt = 0; rt < 4; ++rt) part[(w * 4 + rt) * 64 + lane] = ks[rt];
    lds_barrier();
    f4 x[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int rt = chain_tile<NW>(w, i);
      x[i] = part[rt * 64 + lane];
#pragma unroll
      for (int o = 1; o < NW; ++o) x[i] += part[(o * 4 + rt) * 64 + lane];
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int rt = chain_tile<NW>(w, i);
      float e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = to_f(cur.v[i][r]) - cur.ec[i][r] * x[i][r];
      split4_store(e, Ep + half_at(rt, lane));
    }
    lds_barrier();
    // W = T E, rows of this wave; U' = e^(c_64 - c) lr W
    tri_product_lds<NW>(x, cur.t, Ep, w, lane);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int rt = chain_tile<NW>(w, i);
      float u[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) u[r] = cur.eu[i][r] * x[i][r];
      split4_store(u, Up + half_at(rt, lane));
    }
    lds_barrier();
    const float ge = cur.ge;
    const Fr<3> u0 = load_frag<3>(Up, lane), u1 = load_frag<3>(Up + 1536, lane);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float* wp = a.W + (hat * DC + 16 * chain_tile<NW>(w, i)) * pitch + (uint32_t)(4 * q * pitch + col);
#pragma unroll
      for (int r = 0; r < 4; ++r) wp[(uint32_t)(r * pitch)] = x[i][r];
    }
    f4 up[SR];
    Fr<X::NP> k0[SR], k1[SR];
#pragma unroll
    for (int t = 0; t < SR; ++t) {
      up[t] = zero4();
      S[t] *= ge;
      k0[t] = cur.kt[t][0];
      k1[t] = cur.kt[t][1];
    }
    mma_terms_2(S, k0, u0, up, k1, u1);
#pragma unroll
    for (int t = 0; t < SR; ++t) S[t] += up[t];
  };
  X x0, x1;  // in turn, so that no fragment moves between registers
  if (k.s0 < k.s1) chain_load<E, DK>(a, x0, k, k.s0, h, w, lane, col);
  for (int slot = k.s0; slot < k.s1; slot += 2) {
    chunk(x0, x1, slot);
    if (slot + 1 < k.s1) chunk(x1, x0, slot + 1);
  }
  if (a.fin)
#pragma unroll
    for (int t = 0; t < SR; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * (SR * w + t) + 4 * q + r;
        if (row < a.d_k && col < a.d_v)
          a.fin[((size_t)seq * a.H + h) * a.d_k * a.d_v + row * a.d_v + col] = S[t][r];
      }
}

// ---------------------------------------------------------------------------------
// Outputs, every (chunk, head) at once: O = scale (e^c (Q S) + (D * Q K^T)(lr W)).
// Wave i forms the products of query tile i with the keys up to it as tiles of the
// transpose, which are the operand of the second product as they stand; the waves then
// share them through LDS, each taking its own columns of the values.
// ---------------------------------------------------------------------------------
template <typename E, int DK>
__global__ __launch_bounds__(256, 3) void delta_out_kernel(DeltaArgs a) {
  constexpr int NP = terms_of<E>(), KS = DK / 32;
  __shared__ __attribute__((aligned(16))) __bf16 Pl[4 * 2 * 1536], Ql[4 * KS * 512 * NP];
  __shared__ float2 cl[DC];
  __shared__ float ll[DC], el[DC];
  Chunk ch;
  const int slot = blockIdx.x / a.H, h = blockIdx.x - slot * a.H;
  if (!chunk_of(a, slot, ch)) return;
  const int hk = h / a.per, tid = threadIdx.x, lane = tid & 63, w = wave_id_uniform();
  const int q = lane >> 4, c = lane & 15, pitch = a.pitch;
  const size_t hat = (size_t)slot * a.H + h;
  const size_t kat = ((size_t)slot * a.Hk + hk) * DC * DK * NP;
  const E* qp = (const E*)a.q + ch.b * a.sq.b + hk * a.sq.h + (int64_t)ch.t0 * a.sq.l;
  // rows past the chunk's end repeat its last: their outputs are not written
  const uint32_t q_at = (uint32_t)min(16 * w + c, ch.n - 1) * (uint32_t)a.sq.l;
  Raw<E> qr[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qr[s] = row_raw<E>(qp, q_at, 32 * s, q, a.d_k);
  if (tid < DC) {
    const float2 cc = a.cum[hat * DC + tid];
    cl[tid] = cc;
    el[tid] = a.scale * a.ec[hat * DC + tid];
    ll[tid] = tid < ch.n ? a.lr[ch.b * a.sl.b + h * a.sl.h + (int64_t)(ch.t0 + tid) * a.sl.l] : 0.f;
  }
  f4 p[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = zero4();
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const Fr<NP> fq = raw_frag<E>(qr[s], 32 * s, q, a.d_k);
    store_frag<NP>(Ql + (w * KS + s) * 512 * NP, lane, fq);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j <= w) mma_terms(p[j], load_frag<NP>(a.KF + kat + (size_t)(j * KS + s) * 512 * NP, lane), fq);
  }
  lds_barrier();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float x[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int key = 16 * j + 4 * q + r, qry = 16 * w + c;
      const float d = a.scale * p[j][r] * exp_diff(cl[qry], cl[key]);
      x[r] = key <= qry ? d : 0.f;
    }
    split4_store(x, Pl + w * 3072 + (j >> 1) * 1536 + lane * 8 + 4 * (j & 1));
  }
  lds_barrier();
#pragma unroll 1
  for (int ct = w; ct < a.dvt; ct += 4) {
    const int col = 16 * ct + c;
    const float* sp = a.S + hat * DK * pitch + (uint32_t)(4 * q * pitch + col);
    const float* wp = a.W + hat * DC * pitch + (uint32_t)(4 * q * pitch + col);
    float sx[KS][8], wx[2][8];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) sx[s][j] = sp[(uint32_t)((32 * s + (j & 3) + 16 * (j >> 2)) * pitch)];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) wx[s][j] = wp[(uint32_t)((32 * s + (j & 3) + 16 * (j >> 2)) * pitch)];
    f4 acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = zero4();
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const Fr<3> fs = split8(sx[s]);
      Fr<NP> f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = load_frag<NP>(Ql + (i * KS + s) * 512 * NP, lane);
      mma_terms_n(acc, f, fs);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= *reinterpret_cast<const f4*>(el + 16 * i + 4 * q);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int j = 0; j < 8; ++j) wx[s][j] *= ll[32 * s + 4 * q + (j & 3) + 16 * (j >> 2)];
      const Fr<3> fu = split8(wx[s]);
#pragma unroll
      for (int i = 2 * s; i < 4; ++i) mma_terms(acc[i], load_frag<3>(Pl + i * 3072 + s * 1536, lane), fu);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (col < a.d_v) {
      E* op = (E*)a.o + ch.b * a.so.b + h * a.so.h + (int64_t)ch.t0 * a.so.l;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * i + 4 * q + r;
          if (row < ch.n) op[(uint32_t)row * (uint32_t)a.so.l + (uint32_t)col] = from_f<E>(acc[i][r]);
        }
    }
  }
}

template <typename F> hipError_t by_size(const DeltaArgs& a, bool bf16, F&& f) {
  if (bf16) {
    if (a.DK == 32) f((__bf16)0.f, std::integral_constant<int, 32>());
    else if (a.DK == 64) f((__bf16)0.f, std::integral_constant<int, 64>());
    else f((__bf16)0.f, std::integral_constant<int, 128>());
  } else {
    if (a.DK == 32) f(0.f, std::integral_constant<int, 32>());
    else if (a.DK == 64) f(0.f, std::integral_constant<int, 64>());
    else f(0.f, std::integral_constant<int, 128>());
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_plan(const DeltaArgs& a, hipStream_t st) {
  delta_plan_kernel<<<1, 1024, 0, st>>>(a.seq_start, a.nseq, a.L, a.slots, a.first, a.table);
  return hipGetLastError();
}

hipError_t launch_delta_prep(const DeltaArgs& a, bool bf16, bool bwd, hipStream_t st) {
  return by_size(a, bf16, [&](auto e, auto n) {
    typedef decltype(e) E;
    constexpr int DK = decltype(n)::value;
    if (bwd) delta_prep_kernel<E, DK, true><<<a.slots * a.H, 256, 0, st>>>(a);
    else delta_prep_kernel<E, DK, false><<<a.slots * a.H, 256, 0, st>>>(a);
  });
}

hipError_t launch_delta_chain(const DeltaArgs& a, bool bf16, hipStream_t st) {
  const int blocks = (a.nseq * a.H + 7) / 8 * 8 * a.dvt;
  return by_size(a, bf16, [&](auto e, auto n) {
    typedef decltype(e) E;
    constexpr int DK = decltype(n)::value;
    if (a.pitch == 32) delta_chain_kernel<E, DK, 32><<<blocks, 64 * ChainShape<DK>::NW, 0, st>>>(a);
    else if (a.pitch == 64) delta_chain_kernel<E, DK, 64><<<blocks, 64 * ChainShape<DK>::NW, 0, st>>>(a);
    else delta_chain_kernel<E, DK, 128><<<blocks, 64 * ChainShape<DK>::NW, 0, st>>>(a);
  });
}

hipError_t launch_delta_out(const DeltaArgs& a, bool bf16, hipStream_t st) {
  return by_size(a, bf16, [&](auto e, auto n) {
    delta_out_kernel<decltype(e), decltype(n)::value><<<a.slots * a.H, 256, 0, st>>>(a);
  });
}

}  // namespace tnt
