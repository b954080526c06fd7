// The gated delta rule, backward.  With U = lr W, T = (I + diag(lr) kk)^-1 and the
// adjoint dS of the state leaving the chunk:
//     dU  = (scale D * Q K^T)^T dO + e^(c_64 - c) (K dS)
//     dR  = T^T dU                                   dV = lr dR
//     dS <- e^(c_64) dS + scale (e^c Q)^T dO - (lr e^c K)^T dR
//     dqk = scale D * lower(dO U^T),  M = -lr D * strict(dR U^T)
//     dQ  = scale e^c (dO S^T) + dqk K
//     dK  = e^(c_64 - c) (U dS^T) - lr e^c (dR S^T) + dqk^T Q + (M + M^T) K
//     dlr = rows of dR * W
// and, since c enters every product it scales as a factor of that product's own
// gradient, the adjoint of c_t needs no products of its own:
//     dc_t = q_t.dq_t - k_t.dk_t - 2 dv_t.(v_t - W_t)
// plus, at the chunk's end, what the leaving state asks of c_64; dg is its suffix sum.
// Two terms of it cancel and are left out: the diagonal of dqk (in q.dq and k.dk alike),
// and of the exit e^(c_64 - c) U dS^T the tokens from t on (in k.dk and in c_64's), so that
// dg of a lone token whose decay scales a zero state is zero and not their rounding.
#include "tnt_delta.h"

namespace tnt {
namespace {

// ---------------------------------------------------------------------------------
// dU's part that the chunk's own outputs ask for: P^T dO, every (chunk, head) at once.
// ---------------------------------------------------------------------------------
template <typename E, int DK>
__global__ __launch_bounds__(256) void delta_dlocal_kernel(DeltaArgs a) {
  constexpr int NP = terms_of<E>(), KS = DK / 32;
  __shared__ __attribute__((aligned(16))) __bf16 Pl[4 * 2 * 1536];
  __shared__ float2 cl[DC];
  Chunk ch;
  const int slot = blockIdx.x / a.H, h = blockIdx.x - slot * a.H;
  if (!chunk_of(a, slot, ch)) return;
  const int hk = h / a.per, tid = threadIdx.x, lane = tid & 63, w = wave_id_uniform();
  const int q = lane >> 4, c = lane & 15, pitch = a.pitch;
  const size_t hat = (size_t)slot * a.H + h;
  const size_t kat = ((size_t)slot * a.Hk + hk) * DC * DK * NP;
  const E* qp = (const E*)a.q + ch.b * a.sq.b + hk * a.sq.h + ch.t0 * a.sq.l;
  if (tid < DC) cl[tid] = a.cum[hat * DC + tid];
  // key tile w against the queries from it on: tiles of P, the operand of P^T dO
  f4 p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = zero4();
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const Fr<NP> fk = load_frag<NP>(a.KF + kat + (size_t)(w * KS + s) * 512 * NP, lane);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i >= w) {
        const uint32_t at = (uint32_t)min(16 * i + c, ch.n - 1) * (uint32_t)a.sq.l;
        mma_terms(p[i], row_frag<E>(qp, at, 32 * s, q, a.d_k), fk);
      }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int key = 16 * w + c, qry = 16 * i + 4 * q + r;
      const float d = a.scale * p[i][r] * exp_diff(cl[qry], cl[key]);
      x[r] = key <= qry && qry < ch.n ? d : 0.f;
    }
    split4_store(x, Pl + w * 3072 + (i >> 1) * 1536 + lane * 8 + 4 * (i & 1));
  }
  __syncthreads();
  const E* dop = (const E*)a.dO + ch.b * a.sdO.b + h * a.sdO.h + ch.t0 * a.sdO.l;
  for (int ct = w; ct < a.dvt; ct += 4) {
    const int col = 16 * ct + c;
    f4 acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = zero4();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      typename V4<E>::t x, y;
      const uint32_t cc = (uint32_t)min(col, a.d_v - 1), ld = (uint32_t)a.sdO.l;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = 32 * s + 4 * q + j;
        x[j] = dop[(uint32_t)min(row, ch.n - 1) * ld + cc];
        y[j] = dop[(uint32_t)min(row + 16, ch.n - 1) * ld + cc];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = 32 * s + 4 * q + j;
        if (row >= ch.n || col >= a.d_v) x[j] = (E)0.f;
        if (row + 16 >= ch.n || col >= a.d_v) y[j] = (E)0.f;
      }
      const Fr<NP> fo = frag_of(x, y);
#pragma unroll
      for (int i = 0; i < 2 * s + 2; ++i) mma_terms(acc[i], load_frag<3>(Pl + i * 3072 + s * 1536, lane), fo);
    }
    float* up = a.dU + hat * DC * pitch + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) up[(16 * i + 4 * q + r) * pitch] = acc[i][r];
  }
}

// ---------------------------------------------------------------------------------
// The chain of adjoints, from the last chunk to the first.  One wave walks a (sequence,
// head) for 16 columns of the values, its part of the adjoint in fp32 tiles throughout.
// Every product takes its right operand from the registers of the one before (accumulator
// tiles as they stand), so a chunk needs no LDS and no barrier; each set of fragments is
// requested for the next chunk as soon as this one has used it.  108 MFMAs a chunk at
// dk 64, 180 at 128; bound by the instructions of a wave alone on its SIMD: 2.0 us a chunk
// of 32 x 4 column tiles at dk 64, 3.1 us of 16 x 8 at 128, issuing in 74 and 65 % of its
// cycles.  Cut by rows over four waves as the forward's chain is, it took 2.1 and 2.9 us
// with few tiles (2.0 and 2.9 here at the time) and a third longer with many (1408 tiles of
// 23 chunks at 128: 454 us, 339 here).
// ---------------------------------------------------------------------------------
template <typename E, int DK, int PV>
__global__ __launch_bounds__(64) void delta_bchain_kernel(DeltaArgs a) {
  constexpr int NP = terms_of<E>(), KS = DK / 32, DT = DK / 16;
  // fp32 inputs from dk 64: the three sets of key and query fragments (288 registers, 576
  // at dk 128) do not fit together; each half of a set is requested when half a set before
  // it has been used, one set's registers in all (8 heads of 8192 tokens, the whole
  // training call: 1.10 -> 0.79 ms at 64, 5.80 -> 1.58 at 128)
  constexpr bool ONE = NP == 3 && DK >= 64;
  int seq, h, ct;
  if (!chain_unit(a, seq, h, ct)) return;
  const int lane = threadIdx.x, q = lane >> 4, col = 16 * ct + (lane & 15);
  constexpr int pitch = PV;
  const bool incol = col < a.d_v;
  const Walk k = walk_of(a, seq);
  f4 S[DT];
  const size_t s_at = ((size_t)seq * a.H + h) * a.d_k * a.d_v;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * t + 4 * q + r;
      S[t][r] = a.dfin && row < a.d_k && incol ? a.dfin[s_at + row * a.d_v + col] : 0.f;
    }
  Fr<NP> kf[4][KS], kt[DT][2], qt[DT][2];
  Fr<3> tf[6];
  E o[16];
  float du[16], ec[16], eu[16], el[16], ge;
  auto at = [&](int slot) { return max(slot, k.s0); };
  auto keys = [&](const __bf16* F, int slot) {
    return F + ((size_t)at(slot) * a.Hk + h / a.per) * DC * DK * NP;
  };
  auto load_kf = [&](int slot, int half) {
    const __bf16* p = keys(a.KF, slot);
#pragma unroll
    for (int s = half * KS / 2; s < (half + 1) * KS / 2; ++s)
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) kf[rt][s] = load_frag<NP>(p + (size_t)(rt * KS + s) * 512 * NP, lane);
  };
  auto load_t = [&](Fr<NP> (&f)[DT][2], const __bf16* F, int slot, int s) {
    const __bf16* p = keys(F, slot);
#pragma unroll
    for (int t = 0; t < DT; ++t) f[t][s] = load_frag<NP>(p + (size_t)(t * 2 + s) * 512 * NP, lane);
  };
  auto two = [&](auto&& load) {
    load(0);
    load(1);
  };
  auto load_tf = [&](int slot) {
    const __bf16* p = a.TF + ((size_t)at(slot) * a.H + h) * DELTA_TFRAG;
#pragma unroll
    for (int f = 0; f < 6; ++f) tf[f] = load_frag<3>(p + f * 1536, lane);
  };
  auto load_c = [&](float (&c)[16], const float* F, int slot) {
    const float* p = F + ((size_t)at(slot) * a.H + h) * DC;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      *reinterpret_cast<f4*>(c + 4 * t) = *reinterpret_cast<const f4*>(p + 16 * t + 4 * q);
  };
  auto load_du = [&](int slot) {
    const float* p = a.dU + ((size_t)at(slot) * a.H + h) * DC * pitch + (uint32_t)(4 * q * pitch + col);
#pragma unroll
    for (int e = 0; e < 16; ++e) du[e] = p[(uint32_t)((16 * (e >> 2) + (e & 3)) * pitch)];
    load_c(eu, a.eu, slot);
  };
  auto load_o = [&](int slot) {
    const int past = (at(slot) - k.s0) * DC, n = min(DC, k.len - past);
    const E* p = (const E*)a.dO + k.b * a.sdO.b + h * a.sdO.h + (int64_t)(k.t0 + past) * a.sdO.l;
    load_column(o, p, (uint32_t)a.sdO.l, min(col, a.d_v - 1), n, q);
    load_c(ec, a.ec, slot);
    ge = a.ge[(size_t)at(slot) * a.H + h];
  };
  if (k.s0 < k.s1) {
    const int slot = k.s1 - 1;
    two([&](int i) { load_kf(slot, i); });
    load_du(slot);
    load_tf(slot);
    load_o(slot);
    if (!ONE) two([&](int i) { load_t(qt, a.QT, slot, i); });
    load_c(el, a.el, slot);
    if (!ONE) two([&](int i) { load_t(kt, a.KT, slot, i); });
  }
  for (int slot = k.s1 - 1; slot >= k.s0; --slot) {
    const size_t hat = (size_t)slot * a.H + h;
    f4 x[4] = {zero4(), zero4(), zero4(), zero4()};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const Fr<NP> f[4] = {kf[0][s], kf[1][s], kf[2][s], kf[3][s]};
      mma_terms_n(x, f, frag_of(S[2 * s], S[2 * s + 1]));
      if (ONE && 2 * (s + 1) % KS == 0) load_t(qt, a.QT, slot, 2 * s / KS);
      if (ONE) __builtin_amdgcn_sched_barrier(0);
    }
    if (!ONE) two([&](int i) { load_kf(slot - 1, i); });
    float* sp = a.dS + hat * DK * pitch + (uint32_t)(4 * q * pitch + col);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) sp[(uint32_t)((16 * t + r) * pitch)] = S[t][r];
    Fr<3> y[2];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[t][r] = du[4 * t + r] + eu[4 * t + r] * x[t][r];
    y[0] = frag_of(x[0], x[1]);
    y[1] = frag_of(x[2], x[3]);
    load_du(slot - 1);
    tri_product_t(x, tf, y);
    load_tf(slot - 1);
    // what the chunk's queries ask of the entering state
    f4 z[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        z[t][r] = ec[4 * t + r] * to_f(o[4 * t + r]);
    // (rows past the chunk's end meet zero queries; columns past d_v have to be zero)
    if (16 * ct + 16 > a.d_v && !incol) z[0] = z[1] = z[2] = z[3] = zero4();
    y[0] = frag_of(z[0], z[1]);
    y[1] = frag_of(z[2], z[3]);
#pragma unroll
    for (int t = 0; t < DT; ++t) S[t] *= ge;
    load_o(slot - 1);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Fr<NP> f[DT];
#pragma unroll
      for (int t = 0; t < DT; ++t) f[t] = qt[t][s];
      mma_terms_n(S, f, y[s]);
      if (ONE) load_t(kt, a.KT, slot, s);
      if (ONE) __builtin_amdgcn_sched_barrier(0);
    }
    if (!ONE) two([&](int i) { load_t(qt, a.QT, slot - 1, i); });
    float* rp = a.dR + hat * DC * pitch + (uint32_t)(4 * q * pitch + col);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        rp[(uint32_t)((16 * t + r) * pitch)] = x[t][r];
        x[t][r] *= el[4 * t + r];
      }
    y[0] = frag_of(x[0], x[1]);
    y[1] = frag_of(x[2], x[3]);
    load_c(el, a.el, slot - 1);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      Fr<NP> f[DT];
#pragma unroll
      for (int t = 0; t < DT; ++t) f[t] = kt[t][s];
      mma_terms_n(S, f, y[s]);
      if (ONE) load_kf(slot - 1, s);
      if (ONE) __builtin_amdgcn_sched_barrier(0);
    }
    if (!ONE) two([&](int i) { load_t(kt, a.KT, slot - 1, i); });
  }
  if (a.dS0)
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * t + 4 * q + r;
        if (row < a.d_k && incol) a.dS0[s_at + row * a.d_v + col] = S[t][r];
      }
}

// ---------------------------------------------------------------------------------
// The gradients, every (chunk, key head) at once; the heads that share keys in turn,
// their sums of dq and dk in registers (a fixed order, no atomics).  The values' columns
// are taken 32 at a time: the waves split the rows of U, dR and dO into LDS, where they
// serve as rows (dq, dk) and as columns (dqk, M); a wave takes two row tiles of two
// column tiles of the keys, so that a state's fragment is split by two waves only and a
// row fragment read by a quarter of them.  At dk 128 (1.38 ms for 16 x 32768 tokens) the waves
// wait for memory, LDS and barriers in 57 % of their cycles and issue in 19 %, with one
// workgroup a CU and 0.64 of 1.05 GB written spilled registers; at dk 64 (0.36 ms, 32 x 8192) 46
// and 42 %.
// ---------------------------------------------------------------------------------
template <typename E, int DK> constexpr size_t grads_lds() {
  constexpr int NP = terms_of<E>();
  const size_t stage = (size_t)4 * (3 + 3 + NP) * 512 * 2;      // U, dR, dO of one step
  const size_t prod = (size_t)3 * 4 * 2 * 1536 * 2;             // dqk, dqk^T, M
  return stage > prod ? stage : prod;
}

// tile t of the ten lower ones
__device__ __forceinline__ void lower_tile(int t, int& i, int& j) {
  i = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3;
  j = t - i * (i + 1) / 2;
}

template <typename E, int DK, bool GROUP>
__global__ __launch_bounds__(4 * DK) void delta_grads_kernel(DeltaArgs a) {
  constexpr int NP = terms_of<E>(), NW = DK / 16, CP = DK / 32, NT = 4 * DK;
  constexpr int ITEMS = 8 / NW, TILES = (10 + NW - 1) / NW;
  typedef typename V4<E>::t v4;
  extern __shared__ __attribute__((aligned(16))) __bf16 sm[];
  __shared__ float2 cl[DC];
  __shared__ float ll[DC], lec[DC], leu[DC], lel[DC], diag[DC], rowdot[CP][DC], exdot[CP][DC], vdot[2][DC], wdot[2][DC],
      scal[NW];
  Chunk ch;
  const int slot = blockIdx.x / a.Hk, hk = blockIdx.x - slot * a.Hk;
  if (!chunk_of(a, slot, ch)) return;
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id_uniform();
  const int q = lane >> 4, c = lane & 15, pitch = a.pitch, wide = 16 * a.dvt;  // columns written
  const int cp = w >> 1, i0 = 2 * (w & 1);  // column tiles 2 cp, +1; row tiles i0, i0 + 1
  const size_t kat = ((size_t)slot * a.Hk + hk) * DC * DK * NP;
  __bf16* Uf = sm;
  __bf16* Rf = Uf + 4 * 1536;
  __bf16* Of = Rf + 4 * 1536;
  __bf16* Gq = sm;               // dqk: rows queries
  __bf16* Gk = Gq + 4 * 3072;    // dqk^T: rows keys
  __bf16* Mf = Gk + 4 * 3072;    // M + M^T
  f4 dqt[2][2], dkt[2][2];
  if (GROUP)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) dqt[i][t] = dkt[i][t] = zero4();
  const E* qp = (const E*)a.q + ch.b * a.sq.b + hk * a.sq.h + (int64_t)ch.t0 * a.sq.l;
  const E* kp = (const E*)a.k + ch.b * a.sk.b + hk * a.sk.h + (int64_t)ch.t0 * a.sk.l;

  for (int h = hk * a.per; h < (hk + 1) * a.per; ++h) {
    const size_t hat = (size_t)slot * a.H + h;
    if (tid < DC) {
      cl[tid] = a.cum[hat * DC + tid];
      lec[tid] = a.ec[hat * DC + tid];
      leu[tid] = a.eu[hat * DC + tid];
      lel[tid] = a.el[hat * DC + tid];
      ll[tid] = tid < ch.n ? a.lr[ch.b * a.sl.b + h * a.sl.h + (int64_t)(ch.t0 + tid) * a.sl.l] : 0.f;
    }
    f4 dqs[2][2], dks[2][2], dke[2][2], tp[TILES], ta[TILES];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) dqs[i][t] = dks[i][t] = dke[i][t] = zero4();
#pragma unroll
    for (int i = 0; i < TILES; ++i) tp[i] = ta[i] = zero4();
    float dot_vw[ITEMS], dot_rw[ITEMS], dot_ss = 0.f;
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) dot_vw[n] = dot_rw[n] = 0.f;
    const E* vp = (const E*)a.v + ch.b * a.sv.b + h * a.sv.h + (int64_t)ch.t0 * a.sv.l;
    const E* op = (const E*)a.dO + ch.b * a.sdO.b + h * a.sdO.h + (int64_t)ch.t0 * a.sdO.l;
    E* dvp = (E*)a.dv + ch.b * a.sdv.b + h * a.sdv.h + (int64_t)ch.t0 * a.sdv.l;
    const float* Wp = a.W + hat * DC * pitch;
    const float* Rp = a.dR + hat * DC * pitch;
    const float* Sp = a.S + hat * DK * pitch;
    const float* Dp = a.dS + hat * DK * pitch;
    // A step's data is requested while the one before is multiplied: states by column tile,
    // rows by item (16 columns of 16 rows); past the last step it is requested again.  The
    // eight waves of dk 128 have 256 registers each, too few to hold it: there at the step's
    // start (16 x 32768 tokens: 1.40 ms, ahead 1.62; at dk 64, 32 x 8192: 427 us, ahead 367).
    // At dk 32 a wave has four items of rows and spills as well (whole training call, 32 x
    // 8192 tokens: 775 us, ahead 841).
    constexpr bool AHEAD = DK == 64;
    const int steps = (a.dvt + 1) / 2;
    f4 x[2][2], y[2][2], wv[ITEMS], rv[ITEMS];
    v4 vv[ITEMS], ov[ITEMS];
    auto load_states = [&](int t, int s) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int k0 = 32 * s + 16 * hf + 4 * q;
        const uint32_t at = 4u * (uint32_t)((32 * cp + 16 * t + c) * pitch + min(k0, wide - 4));
        x[t][hf] = load_at<f4>(Sp, at);
        y[t][hf] = load_at<f4>(Dp, at);
      }
    };
    auto load_rows = [&](int n, int s) {
      const int it = w + NW * n, row = 16 * (it >> 1) + c, k0 = 32 * s + 16 * (it & 1) + 4 * q;
      const uint32_t rc = (uint32_t)min(row, ch.n - 1), kc = (uint32_t)min(k0, a.d_v - 4);
      const uint32_t at = 4u * (uint32_t)(row * pitch + min(k0, wide - 4));
      wv[n] = load_at<f4>(Wp, at);
      rv[n] = load_at<f4>(Rp, at);
      vv[n] = load_at<v4>(vp, (uint32_t)sizeof(E) * (rc * (uint32_t)a.sv.l + kc));
      ov[n] = load_at<v4>(op, (uint32_t)sizeof(E) * (rc * (uint32_t)a.sdO.l + kc));
    };
    if (AHEAD) {
#pragma unroll
      for (int n = 0; n < ITEMS; ++n) load_rows(n, 0);
#pragma unroll
      for (int t = 0; t < 2; ++t) load_states(t, 0);
    }
    lds_barrier();  // cl, ll; the previous head's reads of sm
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
      const int next = min(s + 1, steps - 1);
      if (!AHEAD) {
#pragma unroll
        for (int t = 0; t < 2; ++t) load_states(t, s);
#pragma unroll
        for (int n = 0; n < ITEMS; ++n) load_rows(n, s);
      }
      // U, dR, dO; dv and the row sums on the way
#pragma unroll
      for (int n = 0; n < ITEMS; ++n) {
        const int it = w + NW * n, rt = it >> 1, hf = it & 1;
        const int row = 16 * rt + c, k0 = 32 * s + 16 * hf + 4 * q, at = lane * 8 + 4 * hf;
        const bool have = k0 < wide, in = row < ch.n && k0 < a.d_v;
        const float lr = ll[row];
        float u[4], r4[4], o4[4];
        v4 dvv;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float wj = have ? wv[n][j] : 0.f;
          r4[j] = have ? rv[n][j] : 0.f;
          u[j] = lr * wj;
          const float d = lr * r4[j];
          dvv[j] = from_f<E>(d);
          dot_vw[n] += d * ((in ? to_f((E)vv[n][j]) : 0.f) - wj);
          dot_rw[n] += r4[j] * wj;
          o4[j] = in ? to_f((E)ov[n][j]) : 0.f;
        }
        if (AHEAD) load_rows(n, next);
        if (in) *reinterpret_cast<v4*>((char*)dvp + (uint32_t)sizeof(E) * ((uint32_t)row * (uint32_t)a.sdv.l + k0)) = dvv;
        split4_store(u, Uf + rt * 1536 + at);
        split4_store(r4, Rf + rt * 1536 + at);
        if (NP == 1) {
          bf16x4 ob;
#pragma unroll
          for (int j = 0; j < 4; ++j) ob[j] = (__bf16)o4[j];
          *reinterpret_cast<bf16x4*>(Of + rt * 512 + at) = ob;
        } else {
          split4_store(o4, Of + rt * 1536 + at);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      lds_barrier();
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
          if (32 * s + 16 * hf >= wide) x[t][hf] = y[t][hf] = zero4();
        if (i0 == 0)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int j = 0; j < 4; ++j) dot_ss += x[t][hf][j] * y[t][hf][j];
        const Fr<3> fs = frag_of(x[t][0], x[t][1]), fd = frag_of(y[t][0], y[t][1]);
        if (AHEAD) load_states(t, next);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mma_terms(dqs[i][t], load_frag<NP>(Of + (i0 + i) * 512 * NP, lane), fs);
          mma_terms(dks[i][t], load_frag<3>(Rf + (i0 + i) * 1536, lane), fs);
          mma_terms(dke[i][t], load_frag<3>(Uf + (i0 + i) * 1536, lane), fd);
          __builtin_amdgcn_sched_barrier(0);  // limits what is in registers at once
        }
      }
      // lower tiles (i, j) of dO U^T and dR U^T: wave w has tiles w, w + NW, ..
#pragma unroll
      for (int n = 0; n < TILES; ++n) {
        const int t = w + NW * n;
        if (t < 10) {
          int i, j;
          lower_tile(t, i, j);
          const Fr<3> fu = load_frag<3>(Uf + j * 1536, lane);
          mma_terms(tp[n], load_frag<NP>(Of + i * 512 * NP, lane), fu);
          mma_terms(ta[n], load_frag<3>(Rf + i * 1536, lane), fu);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      lds_barrier();
    }
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) {
      const int it = w + NW * n, rt = it >> 1, hf = it & 1;
      const float x = sum_groups(dot_vw[n]), y = sum_groups(dot_rw[n]);
      if (q == 0) {
        vdot[hf][16 * rt + c] = x;
        wdot[hf][16 * rt + c] = y;
      }
    }
    // the masked products into LDS, both ways round; the halves above the diagonal that a
    // step of 32 takes along are zero
    if (w == 0) {
      const f4 z = zero4();
      typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          *reinterpret_cast<f2*>(Gq + i * 3072 + (i >> 1) * 1536 + 512 * p + lane * 8 + 4) = f2{z[0], z[1]};
          *reinterpret_cast<f2*>(Gk + (i + 1) * 3072 + (i >> 1) * 1536 + 512 * p + lane * 8) = f2{z[0], z[1]};
        }
    }
#pragma unroll
    for (int n = 0; n < TILES; ++n) {
      const int t = w + NW * n;
      if (t < 10) {
        int i, j;
        lower_tile(t, i, j);
        float g[4], m[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int qi = 16 * i + 4 * q + r, kj = 16 * j + c;
          const float d = exp_diff(cl[qi], cl[kj]);
          const float x = a.scale * d * tp[n][r];
          g[r] = qi > kj ? x : 0.f;
          if (qi == kj) diag[qi] = x;
          m[r] = qi > kj ? -ll[qi] * d * ta[n][r] : 0.f;
        }
        // as rows of the keys (lane's column c), contraction over the queries 4q + r
        uint32_t tg[3][2], tm[3][2];
        split_n(g, tg);
        split_n(m, tm);
        terms4_store(tg, Gk + j * 3072 + (i >> 1) * 1536 + lane * 8 + 4 * (i & 1));
        if (i != j) terms4_store(tm, Mf + j * 3072 + (i >> 1) * 1536 + lane * 8 + 4 * (i & 1));
        // the other way: row 4q + r, contraction index c of tile j: lane 16 (c / 4) + row
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int rr = 4 * q + r, step = (j >> 1) * 1536, el = 4 * (j & 1);
          const int at = step + (16 * (c >> 2) + rr) * 8 + el + (c & 3);
          terms4_put(tg, r, Gq + i * 3072 + at);
          // of a diagonal tile of M + M^T the lane with row > column writes both places, the
          // lane on the diagonal its zero
          if (i != j || rr >= c) {
            terms4_put(tm, r, Mf + i * 3072 + at);
            if (i == j) terms4_put(tm, r, Mf + i * 3072 + step + (16 * (rr >> 2) + c) * 8 + el + (rr & 3));
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    lds_barrier();
    float dots[2][4], exits[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) dots[i][r] = exits[i][r] = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int dt = 2 * cp + t, col = 16 * dt + c, cc = min(col, a.d_k - 1);
      Fr<NP> kf[2], qf[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        kf[s] = load_frag<NP>(a.KT + kat + (size_t)(dt * 2 + s) * 512 * NP, lane);
        qf[s] = load_frag<NP>(a.QT + kat + (size_t)(dt * 2 + s) * 512 * NP, lane);
      }
#pragma unroll
      for (int ii = 0; ii < 2; ++ii) {
        const int i = i0 + ii;
        E kr[4], qr[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int rw = min(16 * i + 4 * q + r, ch.n - 1);
          kr[r] = load_at<E>(kp, (uint32_t)sizeof(E) * ((uint32_t)rw * (uint32_t)a.sk.l + (uint32_t)cc));
          qr[r] = load_at<E>(qp, (uint32_t)sizeof(E) * ((uint32_t)rw * (uint32_t)a.sq.l + (uint32_t)cc));
        }
        f4 x, y;
        float kv[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int rw = 16 * i + 4 * q + r;
          kv[r] = rw < ch.n && col < a.d_k ? to_f(kr[r]) : 0.f;
          x[r] = lec[rw] * dqs[ii][t][r];
          y[r] = lel[rw] * dks[ii][t][r];
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          if (s <= i / 2) mma_terms(x, load_frag<3>(Gq + i * 3072 + s * 1536, lane), kf[s]);
          if (s >= i / 2) mma_terms(y, load_frag<3>(Gk + i * 3072 + s * 1536, lane), qf[s]);
          mma_terms(y, load_frag<3>(Mf + i * 3072 + s * 1536, lane), kf[s]);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int rw = 16 * i + 4 * q + r;
          const float qv = rw < ch.n && col < a.d_k ? to_f(qr[r]) : 0.f;
          const float ke = leu[rw] * dke[ii][t][r], d = diag[rw];
          dots[ii][r] += qv * x[r] - kv[r] * y[r];
          exits[ii][r] += kv[r] * ke;
          x[r] += d * kv[r];
          y[r] += ke + d * qv;
        }
        if (GROUP) {
          dqt[ii][t] += x;
          dkt[ii][t] += y;
        } else {
          dqs[ii][t] = x;
          dks[ii][t] = y;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = sum16(dots[i][r]), y = sum16(exits[i][r]);
        if (c == 0) {
          rowdot[cp][16 * (i0 + i) + 4 * q + r] = x;
          exdot[cp][16 * (i0 + i) + 4 * q + r] = y;
        }
      }
    {
      const float x = sum_groups(sum16(exp_pair(cl[DC - 1]) * dot_ss));
      if (lane == 0) scal[w] = x;
    }
    lds_barrier();
    if (w == 0) {
      float x = -2.f * (vdot[0][lane] + vdot[1][lane]), y = 0.f, e = 0.f;
#pragma unroll
      for (int i = 0; i < CP; ++i) {
        x += rowdot[i][lane];
        y += exdot[i][lane];
      }
      const float own = y;
      for (int m = 1; m < 64; m <<= 1) {  // suffix sums; the exits: of the tokens before
        const float o = __shfl_down(x, m, 64), u = __shfl_up(y, m, 64);
        if (lane + m < 64) x += o;
        if (lane >= m) y += u;
      }
      x += y - own;
#pragma unroll
      for (int i = 0; i < NW; ++i) e += scal[i];
      if (lane < ch.n) {
        const int64_t t = ch.t0 + lane;
        a.dg[ch.b * a.sdg.b + h * a.sdg.h + t * a.sdg.l] = x + e;
        a.dlr[ch.b * a.sdl.b + h * a.sdl.h + t * a.sdl.l] = wdot[0][lane] + wdot[1][lane];
      }
    }
    if (!GROUP) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          dqt[i][t] = dqs[i][t];
          dkt[i][t] = dks[i][t];
        }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int col = 32 * cp + 16 * t + c;
    if (col >= a.d_k) continue;
    E* dqp = (E*)a.dq + ch.b * a.sdq.b + hk * a.sdq.h + (int64_t)ch.t0 * a.sdq.l + col;
    E* dkp = (E*)a.dk + ch.b * a.sdk.b + hk * a.sdk.h + (int64_t)ch.t0 * a.sdk.l + col;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int rw = 16 * (i0 + i) + 4 * q + r;
        if (rw < ch.n) {
          dqp[(uint32_t)rw * (uint32_t)a.sdq.l] = from_f<E>(dqt[i][t][r]);
          dkp[(uint32_t)rw * (uint32_t)a.sdk.l] = from_f<E>(dkt[i][t][r]);
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

hipError_t launch_delta_dlocal(const DeltaArgs& a, bool bf16, hipStream_t st) {
  return by_size(a, bf16, [&](auto e, auto n) {
    delta_dlocal_kernel<decltype(e), decltype(n)::value><<<a.slots * a.H, 256, 0, st>>>(a);
  });
}

hipError_t launch_delta_bchain(const DeltaArgs& a, bool bf16, hipStream_t st) {
  const int blocks = (a.nseq * a.H + 7) / 8 * 8 * a.dvt;
  return by_size(a, bf16, [&](auto e, auto n) {
    typedef decltype(e) E;
    constexpr int DK = decltype(n)::value;
    if (a.pitch == 32) delta_bchain_kernel<E, DK, 32><<<blocks, 64, 0, st>>>(a);
    else if (a.pitch == 64) delta_bchain_kernel<E, DK, 64><<<blocks, 64, 0, st>>>(a);
    else delta_bchain_kernel<E, DK, 128><<<blocks, 64, 0, st>>>(a);
  });
}

hipError_t launch_delta_grads(const DeltaArgs& a, bool bf16, hipStream_t st) {
  return by_size(a, bf16, [&](auto e, auto n) {
    typedef decltype(e) E;
    constexpr int DK = decltype(n)::value;
    if (a.per > 1) delta_grads_kernel<E, DK, true><<<a.slots * a.Hk, 4 * DK, grads_lds<E, DK>(), st>>>(a);
    else delta_grads_kernel<E, DK, false><<<a.slots * a.Hk, 4 * DK, grads_lds<E, DK>(), st>>>(a);
  });
}

}  // namespace tnt
