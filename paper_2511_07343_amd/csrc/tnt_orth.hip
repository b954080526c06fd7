// Orthogonalising an update by Newton-Schulz products: X = G / (|G| + eps), then
//     A = X X^T,   B = b A + c A^2,   X <- a X + B X
// per step, X [m][k] with m <= k (the transpose where there are more rows).
//
// Number format.  All singular values stay below a bound that the host has checked
// (4), so every entry of X, A and B is bounded and can be held at a fixed power of two
// as fp16: hi + lo, two terms, keep 22 bits of an entry and products
//     hi hi + hi lo + lo hi
// reach the accuracy of fp32 arithmetic at 3 MFMAs (measured against 64 bits: 7e-7 to
// 2e-6 on 64 x 256 to 512 x 512, fp32 itself 1.3e-6 to 2.2e-6; bf16 terms need 6
// products for that, and with 3 are 20 to 40 times worse).  bf16 updates are computed the
// same way and rounded once: one term in the products with X would halve the time of a
// 4096 x 2048 one, but add 1e-3 to 1.7e-3 to that rounding's 1.7e-3.
#include "tnt_orth.h"

#include "tnt_device.h"

namespace tnt {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));

constexpr float SX = 4096.f, SA = 1024.f, SB = 256.f;  // powers of two the planes are held at

__device__ __forceinline__ f4 mma(const h8& a, const h8& b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// The value passes an opaque move: a product that feeds it may otherwise be rounded to
// fp16 directly (one mixed-precision instruction) for h and by way of fp32 for the
// difference, and where the two round to different neighbours h + l is off by 2^-10.
__device__ __forceinline__ void split(float x, _Float16& h, _Float16& l) {
  asm("" : "+v"(x));
  h = (_Float16)x;
  l = (_Float16)(x - (float)h);
}
__device__ __forceinline__ float load_g(const OrthArgs& a, int64_t at) {
  return a.bf16 ? (float)((const __bf16*)a.G)[at] : ((const float*)a.G)[at];
}
__device__ __forceinline__ void store_o(const OrthArgs& a, int64_t at, float x) {
  if (a.bf16) ((__bf16*)a.out)[at] = (__bf16)x;
  else ((float*)a.out)[at] = x;
}

// lower tile t of a symmetric array: row tile i >= column tile j
__device__ __forceinline__ void lower(int t, int& i, int& j) {
  i = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while ((i + 1) * (i + 2) / 2 <= t) ++i;
  while (i * (i + 1) / 2 > t) --i;
  j = t - i * (i + 1) / 2;
}

// ---------------------------------------------------------------------------------
// One workgroup a matrix, every step in one launch.  T = X^T [k][m] lies across eight
// waves: wave w has 32 RP rows as accumulator tiles, held as their two fp16 terms (the
// registers of the fp32 value).  A tile pair stacked along its rows is an operand over
// those rows, for either side: T^T T needs no move, only the sum of the waves' parts
// through LDS.  A and B are symmetric, so a tile's rows are another's columns and they
// lie in LDS as whole fragments.  T B contracts over T's columns: the tiles are turned
// by a product with the identity (exact, 1 MFMA a tile and term).  Bound by one CU's
// instructions a matrix, so its time is that of one matrix up to 256 of them: 16 matrices
// of 256 x 64 in 29 us.
// ---------------------------------------------------------------------------------
template <int MT> constexpr int tile_group() { return MT == 4 ? 5 : 3; }
template <int MT> constexpr size_t small_lds() {
  const size_t frags = (size_t)MT * (MT / 2) * 2 * 1024, part = (size_t)tile_group<MT>() * 8 * 1024;
  return frags + (part > frags ? part : frags);
}

// symmetric tile (i, j), rows 4q + r of column c in `v`, into fragments [tile][step][2][64][8]
template <int MT>
__device__ __forceinline__ void put_sym(_Float16* F, int i, int j, const float (&v)[4], int lane) {
  const int q = lane >> 4, c = lane & 15;
  h4 hi, lo;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    _Float16 h, l;
    split(v[r], h, l);
    hi[r] = h;
    lo[r] = l;
  }
  _Float16* p = F + ((size_t)(j * (MT / 2) + (i >> 1)) * 2) * 512 + lane * 8 + 4 * (i & 1);
  *reinterpret_cast<h4*>(p) = hi;
  *reinterpret_cast<h4*>(p + 512) = lo;
  if (i != j) {
    p = F + ((size_t)(i * (MT / 2) + (j >> 1)) * 2) * 512 + (16 * (c >> 2) + 4 * q) * 8 + 4 * (j & 1) + (c & 3);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      p[8 * r] = hi[r];
      p[8 * r + 512] = lo[r];
    }
  }
}

template <int MT, int RP>
__global__ __launch_bounds__(512) void orth_small_kernel(OrthArgs a) {
  constexpr int KS = MT / 2, NT = MT * (MT + 1) / 2, TG = tile_group<MT>();
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ double red[8];
  _Float16* PA = (_Float16*)smem;
  f4* part = (f4*)(smem + (size_t)MT * KS * 2 * 1024);
  _Float16* PB = (_Float16*)part;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane >> 4, c = lane & 15;
  const int64_t g0 = (int64_t)blockIdx.x * a.gb, o0 = (int64_t)blockIdx.x * a.ob;
  float x[RP][MT][8];
  double ss = 0.;
#pragma unroll
  for (int p = 0; p < RP; ++p)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int row = (w * RP + p) * 32 + 16 * (e >> 2) + 4 * q + (e & 3), col = 16 * j + c;
        const bool in = row < a.k && col < a.m;
        const int rr = min(row, a.k - 1), cc = min(col, a.m - 1);
        const float v = load_g(a, g0 + (uint32_t)(a.flip ? rr * (int)a.gr + cc : cc * (int)a.gr + rr));
        x[p][j][e] = in ? v : 0.f;
      }
#pragma unroll
  for (int p = 0; p < RP; ++p)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += (double)x[p][j][e] * (double)x[p][j][e];
  for (int s = 1; s < 64; s <<= 1) ss += __shfl_xor(ss, s, 64);
  if (lane == 0) red[w] = ss;
  __syncthreads();
  ss = 0.;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss += red[i];
  const double inv = (double)SX / (sqrt(ss) + (double)a.eps);  // of a small norm, past fp32
  h8 xh[RP][MT], xl[RP][MT];
#pragma unroll
  for (int p = 0; p < RP; ++p)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        _Float16 h, l;
        split((float)(x[p][j][e] * inv), h, l);
        xh[p][j][e] = h;
        xl[p][j][e] = l;
      }
  h8 ident[2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) ident[t][e] = (_Float16)(16 * (e >> 2) + 4 * q + (e & 3) == 16 * t + c ? 1.f : 0.f);

  for (int step = 0; step < a.steps; ++step) {
    const float ca = a.coef[3 * step], cb = a.coef[3 * step + 1], cc = a.coef[3 * step + 2];
    // A = T^T T: parts of the lower tiles, TG at a time
#pragma unroll
    for (int t0 = 0; t0 < NT; t0 += TG) {
#pragma unroll
      for (int tt = 0; tt < TG; ++tt) {
        const int t = t0 + tt;
        if (t < NT) {
          int i = 0;
#pragma unroll
          for (int u = 1; u < MT; ++u)
            if (t >= u * (u + 1) / 2) i = u;
          const int j = t - i * (i + 1) / 2;
          f4 acc = zero4();
#pragma unroll
          for (int p = 0; p < RP; ++p) {
            acc = mma(xl[p][i], xh[p][j], acc);
            acc = mma(xh[p][i], xl[p][j], acc);
            acc = mma(xh[p][i], xh[p][j], acc);
          }
          part[(tt * 8 + w) * 64 + lane] = acc;
        }
      }
      __syncthreads();
      for (int tt = w; tt < TG && t0 + tt < NT; tt += 8) {
        f4 s = part[tt * 512 + lane];
#pragma unroll
        for (int o = 1; o < 8; ++o) s += part[tt * 512 + o * 64 + lane];
        int i, j;
        lower(t0 + tt, i, j);
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = s[r] * (SA / (SX * SX));
        put_sym<MT>(PA, i, j, v, lane);
      }
      __syncthreads();
    }
    // B = b A + c A^2
    for (int t = w; t < NT; t += 8) {
      int i, j;
      lower(t, i, j);
      f4 acc = zero4();
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const h8* fi = reinterpret_cast<const h8*>(PA + (size_t)(i * KS + s) * 1024) + lane;
        const h8* fj = reinterpret_cast<const h8*>(PA + (size_t)(j * KS + s) * 1024) + lane;
        const h8 ih = fi[0], il = fi[64], jh = fj[0], jl = fj[64];
        acc = mma(il, jh, acc);
        acc = mma(ih, jl, acc);
        acc = mma(ih, jh, acc);
      }
      const _Float16* p = PA + (size_t)(j * KS + (i >> 1)) * 1024 + lane * 8 + 4 * (i & 1);
      const h4 ah = *reinterpret_cast<const h4*>(p), al = *reinterpret_cast<const h4*>(p + 512);
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v[r] = cb * (SB / SA) * ((float)ah[r] + (float)al[r]) + cc * (SB / (SA * SA)) * acc[r];
      put_sym<MT>(PB, i, j, v, lane);
    }
    __syncthreads();
    // T <- a T + T B, 32 rows at a time
#pragma unroll
    for (int p = 0; p < RP; ++p) {
      h8 th[2][KS], tl[2][KS];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          const f4 u = mma(xh[p][j], ident[t], zero4()), v = mma(xl[p][j], ident[t], zero4());
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            th[t][j >> 1][4 * (j & 1) + r] = (_Float16)u[r];
            tl[t][j >> 1][4 * (j & 1) + r] = (_Float16)v[r];
          }
        }
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        f4 acc[2] = {zero4(), zero4()};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const h8* f = reinterpret_cast<const h8*>(PB + (size_t)(j * KS + s) * 1024) + lane;
          const h8 bh = f[0], bl = f[64];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            acc[t] = mma(tl[t][s], bh, acc[t]);
            acc[t] = mma(th[t][s], bl, acc[t]);
            acc[t] = mma(th[t][s], bh, acc[t]);
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = ca * ((float)xh[p][j][e] + (float)xl[p][j][e]) + acc[e >> 2][e & 3] * (1.f / SB);
          _Float16 h, l;
          split(y, h, l);
          xh[p][j][e] = h;
          xl[p][j][e] = l;
        }
      }
    }
    __syncthreads();  // PB lies where the next step's parts go
  }
  const float os = a.scale / SX;
#pragma unroll
  for (int p = 0; p < RP; ++p)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int row = (w * RP + p) * 32 + 16 * (e >> 2) + 4 * q + (e & 3), col = 16 * j + c;
        if (row < a.k && col < a.m)
          store_o(a, o0 + (uint32_t)(a.flip ? row * (int)a.orow + col : col * (int)a.orow + row),
                  os * ((float)xh[p][j][e] + (float)xl[p][j][e]));
      }
}

// ---------------------------------------------------------------------------------
// Large matrices.  The norm, in 64 bits: up to ORTH_PART parts a matrix, summed in a fixed
// order by every workgroup that scales.
// ---------------------------------------------------------------------------------
__device__ __forceinline__ void norm_part(const OrthArgs& a, double ss, double* red) {
  const int tid = threadIdx.x;
  for (int m = 1; m < 64; m <<= 1) ss += __shfl_xor(ss, m, 64);
  if ((tid & 63) == 0) red[tid >> 6] = ss;
  __syncthreads();
  if (tid == 0) a.part[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(256) void orth_norm_kernel(OrthArgs a) {
  __shared__ double red[4];
  const int b = blockIdx.x / a.parts, s = blockIdx.x - b * a.parts, tid = threadIdx.x;
  const int64_t g0 = (int64_t)b * a.gb;
  double ss = 0.;
  // rows of whole 16-byte pieces at 16 bytes: 4 of them a lane at once
  const int64_t el = a.bf16 ? 8 : 4;
  if ((uintptr_t)a.G % 16 == 0 && a.cols % el == 0 && a.gr % el == 0 && a.gb % el == 0) {
    const uint32_t per = a.cols / (int)el, all = a.rows * per, hop = a.parts * 256;  // all <= 2^28
    for (uint32_t i0 = s * 256 + tid; i0 < all; i0 += 4 * hop) {
      f4 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t i = min(i0 + e * hop, all - 1), row = i / per, col = i - row * per;
        const char* p = (const char*)a.G + (g0 + row * a.gr + col * el) * (a.bf16 ? 2 : 4);
        v[e] = *reinterpret_cast<const f4*>(p);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (i0 + e * hop >= all) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (a.bf16) {
            const uint32_t u = __float_as_uint(v[e][r]);
            const double x = __uint_as_float(u << 16), y = __uint_as_float(u & 0xffff0000u);
            ss += x * x + y * y;
          } else {
            ss += (double)v[e][r] * (double)v[e][r];
          }
        }
      }
    }
    norm_part(a, ss, red);
    return;
  }
  // 256 columns of a row an item; the loads of eight items at once
  const int across = (a.cols + 255) / 256, items = a.rows * across;
  for (int i0 = s; i0 < items; i0 += 8 * a.parts) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = min(i0 + e * a.parts, items - 1), row = i / across;
      v[e] = load_g(a, g0 + (int64_t)row * a.gr + min((i - row * across) * 256 + tid, a.cols - 1));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = i0 + e * a.parts, row = i / across;
      if (i < items && (i - row * across) * 256 + tid < a.cols) ss += (double)v[e] * (double)v[e];
    }
  }
  norm_part(a, ss, red);
}

// G, scaled, into both orientations' planes; zeros in the padding.  64 x 64 a workgroup:
// its loads are all on their way before the parts of the norm are summed, its stores are
// 8 bytes a lane.
__global__ __launch_bounds__(256) void orth_scale_kernel(OrthArgs a) {
  __shared__ float t[64][65];
  const int tid = threadIdx.x, b = blockIdx.z;
  const int m0 = 64 * blockIdx.y, k0 = 64 * blockIdx.x;
  const int64_t g0 = (int64_t)b * a.gb;
  // along the memory's rows
  const int u0 = tid >> 6, v0 = tid & 63;
  const int nu = a.flip ? a.k - k0 : a.m - m0, nv = a.flip ? a.m - m0 : a.k - k0;  // inside
  const int64_t at0 = g0 + (a.flip ? (int64_t)k0 * a.gr + m0 : (int64_t)m0 * a.gr + k0);
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    // past the matrix: its last element (every tile has one at least)
    x[i] = load_g(a, at0 + (int64_t)min(u0 + 4 * i, nu - 1) * a.gr + min(v0, nv - 1));
  }
  // every wave sums the parts, in the same order
  double ss = 0.;
  for (int i = v0; i < a.parts; i += 64) ss += a.part[b * a.parts + i];
  for (int m = 1; m < 64; m <<= 1) ss += __shfl_xor(ss, m, 64);
  const double inv = (double)SX / (sqrt(ss) + (double)a.eps);  // of a small norm, past fp32
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int u = u0 + 4 * i;
    const float y = u < nu && v0 < nv ? (float)(inv * x[i]) : 0.f;
    if (a.flip) t[v0][u] = y;
    else t[u][v0] = y;
  }
  __syncthreads();
  const size_t pl = (size_t)a.mp * a.lk, pt = (size_t)a.kp * a.lm;
  _Float16* X = a.X + 2 * pl * b + (size_t)m0 * a.lk + k0;
  _Float16* XT = a.XT + 2 * pt * b + (size_t)k0 * a.lm + m0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int u = (tid >> 4) + 16 * i, v = 4 * (tid & 15);
    h4 h, l, ht, lt;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      _Float16 p, q;
      split(t[u][v + j], p, q);
      h[j] = p;
      l[j] = q;
      split(t[v + j][u], p, q);
      ht[j] = p;
      lt[j] = q;
    }
    const size_t at = (size_t)u * a.lk + v, tt = (size_t)u * a.lm + v;
    *reinterpret_cast<h4*>(X + at) = h;
    *reinterpret_cast<h4*>(X + pl + at) = l;
    *reinterpret_cast<h4*>(XT + tt) = ht;
    *reinterpret_cast<h4*>(XT + pt + tt) = lt;
  }
}

// ---------------------------------------------------------------------------------
// C = P Q^T, both with the contraction along the rows of memory, TM x TM a workgroup of
// four waves (2 x 2).  Steps of 64: the planes' rows go straight from global memory to
// LDS (16 bytes a lane, 128-byte rows, the 16-byte pieces of a row permuted by the row so
// that a wave's fragment reads meet no bank twice), the next step's while this one is
// multiplied.  Tiles of 64, two workgroups a CU: of 128, one a CU, GRAM and SQUARE are slower
// at every size (five steps with those of 4096 x 2048 so: 1.50 ms against 1.41; 64 matrices of
// 510 x 500: 1.23 / 1.12); UPDATE is 3 to 9 % faster from 1024 rows on (4096 x 2048: 1.37)
// and up to a fifth slower below (16 of 520 x 510: 0.43 / 0.36).
//   GRAM    A = X X^T           lower tiles, written both ways round
//   SQUARE  B = b A + c A A     lower tiles, written both ways round
//   UPDATE  X^T <- a X^T + X^T B, both orientations (X in place: a tile reads its own
//           place only; X^T, an operand, from one buffer to the other)
//   LAST    the same into the caller's tensor
// 4096 x 2048: UPDATE 131 us (the matrix units at work in 36 % of the cycles), GRAM 95 (23 %), SQUARE
// 52 (20 %, 528 workgroups); a wave issues in 30 %, waits for issue in 35 % and for LDS and
// barriers in a third.
// ---------------------------------------------------------------------------------
enum { GRAM = 0, SQUARE = 1, UPDATE = 2, LAST = 3 };

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

// every load into LDS has arrived, and every wave is done reading what the next one overwrites
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

constexpr int TM = ORTH_TILE, BK = 64;  // sides of a tile; contraction elements a stage

template <int EPI>
__global__ __launch_bounds__(256) void orth_gemm_kernel(OrthArgs a, int step, int tiles, int share) {
  constexpr int WT = TM / 32;                      // 16-row tiles a wave and side
  constexpr int SIDE = TM * BK, STAGE = 4 * SIDE;  // elements a plane and side; a stage
  extern __shared__ __attribute__((aligned(16))) _Float16 sh[];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = lane >> 4, c = lane & 15;
  // an XCD (block number modulo 8) takes neighbouring tiles, which share operand rows
  const int unit = (blockIdx.x & 7) * share + (blockIdx.x >> 3);
  const int b = unit / tiles, tile = unit - b * tiles;
  if (b >= a.n) return;
  const size_t px = (size_t)a.mp * a.lk, pt = (size_t)a.kp * a.lm, pa = (size_t)a.mp * a.lm;
  const bool odd = step & 1;
  _Float16* X = a.X + 2 * px * b;
  const _Float16* XT = (odd ? a.XT2 : a.XT) + 2 * pt * b;
  _Float16* XTn = (odd ? a.XT : a.XT2) + 2 * pt * b;
  _Float16* A = a.A + 2 * pa * b;
  _Float16* B = a.B + 2 * pa * b;
  int ti, tj;
  if (EPI <= SQUARE) {
    lower(tile, ti, tj);
  } else {
    const int tn = a.mp / TM;
    ti = tile / tn;
    tj = tile - ti * tn;
  }
  const _Float16* P = EPI == GRAM ? X : EPI == SQUARE ? A : XT;
  const _Float16* Q = EPI == GRAM ? X : EPI == SQUARE ? A : B;
  const size_t pp = EPI == SQUARE ? pa : EPI == GRAM ? px : pt, pq = EPI == GRAM ? px : pa;
  const int ld = EPI == GRAM ? a.lk : a.lm, nk = (EPI == GRAM ? a.kp : a.mp) / BK;
  // loads: a wave brings 1 KB, RR rows of BK, a request
  constexpr int PC = BK / 8, RR = 64 / PC, REQ = 4 * TM / RR, PER = REQ / 4;
  const int lrow = lane / PC, piece = (lane % PC) ^ (lrow & 7);
  const _Float16* src[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = w * PER + i, side = r / (2 * TM / RR), rem = r - side * (2 * TM / RR);
    const int pl = rem / (TM / RR), rr = rem - pl * (TM / RR);
    src[i] = (side ? Q + pl * pq : P + pl * pp) +
             (size_t)((side ? tj : ti) * TM + RR * rr + lrow) * ld + 8 * piece;
  }
  auto fetch = [&](int stage, int ks) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      __builtin_amdgcn_global_load_lds((global_void*)(src[i] + ks * BK),
                                       (lds_void*)(sh + stage * STAGE + (w * PER + i) * 512), 16, 0, 0);
  };
  f4 acc[WT][WT];
#pragma unroll
  for (int i = 0; i < WT; ++i)
#pragma unroll
    for (int j = 0; j < WT; ++j) acc[i][j] = zero4();
  const int wi = (w >> 1) * (TM / 2), wj = (w & 1) * (TM / 2);
  fetch(0, 0);
  for (int ks = 0; ks < nk; ++ks) {
    wait_loads();
    fetch((ks + 1) & 1, min(ks + 1, nk - 1));  // (past the last step: again, into the stage not read)
    const _Float16* sp = sh + (ks & 1) * STAGE;
#pragma unroll
    for (int kk = 0; kk < BK / 32; ++kk) {
      const int frag = c * BK + 8 * ((4 * kk + q) ^ (c & 7));
      h8 pf[WT][2], qf[WT][2];
#pragma unroll
      for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          pf[i][p] = *reinterpret_cast<const h8*>(sp + p * SIDE + (wi + 16 * i) * BK + frag);
          qf[i][p] = *reinterpret_cast<const h8*>(sp + (2 + p) * SIDE + (wj + 16 * i) * BK + frag);
        }
#pragma unroll
      for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j) {
          acc[i][j] = mma(pf[i][1], qf[j][0], acc[i][j]);
          acc[i][j] = mma(pf[i][0], qf[j][1], acc[i][j]);
          acc[i][j] = mma(pf[i][0], qf[j][0], acc[i][j]);
        }
    }
  }
  wait_loads();
  // The tile through LDS: both orientations leave in 16-byte stores of whole rows, by loops
  // over rows instead of code for every accumulator (with that, 20 us of a launch whose
  // products take 5 went to fetching its instructions).
  float* T = (float*)sh;
  constexpr int PT = TM + 1, CH = TM / 8;
#pragma unroll
  for (int i = 0; i < WT; ++i)
#pragma unroll
    for (int j = 0; j < WT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) T[(wi + 16 * i + 4 * q + r) * PT + wj + 16 * j + c] = acc[i][j][r];
  __syncthreads();
  const float ca = a.coef[3 * step], cb = a.coef[3 * step + 1], cc = a.coef[3 * step + 2];
  const int64_t o0 = (int64_t)b * a.ob;
  // rows of the transpose: column `col` of the tile, 8 of its rows
#pragma unroll 1
  for (int it = tid; it < TM * CH; it += 256) {
    const int u = it / CH, v = 8 * (it - u * CH), col = tj * TM + u, row = ti * TM + v;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = T[(v + e) * PT + u];
    const size_t mir = (size_t)col * (EPI <= SQUARE ? a.lm : a.lk) + row;
    if (EPI == GRAM) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= SA / (SX * SX);
    } else {
      const _Float16* old = EPI == SQUARE ? A : X;
      const h8 hi = *reinterpret_cast<const h8*>(old + mir);
      const h8 lo = *reinterpret_cast<const h8*>(old + (EPI == SQUARE ? pa : px) + mir);
      const float f = EPI == SQUARE ? cb * (SB / SA) : ca, g = EPI == SQUARE ? cc * (SB / (SA * SA)) : 1.f / SB;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = f * ((float)hi[e] + (float)lo[e]) + g * y[e];
    }
    if (EPI != LAST) {
      h8 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        _Float16 h, l;
        split(y[e], h, l);
        hi[e] = h;
        lo[e] = l;
      }
      _Float16* D = EPI == GRAM ? A : EPI == SQUARE ? B : X;
      *reinterpret_cast<h8*>(D + mir) = hi;
      *reinterpret_cast<h8*>(D + (EPI <= SQUARE ? pa : px) + mir) = lo;
    } else if (!a.flip && col < a.m) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (row + e < a.k) store_o(a, o0 + (int64_t)col * a.orow + row + e, (a.scale / SX) * y[e]);
    }
    if (EPI == UPDATE || (EPI <= SQUARE ? ti != tj : a.flip))
#pragma unroll
      for (int e = 0; e < 8; ++e) T[(v + e) * PT + u] = y[e];
  }
  if (EPI <= SQUARE ? ti == tj : EPI == LAST && !a.flip) return;
  __syncthreads();
#pragma unroll 1
  for (int it = tid; it < TM * CH; it += 256) {
    const int u = it / CH, v = 8 * (it - u * CH), row = ti * TM + u, col = tj * TM + v;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = T[u * PT + v + e];
    if (EPI != LAST) {
      h8 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        _Float16 h, l;
        split(y[e], h, l);
        hi[e] = h;
        lo[e] = l;
      }
      _Float16* D = EPI == GRAM ? A : EPI == SQUARE ? B : XTn;
      const size_t at = (size_t)row * a.lm + col;
      *reinterpret_cast<h8*>(D + at) = hi;
      *reinterpret_cast<h8*>(D + (EPI <= SQUARE ? pa : pt) + at) = lo;
    } else if (row < a.k) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < a.m) store_o(a, o0 + (int64_t)row * a.orow + col + e, (a.scale / SX) * y[e]);
    }
  }
}

template <int EPI> void gemm(const OrthArgs& a, int step, hipStream_t st) {
  constexpr size_t stages = (size_t)2 * 4 * TM * BK * 2, tile = (size_t)TM * (TM + 1) * 4;
  constexpr size_t lds = stages > tile ? stages : tile;
  const int tm = a.mp / TM, tiles = EPI <= SQUARE ? tm * (tm + 1) / 2 : (a.kp / TM) * tm;
  const int share = (a.n * tiles + 7) / 8;
  orth_gemm_kernel<EPI><<<8 * share, 256, lds, st>>>(a, step, tiles, share);
}

template <int MT, int RP>
hipError_t small(const OrthArgs& a, hipStream_t st) {
  orth_small_kernel<MT, RP><<<a.n, 512, small_lds<MT>(), st>>>(a);
  return hipGetLastError();
}

}  // namespace

// Shorter sides of up to 64.  (65 to 128 fit too, in 256 registers of eight waves with spills, but
// one CU a matrix is then the slower form: 32 matrices of 128 x 512 in 212 us against 126.)  Longer
// sides of up to 512, or 1024 with a shorter one of up to 32, take less than the tiles' 17
// launches at any number of matrices (one of 64 x 512: 59 us against 86, 16 x 1024: 38 / 107).
// 33 to 64 by 513 to 1024 spill, 135 to 175 us for up to 64 matrices, where the tiles take 88
// to 118 for 16, 108 to 155 for 48, 127 to 168 for 64 and 600 to 1000 for 256 (here 184 to 222).
bool orth_small(int n, int m, int k) { return m <= 64 && k <= (m <= 32 || n > 48 ? 1024 : 512); }

hipError_t launch_orth_small(const OrthArgs& a, hipStream_t st) {
  const int rp = a.k <= 256 ? 1 : a.k <= 512 ? 2 : 4;
  if (a.m <= 32) return rp == 1 ? small<2, 1>(a, st) : rp == 2 ? small<2, 2>(a, st) : small<2, 4>(a, st);
  return rp == 1 ? small<4, 1>(a, st) : rp == 2 ? small<4, 2>(a, st) : small<4, 4>(a, st);
}

hipError_t launch_orth_large(const OrthArgs& a, hipStream_t st) {
  orth_norm_kernel<<<a.n * a.parts, 256, 0, st>>>(a);
  orth_scale_kernel<<<dim3(a.kp / 64, a.mp / 64, a.n), 256, 0, st>>>(a);
  for (int s = 0; s < a.steps; ++s) {
    gemm<GRAM>(a, s, st);
    gemm<SQUARE>(a, s, st);
    if (s + 1 < a.steps) gemm<UPDATE>(a, s, st);
    else gemm<LAST>(a, s, st);
  }
  return hipGetLastError();
}

}  // namespace tnt
