// The gated delta rule token by token, the state updated where it lies.
//
// A wave holds 32 columns of one (sequence, head) state in registers: 8 lanes of 4
// columns by 8 groups of rows, row = group + 8 i, so that a row's 32 columns are one
// 128-byte line.  Per token: the two contractions over the rows (of the decayed state
// with the key, and of the state with the query) are sums over a lane's rows and three
// shuffles; with
//     o = scale (e^g S^T q + lr (k.q) e),   e = v - e^g S^T k
// both contractions are over the entering state and run in one pass.  Bound by the
// state's bytes, read and written once a call, past the caches: between two tokens of a
// sequence lie the other layers' states.  248 sequences of 16 heads at 128 x 128, 260 MB
// read and written: 117 us (4.5 TB/s; a large copy reaches 5.1).  Past the caches / through
// them, us a launch in a graph, with three other pools in between or (again) the same one at
// once: 0.5 MB 4.9 / 4.9, 8 MB 5.9 / 6.3 (5.9 / 6.1), 34 MB 14.6 / 15.6 (12.2 / 13.4), 67 MB
// 28 / 31 (27 / 31), 134 MB 56 / 66 (56 / 53), 260 MB 105 / 121 (104 / 109).  A few sequences
// cost a launch.
#include "tnt_delta.h"

namespace tnt {
namespace {

template <typename E> __device__ __forceinline__ float at(const E* p, bool in) { return in ? to_f(*p) : 0.f; }

// sum over the 8 row groups (lane bits 3..5)
__device__ __forceinline__ float sum_rows(float x) {
  x += __shfl_xor(x, 8, 64);
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

template <typename E, int DK>
__global__ __launch_bounds__(64) void delta_step_kernel(DeltaStepArgs a, int tiles) {
  constexpr int R = DK / 8;
  const int lane = threadIdx.x, grp = lane >> 3;
  const int ct = blockIdx.x % tiles, bh = blockIdx.x / tiles;
  const int b = bh / a.H, h = bh - b * a.H, hk = h / a.per;
  const int col = 32 * ct + 4 * (lane & 7);
  const bool incol = col < a.d_v;  // d_v is a multiple of 8: a lane's 4 columns are in or out
  typedef typename V4<E>::t v4;
  E* op = (E*)a.o + b * a.so.b + h * a.so.h + col;
  const int sl = a.slot ? a.slot[b] : b;
  if (sl < 0 || sl >= a.nslots) {  // padding: no state, outputs of zero
    if (grp == 0 && incol)
      for (int t = 0; t < a.T; ++t) *reinterpret_cast<v4*>(op + t * a.so.l) = zero_v4<E>();
    return;
  }
  float* sp = a.state + ((size_t)sl * a.H + h) * a.d_k * a.d_v + col;
  f4 S[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = grp + 8 * i;
    S[i] = row < a.d_k && incol ? __builtin_nontemporal_load(reinterpret_cast<const f4*>(sp + row * a.d_v)) : zero4();
  }
  const E* kp = (const E*)a.k + b * a.sk.b + hk * a.sk.h;
  const E* qp = (const E*)a.q + b * a.sq.b + hk * a.sq.h;
  const E* vp = (const E*)a.v + b * a.sv.b + h * a.sv.h + col;
  for (int t = 0; t < a.T; ++t) {
    float g = a.g[b * a.sg.b + h * a.sg.h + t * a.sg.l];
    const float lr = a.lr[b * a.sl.b + h * a.sl.h + t * a.sl.l];
    g = g < DELTA_GMIN ? DELTA_GMIN : g;
    const float eg = expf(g);
    float kr[R], sk[4], sq[4], kq = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) sk[j] = sq[j] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = grp + 8 * i;
      kr[i] = at(kp + t * a.sk.l + row, row < a.d_k);
      const float qr = at(qp + t * a.sq.l + row, row < a.d_k);
      kq += kr[i] * qr;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sk[j] += S[i][j] * kr[i];
        sq[j] += S[i][j] * qr;
      }
    }
    kq = sum_rows(kq);
    v4 v = zero_v4<E>(), out;
    if (incol) v = *reinterpret_cast<const v4*>(vp + t * a.sv.l);
    float u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] = lr * (to_f((E)v[j]) - eg * sum_rows(sk[j]));
      out[j] = from_f<E>(a.scale * (eg * sum_rows(sq[j]) + kq * u[j]));
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) S[i][j] = eg * S[i][j] + kr[i] * u[j];
    if (grp == 0 && incol) *reinterpret_cast<v4*>(op + t * a.so.l) = out;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = grp + 8 * i;
    if (row < a.d_k && incol) __builtin_nontemporal_store(S[i], reinterpret_cast<f4*>(sp + row * a.d_v));
  }
}

}  // namespace

hipError_t launch_delta_step(const DeltaStepArgs& a, bool bf16, hipStream_t st) {
  const int tiles = (a.d_v + 31) / 32, blocks = a.B * a.H * tiles;
  auto go = [&](auto e) {
    typedef decltype(e) E;
    if (a.d_k <= 32) delta_step_kernel<E, 32><<<blocks, 64, 0, st>>>(a, tiles);
    else if (a.d_k <= 64) delta_step_kernel<E, 64><<<blocks, 64, 0, st>>>(a, tiles);
    else delta_step_kernel<E, 128><<<blocks, 64, 0, st>>>(a, tiles);
  };
  if (bf16) go((__bf16)0.f);
  else go(0.f);
  return hipGetLastError();
}

}  // namespace tnt
