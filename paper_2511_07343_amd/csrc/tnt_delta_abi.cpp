// C ABI of the gated delta rule: validation, workspace layout and launch sequence.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/tnt.h"
#include "tnt_delta.h"
#include "tnt_kernels.h"

using namespace tnt;

namespace {

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

tnt_status validate(const tnt_delta_config* c) {
  if (!c) return TNT_ERR_NULL;
  if (c->dtype < 0 || c->dtype > 1) return TNT_ERR_ARG;
  if (c->B <= 0 || c->H <= 0 || c->Hk <= 0 || c->H % c->Hk || c->L < 0 || c->n_seq < 0 ||
      c->d_k <= 0 || c->d_v <= 0)
    return TNT_ERR_SHAPE;
  if (c->n_seq > 0 && c->B != 1) return TNT_ERR_SHAPE;
  if (c->d_k % 8 || c->d_k > 128 || c->d_v % 8 || c->d_v > 128) return TNT_ERR_UNSUPPORTED;
  return TNT_OK;
}

struct Plan {
  int DK, dvt, nseq, nc, slots;
  size_t pitch, chunks, w_first, w_table, w_cum, w_co, w_ge, w_kf, w_kt, w_qt, w_tf, w_du, w_dr, w_ds, w_sv,
      sv_w, sv_s, saved, fwd, bwd, bwd_re;
};

constexpr int64_t MAX_THREADS = UINT32_MAX;  // of a launch

// false: does not fit the grids of the launches
bool plan_of(const tnt_delta_config* c, Plan* p) {
  p->DK = c->d_k <= 32 ? 32 : c->d_k <= 64 ? 64 : 128;
  p->dvt = (c->d_v + 15) / 16;
  p->nseq = c->n_seq ? c->n_seq : c->B;
  p->nc = (int)(((int64_t)c->L + DC - 1) / DC);
  const int64_t slots = c->n_seq ? (int64_t)c->L / DC + c->n_seq : (int64_t)c->B * p->nc;
  // threads of the passes over chunks (grads: 4 DK a key head) and of the chains
  const int64_t chunk = std::max<int64_t>(256 * (int64_t)c->H, 4 * p->DK * (int64_t)c->Hk);
  if (slots > MAX_THREADS / chunk || ((int64_t)p->nseq * c->H + 7) * p->dvt > MAX_THREADS / 256) return false;
  p->slots = (int)slots;
  p->pitch = c->d_v <= 32 ? 32 : c->d_v <= 64 ? 64 : 128;
  p->chunks = (size_t)slots * c->H;
  const bool bf = c->dtype == TNT_BF16;
  const size_t kfrag = up256((size_t)slots * c->Hk * delta_kfrag(p->DK, bf) * 2);
  size_t o = 0;
  auto take = [&](size_t n) { const size_t at = o; o += up256(n); return at; };
  p->sv_w = take(p->chunks * DC * p->pitch * 4);
  p->sv_s = take(p->chunks * p->DK * p->pitch * 4);
  p->saved = o;
  o = 0;
  p->w_first = take(c->n_seq ? (c->n_seq + 1) * sizeof(int) : 0);
  p->w_table = take(c->n_seq ? slots * sizeof(int4) : 0);
  p->w_cum = take(p->chunks * DC * sizeof(float2));
  p->w_co = take(p->chunks * DC * 3 * sizeof(float));
  p->w_ge = take(p->chunks * sizeof(float));
  p->w_kf = take(kfrag);
  p->w_kt = take(kfrag);
  p->w_tf = take(p->chunks * DELTA_TFRAG * 2);
  const size_t common = o;
  p->w_sv = take(p->saved);
  p->fwd = o;
  o = common;
  p->w_qt = take(kfrag);
  p->w_du = take(p->chunks * DC * p->pitch * 4);
  p->w_dr = take(p->chunks * DC * p->pitch * 4);
  p->w_ds = take(p->chunks * p->DK * p->pitch * 4);
  p->bwd = o;
  // recomputing: the forward's states past everything that the backward itself uses
  p->bwd_re = o + p->saved;
  return true;
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }
// read and written an element of four bytes at a time
bool split_element(const void* p) { return ((uintptr_t)p & 3u) != 0; }

// element strides of [B][heads][L][d] or, d = 0, of the gates [B][heads][L]
Str contiguous(int heads, int L, int d) {
  const int64_t e = d ? d : 1;
  return Str{(int64_t)heads * L * e, (int64_t)L * e, e};
}
Str str_of(const tnt_stride& s) { return Str{s.b, s.h, s.l}; }

// rows are read in 16-byte pieces (a tensor's extents of one element have no stride)
bool rows_misaligned(const Str& s, int B, int heads, int L, size_t elem) {
  return (B > 1 && (s.b * elem) % 16) || (heads > 1 && (s.h * elem) % 16) || (L > 1 && (s.l * elem) % 16);
}
// an output may not have two elements in one place
bool broadcast(const Str& s, int B, int heads, int L) {
  return (B > 1 && !s.b) || (heads > 1 && !s.h) || (L > 1 && !s.l);
}

// a chunk's rows are addressed by 32-bit offsets from its first
bool tokens_apart(const Str& s, int L) { return L > 1 && (s.l < 0 || s.l > (int64_t)1 << 24); }

struct Call {
  DeltaArgs a{};
  Plan p{};
  bool bf = false;
};

tnt_status begin(const tnt_delta_config* c, const tnt_delta_strides* s, bool bwd, Call* k) {
  tnt_status st = validate(c);
  if (st != TNT_OK) return st;
  if (!plan_of(c, &k->p)) return TNT_ERR_UNSUPPORTED;
  DeltaArgs& a = k->a;
  k->bf = c->dtype == TNT_BF16;
  a.B = c->B; a.H = c->H; a.Hk = c->Hk; a.per = c->H / c->Hk; a.L = c->L;
  a.d_k = c->d_k; a.d_v = c->d_v; a.scale = c->scale;
  a.DK = k->p.DK; a.dvt = k->p.dvt; a.pitch = (int)k->p.pitch; a.nseq = k->p.nseq; a.nc = k->p.nc; a.slots = k->p.slots;
  a.sq = a.sk = a.sdq = a.sdk = contiguous(c->Hk, c->L, c->d_k);
  a.sv = a.so = a.sdO = a.sdv = contiguous(c->H, c->L, c->d_v);
  a.sg = a.sl = a.sdg = a.sdl = contiguous(c->H, c->L, 0);
  if (s) {
    a.sq = str_of(s->q); a.sk = str_of(s->k); a.sv = str_of(s->v);
    a.sg = str_of(s->g); a.sl = str_of(s->lr);
    if (!bwd) {
      a.so = str_of(s->o);
    } else {
      a.sdO = str_of(s->dO); a.sdq = str_of(s->dq); a.sdk = str_of(s->dk); a.sdv = str_of(s->dv);
      a.sdg = str_of(s->dg); a.sdl = str_of(s->dlr);
    }
  }
  for (const Str* t : {&a.sq, &a.sk, &a.sv, &a.so, &a.sdO, &a.sdq, &a.sdk, &a.sdv})
    if (tokens_apart(*t, c->L)) return TNT_ERR_UNSUPPORTED;
  const size_t e = k->bf ? 2 : 4;
  if (rows_misaligned(a.sq, c->B, c->Hk, c->L, e) || rows_misaligned(a.sk, c->B, c->Hk, c->L, e) ||
      rows_misaligned(a.sv, c->B, c->H, c->L, e))
    return TNT_ERR_ALIGN;
  if (bwd) {
    if (rows_misaligned(a.sdO, c->B, c->H, c->L, e) || rows_misaligned(a.sdq, c->B, c->Hk, c->L, e) ||
        rows_misaligned(a.sdk, c->B, c->Hk, c->L, e) || rows_misaligned(a.sdv, c->B, c->H, c->L, e))
      return TNT_ERR_ALIGN;
    if (broadcast(a.sdq, c->B, c->Hk, c->L) || broadcast(a.sdk, c->B, c->Hk, c->L) ||
        broadcast(a.sdv, c->B, c->H, c->L) || broadcast(a.sdg, c->B, c->H, c->L) ||
        broadcast(a.sdl, c->B, c->H, c->L))
      return TNT_ERR_ARG;
  } else {
    if (rows_misaligned(a.so, c->B, c->H, c->L, e)) return TNT_ERR_ALIGN;
    if (broadcast(a.so, c->B, c->H, c->L)) return TNT_ERR_ARG;
  }
  return TNT_OK;
}

void place(Call* k, char* ws, char* sv, bool bwd) {
  DeltaArgs& a = k->a;
  const Plan& p = k->p;
  a.first = (int*)(ws + p.w_first);
  a.table = (int4*)(ws + p.w_table);
  a.cum = (float2*)(ws + p.w_cum);
  a.ec = (float*)(ws + p.w_co);  // the forward's, then the backward's in their place
  a.eu = a.ec + p.chunks * DC;
  a.el = a.eu + p.chunks * DC;
  a.ge = (float*)(ws + p.w_ge);
  a.KF = (__bf16*)(ws + p.w_kf);
  a.KT = (__bf16*)(ws + p.w_kt);
  a.TF = (__bf16*)(ws + p.w_tf);
  a.W = (float*)(sv + p.sv_w);
  a.S = (float*)(sv + p.sv_s);
  if (bwd) {
    a.QT = (__bf16*)(ws + p.w_qt);
    a.dU = (float*)(ws + p.w_du);
    a.dR = (float*)(ws + p.w_dr);
    a.dS = (float*)(ws + p.w_ds);
  }
}

template <typename F> hipError_t timed(const char* name, hipStream_t st, F&& f) {
  const int t = section_begin(name, st);
  const hipError_t e = f();
  section_end(t, st);
  return e;
}

#define TRY(name, x)                                                                  \
  do {                                                                                \
    if (timed(name, st, [&]() { return (x); }) != hipSuccess) return TNT_ERR_HIP;     \
  } while (0)

}  // namespace

extern "C" {

size_t tnt_delta_saved_size(const tnt_delta_config* cfg) {
  Plan p;
  return validate(cfg) == TNT_OK && plan_of(cfg, &p) ? (p.saved ? p.saved : 16) : 0;
}

size_t tnt_delta_workspace_size(const tnt_delta_config* cfg, int kind) {
  Plan p;
  if (validate(cfg) != TNT_OK || !plan_of(cfg, &p)) return 0;
  const size_t n = kind == TNT_WS_FWD || kind == TNT_WS_FWD_MIN ? p.fwd
                   : kind == TNT_WS_BWD ? p.bwd : kind == TNT_WS_BWD_RECOMPUTE ? p.bwd_re : 0;
  return n || kind < 0 || kind > TNT_WS_FWD_MIN ? n : 16;
}

tnt_status tnt_delta_fwd(const tnt_delta_config* cfg, const tnt_delta_strides* strides, const void* q,
                         const void* k, const void* v, const float* g, const float* lr,
                         const int32_t* seq_start, const float* S0, void* o, float* final_state,
                         void* saved, size_t saved_bytes, void* workspace, size_t ws_bytes,
                         void* stream) {
  Call c;
  tnt_status s = begin(cfg, strides, false, &c);
  if (s != TNT_OK) return s;
  if ((cfg->L && (!q || !k || !v || !g || !lr || !o)) || !workspace || (cfg->n_seq && !seq_start))
    return TNT_ERR_NULL;
  for (const void* p : {q, k, v, (const void*)S0, (const void*)o, (const void*)final_state,
                        (const void*)saved, (const void*)workspace})
    if (p && misaligned(p)) return TNT_ERR_ALIGN;
  for (const void* p : {(const void*)g, (const void*)lr, (const void*)seq_start})
    if (p && split_element(p)) return TNT_ERR_ALIGN;
  if (ws_bytes < (saved ? c.p.fwd - up256(c.p.saved) : c.p.fwd)) return TNT_ERR_WORKSPACE;
  if (saved && saved_bytes < c.p.saved) return TNT_ERR_WORKSPACE;
  DeltaArgs& a = c.a;
  place(&c, (char*)workspace, saved ? (char*)saved : (char*)workspace + c.p.w_sv, false);
  a.q = q; a.k = k; a.v = v; a.g = g; a.lr = lr; a.S0 = S0; a.o = o; a.fin = final_state;
  a.seq_start = cfg->n_seq ? seq_start : nullptr;
  hipStream_t st = (hipStream_t)stream;
  if (a.seq_start) TRY("delta_plan", launch_delta_plan(a, st));
  if (a.slots) TRY("delta_prep", launch_delta_prep(a, c.bf, false, st));
  TRY("delta_chain", launch_delta_chain(a, c.bf, st));
  if (a.slots) TRY("delta_out", launch_delta_out(a, c.bf, st));
  return TNT_OK;
}

tnt_status tnt_delta_bwd(const tnt_delta_config* cfg, const tnt_delta_strides* strides, const void* q,
                         const void* k, const void* v, const float* g, const float* lr,
                         const int32_t* seq_start, const float* S0, const void* dO,
                         const float* dfinal, const void* saved, size_t saved_bytes, void* dq, void* dk,
                         void* dv, float* dg, float* dlr, float* dS0, void* workspace, size_t ws_bytes,
                         void* stream) {
  Call c;
  tnt_status s = begin(cfg, strides, true, &c);
  if (s != TNT_OK) return s;
  if ((cfg->L && (!q || !k || !v || !g || !lr || !dO || !dq || !dk || !dv || !dg || !dlr)) ||
      !workspace || (cfg->n_seq && !seq_start))
    return TNT_ERR_NULL;
  for (const void* p : {q, k, v, (const void*)S0, dO, (const void*)dfinal, saved, (const void*)dq,
                        (const void*)dk, (const void*)dv, (const void*)dS0, (const void*)workspace})
    if (p && misaligned(p)) return TNT_ERR_ALIGN;
  for (const void* p : {(const void*)g, (const void*)lr, (const void*)seq_start, (const void*)dg, (const void*)dlr})
    if (p && split_element(p)) return TNT_ERR_ALIGN;
  if (ws_bytes < (saved ? c.p.bwd : c.p.bwd_re)) return TNT_ERR_WORKSPACE;
  if (saved && saved_bytes < c.p.saved) return TNT_ERR_WORKSPACE;
  DeltaArgs& a = c.a;
  place(&c, (char*)workspace, saved ? (char*)saved : (char*)workspace + c.p.bwd, true);
  a.q = q; a.k = k; a.v = v; a.g = g; a.lr = lr; a.S0 = S0; a.dO = dO; a.dfin = dfinal;
  a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.dlr = dlr; a.dS0 = dS0;
  a.seq_start = cfg->n_seq ? seq_start : nullptr;
  hipStream_t st = (hipStream_t)stream;
  if (a.seq_start) TRY("delta_plan", launch_delta_plan(a, st));
  if (!saved && a.slots) {
    TRY("delta_prep", launch_delta_prep(a, c.bf, false, st));
    TRY("delta_chain", launch_delta_chain(a, c.bf, st));
  }
  if (a.slots) {
    TRY("delta_bwd_prep", launch_delta_prep(a, c.bf, true, st));
    TRY("delta_dlocal", launch_delta_dlocal(a, c.bf, st));
  }
  TRY("delta_bwd_chain", launch_delta_bchain(a, c.bf, st));
  if (a.slots) TRY("delta_grads", launch_delta_grads(a, c.bf, st));
  return TNT_OK;
}

tnt_status tnt_delta_step(const tnt_delta_config* cfg, const tnt_delta_strides* strides, const void* q,
                          const void* k, const void* v, const float* g, const float* lr, float* state,
                          int32_t n_slots, const int32_t* slots, void* o, void* stream) {
  tnt_status s = validate(cfg);
  if (s != TNT_OK) return s;
  if (cfg->n_seq || n_slots <= 0 || (!slots && n_slots < cfg->B)) return TNT_ERR_SHAPE;
  if (cfg->L == 0) return TNT_OK;
  if (!q || !k || !v || !g || !lr || !state || !o) return TNT_ERR_NULL;
  for (const void* p : {q, k, v, (const void*)state, (const void*)o})
    if (p && misaligned(p)) return TNT_ERR_ALIGN;
  for (const void* p : {(const void*)g, (const void*)lr, (const void*)slots})
    if (p && split_element(p)) return TNT_ERR_ALIGN;
  if ((int64_t)cfg->B * cfg->H * ((cfg->d_v + 31) / 32) > MAX_THREADS / 64) return TNT_ERR_UNSUPPORTED;
  DeltaStepArgs a{};
  a.q = q; a.k = k; a.v = v; a.g = g; a.lr = lr; a.state = state; a.slot = slots; a.o = o;
  a.B = cfg->B; a.H = cfg->H; a.per = cfg->H / cfg->Hk; a.T = cfg->L;
  a.d_k = cfg->d_k; a.d_v = cfg->d_v; a.nslots = n_slots; a.scale = cfg->scale;
  a.sq = a.sk = contiguous(cfg->Hk, cfg->L, cfg->d_k);
  a.sv = a.so = contiguous(cfg->H, cfg->L, cfg->d_v);
  a.sg = a.sl = contiguous(cfg->H, cfg->L, 0);
  if (strides) {
    a.sq = str_of(strides->q); a.sk = str_of(strides->k); a.sv = str_of(strides->v);
    a.so = str_of(strides->o); a.sg = str_of(strides->g); a.sl = str_of(strides->lr);
  }
  const size_t e = cfg->dtype == TNT_BF16 ? 2 : 4;
  if (rows_misaligned(a.sq, cfg->B, cfg->Hk, cfg->L, e) || rows_misaligned(a.sk, cfg->B, cfg->Hk, cfg->L, e) ||
      rows_misaligned(a.sv, cfg->B, cfg->H, cfg->L, e) || rows_misaligned(a.so, cfg->B, cfg->H, cfg->L, e))
    return TNT_ERR_ALIGN;
  if (broadcast(a.so, cfg->B, cfg->H, cfg->L)) return TNT_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  TRY("delta_step", launch_delta_step(a, cfg->dtype == TNT_BF16, st));
  return TNT_OK;
}

}  // extern "C"
