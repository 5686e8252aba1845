// Whole sequences: entry points (checks, then launches) and the forward pass.
#include <algorithm>

#include "dl_prep.hpp"
#include "dl_seq.hpp"

namespace dl {
namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

template <typename K>
hipError_t start(K* kernel, int64_t grid, int block, const SeqParams& p, hipStream_t s) {
  SeqParams q = p;
  void* args[] = {&q};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(unsigned(grid)), dim3(block),
                         args, 0, s);
}

template <int DK, bool BWD, typename TIN>
hipError_t launch_prep_pass(int op, const SeqParams& p, hipStream_t s) {
  const int64_t grid = int64_t(p.max_chunks) * p.H;
  if constexpr (sizeof(TIN) == 2) {
    if (p.raw && p.delta) return start(&raw_prep_kernel<DK, true, BWD>, grid, 64, p, s);
    if (p.raw) return start(&raw_prep_kernel<DK, false, BWD>, grid, 64, p, s);
  } else {
    if (op == DL_OP_GDN) return start(&prep_kernel<DC_SCALAR, DK, true, BWD, TIN>, grid, 256, p, s);
    if (op == DL_OP_RETNET || op == DL_OP_LINATTN)
      return start(&prep_kernel<DC_SCALAR, DK, false, BWD, TIN>, grid, 256, p, s);
  }
  if (op == DL_OP_KDA) return start(&prep_kernel<DC_KEY, DK, true, BWD, TIN>, grid, 256, p, s);
  if (op == DL_OP_GLA) return start(&prep_kernel<DC_KEY, DK, false, BWD, TIN>, grid, 256, p, s);
  return start(&prep_kernel<DC_BONUS, DK, false, BWD, TIN>, grid, 256, p, s);
}
template <int DK, typename TIN>
hipError_t launch_prep(int op, const SeqParams& p, hipStream_t s) {
  return p.bwd ? launch_prep_pass<DK, true, TIN>(op, p, s) : launch_prep_pass<DK, false, TIN>(op, p, s);
}

template <int DK, bool RAW, bool DELTA, typename TIN>
hipError_t launch_walk(const SeqParams& p, hipStream_t s) {
  const int64_t heads = int64_t(p.n) * p.H, tiles = p.dv / 16;
  if (p.seg_len) {
    // columns of values and of M, four tiles a workgroup: one workgroup is of one kind
    const int64_t segs = int64_t(p.segs) * p.H, cols = tiles + (DELTA ? DK / 16 : 0);
    hipError_t e = start(&forward_kernel<DK, 1, 4, RAW, DELTA, PASS_SEG, TIN>, segs * (cols / 4), 256, p, s);
    if (e == hipSuccess) e = start(&join_kernel<DK, RAW, DELTA>, heads * tiles, 4 * DK, p, s);
    if (e != hipSuccess) return e;
    return start(&forward_kernel<DK, 1, 4, RAW, DELTA, PASS_OUT, TIN>, segs * (tiles / 4), 256, p, s);
  }
  int waves = walk_waves(heads, DK, p.dv, RAW);
  // Delta-rule heads of 128 keys with planes: two waves' registers do not hold a chunk on its way to LDS
  // beside what they compute with, and four take the same time (fp32, 2 to 64 heads of 1024 tokens).
  constexpr bool TWO = !(DK == 128 && DELTA && !RAW);
  if (!TWO && waves == 2) waves = 4;
  const int64_t grid = heads * (tiles / waves);
  switch (waves) {
    case 2:
      if constexpr (TWO) return start(&forward_kernel<DK, 1, 2, RAW, DELTA, PASS_OUT, TIN>, grid, 128, p, s);
      return hipErrorInvalidValue;
    case 4: return start(&forward_kernel<DK, 1, 4, RAW, DELTA, PASS_OUT, TIN>, grid, 256, p, s);
    default: return start(&forward_kernel<DK, 1, 8, RAW, DELTA, PASS_OUT, TIN>, grid, 512, p, s);
  }
}

template <int DK, typename TIN>
hipError_t launch_forward_shape(int op, const SeqParams& p, hipStream_t s) {
  const hipError_t e = launch_prep<DK, TIN>(op, p, s);
  if (e != hipSuccess || p.bwd) return e;         // the backward pass has its walks elsewhere
  if constexpr (sizeof(TIN) == 2)
    if (p.raw) return p.delta ? launch_walk<DK, true, true, TIN>(p, s) : launch_walk<DK, true, false, TIN>(p, s);
  return p.delta ? launch_walk<DK, false, true, TIN>(p, s) : launch_walk<DK, false, false, TIN>(p, s);
}

}  // namespace

hipError_t launch_forward(const dl_desc* d, const SeqParams& p, hipStream_t s) {
  if (d->in_dtype == DL_BF16)
    return d->dk == 128 ? launch_forward_shape<128, uint16_t>(d->op, p, s)
                        : launch_forward_shape<64, uint16_t>(d->op, p, s);
  return d->dk == 128 ? launch_forward_shape<128, float>(d->op, p, s)
                      : launch_forward_shape<64, float>(d->op, p, s);
}

namespace {

int check_counts(const dl_desc* d, int32_t n, int32_t tokens) {
  if (n < 0 || tokens < 0 || n > d->num_slots) return DL_E_SHAPE;
  if (d->heads > DL_MAX_HEADS) return DL_E_SHAPE;   // a chunk's rows lie within 32-bit offsets
  // Grids of one workgroup per (chunk, head) and per (sequence, head, 16 value columns).
  const int64_t chunks = int64_t(tokens) / DL_CHUNK + n;
  if (chunks * d->heads > int64_t(0x7fffffff)) return DL_E_SHAPE;
  if (int64_t(n) * d->heads * (d->dv / 16) > int64_t(0x7fffffff)) return DL_E_SHAPE;
  return DL_OK;
}

// bf16 keys and queries with one log-decay per head or none are operands as they are.
bool raw_planes(const dl_desc* d) {
  return d->in_dtype == DL_BF16 &&
         (d->op == DL_OP_GDN || d->op == DL_OP_RETNET || d->op == DL_OP_LINATTN);
}

// The descriptor's own checks are those of a call that drives no rows.
int check_desc_only(const dl_desc* d) { return dl_readout(d, nullptr, nullptr, nullptr, nullptr, 0, nullptr); }

bool is_delta(const dl_desc* d) { return d->op == DL_OP_GDN || d->op == DL_OP_KDA; }

// Workspace: the chunk blocks, then the segment states.
size_t block_bytes(const dl_desc* d, int32_t n, int32_t tokens, bool backward) {
  const WsLayout w{d->dk, d->dv, raw_planes(d), backward};
  return size_t(w.block()) * size_t(tokens / DL_CHUNK + n) * size_t(d->heads);
}
size_t seg_bytes(const dl_desc* d, int32_t n, int32_t tokens) {
  const SegPlan s = seg_plan(n, tokens, d->heads, d->dv, is_delta(d));
  return s.len ? size_t(s.segs) * d->heads * seg_floats(d->dk, d->dv, is_delta(d)) * sizeof(float) : 0;
}

SeqParams params(const dl_desc* d, const void* S_in, const dl_token* tok, const dl_tables* t,
                 int32_t n, int32_t tokens, void* ws) {
  SeqParams p{};
  p.S_in = S_in;
  p.q = tok->q;
  p.k = tok->k;
  p.v = tok->v;
  p.delta = is_delta(d);
  p.beta = p.delta ? tok->beta : nullptr;
  p.lam = d->op == DL_OP_LINATTN ? nullptr : tok->lam;
  p.u = d->op == DL_OP_RWKV6 ? tok->u : nullptr;
  p.cu_tokens = t->cu_tokens;
  p.cu_chunks = t->cu_chunks;
  p.chunks = t->chunks;
  p.seq_slot = t->seq_slot;
  p.order = t->order;
  p.ws = static_cast<unsigned char*>(ws);
  p.n = n;
  p.N = tokens;
  p.B = d->num_slots;
  p.H = d->heads;
  p.dv = d->dv;
  p.max_chunks = tokens / DL_CHUNK + n;
  p.state_bf16 = d->state_dtype == DL_BF16;
  p.raw = raw_planes(d);
  return p;
}

}  // namespace
}  // namespace dl

#define DL_TRY(x)                 \
  do {                            \
    const int rc_ = (x);          \
    if (rc_ != DL_OK) return rc_; \
  } while (0)

extern "C" {

int dl_chunk_tables(const int32_t* lens, const int32_t* slots, int32_t n, int32_t tokens,
                    int32_t num_slots, const dl_tables* t, int32_t* err, hipStream_t stream) {
  if (n < 0 || tokens < 0 || num_slots < 1) return DL_E_SHAPE;
  if (int64_t(tokens) / DL_CHUNK + n > int64_t(0x7fffffff)) return DL_E_SHAPE;
  if (n == 0) return DL_OK;
  if (!slots && n > num_slots) return DL_E_SHAPE;
  if (!lens || !t || !t->cu_tokens || !t->cu_chunks || !t->chunks || !t->seq_slot || !t->order)
    return DL_E_NULL;
  if (tokens > 0 && !t->row_slot) return DL_E_NULL;
  if (!dl::aligned(lens, 4) || !dl::aligned(slots, 4) || !dl::aligned(t->cu_tokens, 4) ||
      !dl::aligned(t->cu_chunks, 4) || !dl::aligned(t->chunks, 16) ||
      !dl::aligned(t->row_slot, 4) || !dl::aligned(t->seq_slot, 4) || !dl::aligned(t->order, 4) ||
      !dl::aligned(err, 4))
    return DL_E_ALIGN;
  const hipError_t e = dl::launch_tables(lens, slots, n, tokens, num_slots, *t, err,
                                         tokens / DL_CHUNK + n, stream);
  return e == hipSuccess ? DL_OK : DL_E_HIP;
}

int dl_prefill_workspace_bytes(const dl_desc* desc, int32_t n, int32_t tokens, int32_t backward,
                               size_t* bytes) {
  DL_TRY(dl::check_desc_only(desc));
  DL_TRY(dl::check_counts(desc, n, tokens));
  if (!bytes) return DL_E_NULL;
  size_t most = dl::block_bytes(desc, n, tokens, false) + dl::seg_bytes(desc, n, tokens);
  if (backward) most = std::max(most, dl::block_bytes(desc, n, tokens, true));
  *bytes = most;
  return DL_OK;
}

int dl_prefill(const dl_desc* desc, const void* S_in, void* S_out, const dl_token* tok, void* o,
               const dl_tables* tables, int32_t n, int32_t tokens, void* workspace,
               size_t workspace_bytes, hipStream_t stream) {
  DL_TRY(dl::check_desc_only(desc));
  DL_TRY(dl::check_counts(desc, n, tokens));
  if (n == 0) return DL_OK;               // nothing to do, whatever the other pointers are
  DL_TRY(dl::check_sequences(desc, tok, tables, n, tokens, workspace, workspace_bytes, false));
  if (!S_out || (tokens > 0 && !o)) return DL_E_NULL;
  if (!dl::aligned(S_in, 16) || !dl::aligned(S_out, 16) || !dl::aligned(o, 16)) return DL_E_ALIGN;
  dl::SeqParams p = dl::params(desc, S_in, tok, tables, n, tokens, workspace);
  p.S_out = S_out;
  p.o = o;
  const dl::SegPlan seg = dl::seg_plan(n, tokens, desc->heads, desc->dv, p.delta);
  p.seg_len = seg.len;
  p.segs = seg.segs;
  p.seg = reinterpret_cast<float*>(p.ws + dl::block_bytes(desc, n, tokens, false));
  return dl::launch_forward(desc, p, stream) == hipSuccess ? DL_OK : DL_E_HIP;
}

int dl_prefill_backward(const dl_desc* desc, const void* S_in, const dl_token* tok,
                        const void* d_o, const void* dS_out, const dl_grads* g,
                        const dl_tables* tables, int32_t n, int32_t tokens, void* workspace,
                        size_t workspace_bytes, hipStream_t stream) {
  DL_TRY(dl::check_desc_only(desc));
  DL_TRY(dl::check_counts(desc, n, tokens));
  if (n == 0) return DL_OK;               // nothing to do, whatever the other pointers are
  DL_TRY(dl::check_sequences(desc, tok, tables, n, tokens, workspace, workspace_bytes, true));
  if (!g || (tokens > 0 && (!d_o || !g->dq || !g->dk || !g->dv))) return DL_E_NULL;
  dl::SeqParams p = dl::params(desc, S_in, tok, tables, n, tokens, workspace);
  if (tokens > 0 && ((p.delta && !g->dbeta) || (p.lam && !g->dlam))) return DL_E_NULL;
  if (p.u && !g->du) return DL_E_NULL;
  if (!dl::aligned(S_in, 16) || !dl::aligned(d_o, 16) || !dl::aligned(dS_out, 16) ||
      !dl::aligned(g->dq, 16) || !dl::aligned(g->dk, 16) || !dl::aligned(g->dv, 16) ||
      !dl::aligned(g->dS, 16) || !dl::aligned(g->dbeta, 4) || !dl::aligned(g->dlam, 4) ||
      !dl::aligned(g->du, 4))
    return DL_E_ALIGN;
  p.bwd = true;
  p.d_o = d_o;
  p.dS_out = dS_out;
  p.S_out = g->dS;
  p.dq = g->dq;
  p.dk_ = g->dk;
  p.dv_ = g->dv;
  p.dbeta = p.delta ? g->dbeta : nullptr;
  p.dlam = p.lam ? g->dlam : nullptr;
  p.du = p.u ? g->du : nullptr;
  if (dl::launch_forward(desc, p, stream) != hipSuccess) return DL_E_HIP;   // the operands
  return dl::launch_backward(desc, p, stream) == hipSuccess ? DL_OK : DL_E_HIP;
}

}  // extern "C"
