// Host layer of the AdamW groups: context, workspace carving, the C ABI.
#include <cfloat>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "lordo_adamw.h"
#include "lordo_embed.h"
#include "lordo_kernels.h"

using namespace lordo;

namespace {

// Tensors [first, first + count) share a launch.
struct Group {
  int first = 0, count = 0;
  unsigned chunks = 0, chunks_before = 0, pieces = 0, blocks = 0;
  AwTable norm, step;           // `G`, and the chunks that the norm's `start` counts, are set by every step
  std::vector<unsigned> outer;  // first block of every tensor
  unsigned* d_outer = nullptr;
};

// A table whose gradient may be given by tokens.
struct Table {
  int tensor = 0;
  TokScratch scratch;
  TokRows rows;
};

}  // namespace

struct lordo_adamw_ctx {
  lordo_adamw_config cfg;
  std::vector<lordo_tensor> tensors;
  std::vector<AwTensor> h_tensors;
  std::vector<Group> groups;
  std::vector<Table> tables;
  std::vector<int> table_of;  // tensor -> table, or -1
  AwTensor* d_tensors = nullptr;
  double* d_partial = nullptr;
  unsigned *d_tickets = nullptr, *d_status = nullptr;
  float* d_coef = nullptr;
  size_t n_tickets = 0;
  unsigned total_chunks = 0;  // most of a worker in one step
  int piece = 0, chunk = 0;
  int64_t steps = 0, outers = 0, launches = 0;
  std::string err;
};

namespace {

int fail(lordo_adamw_ctx* c, int code, const std::string& msg) {
  if (c) c->err = msg;
  return code;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
long long cdiv(long long a, long long b) { return (a + b - 1) / b; }

int validate(const lordo_adamw_config* cfg) {
  if (!cfg || !cfg->tensors || cfg->n_tensors < 1 || cfg->K < 1 || cfg->K > 64) return LORDO_ERR_INVALID_ARG;
  auto dt_ok = [](int d) { return d == LORDO_F32 || d == LORDO_BF16; };
  if (!dt_ok(cfg->w_dtype) || !dt_ok(cfg->g_dtype)) return LORDO_ERR_INVALID_ARG;
  if (cfg->states != LORDO_STATES_F32 && cfg->states != LORDO_STATES_8BIT) return LORDO_ERR_INVALID_ARG;
  if (!(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) || !((float)cfg->eps > 0.f)) return LORDO_ERR_INVALID_ARG;
  // the reciprocal of the 8-bit step takes a subnormal denominator for 0: an element without a gradient would be 0 times infinity
  if (cfg->states == LORDO_STATES_8BIT && (float)cfg->eps < FLT_MIN) return LORDO_ERR_INVALID_ARG;
  if (cfg->clip_scope != 0 && cfg->clip_scope != 1) return LORDO_ERR_INVALID_ARG;
  if (cfg->outer != LORDO_OUTER_AVG && cfg->outer != LORDO_OUTER_NESTEROV) return LORDO_ERR_INVALID_ARG;
  long long elements = 0;
  for (int i = 0; i < cfg->n_tensors; ++i) {
    const lordo_tensor& t = cfg->tensors[i];
    if (t.n < 1 || t.row < 0 || t.max_tokens < 0) return LORDO_ERR_SHAPE;
    if (!std::isfinite(t.weight_decay)) return LORDO_ERR_INVALID_ARG;
    if (t.n > (1ll << 40)) return LORDO_ERR_UNSUPPORTED;
    if (t.row == 0 && t.max_tokens != 0) return LORDO_ERR_SHAPE;
    if (t.row > 0) {
      if (t.n % t.row != 0) return LORDO_ERR_SHAPE;
      const int rc = check_tokens(cfg->K, t.n / t.row, t.row, t.max_tokens, LORDO_I32);
      if (rc != LORDO_OK) return rc;
    }
    elements += t.n;
  }
  // blocks of a launch and partial sums are counted in 32 bits
  if ((elements / 2048 + cfg->n_tensors) * cfg->K > (1ll << 30)) return LORDO_ERR_UNSUPPORTED;
  return LORDO_OK;
}

// Lays the context's tables and workspace out; with base == nullptr only measures.
size_t build(lordo_adamw_ctx* c, const lordo_adamw_buffers* buf, char* base) {
  const lordo_adamw_config& cfg = c->cfg;
  const int nt = cfg.n_tensors, K = cfg.K;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base + off;
    off += (bytes + 255) & ~size_t(255);
    return p;
  };
  c->d_status = reinterpret_cast<unsigned*>(take(4));
  c->n_tickets = cfg.clip_scope ? (size_t)nt * K : (size_t)K;
  c->d_tickets = reinterpret_cast<unsigned*>(take(4 * c->n_tickets));
  c->d_coef = reinterpret_cast<float*>(take(4 * (size_t)nt * K));
  c->d_tensors = reinterpret_cast<AwTensor*>(take(sizeof(AwTensor) * (size_t)nt));
  c->groups.clear(); c->tables.clear(); c->h_tensors.assign(nt, AwTensor());
  c->table_of.assign(nt, -1);
  c->total_chunks = 0;
  long long elements = 0;
  for (int i = 0; i < nt; ++i) elements += cfg.tensors[i].n * K;
  c->piece = (int)aw_piece(elements);
  c->chunk = (int)sq_chunk(elements);
  for (int first = 0; first < nt; first += kAwTable) {
    c->groups.emplace_back();
    Group& g = c->groups.back();
    g.first = first;
    g.count = nt - first < kAwTable ? nt - first : kAwTable;
    for (int x = 0; x < kAwTable; ++x) g.norm.G[x] = g.step.G[x] = nullptr;
    for (int x = 0; x <= kAwTable; ++x) g.norm.start[x] = g.step.start[x] = 0;
    for (int x = 0; x < g.count; ++x) {
      const long long n = cfg.tensors[first + x].n;
      g.step.start[x] = g.pieces;
      g.outer.push_back(g.blocks);
      g.chunks += (unsigned)cdiv(n, c->chunk);
      g.pieces += (unsigned)cdiv(n, c->piece);
      g.blocks += (unsigned)cdiv(n, kAwOuter);
    }
    g.step.start[g.count] = g.pieces;
    g.outer.push_back(g.blocks);
    g.d_outer = reinterpret_cast<unsigned*>(take(4 * g.outer.size()));
    c->total_chunks += g.chunks;
  }
  c->d_partial = reinterpret_cast<double*>(take(8 * (size_t)c->total_chunks * K));
  for (int i = 0; i < nt; ++i) {
    const lordo_tensor& t = cfg.tensors[i];
    AwTensor& a = c->h_tensors[i];
    a.n = t.n; a.nb = cdiv(t.n, kAwBlock); a.wd = (float)t.weight_decay; a.index = i; a.d = t.row; a.cap = t.max_tokens;
    if (buf) {
      a.W = buf->W[i]; a.m = buf->m[i]; a.v = buf->v[i];
      if (cfg.states == LORDO_STATES_8BIT) {
        a.ms = reinterpret_cast<unsigned char*>(buf->ms[i]);
        a.vs = reinterpret_cast<unsigned char*>(buf->vs[i]);
      }
      if (cfg.sync) a.X0 = buf->X0[i];
      if (cfg.sync && cfg.outer == LORDO_OUTER_NESTEROV) a.B = buf->B[i];
    }
    if (t.row > 0) {
      c->table_of[i] = (int)c->tables.size();
      Table tb;
      tb.tensor = i;
      const size_t bytes = (size_t)tok_scratch(nullptr, K, t.n / t.row, t.row, t.max_tokens).bytes;
      tb.scratch = tok_scratch(take(bytes), K, t.n / t.row, t.row, t.max_tokens);
      tb.rows.rows = reinterpret_cast<float*>(take(4 * (size_t)K * t.max_tokens * t.row));
      tb.rows.sq = reinterpret_cast<double*>(take(8 * (size_t)K * tok_row_blocks_max(t.max_tokens, t.row)));
      tb.rows.count = reinterpret_cast<int*>(take(4));
      tb.rows.cap = t.max_tokens;
      if (t.row % 8 == 0 && t.n / 8 < (1ll << 31)) {
        const Divider by = divider((unsigned)(t.row / 8));
        a.row_mul = by.mul;
        a.row_shift = by.shift;
      }
      a.segs = tb.scratch.segs; a.rows = tb.rows.rows; a.rowsq = tb.rows.sq; a.rowsq_count = tb.rows.count;
      c->tables.push_back(tb);
    }
  }
  return off;
}

AwLaunch launch_of(const lordo_adamw_ctx* c, const Group& g, unsigned units, int piece) {
  return AwLaunch{c->d_tensors + g.first, g.count, c->cfg.K, units, c->cfg.w_dtype, c->cfg.g_dtype, c->cfg.states == LORDO_STATES_8BIT, piece};
}

int check_launch(lordo_adamw_ctx* c, const char* what) {
  const cudaError_t e = cudaPeekAtLastError();
  if (e != cudaSuccess) return fail(c, LORDO_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
  return LORDO_OK;
}

// The count of steps and the rates of a call are host values: a replayed graph would repeat the first step's.
int refuse_capture(lordo_adamw_ctx* c, cudaStream_t st) {
  cudaStreamCaptureStatus s = cudaStreamCaptureStatusNone;
  const cudaError_t e = cudaStreamIsCapturing(st, &s);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return fail(c, LORDO_ERR_CUDA, std::string("stream: ") + cudaGetErrorString(e));
  }
  if (s != cudaStreamCaptureStatusNone) return fail(c, LORDO_ERR_UNSUPPORTED, "the stream is being captured: the step count is a host value");
  return LORDO_OK;
}

int step(lordo_adamw_ctx* c, const lordo_grad* G, double lr, double beta1, double omega, const float* coef_dev, cudaStream_t st) {
  const lordo_adamw_config& cfg = c->cfg;
  for (int i = 0; i < cfg.n_tensors; ++i) {
    const lordo_grad& g = G[i];
    if (!g.tokens && !g.G) return fail(c, LORDO_ERR_INVALID_ARG, "null gradient pointer");
    if (!g.tokens) {
      if (!aligned16(g.G)) return fail(c, LORDO_ERR_ALIGN, "gradient not 16-byte aligned");
      continue;
    }
    if (c->table_of[i] < 0) return fail(c, LORDO_ERR_UNSUPPORTED, "tokens for a tensor that was declared without rows");
    if (g.T < 0 || g.T > c->tensors[i].max_tokens) return fail(c, LORDO_ERR_INVALID_ARG, "more tokens than the tensor was declared with");
    if (g.index != LORDO_I32 && g.index != LORDO_I64) return fail(c, LORDO_ERR_INVALID_ARG, "unknown token type");
    if (!g.G && g.T > 0) return fail(c, LORDO_ERR_INVALID_ARG, "null gradient pointer");
    if (misaligned(g.G, cfg.g_dtype) || misaligned_tokens(g.tokens, g.index)) return fail(c, LORDO_ERR_ALIGN, "gradient or tokens misaligned");
  }
  int rc = refuse_capture(c, st);
  if (rc != LORDO_OK) return rc;
  rc = check_launch(c, "before the step");
  if (rc != LORDO_OK) return rc;
  for (int i = 0; i < cfg.n_tensors; ++i) {
    Group& g = c->groups[i / kAwTable];
    const int x = i % kAwTable;
    g.norm.G[x] = g.step.G[x] = G[i].tokens ? nullptr : G[i].G;
    if (!G[i].tokens) continue;
    const Table& tb = c->tables[c->table_of[i]];
    const long long d = c->tensors[i].row;
    const TokProblem p = {G[i].tokens, G[i].index == LORDO_I64, cfg.K, c->tensors[i].n / d, G[i].T, d, G[i].G, cfg.g_dtype, G[i].scale};
    c->launches += tok_rows(p, tb.scratch, tb.rows, st);
  }
  const float* coef = coef_dev;
  int stride = 0;
  if (!coef && cfg.clip_rho > 0.0) {
    // a table whose gradient came by tokens has its sums of squares already: one chunk that adds them
    unsigned total = 0;
    for (Group& g : c->groups) {
      g.chunks_before = total;
      g.chunks = 0;
      for (int x = 0; x < g.count; ++x) {
        g.norm.start[x] = g.chunks;
        g.chunks += G[g.first + x].tokens ? 1u : (unsigned)cdiv(c->tensors[g.first + x].n, c->chunk);
      }
      g.norm.start[g.count] = g.chunks;
      total += g.chunks;
    }
    for (Group& g : c->groups) {
      const AwClip clip = {c->d_partial, c->chunk, total, g.chunks_before, c->d_tickets, cfg.clip_rho, cfg.clip_scope, cfg.n_tensors, c->d_coef, c->d_status};
      launch_aw_norm(launch_of(c, g, g.chunks, c->chunk), g.norm, clip, st);
      c->launches += 1;
    }
    coef = c->d_coef;
    stride = cfg.K;
  }
  const int64_t s = c->steps + 1;
  AwStep a;
  a.lr = (float)lr; a.b1 = (float)beta1; a.a1 = (float)(1.0 - beta1); a.b2 = (float)cfg.beta2; a.a2 = (float)(1.0 - cfg.beta2);
  a.omega = (float)omega; a.a_omega = (float)(1.0 - omega); a.eps = (float)cfg.eps;
  a.inv_bc1 = (float)(1.0 / (1.0 - std::pow(beta1, (double)s)));
  a.inv_bc2 = (float)(1.0 / (1.0 - std::pow(cfg.beta2, (double)s)));
  a.root_inv_bc2 = (float)std::sqrt(1.0 / (1.0 - std::pow(cfg.beta2, (double)s)));
  a.one = 1.f;
  a.key = stream_key(cfg.seed, 3, 0, s, 0);
  for (Group& g : c->groups) {
    launch_aw_step(launch_of(c, g, g.pieces, c->piece), g.step, coef, stride, a, st);
    c->launches += 1;
  }
  rc = check_launch(c, "step");
  if (rc != LORDO_OK) return rc;
  c->steps = s;
  return LORDO_OK;
}

}  // namespace

extern "C" {

int lordo_adamw_query_workspace(const lordo_adamw_config* cfg, size_t* bytes) {
  const int rc = validate(cfg);
  if (rc != LORDO_OK) return rc;
  if (!bytes) return LORDO_ERR_INVALID_ARG;
  try {
    lordo_adamw_ctx tmp;
    tmp.cfg = *cfg;
    *bytes = build(&tmp, nullptr, nullptr);
  } catch (const std::bad_alloc&) {
    return LORDO_ERR_NOMEM;
  }
  return LORDO_OK;
}

int lordo_adamw_init(const lordo_adamw_config* cfg, const lordo_adamw_buffers* buf, void* workspace, size_t workspace_bytes, void* stream,
                     lordo_adamw_ctx** out) {
  const int rc = validate(cfg);
  if (rc != LORDO_OK) return rc;
  if (!buf || !workspace || !out || !buf->W || !buf->m || !buf->v) return LORDO_ERR_INVALID_ARG;
  const bool small = cfg->states == LORDO_STATES_8BIT, nesterov = cfg->sync && cfg->outer == LORDO_OUTER_NESTEROV;
  if (small && (!buf->ms || !buf->vs)) return LORDO_ERR_INVALID_ARG;
  if ((cfg->sync && !buf->X0) || (nesterov && !buf->B)) return LORDO_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return LORDO_ERR_ALIGN;
  void* const any = reinterpret_cast<void*>(16);
  for (int i = 0; i < cfg->n_tensors; ++i) {
    const void* ptrs[7] = {buf->W[i], buf->m[i], buf->v[i], small ? buf->ms[i] : any, small ? buf->vs[i] : any, cfg->sync ? (void*)buf->X0[i] : any,
                           nesterov ? (void*)buf->B[i] : any};
    for (const void* p : ptrs) {
      if (!p) return LORDO_ERR_INVALID_ARG;
      if (!aligned16(p)) return LORDO_ERR_ALIGN;
    }
  }
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  lordo_adamw_ctx* c = nullptr;
  try {
    c = new lordo_adamw_ctx;
    c->cfg = *cfg;
    c->tensors.assign(cfg->tensors, cfg->tensors + cfg->n_tensors);
    c->cfg.tensors = c->tensors.data();
    if (build(c, buf, reinterpret_cast<char*>(workspace)) > workspace_bytes) {
      delete c;
      return LORDO_ERR_NOMEM;
    }
  } catch (const std::bad_alloc&) {
    delete c;
    return LORDO_ERR_NOMEM;
  }
  bool ok = cudaMemcpyAsync(c->d_tensors, c->h_tensors.data(), sizeof(AwTensor) * c->h_tensors.size(), cudaMemcpyHostToDevice, st) == cudaSuccess;
  ok = ok && cudaMemsetAsync(c->d_status, 0, 4, st) == cudaSuccess;
  ok = ok && cudaMemsetAsync(c->d_tickets, 0, 4 * c->n_tickets, st) == cudaSuccess;
  for (Group& g : c->groups) ok = ok && cudaMemcpyAsync(g.d_outer, g.outer.data(), 4 * g.outer.size(), cudaMemcpyHostToDevice, st) == cudaSuccess;
  if (ok) {
    launch_fill_float(c->d_coef, (long long)cfg->n_tensors * cfg->K, 1.f, st);
    for (Group& g : c->groups) launch_aw_init(launch_of(c, g, g.blocks, kAwOuter), g.d_outer, st);
    c->launches += 1 + (int64_t)c->groups.size();
    ok = cudaStreamSynchronize(st) == cudaSuccess && cudaGetLastError() == cudaSuccess;
  }
  if (!ok) {
    cudaGetLastError();
    delete c;
    return LORDO_ERR_CUDA;
  }
  *out = c;
  return LORDO_OK;
}

int lordo_adamw_step(lordo_adamw_ctx* c, const lordo_grad* G, double lr, double beta1, double omega, const float* coef_dev, void* stream) {
  if (!c) return LORDO_ERR_INVALID_ARG;
  if (!G) return fail(c, LORDO_ERR_INVALID_ARG, "G is null");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(omega >= 0.0 && omega <= 1.0)) return fail(c, LORDO_ERR_INVALID_ARG, "beta1 or omega out of range");
  return step(c, G, lr, beta1, omega, coef_dev, reinterpret_cast<cudaStream_t>(stream));
}

int lordo_adamw_outer_step(lordo_adamw_ctx* c, void* stream) {
  if (!c) return LORDO_ERR_INVALID_ARG;
  if (!c->cfg.sync) return fail(c, LORDO_ERR_STATE, "the group was made without synchronisation");
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  int rc = refuse_capture(c, st);
  if (rc != LORDO_OK) return rc;
  rc = check_launch(c, "before the synchronisation");
  if (rc != LORDO_OK) return rc;
  const AwOuter o = {c->cfg.sync_m, c->cfg.sync_v, c->cfg.outer == LORDO_OUTER_NESTEROV, (float)c->cfg.outer_lr, (float)c->cfg.outer_momentum,
                     stream_key(c->cfg.seed, 4, 0, c->outers, 0)};
  for (Group& g : c->groups) {
    launch_aw_outer(launch_of(c, g, g.blocks, kAwOuter), g.d_outer, o, st);
    c->launches += 1;
  }
  rc = check_launch(c, "outer");
  if (rc != LORDO_OK) return rc;
  c->outers += 1;
  return LORDO_OK;
}

int lordo_adamw_poll_status(lordo_adamw_ctx* c, void* stream, uint32_t* flags) {
  if (!c) return LORDO_ERR_INVALID_ARG;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  unsigned word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, c->d_status, sizeof(word), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return fail(c, LORDO_ERR_CUDA, cudaGetErrorString(e));
  if (flags) *flags = word;
  return word ? fail(c, LORDO_ERR_NUMERIC, "device flag word is non-zero") : LORDO_OK;
}

int lordo_adamw_clear_status(lordo_adamw_ctx* c, void* stream) {
  if (!c) return LORDO_ERR_INVALID_ARG;
  const cudaError_t e = cudaMemsetAsync(c->d_status, 0, sizeof(unsigned), reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? LORDO_OK : fail(c, LORDO_ERR_CUDA, cudaGetErrorString(e));
}

int lordo_adamw_get_counters(const lordo_adamw_ctx* c, int64_t out[2]) {
  if (!c || !out) return LORDO_ERR_INVALID_ARG;
  out[0] = c->steps;
  out[1] = c->outers;
  return LORDO_OK;
}

int lordo_adamw_set_counters(lordo_adamw_ctx* c, const int64_t in[2]) {
  if (!c || !in) return LORDO_ERR_INVALID_ARG;
  if (in[0] < 0 || in[1] < 0) return fail(c, LORDO_ERR_INVALID_ARG, "counter out of range");
  c->steps = in[0];
  c->outers = in[1];
  return LORDO_OK;
}

int lordo_adamw_clip_coefficients(const lordo_adamw_ctx* c, const float** device_ptr) {
  if (!c || !device_ptr) return LORDO_ERR_INVALID_ARG;
  *device_ptr = c->d_coef;
  return LORDO_OK;
}

int64_t lordo_adamw_launch_count(const lordo_adamw_ctx* c) { return c ? c->launches : -1; }
const char* lordo_adamw_last_error(const lordo_adamw_ctx* c) { return c ? c->err.c_str() : "null context"; }

int lordo_adamw_destroy(lordo_adamw_ctx* c) {
  if (!c) return LORDO_ERR_INVALID_ARG;
  delete c;
  return LORDO_OK;
}

}  // extern "C"
