// attn.hip -- C-ABI of decoding on a translated cache (kvx_attn.h): argument
// checks, launches, and the kernel that rotates and stores new tokens.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <memory>
#include <new>

#include "attn.h"

using namespace kvx;

namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr double kLog2e = 1.4426950408889634;

// Whether a positive number is a normal one in fp32.
bool normal(double x) {
  return x >= std::numeric_limits<float>::min() && x <= std::numeric_limits<float>::max();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int elem_size(const kvx_attn* at) { return at->dtype == KVX_F32 ? 4 : 2; }

bool fault_injected() {
  const char* f = std::getenv("KVX_FAULT");
  return f && std::strcmp(f, "launch") == 0;
}

bool validating() {
  const char* v = std::getenv("KVX_VALIDATE");
  return v && v[0] == '1';
}

// A cache's pointers, strides and capacity, checked; the layer is applied to
// the base pointers.
kvx_status prepare_cache(const kvx_attn* at, const kvx_cache& in, int32_t batch, int32_t layer,
                         CacheArgs& c) {
  if (!in.k || !in.v) return KVX_EINVAL;
  const bool paged = in.block_table != nullptr;
  if (paged ? in.block_size <= 0 || in.max_blocks <= 0 || in.num_blocks <= 0 : in.capacity <= 0)
    return KVX_EINVAL;
  const int64_t heads = at->model.n_kv_heads, d = at->model.head_dim;
  const int64_t run = paged ? in.block_size : in.capacity;  // rows per block and head
  int64_t s[4];
  for (int i = 0; i < 4; ++i) s[i] = in.stride[i];
  if (!s[0] && !s[1] && !s[2] && !s[3]) {
    s[3] = d;
    s[2] = d * run;
    s[1] = heads * s[2];
    s[0] = (paged ? int64_t(in.num_blocks) : int64_t(batch)) * s[1];
  }
  for (int i = 0; i < 4; ++i)
    if (s[i] < 0) return KVX_ESHAPE;
  if (s[3] < d && run > 1) return KVX_ESHAPE;
  const int es = elem_size(at);
  if (!aligned16(in.k) || !aligned16(in.v)) return KVX_EUNSUPPORTED;
  for (int i = 0; i < 4; ++i)
    if (s[i] * es % 16) return KVX_EUNSUPPORTED;
  const int64_t cap = paged ? int64_t(in.max_blocks) * in.block_size : in.capacity;
  if (cap > INT32_MAX / 2) return KVX_ESHAPE;
  c.k = static_cast<char*>(in.k) + layer * s[0] * es;
  c.v = static_cast<char*>(in.v) + layer * s[0] * es;
  c.sl = s[0];
  c.sb = s[1];
  c.sh = s[2];
  c.st = s[3];
  c.table = in.block_table;
  c.max_blocks = paged ? in.max_blocks : 1;
  c.capacity = static_cast<int32_t>(cap);
  c.bs = fast_div(paged ? in.block_size : in.capacity);
  c.run = 64;
  while (paged && in.block_size % c.run) c.run /= 2;
  if (s[3] * es >= (int64_t(1) << 25)) c.run = 1;
  return KVX_OK;
}

// The polynomial of tanh(y) / y in y^2 below 0.5, for scores of dot products.  No
// range where a coefficient is past fp32 (caps far below a score's scale).
void near_cap(const kvx_attn* at, AttnArgs& a) {
  constexpr double c[4] = {-0.3333314389628958, 0.1332587895825113, -0.053045494297645907,
                           0.017241491495620133};
  const double y = at->scale / at->softcap;
  double factor = at->scale * kLog2e;
  a.near = static_cast<float>(0.5 / y);
  for (int i = 0; i < 4; ++i) {
    factor *= y * y;
    a.near_c[i] = static_cast<float>(c[i] * factor);
    if (!std::isfinite(a.near_c[i])) a.near = 0.f;
  }
}

// Rows of a new tensor: (row, head) strides of `heads` head vectors.
kvx_status check_rows(const kvx_attn* at, const void* p, const int64_t* s, int64_t heads,
                      int64_t rows) {
  const int64_t d = at->model.head_dim;
  if (s[0] < 0 || s[1] < 0) return KVX_ESHAPE;
  if ((heads > 1 && s[1] < d) || (rows > 1 && s[0] < d)) return KVX_ESHAPE;
  const int es = elem_size(at);
  if (!aligned16(p) || s[0] * es % 16 || s[1] * es % 16) return KVX_EUNSUPPORTED;
  return KVX_OK;
}

// Fields that append, forward and mass share; rows == 0 leaves nothing to do.
kvx_status prepare(const kvx_attn* at, const kvx_attn_io* io, AttnArgs& a) {
  if (!at || !io) return KVX_EINVAL;
  if (io->batch < 0 || io->rows < 0 || io->layer < 0 || io->layer >= at->model.n_layers ||
      io->window < 0)
    return KVX_EINVAL;
  a.batch = io->batch;
  a.rows = io->rows;
  if (io->batch == 0 && io->rows > 0) return KVX_ESHAPE;
  if (!io->q_start && io->rows != io->batch) return KVX_ESHAPE;
  if (io->batch == 0) return KVX_OK;
  if (io->rows > 0 && io->max_new < 1) return KVX_EINVAL;
  if (int64_t(io->rows) * at->n_heads > INT32_MAX / 2 || io->batch > (1 << 20)) return KVX_ESHAPE;
  if (!io->tokens) return KVX_EINVAL;
  kvx_status s = prepare_cache(at, io->cache, io->batch, io->layer, a.c);
  if (s != KVX_OK) return s;
  a.q_start = io->q_start;
  a.tokens = io->tokens;
  a.prefix = io->prefix;
  a.pos = io->pos;
  a.hq = at->n_heads;
  a.hkv = at->model.n_kv_heads;
  a.group = at->group;
  a.by_group = fast_div(at->group);
  a.d = at->model.head_dim;
  a.window = io->window;
  a.scale2 = static_cast<float>(at->scale * kLog2e);
  a.cap2 = static_cast<float>(at->softcap * kLog2e);
  if (at->softcap > 0.0) near_cap(at, a);
  a.tanh2 = at->softcap > 0.0 ? static_cast<float>(2.0 * at->scale / at->softcap * kLog2e) : 0.f;
  a.q = static_cast<const char*>(io->q);
  a.q_sr = io->q_stride[0];
  a.q_sh = io->q_stride[1];
  return KVX_OK;
}

template <typename T>
kvx_status fetch(std::unique_ptr<T[]>& host, const T* dev, size_t n) {
  host.reset(new (std::nothrow) T[n > 0 ? n : 1]);
  if (!host) return KVX_ENOMEM;
  return hip_status(hipMemcpy(host.get(), dev, n * sizeof(T), hipMemcpyDeviceToHost));
}

// KVX_VALIDATE=1: lengths, row ranges, prefixes and the block ids of the slots
// that a call may touch (those of a window's reach, when it has one).
kvx_status validate(const kvx_attn_io* io, const AttnArgs& a, bool reads_cache, hipStream_t st) {
  if (!validating()) return KVX_OK;
  kvx_status s = hip_status(hipStreamSynchronize(st));
  if (s != KVX_OK) return s;
  std::unique_ptr<int32_t[]> qs, tok, pre, tab;
  s = fetch(tok, io->tokens, io->batch);
  if (s != KVX_OK) return s;
  if (io->q_start) {
    s = fetch(qs, io->q_start, size_t(io->batch) + 1);
    if (s != KVX_OK) return s;
    if (qs[0] != 0 || qs[io->batch] != io->rows) return KVX_EDATA;
  }
  if (reads_cache && io->prefix) {
    s = fetch(pre, io->prefix, io->batch);
    if (s != KVX_OK) return s;
  }
  const kvx_cache& c = io->cache;
  if (c.block_table) {
    s = fetch(tab, c.block_table, size_t(io->batch) * c.max_blocks);
    if (s != KVX_OK) return s;
  }
  for (int64_t b = 0; b < io->batch; ++b) {
    const int32_t m = qs ? qs[b + 1] - qs[b] : 1, n = tok[b];
    if (m < 0 || n < 0 || n > a.c.capacity || (pre && pre[b] < 0)) return KVX_EDATA;
    if (a.mass && n > a.mass_capacity) return KVX_EDATA;
    if (!tab || m == 0) continue;
    int64_t lo = n - m;
    if (reads_cache) lo = io->window ? lo - io->window + 1 : 0;
    for (int64_t j = (lo > 0 ? lo : 0) / c.block_size; j * c.block_size < n; ++j) {
      const int32_t id = tab[b * c.max_blocks + j];
      if (id < 0 || id >= c.num_blocks) return KVX_EDATA;
    }
  }
  return KVX_OK;
}

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------

// The context of a row: the last whose first row is not after it.
__device__ __forceinline__ int context_of(const AttnArgs& a, int row) {
  if (!a.q_start) return row;
  int lo = 0, hi = a.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.q_start[mid] <= row)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

struct AppendArgs {
  AttnArgs a;
  const double* freq;
  const uint8_t* axis;
  const char* in[3];     // new q, k, v (NULL: none)
  int64_t sr[3], sh[3];  // their strides
  char* q_out;
};

// One 16-byte piece of a head vector.
template <typename T>
struct Piece {
  static constexpr int n = 16 / sizeof(T);
  T x[n];
};

// (x_e, x_{e+D/2}) turned by pos[axis e] * f_e, to the cache or q.  Bound by
// memory: a row is read and written once, with few operations.  One thread: a
// row, 16 bytes of first pair members and the 16 bytes of their partners, of
// every `heads_step`-th head.  The angles (64 bits) are formed once and turn all
// of the thread's heads; heads are shared out only until the card has four
// workgroups a compute unit, so one token's heads turn side by side.
// Measured: 18.6k tokens of 8 contexts, heads 28 / 4 x 128, 3 axes, 350 MB in
// 80 us, 4.4 TB/s; one token 8.3 us, its launch and the latency of three
// dependent loads (lengths, block, row).
template <typename T>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs g, int pieces, int heads_step) {
  constexpr int N = Piece<T>::n;
  const AttnArgs& a = g.a;
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = id / pieces;
  const int e0 = static_cast<int>(id % pieces) * N;
  if (row >= a.rows) return;
  const int b = context_of(a, static_cast<int>(row));
  const Context c = context(a, b);
  const int slot = c.p0 + static_cast<int>(row) - c.q0;
  const int half = a.d / 2;
  float cs[N], sn[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = a.pos ? a.pos[g.axis[e0 + i] * static_cast<int64_t>(a.rows) + row] : slot;
    rope_cs(g.freq[e0 + i], p, cs[i], sn[i]);
  }
  const bool stored = slot >= 0 && slot < a.c.capacity && row < c.q0 + c.m;
  const int64_t at = stored ? cache_offset(a.c, cache_block(a.c, b, slot), slot) : 0;
  const int nq = g.in[0] ? a.hq : 0, nk = g.in[1] ? a.hkv : 0;
  for (int h = blockIdx.y; h < nq + 2 * nk; h += heads_step) {
    const int which = h < nq ? 0 : h < nq + nk ? 1 : 2;
    if (which > 0 && !stored) continue;
    const int hh = h - (which == 0 ? 0 : which == 1 ? nq : nq + nk);
    const T* src = reinterpret_cast<const T*>(g.in[which]) + row * g.sr[which] +
                   hh * g.sh[which] + e0;
    T* dst = which == 0 ? reinterpret_cast<T*>(g.q_out) + row * a.q_sr + hh * a.q_sh + e0
                        : reinterpret_cast<T*>(which == 1 ? a.c.k : a.c.v) + at + hh * a.c.sh + e0;
    Piece<T> x = *reinterpret_cast<const Piece<T>*>(src);
    Piece<T> y = *reinterpret_cast<const Piece<T>*>(src + half);
    if (which < 2) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float u = load_f32<T>(&x.x[i]), w = load_f32<T>(&y.x[i]);
        x.x[i] = store_cvt<T>(u * cs[i] - w * sn[i]);
        y.x[i] = store_cvt<T>(w * cs[i] + u * sn[i]);
      }
    }
    *reinterpret_cast<Piece<T>*>(dst) = x;
    *reinterpret_cast<Piece<T>*>(dst + half) = y;
  }
}

}  // namespace

extern "C" {

kvx_status kvx_attn_create(const kvx_attn_desc* d, kvx_attn** out) {
  if (out) *out = nullptr;
  if (!d || !out) return KVX_EINVAL;
  const kvx_model& m = d->model;
  if (m.n_layers <= 0 || m.n_kv_heads <= 0 || m.head_dim <= 0 || !std::isfinite(m.rope_base) ||
      d->n_heads <= 0 || d->n_heads % m.n_kv_heads || d->n_axes < 1 || d->n_axes > 4 ||
      (d->dtype != KVX_F32 && d->dtype != KVX_BF16) || !std::isfinite(d->scale) || d->scale < 0.0 ||
      !std::isfinite(d->softcap) || d->softcap < 0.0)
    return KVX_EINVAL;
  if (m.head_dim % 16 || m.head_dim > 256) return KVX_EUNSUPPORTED;
  // what the kernels take in fp32 (prepare) is there neither infinite nor zero
  const double scale = d->scale > 0.0 ? d->scale : 1.0 / std::sqrt(double(m.head_dim));
  if (!normal(scale * kLog2e) ||
      (d->softcap > 0.0 && (!normal(d->softcap * kLog2e) || !normal(2.0 * scale / d->softcap * kLog2e))))
    return KVX_EINVAL;
  const int half = m.head_dim / 2;
  for (int i = 0; i < half; ++i) {
    if (m.inv_freq && !std::isfinite(m.inv_freq[i])) return KVX_EINVAL;
    if (d->pair_axis && d->pair_axis[i] >= d->n_axes) return KVX_EINVAL;
  }
  kvx_attn* at = new (std::nothrow) kvx_attn();
  if (!at) return KVX_ENOMEM;
  at->model = m;
  at->model.inv_freq = nullptr;
  at->n_heads = d->n_heads;
  at->group = d->n_heads / m.n_kv_heads;
  at->dtype = d->dtype;
  at->scale = scale;
  at->softcap = d->softcap;
  at->n_axes = d->n_axes;
  // [128] revolutions per position, then [128] axes
  struct Tables {
    double freq[128];
    uint8_t axis[128];
  } host{};
  for (int i = 0; i < half; ++i) {
    const double th = m.inv_freq           ? m.inv_freq[i]
                      : m.rope_base > 0.0  ? std::pow(m.rope_base, -2.0 * i / m.head_dim)
                                           : 0.0;
    host.freq[i] = th / kTwoPi;
    host.axis[i] = d->pair_axis ? d->pair_axis[i] : 0;
  }
  hipError_t e = hipGetDevice(&at->device);
  if (e == hipSuccess)
    e = hipDeviceGetAttribute(&at->n_cu, hipDeviceAttributeMultiprocessorCount, at->device);
  if (e == hipSuccess) e = hipMalloc(&at->tables, sizeof(Tables));
  if (e == hipSuccess) e = hipMemcpy(at->tables, &host, sizeof(Tables), hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    const kvx_status s = hip_status(e);
    kvx_attn_destroy(at);
    return s;
  }
  at->freq = static_cast<const double*>(at->tables);
  at->axis = static_cast<const uint8_t*>(at->tables) + offsetof(Tables, axis);
  *out = at;
  return KVX_OK;
}

void kvx_attn_destroy(kvx_attn* at) {
  if (!at) return;
  if (at->tables) (void)hipFree(at->tables);
  delete at;
}

kvx_status kvx_attn_append(const kvx_attn* at, const kvx_attn_io* io, void* stream) {
  AppendArgs g{};
  kvx_status s = prepare(at, io, g.a);
  if (s != KVX_OK) return s;
  if (!io->new_k != !io->new_v || (!io->new_q && !io->new_k)) return KVX_EINVAL;
  if (io->rows == 0 || io->batch == 0) return KVX_OK;
  const int64_t heads[3] = {at->n_heads, at->model.n_kv_heads, at->model.n_kv_heads};
  const void* in[3] = {io->new_q, io->new_k, io->new_v};
  const int64_t* str[3] = {io->new_q_stride, io->new_k_stride, io->new_v_stride};
  for (int i = 0; i < 3; ++i) {
    g.in[i] = static_cast<const char*>(in[i]);
    if (!in[i]) continue;
    s = check_rows(at, in[i], str[i], heads[i], io->rows);
    if (s != KVX_OK) return s;
    g.sr[i] = str[i][0];
    g.sh[i] = str[i][1];
  }
  if (io->new_q) {
    if (!io->q) return KVX_EINVAL;
    s = check_rows(at, io->q, io->q_stride, at->n_heads, io->rows);
    if (s != KVX_OK) return s;
    g.q_out = static_cast<char*>(io->q);
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  s = validate(io, g.a, false, st);
  if (s != KVX_OK) return s;
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  g.freq = at->freq;
  g.axis = at->axis;
  const int pieces = at->model.head_dim / 2 * elem_size(at) / 16;
  const int total_heads = (io->new_q ? at->n_heads : 0) + (io->new_k ? 2 * at->model.n_kv_heads : 0);
  const int64_t groups = (int64_t(io->rows) * pieces + 255) / 256;
  int split = 1;
  while (split < total_heads && groups * split < 4 * at->n_cu) ++split;
  const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>(split));
  return hip_status(at->dtype == KVX_F32
                        ? launch_on(append_kernel<float>, grid, dim3(256), st, g, pieces, split)
                        : launch_on(append_kernel<bf16_t>, grid, dim3(256), st, g, pieces, split));
}

kvx_status kvx_attn_workspace_bytes(const kvx_attn* at, size_t* bytes) {
  if (bytes) *bytes = 0;
  if (!at || !bytes) return KVX_EINVAL;
  *bytes = forward_workspace(at);
  return KVX_OK;
}

kvx_status kvx_attn_forward(const kvx_attn* at, const kvx_attn_io* io, void* workspace,
                            size_t workspace_bytes, void* stream) {
  AttnArgs a{};
  kvx_status s = prepare(at, io, a);
  if (s != KVX_OK) return s;
  if (io->rows == 0 || io->batch == 0) return KVX_OK;
  if (!io->q || !io->out || !workspace || !aligned16(workspace)) return KVX_EINVAL;
  if (workspace_bytes < forward_workspace(at)) return KVX_ESHAPE;
  s = check_rows(at, io->q, io->q_stride, at->n_heads, io->rows);
  if (s != KVX_OK) return s;
  s = check_rows(at, io->out, io->out_stride, at->n_heads, io->rows);
  if (s != KVX_OK) return s;
  a.out = static_cast<char*>(io->out);
  a.o_sr = io->out_stride[0];
  a.o_sh = io->out_stride[1];
  a.lse = io->lse;
  hipStream_t st = static_cast<hipStream_t>(stream);
  s = validate(io, a, true, st);
  if (s != KVX_OK) return s;
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  return hip_status(launch_forward(at, a, io->max_new, workspace, st));
}

kvx_status kvx_attn_mass(const kvx_attn* at, const kvx_attn_io* io, void* stream) {
  AttnArgs a{};
  kvx_status s = prepare(at, io, a);
  if (s != KVX_OK) return s;
  if (io->batch == 0) return KVX_OK;
  if (!io->mass || io->mass_capacity <= 0) return KVX_EINVAL;
  if (io->mass_capacity > INT32_MAX / 2) return KVX_ESHAPE;
  if (io->rows > 0) {
    if (!io->q || !io->lse) return KVX_EINVAL;
    s = check_rows(at, io->q, io->q_stride, at->n_heads, io->rows);
    if (s != KVX_OK) return s;
  }
  a.lse = io->lse;
  a.mass_in = io->mass_in;
  a.mass = io->mass;
  a.mass_capacity = io->mass_capacity;
  hipStream_t st = static_cast<hipStream_t>(stream);
  s = validate(io, a, true, st);
  if (s != KVX_OK) return s;
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  return hip_status(launch_mass(at, a, io->max_new, st));
}

kvx_status kvx_attn_evict(const kvx_attn* at, const kvx_evict_io* io, void* stream) {
  if (!at || !io) return KVX_EINVAL;
  if (io->batch < 0 || io->keep < 1 || io->sink < 0 || io->recent < 0) return KVX_EINVAL;
  if (io->batch == 0) return KVX_OK;
  if (int64_t(io->sink) + io->recent > io->keep || io->mass_capacity <= 0) return KVX_EINVAL;
  if (!io->tokens || !io->mass || !io->kept || io->tokens_out == io->tokens) return KVX_EINVAL;
  EvictArgs a{};
  kvx_status s = prepare_cache(at, io->src, io->batch, 0, a.src);
  if (s != KVX_OK) return s;
  a.in_place = io->dst.k == nullptr;
  if (a.in_place) {
    a.dst = a.src;
  } else {
    if (io->dst.k == io->src.k || io->dst.v == io->src.v) return KVX_EINVAL;
    s = prepare_cache(at, io->dst, io->batch, 0, a.dst);
    if (s != KVX_OK) return s;
    if (a.dst.capacity < io->keep && a.dst.capacity < a.src.capacity) return KVX_ESHAPE;
  }
  if (io->mass_capacity > INT32_MAX / 2) return KVX_ESHAPE;
  a.tokens = io->tokens;
  a.layers = at->model.n_layers;
  a.batch = io->batch;
  a.heads = at->model.n_kv_heads;
  a.row_bytes = at->model.head_dim * elem_size(at);
  if (int64_t(a.layers) * a.batch * a.heads > INT32_MAX / 16) return KVX_ESHAPE;
  a.keep = io->keep;
  a.sink = io->sink;
  a.recent = io->recent;
  a.mass = io->mass;
  a.mass_out = io->mass_out;
  a.mass_capacity = io->mass_capacity;
  a.kept = io->kept;
  a.tokens_out = io->tokens_out;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validating()) {
    s = hip_status(hipStreamSynchronize(st));
    if (s != KVX_OK) return s;
    std::unique_ptr<int32_t[]> tok, tab[2];
    s = fetch(tok, io->tokens, io->batch);
    if (s != KVX_OK) return s;
    const kvx_cache* cs[2] = {&io->src, a.in_place ? &io->src : &io->dst};
    for (int i = 0; i < 2; ++i)
      if (cs[i]->block_table) {
        s = fetch(tab[i], cs[i]->block_table, size_t(io->batch) * cs[i]->max_blocks);
        if (s != KVX_OK) return s;
      }
    for (int64_t b = 0; b < io->batch; ++b) {
      const int32_t n = tok[b];
      if (n < 0 || n > a.src.capacity || n > io->mass_capacity) return KVX_EDATA;
      const int64_t used[2] = {n, n < io->keep ? n : io->keep};
      for (int i = 0; i < 2; ++i)
        for (int64_t j = 0; tab[i] && j * cs[i]->block_size < used[i]; ++j) {
          const int32_t id = tab[i][b * cs[i]->max_blocks + j];
          if (id < 0 || id >= cs[i]->num_blocks) return KVX_EDATA;
        }
    }
  }
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  return hip_status(launch_evict(at, a, st));
}

}  // extern "C"
