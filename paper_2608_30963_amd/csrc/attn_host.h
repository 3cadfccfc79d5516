// attn_host.h -- argument checks that the entry points of decoding share
// (kvx_attn.h, kvx_serve.h).  Host only.
#pragma once

#include <cmath>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <memory>
#include <new>

#include "attn.h"

namespace kvx {

constexpr double kLog2eHost = 1.4426950408889634;

// Whether a positive number is a normal one in fp32.
inline bool normal(double x) {
  return x >= std::numeric_limits<float>::min() && x <= std::numeric_limits<float>::max();
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline int elem_size(const kvx_attn* at) { return at->dtype == KVX_F32 ? 4 : 2; }

inline bool fault_injected() {
  const char* f = std::getenv("KVX_FAULT");
  return f && std::strcmp(f, "launch") == 0;
}

inline bool validating() {
  const char* v = std::getenv("KVX_VALIDATE");
  return v && v[0] == '1';
}

// A cache's pointers, strides and capacity, checked; the layer is applied to
// the base pointers.  es: bytes of a number.
inline kvx_status prepare_cache(const kvx_attn* at, const kvx_cache& in, int es, int32_t batch,
                                int32_t layer, CacheArgs& c) {
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
inline void near_cap(const kvx_attn* at, AttnArgs& a) {
  constexpr double c[4] = {-0.3333314389628958, 0.1332587895825113, -0.053045494297645907,
                           0.017241491495620133};
  const double y = at->scale / at->softcap;
  double factor = at->scale * kLog2eHost;
  a.near = static_cast<float>(0.5 / y);
  for (int i = 0; i < 4; ++i) {
    factor *= y * y;
    a.near_c[i] = static_cast<float>(c[i] * factor);
    if (!std::isfinite(a.near_c[i])) a.near = 0.f;
  }
}

// Rows of a new tensor: (row, head) strides of `heads` head vectors.
inline kvx_status check_rows(const kvx_attn* at, const void* p, const int64_t* s, int64_t heads,
                             int64_t rows) {
  const int64_t d = at->model.head_dim;
  if (s[0] < 0 || s[1] < 0) return KVX_ESHAPE;
  if ((heads > 1 && s[1] < d) || (rows > 1 && s[0] < d)) return KVX_ESHAPE;
  const int es = elem_size(at);
  if (!aligned16(p) || s[0] * es % 16 || s[1] * es % 16) return KVX_EUNSUPPORTED;
  return KVX_OK;
}

// Fields that append, forward and mass share; rows == 0 leaves nothing to do.
// `codes`: the cache of 8 bits that the call takes instead of io's.
inline kvx_status prepare(const kvx_attn* at, const kvx_attn_io* io, AttnArgs& a,
                          const kvx_cache* codes = nullptr) {
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
  kvx_status s = prepare_cache(at, codes ? *codes : io->cache, codes ? 1 : elem_size(at), io->batch,
                               io->layer, a.c);
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
  a.scale2 = static_cast<float>(at->scale * kLog2eHost);
  a.cap2 = static_cast<float>(at->softcap * kLog2eHost);
  if (at->softcap > 0.0) near_cap(at, a);
  a.tanh2 = at->softcap > 0.0 ? static_cast<float>(2.0 * at->scale / at->softcap * kLog2eHost) : 0.f;
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
// that a call may touch (those of a window's reach, and sinks, when it has one).
inline kvx_status validate(const kvx_attn_io* io, const AttnArgs& a, bool reads_cache, hipStream_t st,
                           const kvx_cache* codes = nullptr, int32_t sink = 0) {
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
  const kvx_cache& c = codes ? *codes : io->cache;
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
    if (lo < 0) lo = 0;
    for (int64_t j = 0; j * c.block_size < n; ++j) {
      if ((j + 1) * c.block_size <= lo && (!reads_cache || j * c.block_size >= sink)) continue;
      const int32_t id = tab[b * c.max_blocks + j];
      if (id < 0 || id >= c.num_blocks) return KVX_EDATA;
    }
  }
  return KVX_OK;
}

}  // namespace kvx
