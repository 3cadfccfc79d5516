// attn_serve.hip -- C-ABI of serving on caches of 8 bits, with sinks and drafted
// trees (kvx_serve.h): argument checks, launches, and the kernel that rotates
// and stores new tokens in 8 bits.
#include <hip/hip_runtime.h>

#include "attn_host.h"
#include "attn_view.h"

using namespace kvx;

namespace {

// cos and sin of r revolutions, |r| <= 1/2: by the nearest quarter and Taylor's
// series of the rest, at most pi / 4 (up to the 11th and 12th power: 7e-12).
__device__ __forceinline__ void turn64(double r, double& c, double& s) {
  const double q = rint(4.0 * r), y = __builtin_fma(4.0, r, -q) * 1.5707963267948966, z = y * y;
  double a = -1.0 / 39916800, b = 1.0 / 479001600;
  a = __builtin_fma(a, z, 1.0 / 362880);
  b = __builtin_fma(b, z, -1.0 / 3628800);
  a = __builtin_fma(a, z, -1.0 / 5040);
  b = __builtin_fma(b, z, 1.0 / 40320);
  a = __builtin_fma(a, z, 1.0 / 120);
  b = __builtin_fma(b, z, -1.0 / 720);
  a = __builtin_fma(a, z, -1.0 / 6);
  b = __builtin_fma(b, z, 1.0 / 24);
  b = __builtin_fma(b, z, -0.5);
  a = __builtin_fma(a * z, y, y);
  b = __builtin_fma(b, z, 1.0);
  const int k = static_cast<int>(q) & 3;
  const double u = k & 1 ? b : a, v = k & 1 ? a : b;  // sin, cos up to their signs
  s = k & 2 ? -u : u;
  c = (k + 1) & 2 ? -v : v;
}

// x in fp32, with an odd last bit where that is not x itself: what is rounded to
// fewer bits after, or compared with a number of fewer, comes out as from x.  (The
// nearest one would take x to the middle of two codes, or to the largest code.)
__device__ __forceinline__ float to_odd(double x) {
  const float near = static_cast<float>(x);
  const double back = near;
  uint32_t u = __float_as_uint(near);
  u -= fabs(back) > fabs(x) ? 1 : 0;
  return __uint_as_float(back == x ? u : u | 1u);
}

struct Append8Args {
  AttnArgs a;  // c: the codes
  ScaleArgs scale;
  const double* freq;
  const uint8_t* axis;
  const char* in[3];     // new q, k, v (NULL: none)
  int64_t sr[3], sh[3];  // their strides
  char* q_out;
};

// As append_kernel, with G lanes a row of which those past head_dim stay idle:
// a row's largest magnitude is taken over them.  Keys are rotated in 64 bits, so
// that their codes are those of the exact angles: an error in fp32 would move
// numbers near the middle of two codes by a whole step.  Bound by memory and, where
// tokens are many, the sines of 64 bits: 4 prompts, 11k tokens, heads 28 / 4 x 128, 92 MB
// in 24.2 us, 3.8 TB/s (with the library's sine and cosine and a workgroup for all heads
// of its rows: 32); one token 6 us, a launch and three loads that wait for each other.
template <typename C, int G>
__global__ void __launch_bounds__(256) append8_kernel(Append8Args g, int heads_step) {
  const AttnArgs& a = g.a;
  const int half = a.d / 2, lane = threadIdx.x % G, e0 = lane * 8;
  const int64_t row = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / G;
  if (row >= a.rows) return;  // all lanes of a row
  const bool active = e0 < half;
  const int b = context_of(a, static_cast<int>(row));
  const Context c = context(a, b);
  const int slot = c.p0 + static_cast<int>(row) - c.q0;
  double cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = active ? e0 + i : 0;
    const int p = a.pos ? a.pos[g.axis[e] * static_cast<int64_t>(a.rows) + row] : slot;
    double r = static_cast<double>(p) * g.freq[e];
    r -= rint(r);
    turn64(r, cs[i], sn[i]);
  }
  const bool stored = slot >= 0 && slot < a.c.capacity && row < c.q0 + c.m;
  const int32_t block = stored ? cache_block(a.c, b, slot) : 0;
  const int64_t at = stored ? cache_offset(a.c, block, slot) : 0;
  const int in_block = a.c.table ? slot - fdiv(a.c.bs, max(slot, 0)) * static_cast<int>(a.c.bs.d) : slot;
  const int nq = g.in[0] ? a.hq : 0, nk = g.in[1] ? a.hkv : 0, heads = stored ? nq + 2 * nk : nq;
  // a head's numbers are asked for before the last one's are worked on
  auto load = [&](int h, uint4 (&x)[2]) {
    const int which = h < nq ? 0 : h < nq + nk ? 1 : 2;
    const int hh = h - (which == 0 ? 0 : which == 1 ? nq : nq + nk);
    const bf16_t* src = reinterpret_cast<const bf16_t*>(g.in[which]) + row * g.sr[which] + hh * g.sh[which] + e0;
    x[0] = x[1] = uint4{0, 0, 0, 0};
    if (h < heads && active) {
      x[0] = *reinterpret_cast<const uint4*>(src);
      x[1] = *reinterpret_cast<const uint4*>(src + half);
    }
  };
  uint4 x[2], next[2];
  load(blockIdx.y, x);
  for (int h = blockIdx.y; h < heads; h += heads_step) {  // all lanes of a row
    load(h + heads_step, next);
    const int which = h < nq ? 0 : h < nq + nk ? 1 : 2;
    const int hh = h - (which == 0 ? 0 : which == 1 ? nq : nq + nk);
    const bf16_t* xs = reinterpret_cast<const bf16_t*>(x);
    if (which == 0) {
      bf16_t y[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = load_f32<bf16_t>(xs + i), w = load_f32<bf16_t>(xs + 8 + i);
        const float cf = static_cast<float>(cs[i]), sf = static_cast<float>(sn[i]);
        y[i] = store_cvt<bf16_t>(u * cf - w * sf);
        y[8 + i] = store_cvt<bf16_t>(w * cf + u * sf);
      }
      if (active) {
        bf16_t* dst = reinterpret_cast<bf16_t*>(g.q_out) + row * a.q_sr + hh * a.q_sh + e0;
        *reinterpret_cast<uint4*>(dst) = reinterpret_cast<const uint4*>(y)[0];
        *reinterpret_cast<uint4*>(dst + half) = reinterpret_cast<const uint4*>(y)[1];
      }
    } else {
      float y[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = load_f32<bf16_t>(xs + i), w = load_f32<bf16_t>(xs + 8 + i);
        y[i] = u;
        y[8 + i] = w;
        if (which == 1) {
          y[i] = to_odd(u * cs[i] - w * sn[i]);
          y[8 + i] = to_odd(w * cs[i] + u * sn[i]);
        }
      }
      uint32_t u[4];
      const uint32_t scale = encode_row<C, G>(y, u);
      if (active) {
        char* dst = (which == 1 ? a.c.k : a.c.v) + at + hh * a.c.sh + e0;
        *reinterpret_cast<uint2*>(dst) = uint2{u[0], u[1]};
        *reinterpret_cast<uint2*>(dst + half) = uint2{u[2], u[3]};
      }
      if (lane == 0) {
        uint16_t* pair = reinterpret_cast<uint16_t*>(g.scale.p + block * g.scale.sb + hh * g.scale.sh + in_block * g.scale.st);
        pair[which - 1] = static_cast<uint16_t>(scale);
      }
    }
    x[0] = next[0];
    x[1] = next[1];
  }
}

template <typename C>
hipError_t launch_append8(const kvx_attn* at, const Append8Args& g, int total_heads, hipStream_t st) {
  const int d = at->model.head_dim, lanes = d <= 64 ? 4 : d <= 128 ? 8 : 16;
  const int64_t groups = (int64_t(g.a.rows) * lanes + 255) / 256;
  int split = 1;
  while (split < total_heads && groups * split < 2 * at->n_cu) ++split;
  const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>(split));
  return lanes == 4   ? launch_on(append8_kernel<C, 4>, grid, dim3(256), st, g, split)
         : lanes == 8 ? launch_on(append8_kernel<C, 8>, grid, dim3(256), st, g, split)
                      : launch_on(append8_kernel<C, 16>, grid, dim3(256), st, g, split);
}

// A cache of 8 bits, checked; the layer is applied to its pointers.
kvx_status prepare_cache8(const kvx_attn* at, const kvx_cache8* in, int32_t batch, int32_t layer,
                          CacheArgs& c, ScaleArgs& sc) {
  if (!in || !in->scale || (in->code != KVX_CODE_I8 && in->code != KVX_CODE_E4M3)) return KVX_EINVAL;
  const kvx_status s = prepare_cache(at, in->codes, 1, batch, layer, c);
  if (s != KVX_OK) return s;
  if (reinterpret_cast<uintptr_t>(in->scale) & 3) return KVX_EUNSUPPORTED;
  int64_t t[4];
  for (int i = 0; i < 4; ++i) t[i] = in->scale_stride[i];
  if (!t[0] && !t[1] && !t[2] && !t[3]) {
    const bool paged = in->codes.block_table != nullptr;
    t[3] = 1;
    t[2] = paged ? in->codes.block_size : in->codes.capacity;
    t[1] = at->model.n_kv_heads * t[2];
    t[0] = (paged ? int64_t(in->codes.num_blocks) : int64_t(batch)) * t[1];
  }
  for (int i = 0; i < 4; ++i)
    if (t[i] < 0) return KVX_ESHAPE;
  const int64_t run = in->codes.block_table ? in->codes.block_size : in->codes.capacity;
  if (t[3] < 1 && run > 1) return KVX_ESHAPE;
  sc.p = static_cast<uint32_t*>(in->scale) + layer * t[0];
  sc.sl = t[0];
  sc.sb = t[1];
  sc.sh = t[2];
  sc.st = t[3];
  return KVX_OK;
}

// Whether n numbers at a and m at b share memory.
bool overlap(const int32_t* a, int64_t n, const int32_t* b, int64_t m) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + 4 * static_cast<uintptr_t>(m) && y < x + 4 * static_cast<uintptr_t>(n);
}

// KVX_VALIDATE=1: block ids of slots [from[b], to[b]) of every context.
kvx_status validate_blocks(const kvx_cache& c, int32_t batch, const int64_t* from, const int64_t* to) {
  if (!c.block_table) return KVX_OK;
  std::unique_ptr<int32_t[]> tab;
  const kvx_status s = fetch(tab, c.block_table, size_t(batch) * c.max_blocks);
  if (s != KVX_OK) return s;
  for (int64_t b = 0; b < batch; ++b)
    for (int64_t j = (from[b] > 0 ? from[b] : 0) / c.block_size; j * c.block_size < to[b]; ++j) {
      const int32_t id = tab[b * c.max_blocks + j];
      if (id < 0 || id >= c.num_blocks) return KVX_EDATA;
    }
  return KVX_OK;
}

kvx_status convert(const kvx_attn* at, const kvx_pack_io* io, bool pack, void* stream) {
  if (!at || !io) return KVX_EINVAL;
  if (io->batch < 0) return KVX_EINVAL;
  if (io->batch == 0) return KVX_OK;
  if (!io->tokens || !io->cache8) return KVX_EINVAL;
  PackArgs a{};
  kvx_status s = prepare_cache(at, io->cache, elem_size(at), io->batch, 0, a.plain);
  if (s != KVX_OK) return s;
  s = prepare_cache8(at, io->cache8, io->batch, 0, a.coded, a.scale);
  if (s != KVX_OK) return s;
  const void* const coded[3] = {io->cache8->codes.k, io->cache8->codes.v, io->cache8->scale};
  for (const void* p : coded)
    if (p == io->cache.k || p == io->cache.v) return KVX_EINVAL;
  a.tokens = io->tokens;
  a.layers = at->model.n_layers;
  a.batch = io->batch;
  a.heads = at->model.n_kv_heads;
  a.d = at->model.head_dim;
  if (int64_t(a.layers) * a.batch * a.heads > INT32_MAX / 16) return KVX_ESHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validating()) {
    s = hip_status(hipStreamSynchronize(st));
    if (s != KVX_OK) return s;
    std::unique_ptr<int32_t[]> tok;
    s = fetch(tok, io->tokens, io->batch);
    if (s != KVX_OK) return s;
    std::unique_ptr<int64_t[]> ends(new (std::nothrow) int64_t[2 * size_t(io->batch)]());
    if (!ends) return KVX_ENOMEM;
    for (int64_t b = 0; b < io->batch; ++b) {
      if (tok[b] < 0 || tok[b] > a.plain.capacity || tok[b] > a.coded.capacity) return KVX_EDATA;
      ends[io->batch + b] = tok[b];
    }
    const kvx_cache* both[2] = {&io->cache, &io->cache8->codes};
    for (const kvx_cache* c : both) {
      s = validate_blocks(*c, io->batch, ends.get(), ends.get() + io->batch);
      if (s != KVX_OK) return s;
    }
  }
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  return hip_status(launch_pack(at, a, io->cache8->code, pack, st));
}

}  // namespace

extern "C" {

kvx_status kvx_attn_append_coded(const kvx_attn* at, const kvx_attn_io* io, const kvx_cache8* cache8,
                            void* stream) {
  if (!at || !io || !cache8) return KVX_EINVAL;
  if (at->dtype != KVX_BF16) return KVX_EUNSUPPORTED;
  Append8Args g{};
  kvx_status s = prepare(at, io, g.a, &cache8->codes);
  if (s != KVX_OK) return s;
  if (!io->new_k != !io->new_v || (!io->new_q && !io->new_k)) return KVX_EINVAL;
  if (io->rows == 0 || io->batch == 0) return KVX_OK;
  s = prepare_cache8(at, cache8, io->batch, io->layer, g.a.c, g.scale);
  if (s != KVX_OK) return s;
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
  s = validate(io, g.a, false, st, &cache8->codes);
  if (s != KVX_OK) return s;
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  g.freq = at->freq;
  g.axis = at->axis;
  const int total = (io->new_q ? at->n_heads : 0) + (io->new_k ? 2 * at->model.n_kv_heads : 0);
  return hip_status(cache8->code == KVX_CODE_I8 ? launch_append8<code_i8>(at, g, total, st)
                                                : launch_append8<code_e4m3>(at, g, total, st));
}

kvx_status kvx_attn_pack(const kvx_attn* at, const kvx_pack_io* io, void* stream) {
  return convert(at, io, true, stream);
}

kvx_status kvx_attn_unpack(const kvx_attn* at, const kvx_pack_io* io, void* stream) {
  return convert(at, io, false, stream);
}

kvx_status kvx_attn_tree(const kvx_attn* at, const kvx_tree_io* io, void* stream) {
  if (!at || !io) return KVX_EINVAL;
  if (io->batch < 0 || io->rows < 0 || io->window < 0 || io->sink < 0 || io->words < 1)
    return KVX_EINVAL;
  if (io->words > 64) return KVX_EUNSUPPORTED;
  if ((io->batch == 0 && io->rows > 0) || (!io->q_start && io->rows != io->batch)) return KVX_ESHAPE;
  if (io->rows > INT32_MAX / 128 || io->batch > (1 << 20)) return KVX_ESHAPE;
  if (io->rows == 0 || io->batch == 0) return KVX_OK;
  if (!io->tokens || !io->parent || !io->mask) return KVX_EINVAL;
  TreeArgs a{};
  a.batch = io->batch;
  a.rows = io->rows;
  a.axes = at->n_axes;
  a.q_start = io->q_start;
  a.tokens = io->tokens;
  a.parent = io->parent;
  a.window = io->window;
  a.sink = io->sink;
  a.shift = io->shift;
  a.words = io->words;
  a.mask = io->mask;
  a.depth = io->depth;
  a.pos = io->pos;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validating()) {
    kvx_status s = hip_status(hipStreamSynchronize(st));
    if (s != KVX_OK) return s;
    std::unique_ptr<int32_t[]> qs, tok, par;
    s = fetch(tok, io->tokens, io->batch);
    if (s == KVX_OK) s = fetch(par, io->parent, io->rows);
    if (s == KVX_OK && io->q_start) s = fetch(qs, io->q_start, size_t(io->batch) + 1);
    if (s != KVX_OK) return s;
    if (qs && (qs[0] != 0 || qs[io->batch] != io->rows)) return KVX_EDATA;
    for (int64_t b = 0; b < io->batch; ++b) {
      const int32_t q0 = qs ? qs[b] : static_cast<int32_t>(b), q1 = qs ? qs[b + 1] : q0 + 1;
      if (q1 < q0 || q0 < 0 || q1 > io->rows || q1 - q0 > 32 * io->words || tok[b] < q1 - q0)
        return KVX_EDATA;
      for (int32_t i = q0; i < q1; ++i)
        if (par[i] >= i - q0) return KVX_EDATA;
    }
  }
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  return hip_status(launch_tree(a, st));
}

kvx_status kvx_attn_forward_view(const kvx_attn* at, const kvx_attn_io* io, const kvx_attn_view* view,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (!view || (!view->cache8 && !view->tree && (view->sink == 0 || (io && io->window == 0)))) {
    if (view && view->sink < 0) return KVX_EINVAL;
    return kvx_attn_forward(at, io, workspace, workspace_bytes, stream);
  }
  if (!at || !io || view->sink < 0) return KVX_EINVAL;
  if (view->cache8 && at->dtype != KVX_BF16) return KVX_EUNSUPPORTED;
  AttnView a{};
  kvx_status s = prepare(at, io, a, view->cache8 ? &view->cache8->codes : nullptr);
  if (s != KVX_OK) return s;
  if (view->tree && (view->tree_words < 1 || io->prefix)) return KVX_EINVAL;
  if (io->rows == 0 || io->batch == 0) return KVX_OK;
  if (view->tree && int64_t(view->tree_words) * 32 < io->max_new) return KVX_ESHAPE;
  if (view->cache8) {
    s = prepare_cache8(at, view->cache8, io->batch, io->layer, a.c, a.scale);
    if (s != KVX_OK) return s;
  }
  if (!io->q || !io->out || !workspace || !aligned16(workspace)) return KVX_EINVAL;
  size_t need = 0;
  s = kvx_attn_workspace_bytes(at, &need);
  if (s != KVX_OK) return s;
  if (workspace_bytes < need) return KVX_ESHAPE;
  s = check_rows(at, io->q, io->q_stride, at->n_heads, io->rows);
  if (s != KVX_OK) return s;
  s = check_rows(at, io->out, io->out_stride, at->n_heads, io->rows);
  if (s != KVX_OK) return s;
  a.out = static_cast<char*>(io->out);
  a.o_sr = io->out_stride[0];
  a.o_sh = io->out_stride[1];
  a.lse = io->lse;
  a.sink = io->window ? view->sink : 0;
  a.tree = view->tree;
  a.words = view->tree_words;
  a.depth = view->depth;
  hipStream_t st = static_cast<hipStream_t>(stream);
  s = validate(io, a, true, st, view->cache8 ? &view->cache8->codes : nullptr, a.sink);
  if (s != KVX_OK) return s;
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  return hip_status(launch_view(at, a, view->cache8 ? view->cache8->code : -1, io->max_new, workspace, st));
}

kvx_status kvx_attn_accept(const kvx_attn* at, const kvx_accept_io* io, void* stream) {
  if (!at || !io) return KVX_EINVAL;
  if (io->batch < 0 || io->max_path < 1) return KVX_EINVAL;
  if (io->batch == 0) return KVX_OK;
  if (!io->tokens || !io->path || !io->count) return KVX_EINVAL;
  // written while other workgroups still read these
  if (overlap(io->tokens_out, io->batch, io->tokens, io->batch) ||
      overlap(io->tokens_out, io->batch, io->count, io->batch) ||
      overlap(io->tokens_out, io->batch, io->path, int64_t(io->batch) * io->max_path) ||
      overlap(io->tokens_out, io->batch, io->q_start, io->batch + int64_t(1)))
    return KVX_EINVAL;
  AcceptArgs a{};
  kvx_status s = io->cache8 ? prepare_cache8(at, io->cache8, io->batch, 0, a.c, a.scale)
                            : prepare_cache(at, io->cache, elem_size(at), io->batch, 0, a.c);
  if (s != KVX_OK) return s;
  a.q_start = io->q_start;
  a.tokens = io->tokens;
  a.path = io->path;
  a.max_path = io->max_path;
  a.count = io->count;
  a.tokens_out = io->tokens_out;
  a.layers = at->model.n_layers;
  a.batch = io->batch;
  a.heads = at->model.n_kv_heads;
  a.es = io->cache8 ? 1 : elem_size(at);
  a.row_bytes = at->model.head_dim * a.es;
  if (int64_t(a.layers) * a.batch * a.heads > INT32_MAX / 16) return KVX_ESHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (validating()) {
    s = hip_status(hipStreamSynchronize(st));
    if (s != KVX_OK) return s;
    std::unique_ptr<int32_t[]> qs, tok, path, cnt;
    s = fetch(tok, io->tokens, io->batch);
    if (s == KVX_OK) s = fetch(cnt, io->count, io->batch);
    if (s == KVX_OK) s = fetch(path, io->path, size_t(io->batch) * io->max_path);
    if (s == KVX_OK && io->q_start) s = fetch(qs, io->q_start, size_t(io->batch) + 1);
    if (s != KVX_OK) return s;
    std::unique_ptr<int64_t[]> ends(new (std::nothrow) int64_t[2 * size_t(io->batch)]());
    if (!ends) return KVX_ENOMEM;
    for (int64_t b = 0; b < io->batch; ++b) {
      const int32_t m = qs ? qs[b + 1] - qs[b] : 1;
      if (m < 0 || tok[b] < m || tok[b] > a.c.capacity || cnt[b] < 0 || cnt[b] > m ||
          cnt[b] > io->max_path)
        return KVX_EDATA;
      for (int32_t i = 0, last = -1; i < cnt[b]; ++i) {
        const int32_t k = path[b * io->max_path + i];
        if (k <= last || k >= m) return KVX_EDATA;
        last = k;
      }
      ends[b] = cnt[b] ? tok[b] - m : tok[b];
      ends[io->batch + b] = tok[b];
    }
    s = validate_blocks(io->cache8 ? io->cache8->codes : io->cache, io->batch, ends.get(),
                        ends.get() + io->batch);
    if (s != KVX_OK) return s;
  }
  if (fault_injected()) return hip_status(hipErrorLaunchFailure);
  return hip_status(launch_accept(at, a, st));
}

}  // extern "C"
