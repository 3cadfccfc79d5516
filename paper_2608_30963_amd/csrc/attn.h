// attn.h -- what the kernels of decoding on a translated cache share
// (kvx_attn.h): their arguments, cache addressing and visibility.
#pragma once

#include "common.h"
#include "kvx_attn.h"

struct kvx_attn {
  int device = 0;
  int n_cu = 0;
  kvx_model model{};
  int32_t n_heads = 0, group = 0;  // query heads, and per KV head
  int32_t dtype = KVX_BF16;
  double scale = 0.0, softcap = 0.0;
  int32_t n_axes = 1;
  void* tables = nullptr;          // device: the two tables below
  const double* freq = nullptr;    // [head_dim/2] theta / (2 pi)
  const uint8_t* axis = nullptr;   // [head_dim/2]
};

namespace kvx {

// floor(n / d) for 0 <= n < 2^31 by a product: mul = floor(2^(31+l) / d) + 1,
// l = ceil(log2 d); its excess over 2^(31+l)/d is at most 1, and n < 2^31
// times that stays below 2^(31+l) / d, less than a quotient's step.
struct FastDiv {
  uint32_t mul, shift, d;
};

inline FastDiv fast_div(int32_t d) {
  uint32_t l = 0;
  while ((int64_t(1) << l) < d) ++l;
  return FastDiv{static_cast<uint32_t>((uint64_t(1) << (31 + l)) / uint32_t(d) + 1), 31 + l,
                 static_cast<uint32_t>(d)};
}

__device__ __forceinline__ int fdiv(const FastDiv& f, int n) {
  return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(n)) * f.mul) >> f.shift);
}

// One layer's cache (or the first layer's, sl elements a layer): the row of
// slot j of context b and head h starts at element block * sb + h * sh +
// (j % block_size) * st, block the table's entry; without a table (contiguous)
// the block is the context and block_size exceeds every slot.
struct CacheArgs {
  char* k;
  char* v;
  int64_t sl, sb, sh, st;
  const int32_t* table;
  int32_t max_blocks;
  int32_t capacity;  // slots of a context
  FastDiv bs;
  int32_t run;       // power of two up to 64: that many slots, from a multiple of
                     // it on, lie in one block, at 32-bit offsets; 1 otherwise
};

__device__ __forceinline__ int32_t cache_block(const CacheArgs& c, int b, int j) {
  return c.table ? c.table[static_cast<int64_t>(b) * c.max_blocks + fdiv(c.bs, j)] : b;
}

// Element offset of slot j within its block's rows of one head.
__device__ __forceinline__ int64_t cache_offset(const CacheArgs& c, int32_t block, int j) {
  const int slot = c.table ? j - fdiv(c.bs, j) * static_cast<int>(c.bs.d) : j;
  return static_cast<int64_t>(block) * c.sb + static_cast<int64_t>(slot) * c.st;
}

// One layer's append, forward or mass.
struct AttnArgs {
  CacheArgs c;
  const int32_t* q_start;  // NULL: one row per context
  const int32_t* tokens;
  const int32_t* prefix;   // NULL: none
  const int32_t* pos;      // append: [axes][rows], NULL: slots
  int32_t batch, rows, hq, hkv, group, d;
  FastDiv by_group;        // division by group
  int32_t window;          // 0: none
  float scale2;            // score scale * log2(e)
  float cap2;              // cap * log2(e), 0: none
  float tanh2;             // 2 scale / cap * log2(e)
  const char* q;           // forward, mass
  int64_t q_sr, q_sh;      // elements
  char* out;
  int64_t o_sr, o_sh;
  float* lse;              // [rows][hq]
  const float* mass_in;
  float* mass;
  int32_t mass_capacity;
  float near, near_c[4];   // cap_near's range and coefficients
};

// A context's rows and slots, clamped to what the caller's buffers hold.  New
// token i has slot p0 + i by the length that the caller gave, also where that
// is past the cache's capacity: then the first n = capacity slots are there.
struct Context {
  int q0, m, n;  // first row, new tokens, slots that the cache holds
  int p0;        // slot of the first new token, n - m or more
  int prefix;    // slots that every new token sees
};

__device__ __forceinline__ Context context(const AttnArgs& a, int b) {
  Context c;
  c.q0 = a.q_start ? min(max(a.q_start[b], 0), a.rows) : b;
  const int q1 = a.q_start ? min(max(a.q_start[b + 1], c.q0), a.rows) : b + 1;
  c.m = q1 - c.q0;
  // room above for the rows that pad a tile past the last new token
  const int all = min(max(a.tokens[b], 0), INT32_MAX - 1024);
  c.n = min(all, a.c.capacity);
  c.p0 = all - c.m;
  c.prefix = a.prefix ? min(max(a.prefix[b], 0), c.n) : 0;
  return c;
}

// Slots [lo, hi) that the new token of slot p sees; empty for p < 0, and where
// a window starts past the cache's last slot.
__device__ __forceinline__ int first_seen(const AttnArgs& a, int p) {
  return a.window && p >= a.window ? p - a.window + 1 : 0;
}
__device__ __forceinline__ int end_seen(const Context& c, int p) {
  return p < 0 ? 0 : min(max(p + 1, c.prefix), c.n);
}

// A capped score is cap tanh(y), y = dot scale / cap, x the dot product q.k.
//
// cap_part: the r of tanh(y) = 1 - 2 r, r = 1 / (1 + exp(2 y)).  Its absolute
// error is 2^-24 or so, and the score's at most 2^-22 times the cap: up to
// kPartCap below 2^-15, far less than bf16 weights are rounded by, for which
// it serves there.
constexpr double kPartCap = 128.0;
__device__ __forceinline__ float cap_part(const AttnArgs& a, float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * a.tanh2));
}

// tanh(y) with a relative error of 2^-22: below 0.6, where 1 - 2 r loses digits,
// y + y^3 P(y^2), P a polynomial of small relative error there (4.7e-9).
__device__ __forceinline__ float cap_tanh(const AttnArgs& a, float x) {
  constexpr float kHalfLn2 = 0.34657359f;
  const float y = x * (a.tanh2 * kHalfLn2), z = y * y;
  float p = __builtin_fmaf(z, -0.005895158275961876f, 0.020795971155166626f);
  p = __builtin_fmaf(z, p, -0.053783830255270004f);
  p = __builtin_fmaf(z, p, 0.13331924378871918f);
  p = __builtin_fmaf(z, p, -0.33333298563957214f);
  return z < 0.36f ? __builtin_fmaf(y * z, p, y) : __builtin_fmaf(-2.f, cap_part(a, x), 1.f);
}

// cap2 tanh(y) + add for |x| < a.near, |y| < 0.5: x times a polynomial of x^2 whose
// coefficients hold scale and cap (relative error 1.5e-8 and its roundings).
__device__ __forceinline__ float cap_near(const AttnArgs& a, float x, float add) {
  const float z = x * x;
  float p = __builtin_fmaf(z, a.near_c[3], a.near_c[2]);
  p = __builtin_fmaf(z, p, a.near_c[1]);
  p = __builtin_fmaf(z, p, a.near_c[0]);
  return __builtin_fmaf(x, __builtin_fmaf(z, p, a.scale2), add);
}

// Score in units of log2.
__device__ __forceinline__ float score2(const AttnArgs& a, float x) {
  return a.cap2 == 0.f ? x * a.scale2 : a.cap2 * cap_tanh(a, x);
}

// Launchers; each returns the launch's own status.
hipError_t launch_forward(const kvx_attn* at, const AttnArgs& a, int max_new, void* workspace,
                          hipStream_t st);
size_t forward_workspace(const kvx_attn* at);
hipError_t launch_mass(const kvx_attn* at, const AttnArgs& a, int max_new, hipStream_t st);

struct EvictArgs {
  CacheArgs src, dst;
  const int32_t* tokens;
  int32_t layers, batch, heads, row_bytes;
  int32_t set0;  // (layer, context, KV head) of a launch's first workgroup
  int32_t keep, sink, recent;
  bool in_place;
  const float* mass;
  float* mass_out;
  int32_t mass_capacity;
  int32_t* kept;
  int32_t* tokens_out;
};
hipError_t launch_evict(const kvx_attn* at, const EvictArgs& a, hipStream_t st);

// Whether a launch has less than 2^32 threads along x.  The runtime takes more
// without an error and runs a part of them.
inline bool launchable(int64_t groups, int threads) {
  return groups * threads <= int64_t(UINT32_MAX);
}

// A launch with its own status: the runtime's last error may be another
// call's.  Each argument is converted to the kernel's parameter type.
template <typename... P, typename... A>
hipError_t launch_on(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t st, const A&... a) {
  if (!launchable(grid.x, block.x)) return hipErrorInvalidConfiguration;
  return [&](P... p) {
    void* args[] = {&p...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, args, 0, st);
  }(static_cast<P>(a)...);
}

}  // namespace kvx
