// Optimizer step for gfx950: AdamW over a table of tensors, and the norm of their gradients.
//
// Both stream memory once: per element AdamW reads weight, gradient and two states and writes weight and states back.  A thread has eight consecutive elements, in
// 16-byte loads; 32 threads have a block of 256, whose magnitudes meet in registers where the states have 8 bits.
// What bounds it: memory, with 32-bit states by far.  With 8-bit states and bf16 weights and gradients an element is 10 bytes, in whose time the chip does about 60 vector
// instructions, so those are counted (executed ones, the launch's beginning among them): by its code 86 an element in the first form of this kernel, with the library's root and quotient, 4.5 TB/s; 60 with the
// hardware's and with one product for eight random words; 49.5 with constants folded, what is rare (values not finite, v below the normal range) done again for the wave that has it, and what
// the host can compute computed there: 545 M elements 910 -> 875 us.
// Measured: 233 M elements with fp32 states and master copies 1311 us, 5.7 TB/s of the bytes above (a large copy runs at 4.8 TB/s); 545 M with 8-bit states 866 us, 6.3 TB/s.
// The norm reads 933 MB of fp32 gradients in 155 us and 477 MB of bf16 ones in 75 us, 6.0 and 6.4 TB/s.
#include "optim.h"
#include "device.h"

namespace sbp {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256, PER = 8, TILE = THREADS * PER;      // elements of a thread, of a pass of the workgroup

struct AdamwTable { AdamwArgs a; int n; AdamwTensor t[ADAMW_TABLE]; };
struct NormTable { double* part; int64_t span; int n; NormTensor t[NORM_TABLE]; };
static_assert(sizeof(AdamwTable) <= 4096 && sizeof(NormTable) <= 4096, "arguments of a launch");

// The tensor of a workgroup: the last one that begins at or before it
template <typename Table>
__device__ __forceinline__ int tensor_of(const Table& table, uint32_t group) {
  int lo = 0, hi = table.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (table.t[mid].first_group <= group) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// ---- eight elements ---------------------------------------------------------------------------------------------
// WHOLE: all eight exist and their address is a multiple of 16 (bytes: 8); else `n` of them, element by element.
// PAST: what passes the caches by, because it is more than they hold until it is read again (OPTIM_PAST).
template <bool PAST, typename T> __device__ __forceinline__ T load(const T* p) {
  if constexpr (PAST) return __builtin_nontemporal_load(p); else return *p;
}
template <bool PAST, typename T> __device__ __forceinline__ void store(T* p, T x) {
  if constexpr (PAST) __builtin_nontemporal_store(x, p); else *p = x;
}
template <bool PAST> __device__ __forceinline__ void load8(float (&x)[8], const float* p) {
  const f32x4 a = load<PAST>((const f32x4*)p), b = load<PAST>((const f32x4*)(p + 4));
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
template <bool PAST> __device__ __forceinline__ void load8(float (&x)[8], const bf16_t* p) {
  const u32x4 a = load<PAST>((const u32x4*)p);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(a[i] << 16); x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u); }
}
template <bool PAST> __device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  store<PAST>((f32x4*)p, f32x4{x[0], x[1], x[2], x[3]});
  store<PAST>((f32x4*)(p + 4), f32x4{x[4], x[5], x[6], x[7]});
}
template <bool PAST> __device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8]) {      // to nearest
  bf16x8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (bf16_t)x[i];
  store<PAST>((bf16x8*)p, a);
}
template <bool WHOLE, bool PAST, typename T> __device__ __forceinline__ void get(float (&x)[8], const T* p, int n) {
  if constexpr (WHOLE) { load8<PAST>(x, p); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = i < n ? ldf(p + i) : 0.f;
}
template <bool WHOLE, bool PAST, typename T> __device__ __forceinline__ void put(T* p, const float (&x)[8], int n) {
  if constexpr (WHOLE) { store8<PAST>(p, x); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) stf(p + i, x[i]);
}
template <bool WHOLE, bool PAST> __device__ __forceinline__ u32x2 get_bytes(const uint8_t* p, int n) {
  if constexpr (WHOLE) return load<PAST>((const u32x2*)p);
  u32x2 w = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return w;
}
template <bool WHOLE, bool PAST> __device__ __forceinline__ void put_bytes(uint8_t* p, const u32x2& w, int n) {
  if constexpr (WHOLE) { store<PAST>((u32x2*)p, w); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
}

// ---- random bits: see the public header
constexpr uint32_t MIX1 = 0x9E3779B1u, MIX2 = 0xB504F333u;
__device__ __forceinline__ uint32_t mix_end(uint32_t x) {      // ... from the first product on
  x = (x ^ (x >> 15)) * MIX2;
  return x ^ (x >> 16);
}
__device__ __forceinline__ uint32_t mix(uint32_t x) { return mix_end((x ^ (x >> 16)) * MIX1); }

// ---- e4m3 times a power of two ----------------------------------------------------------------------------------
// Largest bit pattern of non-negative floats over the 32 lanes that share a block: the order of the patterns is that of the values, NaN above infinity.
__device__ __forceinline__ uint32_t max_of_block(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));       // lane ^ 1
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));       // lane ^ 2
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));      // mirrored within 8 lanes
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, true));      // ... within 16
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x, x, false, false));
  return max(r[0], r[1]);
}
constexpr uint32_t NOT_FINITE = 0x7f800000u;
// The byte of a block whose largest magnitude has this pattern: 2^(byte - 127) brings it to [128, 256)
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest) { return max(largest >> 23, 8u) - 7u; }
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(max(byte << 23, 0x00400000u)); }      // (byte 0: 2^-127, below the normal range)
// A magnitude as the code of an e4m3 value of 2^(byte - 127): a float 2^120 times smaller than the value has the e4m3 value's exponent, and below its smallest normal
// one its fixed point, in bits 20 to 26.  u / 2^20 of a step is added before the rest is cut off.
__device__ __forceinline__ uint32_t e4m3_bits(float x, uint32_t byte) { return __float_as_uint(__builtin_amdgcn_ldexpf(fabsf(x), 7 - (int)byte)); }
__device__ __forceinline__ uint32_t median(uint32_t a, uint32_t b, uint32_t c) { return max(min(a, b), min(max(a, b), c)); }
// the top bytes of four words
__device__ __forceinline__ uint32_t top_bytes(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
  return __builtin_amdgcn_perm(x1, x0, 0x0c0c0703u) | __builtin_amdgcn_perm(x3, x2, 0x07030c0cu);
}
// Root and reciprocal by the hardware's instructions, a unit in the last place off at most.  They take no numbers below the normal range: a v of less is scaled up; the reciprocal's
// argument is a root or more.
__device__ __forceinline__ float root_of(float v) {
  const bool tiny = v < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(v * (tiny ? 0x1p64f : 1.f)) * (tiny ? 0x1p-32f : 1.f);
}

struct Consts { float bias1, bias2, keep; uint32_t key; float grad_scale; };

template <bool WHOLE, typename P, bool MASTER, typename G, bool EIGHT, bool PAST>
__device__ __forceinline__ void eight_elements(const AdamwTensor& t, const AdamwArgs& a, const Consts& c, int64_t e, int n, bool zero) {
  float g[8], w[8], m[8], v[8], root[8];
  if constexpr (MASTER) get<WHOLE, PAST>(w, t.master + e, n); else get<WHOLE, PAST>(w, (const P*)t.param + e, n);
  get<WHOLE, PAST>(g, (const G*)t.grad + e, n);
  if constexpr (EIGHT) {
    const u32x2 mb = get_bytes<WHOLE, PAST>((const uint8_t*)t.m + e, n), vb = get_bytes<WHOLE, PAST>((const uint8_t*)t.v + e, n);
    const bool in = WHOLE || n > 0;
    // the factors that an element's code and gradient meet, of m and of v's root: products of constants, so that m and v are a product and a sum each
    const float ms = in ? scale_of(t.m_scale[e / ADAMW_BLOCK]) * a.beta1 : 0.f, vs = in ? scale_of(t.v_scale[e / ADAMW_BLOCK]) * a.root2 : 0.f;
    const float gm = c.grad_scale * a.rest1, gv = c.grad_scale * a.root_rest2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const f32x2 m0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mb[i], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mb[i], true);
      const f32x2 v0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vb[i], false), v1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vb[i], true);
      m[4 * i] = m0[0] * ms; m[4 * i + 1] = m0[1] * ms; m[4 * i + 2] = m1[0] * ms; m[4 * i + 3] = m1[1] * ms;
      v[4 * i] = v0[0] * vs; v[4 * i + 1] = v0[1] * vs; v[4 * i + 2] = v1[0] * vs; v[4 * i + 3] = v1[1] * vs;
    }
    bool small = false;      // a v below the normal range, which the root's instruction takes for zero
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = g[i] * gv;
      m[i] = fmaf(g[i], gm, m[i]);      // (sums of products are written out: every copy of this code rounds alike)
      v[i] = fmaf(y, y, v[i] * v[i]);
      root[i] = __builtin_amdgcn_sqrtf(v[i]);
      small |= __builtin_amdgcn_classf(v[i], 0x80);
    }
    if (__builtin_amdgcn_ballot_w64(small) != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) root[i] = root_of(v[i]);
    }
  } else {
    get<WHOLE, PAST>(m, (const float*)t.m + e, n);
    get<WHOLE, PAST>(v, (const float*)t.v + e, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = g[i] * c.grad_scale;
      m[i] = fmaf(x, a.rest1, m[i] * a.beta1);
      v[i] = fmaf(x * x, a.rest2, v[i] * a.beta2);
      root[i] = root_of(v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = fmaf(-(c.bias1 * m[i]), __builtin_amdgcn_rcpf(fmaf(root[i], c.bias2, a.eps)), w[i] * c.keep);
  uint32_t r[8];
  constexpr bool ROUNDS = sizeof(P) == 2 && !MASTER;
  if constexpr (EIGHT || ROUNDS) {
    const uint32_t key = e >> 32 ? mix(c.key + (uint32_t)(e >> 32)) : c.key;
    // mix((e + i) ^ key), e a multiple of eight: the first shift moves the same bits for all eight, and each bit of i adds its multiple of the first factor to their product or takes
    // it away, so that eight words cost one first product instead of eight (a product of 32 bits is four other instructions)
    const uint32_t x = (uint32_t)e ^ key, y = x ^ (x >> 16);
    r[0] = y * MIX1;
#pragma unroll
    for (int b = 0; b < 3; ++b) {
      const uint32_t d = y >> b & 1 ? 0u - (MIX1 << b) : MIX1 << b;
#pragma unroll
      for (int i = 0; i < 1 << b; ++i) r[i + (1 << b)] = r[i] + d;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = mix_end(r[i]);
  }
  bool odd = !EIGHT;
  if constexpr (EIGHT) {
    uint32_t mx = 0, vx = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)      // (a root has a sign only as NaN, which is above all others with it too)
      if (WHOLE || i < n) { mx = max(mx, __float_as_uint(m[i]) & 0x7fffffffu); vx = max(vx, __float_as_uint(root[i])); }
    mx = max_of_block(mx);
    vx = max_of_block(vx);
    odd = __builtin_amdgcn_ballot_w64(max(mx, vx) >= NOT_FINITE) != 0;      // some element of the wave is not finite: it becomes NaN, and the scale is that of the others
    if (odd) {
      mx = vx = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t x = __float_as_uint(m[i]) & 0x7fffffffu, y = __float_as_uint(root[i]) & 0x7fffffffu;
        if ((WHOLE || i < n) && x < NOT_FINITE) mx = max(mx, x);
        if ((WHOLE || i < n) && y < NOT_FINITE) vx = max(vx, y);
      }
      mx = max_of_block(mx);
      vx = max_of_block(vx);
    }
    const uint32_t mb = scale_byte(mx), vb = scale_byte(vx);
    uint32_t d[8], b[8];      // the codes, in the top bytes
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      d[i] = (((e4m3_bits(m[i], mb) + (r[i] >> 12)) << 4) & 0x7fffffffu) | (__float_as_uint(m[i]) & 0x80000000u);
      // A root that is not zero gets code 1 at least.  The median of its code's pattern, 2^20, which is code 1, and its own pattern: zero, or, as a root is 2^-75 or more and a block's byte then
      // 45 or more, larger than both.
      b[i] = median(e4m3_bits(root[i], vb) + (r[i] & 0xfffffu), 1u << 20, __float_as_uint(root[i])) << 4;
    }
    if (odd) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if ((__float_as_uint(m[i]) & 0x7fffffffu) >= NOT_FINITE) d[i] = 0x7f000000u;
        if ((__float_as_uint(root[i]) & 0x7fffffffu) >= NOT_FINITE) b[i] = 0x7f000000u;
      }
    }
    const u32x2 mc = {top_bytes(d[0], d[1], d[2], d[3]), top_bytes(d[4], d[5], d[6], d[7])}, vc = {top_bytes(b[0], b[1], b[2], b[3]), top_bytes(b[4], b[5], b[6], b[7])};
    put_bytes<WHOLE, PAST>((uint8_t*)t.m + e, mc, n);
    put_bytes<WHOLE, PAST>((uint8_t*)t.v + e, vc, n);
    if ((threadIdx.x & 31) == 0 && (WHOLE || n > 0)) { t.m_scale[e / ADAMW_BLOCK] = (uint8_t)mb; t.v_scale[e / ADAMW_BLOCK] = (uint8_t)vb; }
  } else {
    put<WHOLE, PAST>((float*)t.m + e, m, n);
    put<WHOLE, PAST>((float*)t.v + e, v, n);
  }
  if constexpr (MASTER) put<WHOLE, PAST>(t.master + e, w, n);
  if constexpr (ROUNDS) {
    float up[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) up[i] = __uint_as_float((__float_as_uint(w[i]) + (r[i] & 0xffffu)) & 0xffff0000u);      // (then exact; an infinity has nothing below its last bit)
    // NaN stays NaN: with finite m and root it is the weight's own, or of 0 / 0, and has nothing in its lower half that would carry into the sign
    if (odd) {
#pragma unroll
      for (int i = 0; i < 8; ++i) up[i] = w[i] != w[i] ? w[i] : up[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = up[i];
  }
  put<WHOLE, PAST>((P*)t.param + e, w, n);
  if (zero) {
    const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    put<WHOLE, PAST>((G*)t.grad + e, none, n);
  }
}

template <typename P, bool MASTER, typename G, bool EIGHT, bool PAST>
__device__ __forceinline__ void span_of(const AdamwTensor& t, const AdamwArgs& a, const Consts& c, int64_t first, bool zero) {
  auto whole16 = [](const void* p) { return ((uintptr_t)p & 15) == 0; };
  auto whole8 = [](const void* p) { return ((uintptr_t)p & 7) == 0; };
  const bool aligned = whole16(t.param) && whole16(t.master) && whole16(t.grad) && (EIGHT ? whole8(t.m) && whole8(t.v) : whole16(t.m) && whole16(t.v));
  static_assert(ADAMW_SPAN == TILE, "one pass");
  const int64_t e = first + threadIdx.x * PER;
  if (aligned && first + TILE <= t.n) eight_elements<true, P, MASTER, G, EIGHT, PAST>(t, a, c, e, PER, zero);
  else eight_elements<false, P, MASTER, G, EIGHT, PAST>(t, a, c, e, (int)min((int64_t)PER, max((int64_t)0, t.n - e)), zero);
}

template <bool EIGHT, bool PAST>
__global__ __launch_bounds__(THREADS) void adamw_k(const AdamwTable table) {
  const AdamwArgs& a = table.a;
  const AdamwTensor& t = table.t[tensor_of(table, blockIdx.x)];
  const int64_t first = (int64_t)(blockIdx.x - t.first_group) * ADAMW_SPAN;
  Consts c;
  c.bias1 = a.bias1; c.bias2 = a.bias2; c.keep = t.keep;
  c.grad_scale = a.grad_scale ? *a.grad_scale : 1.f;
  int step = a.step;
  if (a.now) {
    step = max(1, a.now->step);
    const double lr = a.now->lr;
    __shared__ float bias[2];      // (by one wave: some hundred instructions in fp64)
    if (threadIdx.x < WAVE) {
      const double t1 = -expm1(step * a.log1), t2 = -expm1(step * a.log2);
      bias[0] = (float)(lr / t1);
      bias[1] = (float)(1.0 / sqrt(t2));
    }
    __syncthreads();
    c.bias1 = bias[0];
    c.bias2 = bias[1];
    c.keep = (float)(1.0 - lr * t.weight_decay);
  }
  c.key = mix(mix(mix(a.seed) + (uint32_t)step) + t.index);
  const bool zero = a.zero_grads != 0;
  if (!(fabsf(c.grad_scale) < INFINITY)) {      // nothing is known of the gradients: nothing moves
    if (!zero) return;
    const int64_t end = min(first + ADAMW_SPAN, t.n);
    for (int64_t e = first + threadIdx.x; e < end; e += THREADS) {
      if (t.grad_dtype == DT_BF16) stf((bf16_t*)t.grad + e, 0.f); else stf((float*)t.grad + e, 0.f);
    }
    return;
  }
  const bool gb = t.grad_dtype == DT_BF16;
  if (t.dtype == DT_F32) { if (gb) span_of<float, false, bf16_t, EIGHT, PAST>(t, a, c, first, zero); else span_of<float, false, float, EIGHT, PAST>(t, a, c, first, zero); }
  else if (t.master) { if (gb) span_of<bf16_t, true, bf16_t, EIGHT, PAST>(t, a, c, first, zero); else span_of<bf16_t, true, float, EIGHT, PAST>(t, a, c, first, zero); }
  else { if (gb) span_of<bf16_t, false, bf16_t, EIGHT, PAST>(t, a, c, first, zero); else span_of<bf16_t, false, float, EIGHT, PAST>(t, a, c, first, zero); }
}

hipError_t adamw_step(const AdamwArgs& a, const AdamwTensor* t, int n, hipStream_t st) {
  if (n < 1 || n > ADAMW_TABLE) return hipErrorInvalidValue;
  AdamwTable table{};
  table.a = a;
  table.n = n;
  int64_t groups = 0;
  for (int i = 0; i < n; ++i) {
    table.t[i] = t[i];
    table.t[i].first_group = (uint32_t)groups;
    groups += cdiv(t[i].n, ADAMW_SPAN);
  }
  if (a.eight && a.past) adamw_k<true, true><<<(unsigned)groups, THREADS, 0, st>>>(table);
  else if (a.eight) adamw_k<true, false><<<(unsigned)groups, THREADS, 0, st>>>(table);
  else adamw_k<false, false><<<(unsigned)groups, THREADS, 0, st>>>(table);
  return hipGetLastError();
}

// ---- norm -------------------------------------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, WAVE);
  return v;
}
template <int N>
__device__ __forceinline__ double group_sum(double v) {      // of N threads, the same for all of them
  __shared__ double red[N / WAVE];
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < N / WAVE; ++i) s += red[i];
  return s;
}

template <bool PAST, typename G>
__device__ __forceinline__ double squares(const NormTensor& t, int64_t first, int64_t span) {
  const G* g = (const G*)t.grad;
  const bool aligned = ((uintptr_t)g & 15) == 0;
  const int64_t end = min(first + span, t.n);
  double sum = 0.0;
  auto add = [&](const float (&x)[8]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i] * x[i];
    sum += (double)s;
  };
  constexpr int DEEP = NORM_SPAN / TILE;      // passes whose loads are under way at once: one by one, bf16 gradients took 109 us in place of 84
  int64_t at = first;
  for (; aligned && at + NORM_SPAN <= end; at += NORM_SPAN) {
    float x[DEEP][8];
#pragma unroll
    for (int i = 0; i < DEEP; ++i) get<true, PAST>(x[i], g + at + i * TILE + threadIdx.x * PER, PER);
#pragma unroll
    for (int i = 0; i < DEEP; ++i) add(x[i]);
  }
  for (; at < end; at += TILE) {
    const int64_t e = at + threadIdx.x * PER;
    float x[8];
    if (aligned && at + TILE <= t.n) get<true, PAST>(x, g + e, PER);
    else get<false, PAST>(x, g + e, (int)min((int64_t)PER, max((int64_t)0, t.n - e)));
    add(x);
  }
  return sum;
}
template <bool PAST>
__global__ __launch_bounds__(THREADS) void grad_squares_k(const NormTable table) {
  const NormTensor& t = table.t[tensor_of(table, blockIdx.x)];
  const int64_t first = (int64_t)(blockIdx.x - t.first_group) * table.span;
  const double s = group_sum<THREADS>(t.dtype == DT_BF16 ? squares<PAST, bf16_t>(t, first, table.span) : squares<PAST, float>(t, first, table.span));
  if (threadIdx.x == 0) table.part[blockIdx.x] = s;
}
hipError_t norm_parts(const NormTensor* t, int n, int64_t span, bool past, double* part, int* n_parts, hipStream_t st) {
  if (n < 1 || n > NORM_TABLE || span < NORM_SPAN || span % NORM_SPAN) return hipErrorInvalidValue;
  NormTable table{};
  table.part = part;
  table.span = span;
  table.n = n;
  int64_t groups = 0;
  for (int i = 0; i < n; ++i) {
    table.t[i] = t[i];
    table.t[i].first_group = (uint32_t)groups;
    groups += cdiv(t[i].n, span);
  }
  if (past) grad_squares_k<true><<<(unsigned)groups, THREADS, 0, st>>>(table);
  else grad_squares_k<false><<<(unsigned)groups, THREADS, 0, st>>>(table);
  *n_parts = (int)groups;
  return hipGetLastError();
}

constexpr int FINISH_THREADS = 1024;
__global__ __launch_bounds__(FINISH_THREADS) void norm_finish_k(const double* __restrict__ part, int n, float max_norm, float* __restrict__ norm,
                                                                float* __restrict__ scale) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += FINISH_THREADS) s += part[i];
  s = group_sum<FINISH_THREADS>(s);
  if (threadIdx.x != 0) return;
  const float x = (float)sqrt(s);
  *norm = x;
  if (scale) *scale = !(x < INFINITY) ? __builtin_nanf("") : max_norm > 0.f && x > max_norm ? max_norm / x : 1.f;
}
hipError_t norm_finish(const double* part, int n, float max_norm, float* norm, float* scale, hipStream_t st) {
  norm_finish_k<<<1, FINISH_THREADS, 0, st>>>(part, n, max_norm, norm, scale);
  return hipGetLastError();
}

}  // namespace sbp
