// Paged 8-bit caches: the kernels that keep the pages (fork, compact) and write new tokens into them (append).  The
// attention over them is in pages_attn.cuh.  Contracts: include/tabed.h.
//
// A cached value is an e4m3 code times the scale of its page, layer and KV head.  Scales written here are powers of two: bringing codes to a larger scale only
// moves the exponent, so a page that fills up token by token holds, but for values that become subnormal, what one rounding
// of every value would have given, and the 3 bits of mantissa lose nothing against a scale amax / 448.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ptx.cuh"

namespace tabed {

enum { PGERR_NUMERIC = 1, PGERR_INVALID = 32 };       // beside PERR_KV and PERR_COPY

struct PagesDev {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int *table, *ref, *err;
  int L, NP, Hkv, ps, ls, hd, n_seqs, max_pages;      // ps = 1 << ls tokens a page
};

// ---- e4m3 ------------------------------------------------------------------------------------------
// four codes of a word: (0, 1) and (2, 3) as pairs of fp16 values (exact)
__device__ __forceinline__ void e4m3x4_to_f16x4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {      // to nearest even, saturating
  uint32_t r;
  asm("{\n .reg .b16 x, y;\n cvt.rn.satfinite.e4m3x2.f32 x, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 y, %4, %3;\n mov.b32 %0, {x, y};\n}\n"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ float2 f16x2_to_float2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// the codes of a word at `ratio` times their scale's inverse
__device__ __forceinline__ uint32_t e4m3x4_rescale(uint32_t w, float ratio) {
  uint32_t lo, hi;
  e4m3x4_to_f16x4(w, lo, hi);
  const float2 a = f16x2_to_float2(lo), b = f16x2_to_float2(hi);
  return to_e4m3x4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
}
// the least 2^e, -126 <= e <= 120, with amax <= 448 * 2^e  (448 = 1.75 * 2^8)
__device__ __forceinline__ float least_scale(float amax) {
  const uint32_t b = __float_as_uint(amax);
  int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = min(max(e, -126), 120);
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// ---- append ----------------------------------------------------------------------------------------
struct AppendArgs {
  PagesDev P;
  int layer, n, n_tokens, max_new, n_heads, nblk, hpc, n_axes, has_q;
  const int *seq, *first, *start, *positions;      // seq null: entry e is sequence seq0 + e; first null: one entry, all tokens, from start0 on
  int seq0, start0;
  const int* held;                    // tokens that the rows come from (null: any number): none behind them are taken
  const void *k, *v, *q;
  void* q_out;
  long long kv_stride, kv_head, q_stride, q_out_stride;      // elements between tokens; between heads of K and V
  int vec_kv, vec_q;                  // rows start on 16-byte boundaries
  int sections[4];
  double turns[64];                   // theta^(-2 i / hd) / (2 pi)
};

__device__ __forceinline__ void load8(const __nv_bfloat16* p, bool vec, float (&f)[8]) {
  if (vec) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __bfloat162float(p[i]);
  }
}
__device__ __forceinline__ void load8(const float* p, bool vec, float (&f)[8]) {
  if (vec) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = p[i];
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, bool vec, const float (&f)[8]) {
  if (vec) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(f[i]);
  }
}
__device__ __forceinline__ void store8(float* p, bool vec, const float (&f)[8]) {
  if (vec) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = f[i];
  }
}

// Whether another of the n entries names the sequence of entry e (all threads of the block take part; n_threads of them).
__device__ __forceinline__ bool named_twice(const int* seq, int e, int n) {
  int twice = 0;
  const int s = seq[e];
  for (int i = threadIdx.x; i < n; i += blockDim.x) twice |= (i != e && seq[i] == s);
  return __syncthreads_or(twice) != 0;
}

constexpr int kAppendThreads = 256;

// eight values as they lie in memory: asked for early, turned into fp32 late
template <typename T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw8<T> raw8(const T* p, bool vec) {
  Raw8<T> r;
  if (vec) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.v[i] = reinterpret_cast<const uint4*>(p)[i];
  } else {
    uint32_t w[4 * (sizeof(T) / 2)];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
      else if (i % 2 == 0) w[i / 2] = reinterpret_cast<const unsigned short*>(p)[i] | (uint32_t)reinterpret_cast<const unsigned short*>(p)[i + 1] << 16;
    }
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
  return r;
}
__device__ __forceinline__ void open8(const Raw8<__nv_bfloat16>& r, float (&f)[8]) {
  const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void open8(const Raw8<float>& r, float (&f)[8]) {
  const uint32_t w[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
}

// A CTA has one block of page_tokens tokens of one entry and hpc of the K, V and query heads: the cosines and sines of
// its tokens are taken once (the angle's turns in fp64: positions of any size) and serve all of those heads.  A unit (a head's
// tokens of the block) is worked by TPU threads, each with up to MAXI items of 8 rotated pairs in registers between the
// block's maximum and the rounding: k, v and q are read once, the next unit's while this one is worked.  Short units (single
// tokens) take a warp each, 8 at once; long ones the whole CTA, of 256 or 512 threads: an item a thread keeps most warps on an SM (64
// tokens of 128 values: two items on 256 threads 144 us, one on 512 113 us, 424 MB, at 18,800 tokens of 48 heads; fp32 156 us, 809 MB, 5.2 TB/s).
template <typename T, int TPU, int MAXI>
__global__ void __launch_bounds__(TPU == 32 ? kAppendThreads : TPU, TPU == 512 && MAXI == 1 ? 2 : 1) k_pages_append(const AppendArgs A) {
  extern __shared__ float4 ap_cs[];               // [4][items] cosine and sine of two frequencies: the lanes' places are neighbours
  constexpr int THREADS = TPU == 32 ? kAppendThreads : TPU, WARPS = THREADS / 32;
  __shared__ float s_red[2][WARPS];
  const PagesDev& P = A.P;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int e = blockIdx.x / A.nblk, slot = blockIdx.x - e * A.nblk;
  pdl_trigger();
  pdl_wait();
  const int s = A.seq ? A.seq[e] : A.seq0 + e, f0 = A.first ? A.first[e] : 0, f1 = A.first ? A.first[e + 1] : A.n_tokens, p0 = A.start ? A.start[e] : A.start0;
  const int ps = P.ps, hd = P.hd, half = hd >> 1;
  if (f0 < 0 || f1 < f0 || f1 > A.n_tokens || s < 0 || s >= P.n_seqs || p0 < 0 || f1 - f0 > A.max_new || (A.held && p0 > *A.held - (f1 - f0))) {
    if (tid == 0) atomicOr(P.err, PGERR_INVALID);
    return;
  }
  if ((long long)p0 + (f1 - f0) > (long long)P.max_pages * ps) {
    if (tid == 0) atomicOr(P.err, PERR_KV);
    return;
  }
  const int p1 = p0 + (f1 - f0), bi = (p0 >> P.ls) + slot;
  if (f1 == f0 || slot > ((p1 - 1) >> P.ls) - (p0 >> P.ls)) return;      // (not by bi * page_tokens, which may pass 2^31)
  const int lo = max(p0, bi * ps), cnt = min(p1, (bi + 1) * ps) - lo, off = lo - bi * ps, t0 = f0 + (lo - p0);
  const int u0 = blockIdx.y * A.hpc, u1 = min(u0 + A.hpc, 2 * P.Hkv + (A.has_q ? A.n_heads : 0));
  const int lt = 31 - __clz(hd >> 4), n_items = cnt << lt;      // hd / 16 = 2^lt items a token
  constexpr int UNITS = THREADS / TPU;
  const int me = TPU == 32 ? lane : tid;
  Raw8<T> ra[MAXI], rb[MAXI];
  auto ask = [&](int u) {                         // unit u's values
    const bool is_q = u >= 2 * P.Hkv, is_v = !is_q && u >= P.Hkv;
    const T* in = reinterpret_cast<const T*>(is_q ? A.q : (is_v ? A.v : A.k)) + (is_q ? (size_t)(u - 2 * P.Hkv) * hd : (size_t)(is_v ? u - P.Hkv : u) * A.kv_head);
    const long long stride = is_q ? A.q_stride : A.kv_stride;
    const bool vec = is_q ? A.vec_q : A.vec_kv;
#pragma unroll
    for (int j = 0; j < MAXI; ++j) {
      const int it = me + j * TPU;
      if (it < n_items) {
        const T* row = in + (long long)(t0 + (it >> lt)) * stride + (it & ((1 << lt) - 1)) * 8;
        ra[j] = raw8(row, vec);
        rb[j] = raw8(row + half, vec);
      }
    }
  };
  int u = u0 + (TPU == 32 ? warp : 0);
  if (u < u1) ask(u);
  const int page = P.table[(size_t)s * P.max_pages + bi];
  bool own = page >= 0 && page < P.NP;
  if (own) own = P.ref[page] == 1;
  if (A.n_axes) {
    for (int i = tid; i < n_items * 4; i += THREADS) {
      const int k = i / n_items, it = i - k * n_items, tok = it >> lt, f = (it & ((1 << lt) - 1)) * 8 + 2 * k;
      float c[4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        int axis = 0, upto = A.sections[0];
        while (f + x >= upto && axis < A.n_axes - 1) upto += A.sections[++axis];
        double turn = (double)A.positions[(size_t)axis * A.n_tokens + t0 + tok] * A.turns[f + x];
        turn -= rint(turn);
        // What the angle loses in fp32 is put back to first order (the rest is below 2^-46): without it fp32 queries are 1.24 times as far off as
        // with cosines rounded once, with it 0.95 times (images' prompts 111.9 -> 112.7 us; both in fp64 0.87 times, 114.7 us).
        const float at = (float)(2.0 * turn), r = (float)(2.0 * turn - (double)at) * 3.14159265f;
        float sn, cn;
        sincospif(at, &sn, &cn);
        c[2 * x] = fmaf(-sn, r, cn); c[2 * x + 1] = fmaf(cn, r, sn);
      }
      ap_cs[i] = make_float4(c[0], c[1], c[2], c[3]);
    }
  }
  if (A.seq && named_twice(A.seq, e, A.n)) {      // (a barrier, too)
    if (tid == 0) atomicOr(P.err, PGERR_INVALID);
    return;
  }
  __syncthreads();
  if (!own && tid == 0) atomicOr(P.err, PGERR_INVALID);
  for (int n = 0; u < u1; u += UNITS, n ^= 1) {
    const bool is_q = u >= 2 * P.Hkv, is_v = !is_q && u >= P.Hkv;
    const int head = is_q ? u - 2 * P.Hkv : (is_v ? u - P.Hkv : u);
    const bool turned = A.n_axes && !is_v;
    float x[MAXI][16], amax = 0.0f;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < MAXI; ++j) {
      const int it = me + j * TPU;
      if (it < n_items) {
        float a[8], b[8];
        open8(ra[j], a);
        open8(rb[j], b);
        if (turned) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float4 cs = ap_cs[k * n_items + it];
            const int i = 2 * k;
            const float y0 = a[i] * cs.x - b[i] * cs.y, y1 = a[i + 1] * cs.z - b[i + 1] * cs.w;
            b[i] = b[i] * cs.x + a[i] * cs.y;
            b[i + 1] = b[i + 1] * cs.z + a[i + 1] * cs.w;
            a[i] = y0; a[i + 1] = y1;
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) { x[j][i] = a[i]; x[j][8 + i] = b[i]; }
        if (is_q) {
          T* o = reinterpret_cast<T*>(A.q_out) + (size_t)head * hd + (long long)(t0 + (it >> lt)) * A.q_out_stride + (it & ((1 << lt) - 1)) * 8;
          store8(o, A.vec_q, a);
          store8(o + half, A.vec_q, b);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float m = fabsf(x[j][i]);
            if (m < INFINITY) amax = fmaxf(amax, m); else odd = true;
          }
        }
      }
    }
    if (u + UNITS < u1) ask(u + UNITS);
    if (is_q || !own) continue;                   // (the same for all threads of the unit)
    const size_t at = ((size_t)A.layer * P.NP + page) * P.Hkv + head;
    float* scale = (is_v ? P.v_scale : P.k_scale) + at;
    uint8_t* codes = (is_v ? P.v : P.k) + at * ps * hd;
    const float old = off > 0 ? *scale : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if (TPU > 32) {
      if (lane == 0) s_red[n][warp] = amax;
      __syncthreads();                            // (everybody has read the old scale, too)
      amax = s_red[n][lane & (WARPS - 1)];
#pragma unroll
      for (int o = WARPS / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    } else {
      __syncwarp();
    }
    const float now = fmaxf(least_scale(amax), old), inv = 1.0f / now;
    if (me == 0) *scale = now;
    if (odd) atomicOr(P.err, PGERR_NUMERIC);
    if (off > 0 && now != old) {
      const float ratio = old / now;
      for (int i = me; i < off * (hd >> 3); i += TPU) {
        uint2* w = reinterpret_cast<uint2*>(codes) + i;
        uint2 c = *w;
        c.x = e4m3x4_rescale(c.x, ratio);
        c.y = e4m3x4_rescale(c.y, ratio);
        *w = c;
      }
    }
#pragma unroll
    for (int j = 0; j < MAXI; ++j) {
      const int it = me + j * TPU;
      if (it < n_items) {
        uint8_t* row = codes + (size_t)(off + (it >> lt)) * hd + (it & ((1 << lt) - 1)) * 8;
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = x[j][i] != x[j][i] ? 0.0f : x[j][i] * inv;     // (the conversion saturates)
        *reinterpret_cast<uint2*>(row) = make_uint2(to_e4m3x4(y[0], y[1], y[2], y[3]), to_e4m3x4(y[4], y[5], y[6], y[7]));
        *reinterpret_cast<uint2*>(row + half) = make_uint2(to_e4m3x4(y[8], y[9], y[10], y[11]), to_e4m3x4(y[12], y[13], y[14], y[15]));
      }
    }
  }
}

// The other way: the first `len` tokens of a sequence into a dense cache row [L][Hkv][cap][hd] (a code times a power of two is a bf16 value
// already).  Blocks without a page become zeros.  Measured: 4 layers of 12 heads of 64, 704 tokens 8.2 us, 8192 32 us (151 MB, 4.7 TB/s).  grid (ceil(len / page_tokens), 2 Hkv, L)
template <typename T>
__global__ void __launch_bounds__(128) k_pages_load_row(const PagesDev P, int seq, int len, T* __restrict__ k, T* __restrict__ v, int cap, int* kv_len) {
  const int b = blockIdx.x, head = blockIdx.y >> 1, layer = blockIdx.z, hd = P.hd, tid = threadIdx.x;
  const bool is_v = blockIdx.y & 1;
  pdl_trigger();
  pdl_wait();
  int page = P.table[(size_t)seq * P.max_pages + b];
  if (page < 0 || page >= P.NP) {
    if (tid == 0) atomicOr(P.err, PGERR_INVALID);
    page = -1;
  }
  if (tid == 0 && b == 0 && blockIdx.y == 0 && layer == 0) *kv_len = len;
  const size_t at = ((size_t)layer * P.NP + max(page, 0)) * P.Hkv + head;
  const uint8_t* codes = (is_v ? P.v : P.k) + at * P.ps * hd;
  const float scale = page >= 0 ? (is_v ? P.v_scale : P.k_scale)[at] : 0.0f;
  T* out = (is_v ? v : k) + (((size_t)layer * P.Hkv + head) * cap + (size_t)b * P.ps) * hd;
  const int n = min(P.ps, len - b * P.ps) * hd;
  for (int i = tid * 8; i < n; i += 128 * 8) {
    const uint2 c = page >= 0 ? *reinterpret_cast<const uint2*>(codes + i) : make_uint2(0u, 0u);
    uint32_t h[4];
    e4m3x4_to_f16x4(c.x, h[0], h[1]);
    e4m3x4_to_f16x4(c.y, h[2], h[3]);
    float f[8];
#pragma unroll
    for (int x = 0; x < 4; ++x) { const float2 y = f16x2_to_float2(h[x]); f[2 * x] = y.x * scale; f[2 * x + 1] = y.y * scale; }
    store8(out + i, true, f);
  }
}

// ---- fork ------------------------------------------------------------------------------------------
// Three launches: the references of the pages shared, marked and given back (a CTA an entry; atomic operations whose order does
// not matter), the free pages (one CTA: who needs how many, and the lowest-numbered ones in order), the tables and the copies.  The
// first two are one CTA's launch for few and short tables.
// While the call runs a page's word in `ref` holds its references in the low half, above them how many entries keep a part of it in place (src
// == dst), and in the sign whether others copy from it: such a page is not handed out even where nobody names it any longer.
struct ForkEntry { int valid, stays, first_new, tail; };     // tail: page of the block that keep ends in, -1 if it ends with a block

struct ForkArgs {
  PagesDev P;
  int n;
  const int *src, *dst, *keep, *len;
  ForkEntry* ent;                     // [n_seqs]
  int* found;                         // [4]: free pages found
  int* rows;                          // [n_seqs][max_pages] the kept blocks of an entry, as they were before the call
  int* free_list;                     // [min(n_pages, n_seqs * max_pages)]
  int vec_ref;                        // ref starts on a 16-byte boundary
};

constexpr int kForkThreads = 256;
constexpr int kForkKeeps = 1 << 16, kForkCopies = (int)0x80000000;
__device__ __forceinline__ void fork_mark(int* word, bool keeps) { if (keeps) atomicAdd(word, kForkKeeps); else atomicOr(word, kForkCopies); }
__device__ __forceinline__ void fork_unmark(int* word, bool keeps) { if (keeps) atomicAdd(word, -kForkKeeps); else atomicAnd(word, ~kForkCopies); }
constexpr int kForkAllocThreads = 1024;

__global__ void __launch_bounds__(kForkThreads) k_pages_share(const ForkArgs A) {
  const PagesDev& P = A.P;
  const int e = blockIdx.x, tid = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  const int src = A.src[e], dst = A.dst[e], keep = A.keep[e], len = A.len[e];
  int bad = src < 0 || src >= P.n_seqs || dst < 0 || dst >= P.n_seqs || keep < 0 || len < keep;
  const bool over = !bad && len > P.max_pages * P.ps;
  bad |= over;
  const int full = bad ? 0 : keep / P.ps, part = bad ? 0 : keep % P.ps;
  const int* from = P.table + (size_t)(bad ? 0 : src) * P.max_pages;
  int lost = 0;
  for (int b = tid; b < full + (part > 0); b += kForkThreads) { const int pg = from[b]; lost |= pg < 0 || pg >= P.NP; }
  bad |= __syncthreads_or(lost);
  bad |= named_twice(A.dst, e, A.n);
  if (tid == 0) {
    A.ent[e] = ForkEntry{!bad, 0, 0, bad || part == 0 ? -1 : from[full]};
    if (bad) atomicOr(P.err, over ? PERR_KV : PGERR_INVALID);
  }
  if (bad) return;
  int* row = A.rows + (size_t)e * P.max_pages;
  for (int b = tid; b < full; b += kForkThreads) {
    const int pg = from[b];
    row[b] = pg;
    atomicAdd(P.ref + pg, 1);
  }
  if (tid == 0 && part > 0) fork_mark(P.ref + from[full], src == dst);
  const int* to = P.table + (size_t)dst * P.max_pages;
  for (int b = tid; b < P.max_pages; b += kForkThreads) {
    const int pg = to[b];
    if (pg >= 0 && pg < P.NP) atomicAdd(P.ref + pg, -1);
  }
}

// the sum of v over the threads before this one; *total over all (1024 threads; s_scan of 33 words)
__device__ __forceinline__ int block_scan(int v, int* s_scan, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
  if (lane == 31) s_scan[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int w = s_scan[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, w, o); if (lane >= o) w += y; }
    s_scan[lane] = w;
  }
  __syncthreads();
  *total = s_scan[31];
  const int before = (warp ? s_scan[warp - 1] : 0) + x - v;
  __syncthreads();
  return before;
}

// Who needs how many pages, and the free ones in order: one CTA.
// An entry that keeps a part of its own page stays in it if nobody names the page after all have given theirs back; of several that were cut
// inside a page they shared, the first stays and the others copy.  Where there are such, they bid for the page in its word's low half, which is
// 0: 0xFFFF - entry, above any count of references; the largest is the first entry's.
__device__ __forceinline__ void fork_alloc(const ForkArgs& A, int* s_scan) {
  const PagesDev& P = A.P;
  const int tid = threadIdx.x;
  int shared = 0;
  for (int e = tid; e < A.n; e += kForkAllocThreads) {
    const ForkEntry E = A.ent[e];
    if (!E.valid || E.tail < 0 || A.src[e] != A.dst[e]) continue;
    const int w = __ldcg(P.ref + E.tail);
    if ((w & 0xFFFF) != 0) continue;
    A.ent[e].stays = 1;
    shared |= (w & ~kForkCopies) >= 2 * kForkKeeps;
  }
  const bool bids = __syncthreads_or(shared) != 0;
  if (bids) {
    for (int e = tid; e < A.n; e += kForkAllocThreads)
      if (A.ent[e].stays) {
        int* word = P.ref + A.ent[e].tail;
        atomicMax(word, (__ldcg(word) & ~0xFFFF) | (0xFFFF - e));
      }
    __syncthreads();
    for (int e = tid; e < A.n; e += kForkAllocThreads)
      if (A.ent[e].stays) A.ent[e].stays = (__ldcg(P.ref + A.ent[e].tail) & 0xFFFF) == 0xFFFF - e;
  }
  int need_all = 0;
  for (int base = 0; base < A.n; base += kForkAllocThreads) {
    const int e = base + tid;
    int need = 0;
    if (e < A.n && A.ent[e].valid) need = (A.len[e] + P.ps - 1) / P.ps - A.keep[e] / P.ps - A.ent[e].stays;
    int total;
    const int before = block_scan(need, s_scan, &total);
    if (e < A.n) A.ent[e].first_new = need_all + before;
    need_all += total;
  }
  // (every bid has been read: the pages that stay with their sequence get their reference)
  for (int e = tid; e < A.n; e += kForkAllocThreads)
    if (A.ent[e].valid && A.ent[e].stays) atomicAdd(P.ref + A.ent[e].tail, bids ? 1 - (0xFFFF - e) : 1);
  __syncthreads();
  constexpr int PER = 8;
  int found = 0;
  for (long long base = 0; base < P.NP && found < need_all; base += kForkAllocThreads * PER) {
    const long long p0 = base + (long long)tid * PER;
    int r[PER], mine = 0;
    if (A.vec_ref && p0 + PER <= P.NP) {
#pragma unroll
      for (int j = 0; j < PER; j += 4) *reinterpret_cast<int4*>(r + j) = __ldcg(reinterpret_cast<const int4*>(P.ref + p0 + j));
    } else {
#pragma unroll
      for (int j = 0; j < PER; ++j) r[j] = p0 + j < P.NP ? __ldcg(P.ref + p0 + j) : 1;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) mine += r[j] == 0;
    int total, at = found + block_scan(mine, s_scan, &total);
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (r[j] == 0) { if (at < need_all) A.free_list[at] = (int)(p0 + j); ++at; }
    found += total;
  }
  if (tid == 0) {
    A.found[0] = min(found, need_all);
    if (found < need_all) atomicOr(P.err, PERR_KV);
  }
}

__global__ void __launch_bounds__(kForkAllocThreads) k_pages_alloc(const ForkArgs A) {
  __shared__ int s_scan[33];
  pdl_trigger();
  pdl_wait();
  fork_alloc(A, s_scan);
}

// k_pages_share and k_pages_alloc in one launch of one CTA, for few and short tables (the threads go over all entries' blocks together).
constexpr int kPlanEntries = kForkAllocThreads, kPlanBlocks = 1024;
__global__ void __launch_bounds__(kForkAllocThreads) k_pages_plan(const ForkArgs A) {
  __shared__ int s_scan[33], s_src[kPlanEntries], s_dst[kPlanEntries], s_keep[kPlanEntries], s_bad[kPlanEntries];
  const PagesDev& P = A.P;
  const int tid = threadIdx.x, W = P.max_pages;
  pdl_trigger();
  pdl_wait();
  bool over = false;
  if (tid < A.n) {
    const int src = A.src[tid], dst = A.dst[tid], keep = A.keep[tid], len = A.len[tid];
    bool bad = src < 0 || src >= P.n_seqs || dst < 0 || dst >= P.n_seqs || keep < 0 || len < keep;
    over = !bad && len > W * P.ps;
    bad |= over;
    s_src[tid] = bad ? 0 : src; s_keep[tid] = bad ? 0 : keep; s_dst[tid] = dst; s_bad[tid] = bad;
  }
  __syncthreads();
  if (tid < A.n) {
    const int dst = s_dst[tid];
    bool twice = false;
    for (int i = 0; i < A.n; ++i) twice |= i != tid && s_dst[i] == dst;
    if (twice) s_bad[tid] = 1;
  }
  for (int i = tid; i < A.n * W; i += kForkAllocThreads) {
    const int e = i / W, b = i - e * W;
    if (b < (s_keep[e] + P.ps - 1) >> P.ls) { const int pg = P.table[(size_t)s_src[e] * W + b]; if (pg < 0 || pg >= P.NP) s_bad[e] = 1; }
  }
  __syncthreads();
  if (tid < A.n) {
    const bool bad = s_bad[tid];
    const int keep = s_keep[tid], tail = bad || (keep & (P.ps - 1)) == 0 ? -1 : P.table[(size_t)s_src[tid] * W + (keep >> P.ls)];
    A.ent[tid] = ForkEntry{!bad, 0, 0, tail};
    if (bad) atomicOr(P.err, over ? PERR_KV : PGERR_INVALID);
    if (tail >= 0) fork_mark(P.ref + tail, s_src[tid] == s_dst[tid]);
  }
  for (int i = tid; i < A.n * W; i += kForkAllocThreads) {
    const int e = i / W, b = i - e * W;
    if (s_bad[e]) continue;
    if (b < s_keep[e] >> P.ls) {
      const int pg = P.table[(size_t)s_src[e] * W + b];
      A.rows[(size_t)e * W + b] = pg;
      atomicAdd(P.ref + pg, 1);
    }
    const int pg = P.table[(size_t)s_dst[e] * W + b];
    if (pg >= 0 && pg < P.NP) atomicAdd(P.ref + pg, -1);
  }
  __syncthreads();
  fork_alloc(A, s_scan);
}

// grid (n, 1 + 2 L): the table, then K and V of a layer
__global__ void __launch_bounds__(kForkThreads) k_pages_settle(const ForkArgs A) {
  const PagesDev& P = A.P;
  const int e = blockIdx.x, tid = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  const ForkEntry E = A.ent[e];
  if (!E.valid) return;
  const int keep = A.keep[e], full = keep / P.ps, part = keep % P.ps, nb = (A.len[e] + P.ps - 1) / P.ps, kept = full + E.stays, found = A.found[0];
  if (blockIdx.y == 0) {
    int* to = P.table + (size_t)A.dst[e] * P.max_pages;
    const int* row = A.rows + (size_t)e * P.max_pages;
    for (int b = tid; b < P.max_pages; b += kForkThreads) {
      int pg = -1;
      if (b < full) pg = row[b];
      else if (b < kept) pg = E.tail;
      else if (b < nb) {
        const int at = E.first_new + b - kept;
        if (at < found) { pg = A.free_list[at]; P.ref[pg] = 1; }
      }
      to[b] = pg;
    }
    if (tid == 0 && E.tail >= 0) fork_unmark(P.ref + E.tail, A.src[e] == A.dst[e]);
    return;
  }
  if (E.tail < 0 || E.stays || E.first_new >= found) return;
  const int page = A.free_list[E.first_new], layer = (blockIdx.y - 1) >> 1;
  const bool is_v = (blockIdx.y - 1) & 1;
  uint8_t* codes = is_v ? P.v : P.k;
  float* scale = is_v ? P.v_scale : P.k_scale;
  const size_t of = ((size_t)layer * P.NP + E.tail) * P.Hkv, at = ((size_t)layer * P.NP + page) * P.Hkv;
  for (int i = tid; i < P.Hkv; i += kForkThreads) scale[at + i] = scale[of + i];
  const int head_bytes = P.ps * P.hd, vecs = part * P.hd >> 4;          // 16-byte pieces of a head's kept tokens
  for (int i = tid; i < P.Hkv * vecs; i += kForkThreads) {
    const int h = i / vecs, x = (i - h * vecs) << 4;
    *reinterpret_cast<uint4*>(codes + (at + h) * head_bytes + x) = *reinterpret_cast<const uint4*>(codes + (of + h) * head_bytes + x);
  }
}

// ---- compact ---------------------------------------------------------------------------------------
struct CompactArgs {
  PagesDev P;
  const int *seq, *start, *count, *index;
  int n, width;
};
constexpr int kCompactThreads = 256;
constexpr int kCompactTile = 1024;        // tokens whose places are looked up at once (a multiple of page_tokens)

// A CTA has one entry and layer and up to 8 units (a KV head of K or V), each worked by UW warps that fill its target blocks one by one; the
// places of the tokens are looked up once for all of them.  Sources lie at or behind their targets in ascending order, so no source of a block lies in a
// block filled before it: reads may run ahead at will (two blocks here), and a block's reads and writes are parted by the maximum of its scales.
// MAXV: 16-byte pieces of a block per thread.  Bound by the instructions and trips to memory of a unit's blocks, one after the other.
// grid (n, L, ceil(2 Hkv UW / 8))
template <int UW, int MAXV>
__global__ void __launch_bounds__(kCompactThreads) k_pages_compact(const CompactArgs A) {
  const PagesDev& P = A.P;
  constexpr int UNITS = kCompactThreads / 32 / UW, TPU = 32 * UW;
  const int e = blockIdx.x, layer = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, mine = warp / UW, me = tid - mine * TPU;
  const int unit = blockIdx.z * UNITS + mine, head = unit >> 1;
  const bool is_v = unit & 1, there = unit < 2 * P.Hkv;
  __shared__ int2 s_src[kCompactTile];            // a token's page, and its place in the page
  __shared__ float s_red[2][kCompactThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int s = A.seq[e], start = A.start[e], count = A.count[e], ps = P.ps, ls = P.ls, hd = P.hd, cap = P.max_pages * ps;
  const int* index = A.index + (size_t)e * A.width;
  int bad = s < 0 || s >= P.n_seqs || start < 0 || count < 0 || count > A.width || start > cap - count;
  const int* table = P.table + (size_t)(bad ? 0 : s) * P.max_pages;
  // places of the tokens i0 .. of the next tile
  int tile0 = 0;
  auto look_up = [&](int i0) {
    tile0 = i0;
    for (int i = tid; i < kCompactTile && i0 + i < count; i += kCompactThreads) {
      const int x = index[i0 + i];
      s_src[i] = make_int2(table[x >> ls], x & (ps - 1));
    }
    __syncthreads();
  };
  if (!bad) {
    for (int i = tid; i < count; i += kCompactThreads) {
      const int x = index[i];
      int wrong = x < start + i || x >= cap || (i > 0 && index[i - 1] >= x);
      if (!wrong) {
        const int pg = table[x >> ls];
        wrong = pg < 0 || pg >= P.NP;
        if (i < kCompactTile) s_src[i] = make_int2(pg, x & (ps - 1));
      }
      bad |= wrong;
    }
    if (count > 0)
      for (int b = (start >> ls) + tid; b <= (start + count - 1) >> ls; b += kCompactThreads) {
        const int pg = table[b];
        bad |= pg < 0 || pg >= P.NP || P.ref[pg] != 1;
      }
    for (int i = tid; i < A.n; i += kCompactThreads) bad |= i != e && A.seq[i] == s;      // (named twice)
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicOr(P.err, PGERR_INVALID);
    return;
  }
  if (count == 0) return;
  uint8_t* codes = (is_v ? P.v : P.k) + ((size_t)layer * P.NP * P.Hkv + (there ? head : 0)) * ps * hd;        // + page * Hkv * ps * hd
  float* scale = (is_v ? P.v_scale : P.k_scale) + (size_t)layer * P.NP * P.Hkv + (there ? head : 0);          // + page * Hkv
  const size_t page_codes = (size_t)P.Hkv * ps * hd;
  const int lv = 31 - __clz(hd >> 4);             // 16-byte pieces of a token: 2^lv
  // first token (of the entry's moved ones), tokens and place of target block b
  auto span = [&](int b, int& i0, int& cnt, int& off) {
    const int lo = max(start, b << ls), hi = min(start + count, (b + 1) << ls);
    i0 = lo - start; cnt = hi - lo; off = lo - (b << ls);
  };
  struct Block { uint4 w[MAXV]; float s[MAXV]; };
  auto fetch = [&](int b, Block& B) {
    int i0, cnt, off;
    span(b, i0, cnt, off);
#pragma unroll
    for (int j = 0; j < MAXV; ++j) {
      const int x = me + j * TPU;
      B.s[j] = 0.0f;
      if (there && x < cnt << lv) {
        const int2 at = s_src[i0 - tile0 + (x >> lv)];
        B.w[j] = *reinterpret_cast<const uint4*>(codes + at.x * page_codes + at.y * hd + ((x & ((1 << lv) - 1)) << 4));
        B.s[j] = scale[(size_t)at.x * P.Hkv];
      }
    }
  };
  const int b0 = start >> ls, b1 = (start + count - 1) >> ls;
  int known = b0;                                 // blocks before this one have been asked for
  auto ask = [&](Block& B) {                      // the next block's values; the whole CTA comes here together
    if (known > b1) return;
    int i0, cnt, off;
    span(known, i0, cnt, off);
    if (i0 + cnt > tile0 + kCompactTile) { __syncthreads(); look_up(i0); }
    fetch(known++, B);
  };
  auto settle = [&](int b, const Block& B) {
    int i0, cnt, off;
    span(b, i0, cnt, off);
    const int page = table[b];
    const float old = there && off > 0 ? scale[(size_t)page * P.Hkv] : 0.0f;
    float most = old;
#pragma unroll
    for (int j = 0; j < MAXV; ++j) most = fmaxf(most, B.s[j]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (UW > 1) {                                 // (all of this block's sources have been read behind it)
      float* red = s_red[b & 1];
      if (lane == 0) red[warp] = most;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "n"(TPU) : "memory");
#pragma unroll
      for (int i = 0; i < UW; ++i) most = fmaxf(most, red[mine * UW + i]);
    } else {
      __syncwarp();
    }
    if (!there) return;
    uint8_t* to = codes + (size_t)page * page_codes;
    if (off > 0 && old != most) {
      const float ratio = old / most;
      for (int i = me; i < off << lv; i += TPU) {
        uint4 w = *reinterpret_cast<uint4*>(to + ((size_t)i << 4));
        w.x = e4m3x4_rescale(w.x, ratio); w.y = e4m3x4_rescale(w.y, ratio);
        w.z = e4m3x4_rescale(w.z, ratio); w.w = e4m3x4_rescale(w.w, ratio);
        *reinterpret_cast<uint4*>(to + ((size_t)i << 4)) = w;
      }
    }
#pragma unroll
    for (int j = 0; j < MAXV; ++j) {
      const int x = me + j * TPU;
      if (x < cnt << lv) {
        uint4 w = B.w[j];
        if (B.s[j] != most) {
          const float ratio = B.s[j] / most;
          w.x = e4m3x4_rescale(w.x, ratio); w.y = e4m3x4_rescale(w.y, ratio);
          w.z = e4m3x4_rescale(w.z, ratio); w.w = e4m3x4_rescale(w.w, ratio);
        }
        *reinterpret_cast<uint4*>(to + (size_t)off * hd + ((size_t)x << 4)) = w;
      }
    }
    if (me == 0) scale[(size_t)page * P.Hkv] = most;
  };
  Block A0, A1, A2;
  ask(A0);
  ask(A1);
#pragma unroll 1
  for (int b = b0; b <= b1; b += 3) {
    ask(A2);
    settle(b, A0);
    if (b + 1 > b1) break;
    ask(A0);
    settle(b + 1, A1);
    if (b + 2 > b1) break;
    ask(A1);
    settle(b + 2, A2);
  }
}

}  // namespace tabed
