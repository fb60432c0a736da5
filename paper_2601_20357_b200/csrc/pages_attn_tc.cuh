// Attention over a paged 8-bit cache on the fifth-generation tensor cores, for many bf16 query rows a KV head (more than 16, of head sizes 32 and
// 64 more than 32): token trees, verified blocks, chunks of prompts.  The same list of chunks (here of 128 positions), numbers and partial results as pages_attn.cuh.
//
//   S [128 rows][128 positions] = Q K^T        Q, K in shared memory (kind::f16, fp32 sums in tensor memory)
//   O [128 rows][hd]           += P V          P in tensor memory (over its S), V in shared memory
//
// * A softmax thread has one row: its limits and its running maximum are scalars, and a position's scales are the same for 16 columns.
//   MT = 2 tiles of 128 rows share the converted K and V, and one's softmax runs under the other's products; with MT = 1 two threads have a
//   row, half of a chunk's positions each, and the scores of the next chunk are computed meanwhile.  Items of up to 64 rows have them twice in
//   the tile, and a copy takes half of the positions: the products cost the same, the softmax a half; the copies are put together at the end.
// * Eight warps load codes straight into registers, a chunk ahead (through a ring in shared memory the codes would cost its bandwidth
//   twice more), turn them into fp16 and store K and V alike as [dims / 8][128 positions][8 dims]: that is
//   K's K-major layout and V's MN-major one.  Half of the codes go through the conversion unit (16 a clock and SM, which the
//   exponentials need too), half are shifted into place, which leaves them 2^8 too small: undone in q and in the output.
// * One warp walks the list, looks pages and scales up and tells the others; one issues the products.
// q is scaled by a power of two per row: bf16 values are exact in fp16 down to 2^-21 of their row's largest.  Weights have 11 bits.
//
// Measured (B200): the trees of 32 requests (16 rows, 32 / 8 heads of 128, 500 - 8192 tokens, capped scores) 162 us with the join, where the
// kernel of pages_attn.cuh took 434 and the bytes take 45; two chunks of 2048 rows against 2111 - 4096 tokens 266 us, 480 TFLOP/s (1514 there);
// against 8192 tokens 650 TFLOP/s, 0.4 of the measured rate.  Four converting warps instead of eight: trees 190 us, prompts 285.  Chunks asked for two ahead
// spill registers: trees 198.  Parts of equal length instead of equal cost, before that: trees 212, prompts 365 against 188 and 281.
#pragma once
#include "pages_attn.cuh"

namespace tabed {

constexpr int kPtChunk = 128;
constexpr int kPtStart = 2;                    // chunks that an item's beginning and end cost
constexpr int kPtInfo = 8;                     // chunks that are known ahead
constexpr int kPtMaxCtas = 160, kPtMaxRows = 256;
constexpr size_t kPtSmem = 213u * 1024u;       // (too much for any other CTA with tensor memory beside it, which would wait for columns: proj_plan.h, tc_least_smem)

struct PtTile {
  int first, ends, whole, slot, to_end, j0, lim_min, lim_max, q0, nq, len, pre, rt, kvh, e, gaps;      // gaps: positions without a page
  int k_page[8], v_page[8];                    // of 16 positions each; -1: none, zeros
  float4 meta[8];                              // (pga_meta)
};

template <int HD, int MT> struct Pt {
  static constexpr int kThreads = 32 * 18;                             // 8 warps each for the softmax and the conversion, 1, 1
  static constexpr int kOp = kPtChunk * HD * 2;                        // fp16 operand of 128 rows or positions
  static constexpr int kQOff = 0, kKOff = MT * kOp, kVOff = kKOff + 2 * kOp, kEnd = kVOff + 2 * kOp;
  static_assert(1024 + kEnd <= (int)kPtSmem, "shared memory");
};

__device__ __forceinline__ void pt_ld16(uint32_t taddr, float* v) {
  uint32_t* u = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
                 "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]) : "r"(taddr));
}
__device__ __forceinline__ void pt_st16(uint32_t taddr, const uint32_t* u) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]),
                 "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]) : "memory");
}
__device__ __forceinline__ void pt_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pt_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pt_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void pt_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void pt_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void pt_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void pt_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void pt_fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
template <int ID, int N> __device__ __forceinline__ void pt_sync() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(N) : "memory"); }
__device__ __forceinline__ bool pt_elect() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}\n" : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// two fp32 operations at a time
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)), "l"(*reinterpret_cast<uint64_t*>(&c)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
  return *reinterpret_cast<float2*>(&d);
}
// the four codes of a word as fp16, 2^-8 of their values: sign to bit 15, the rest to bits 7 - 13 (subnormals too).
// (The codes that are no numbers come out as 480.)  In order: (0, 1), (2, 3).
__device__ __forceinline__ void e4m3x4_shifted(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t a = __byte_perm(w, 0, 0x1404), b = __byte_perm(w, 0, 0x3424);      // codes in the upper bytes of the halves
  lo = ((a >> 1) & 0x3F803F80u) | (a & 0x80008000u);
  hi = ((b >> 1) & 0x3F803F80u) | (b & 0x80008000u);
}
struct Row32 { uint32_t w[8]; };
// 32 bytes, 32-byte aligned, or zeros.  (One predicated load: behind a branch around it the warp would wait for the value.)
__device__ __forceinline__ Row32 ldg32_if(const uint8_t* p, bool there) {
  Row32 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.w[i] = 0;
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %9, 0;\n @p ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n}\n"
               : "+r"(r.w[0]), "+r"(r.w[1]), "+r"(r.w[2]), "+r"(r.w[3]), "+r"(r.w[4]), "+r"(r.w[5]), "+r"(r.w[6]), "+r"(r.w[7]) : "l"(p), "r"((int)there));
  return r;
}
__device__ __forceinline__ void stg32(void* p, const uint32_t* u) {                 // 32 bytes, 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]) : "memory");
}

template <int HD, int MT, int COPIES>
__global__ void __launch_bounds__(Pt<HD, MT>::kThreads, 1) k_pages_attn_tc(const PagesAttnArgs A) {
  using L = Pt<HD, MT>;
  constexpr unsigned FULL = 0xffffffffu;
  constexpr int W_CONV = 8, W_LOOK = 16, W_MMA = 17;
  extern __shared__ __align__(128) unsigned char pt_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(pt_raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t i_full[kPtInfo], i_empty[kPtInfo], k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_done[2];
  __shared__ PtTile info[kPtInfo];
  __shared__ PgaShare s_share;
  // 1 / scale of the query rows, of four items: an item may be one chunk, and the conversion is up to two chunks ahead of the softmax
  __shared__ float s_cr[4][128 * MT];
  __shared__ float s_top[2][2][128];             // MT = 1: the largest exponents of both halves of the positions
  __shared__ float2 s_ml[2][128];                // ... and (maximum, sum) at an item's end
  __shared__ uint32_t s_tmem;
  __shared__ int s_dead;
  const PagesDev& P = A.P;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0), cta = blockIdx.x;      // (the warp's number as a uniform value)
  const int Hkv = P.Hkv, grp = A.H / Hkv, ps = P.ps, RB = A.RB;
  constexpr int RP = 128 / COPIES;               // rows of a tile before they repeat
  if (tid == 0) {
    for (int i = 0; i < kPtInfo; ++i) { mbar_init(&i_full[i], 1); mbar_init(&i_empty[i], 9); }       // (read by the softmax warps and the products')
    for (int i = 0; i < 2; ++i) { mbar_init(&k_full[i], 8); mbar_init(&k_empty[i], 1); mbar_init(&v_full[i], 8); mbar_init(&v_empty[i], 1); mbar_init(&s_full[i], 1); mbar_init(&p_full[i], MT == 2 ? 4 : 8); mbar_init(&o_done[i], 1); }
    s_dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pt_fence_before();
  __syncthreads();
  pt_fence_after();
  pdl_trigger();                                  // (behind the allocation, as in the other kernels with tensor memory)
  // S: two of 128 columns (of two tiles, or of two chunks); O: one or two.  The weights lie over their scores, whose halves two threads
  // read with MT = 1: there they have columns of their own.
  const uint32_t tmem = s_tmem, tm_o = tmem + 256;
  pdl_wait();
  if (tid < 2) A.desc[cta * 2 + tid] = make_int4(0, 0, 0, 0);
  PgaWalk<kPtChunk> w;
  const int total = pga_begin<kPtChunk, kPtStart, L::kThreads>(A, s_share, w);
  volatile int* dead = &s_dead;
  const float log2e = 1.4426950408889634f;
  const bool cap = A.softcap > 0.0f;

  if (warp == W_LOOK && total > 0) {
    // ---- the list ----
    int cb = -1, ce = -1, ck = -1, pg = -1;       // block that lane 0 has looked up, entry, KV head
    float pks = 1.0f, pvs = 1.0f;
    bool fresh = true, from_start = false, ok = true;
#pragma unroll 1
    for (int c = 0; c < total; ++c) {
      const PgaEntry& E = w.E;
      const int p0 = w.ch * kPtChunk, blk0 = p0 >> P.ls, nblk = (E.len + ps - 1) >> P.ls;
      if (w.e != ce || blk0 < cb || blk0 + (kPtChunk >> P.ls) > cb + 32) {
        cb = blk0; ce = w.e; ck = -1;
        const int b = cb + lane;
        pg = b < nblk ? P.table[(size_t)E.seq * P.max_pages + b] : -1;
        if (b < nblk && (pg < 0 || pg >= P.NP)) { atomicOr(P.err, PGERR_INVALID); pg = -1; }
      }
      if (w.kvh != ck) {
        ck = w.kvh;
        if (pg >= 0) {
          const size_t at = ((size_t)A.layer * P.NP + pg) * Hkv + w.kvh;
          pks = P.k_scale[at]; pvs = P.v_scale[at];
        }
      }
      const int src = (((p0 + lane * 16) >> P.ls) - cb) & 31;
      const float ks = __shfl_sync(FULL, pks, src), vs = __shfl_sync(FULL, pvs, src);
      const int gp = __shfl_sync(FULL, pg, src);
      PtTile& T = info[c % kPtInfo];
      if (c >= kPtInfo) { ok = pga_wait(&i_empty[c % kPtInfo], (unsigned)(c / kPtInfo - 1) & 1u, dead, P.err); ok = __all_sync(FULL, ok); if (!ok) break; }
      if (lane < 8) {
        T.k_page[lane] = gp; T.v_page[lane] = vs < kPgaLeastV ? -1 : gp;
        T.meta[lane] = pga_meta(ks, vs, gp >= 0);
      }
      if (fresh) from_start = w.ch == 0;
      const bool gaps = __any_sync(FULL, lane < 8 && gp < 0);
      if (lane == 0) {
        T.gaps = gaps;
        T.first = fresh; T.to_end = w.ch == w.nch - 1; T.ends = T.to_end || c == total - 1;
        T.whole = from_start && T.to_end; T.slot = from_start;
        T.j0 = p0; T.lim_min = pga_limit(A, E, w.rt * RB, grp); T.lim_max = w.last;
        T.q0 = E.q0; T.nq = E.nq; T.len = E.len; T.pre = E.pre; T.rt = w.rt; T.kvh = w.kvh; T.e = w.e;
      }
      fresh = w.ch == w.nch - 1;
      __syncwarp();
      if (lane == 0) mbar_arrive(&i_full[c % kPtInfo]);
      if (c + 1 < total) w.step(A, grp);
    }
  } else if (warp == W_MMA && total > 0) {
    // ---- products (the whole warp walks the loop, so that descriptors and flags stay in uniform registers; one elected lane issues) ----
    const uint32_t id_s = (1u << 4) | (16u << 17) | (8u << 24);                                      // f16 x f16, both K-major, 128 x 128
    const uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | (8u << 24);           // B MN-major, 128 x hd
    // a step of 16 in the summed index is a constant on the descriptor's address field (16-byte units)
    const uint64_t d_q = tc_smem_desc(smem_u32(sm + L::kQOff), 2048, 128), d_k = tc_smem_desc(smem_u32(sm + L::kKOff), 2048, 128);
    const uint64_t d_v = tc_smem_desc(smem_u32(sm + L::kVOff), 128, 2048);
    const bool one = pt_elect();
    bool ok = true;
    auto scores = [&](int j, int m) {             // S of chunk j for tile m, into buffer b
      const uint32_t d = tmem + (MT == 2 ? m : (j & 1)) * 128;
      const uint64_t dq = d_q + (uint64_t)(m * (L::kOp >> 4)), dk = d_k + (uint64_t)((j & 1) * (L::kOp >> 4));
      if (one) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) pt_mma_ss(d, dq + k * 256, dk + k * 256, id_s, k > 0);
        if (m == MT - 1) pt_commit(&k_empty[j & 1]);
        pt_commit(&s_full[MT == 2 ? m : (j & 1)]);
      }
      __syncwarp();
    };
    auto output = [&](int j, int m, uint32_t fresh) {      // O of tile m, chunk j
      const int b = MT == 2 ? m : (j & 1);
      const uint32_t d = tm_o + m * 128, a = MT == 2 ? tmem + b * 128 : tmem + 384 + b * 64;
      const uint64_t dv = d_v + (uint64_t)((j & 1) * (L::kOp >> 4));
      if (one) {
#pragma unroll
        for (int k = 0; k < kPtChunk / 16; ++k) pt_mma_ts(d, a + k * 8, dv + k * 16, id_o, k > 0 || !fresh);
        if (m == MT - 1) pt_commit(&v_empty[j & 1]);
        pt_commit(&o_done[m]);
      }
      __syncwarp();
    };
    auto wait = [&](uint64_t* bar, unsigned parity) { if (ok) { ok = pga_wait(bar, parity, dead, P.err); ok = __all_sync(FULL, ok); } };
    auto k_ready = [&](int j) { wait(&k_full[j & 1], (unsigned)(j >> 1) & 1u); pt_fence_after(); };
    const int ahead = MT == 2 ? 1 : 2;            // chunks whose scores are asked for before the first output
    for (int j = 0; j < ahead && j < total && ok; ++j) {
      k_ready(j);
      for (int m = 0; m < MT && ok; ++m) scores(j, m);
    }
#pragma unroll 1
    for (int j = 0; j < total && ok; ++j) {
      wait(&i_full[j % kPtInfo], (unsigned)(j / kPtInfo) & 1u);
      const uint32_t fresh = __shfl_sync(FULL, info[j % kPtInfo].first, 0);
      if (lane == 0) mbar_arrive(&i_empty[j % kPtInfo]);
      const bool more = j + ahead < total;
#pragma unroll 1
      for (int m = 0; m < MT && ok; ++m) {
        if (m == 0) wait(&v_full[j & 1], (unsigned)(j >> 1) & 1u);
        if (MT == 2) wait(&p_full[m], (unsigned)j & 1u);
        else wait(&p_full[j & 1], (unsigned)(j >> 1) & 1u);
        if (!ok) break;
        pt_fence_after();
        output(j, m, fresh);
        if (more) {
          if (m == 0) k_ready(j + ahead);
          if (ok) scores(j + ahead, m);
        }
      }
    }
    // (the products read shared memory and write tensor memory until then)
    for (int m = 0; m < MT; ++m) wait(&o_done[m], (unsigned)(total - 1) & 1u);
    if (!ok) __nanosleep(100000);
  } else if (warp >= W_CONV && warp < W_LOOK) {
    // ---- conversion ----
    // A warp has 16 positions (one page's).  A lane has one 32-byte piece of every (16 / RS)th of them: eight neighbouring lanes have
    // neighbouring positions (stores free of bank conflicts), and together the lanes read whole rows (few lines a load).
    const int cw = warp - W_CONV;
    constexpr int NP = HD / 32, RS = NP == 4 ? 8 : 16, NI = 16 / RS;
    const int piece = lane / RS % NP, row0 = cw * 16 + lane % RS;
    const bool works = NP > 1 || lane < 16;       // (a row of 32 bytes: 16 lanes)
    const bool vec = A.vec_q;
    int item = -1;
    Row32 kr[NI], vr[NI];
    auto fetch = [&](const uint8_t* codes, const int (&pages)[8], const PtTile& T, Row32 (&r)[NI]) {
      const int page = pages[cw], j = T.j0 + cw * 16;
      const uint8_t* p = codes + (((size_t)A.layer * P.NP + max(page, 0)) * Hkv + T.kvh) * (ps * HD) + ((j & (ps - 1)) + lane % RS) * HD + piece * 32;
      const int live = page >= 0 ? T.lim_max - j - lane % RS : 0;      // (what nobody sees becomes zeros: 0 * NaN is not 0)
#pragma unroll
      for (int i = 0; i < NI; ++i) r[i] = ldg32_if(p + i * RS * HD, works && i * RS < live);
    };
    auto put = [&](unsigned char* dst, const Row32 (&r)[NI]) {      // 16 codes through the conversion unit, 16 shifted
      unsigned char* o = dst + piece * 4 * 2048 + row0 * 16;
      if (!works) return;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        uint4 a, b, c, d;
        e4m3x4_to_f16x4(r[i].w[0], a.x, a.y); e4m3x4_to_f16x4(r[i].w[1], a.z, a.w);
        e4m3x4_to_f16x4(r[i].w[2], b.x, b.y); e4m3x4_to_f16x4(r[i].w[3], b.z, b.w);
        e4m3x4_shifted(r[i].w[4], c.x, c.y); e4m3x4_shifted(r[i].w[5], c.z, c.w);
        e4m3x4_shifted(r[i].w[6], d.x, d.y); e4m3x4_shifted(r[i].w[7], d.z, d.w);
        *reinterpret_cast<uint4*>(o + i * RS * 16) = a;
        *reinterpret_cast<uint4*>(o + i * RS * 16 + 2048) = b;
        *reinterpret_cast<uint4*>(o + i * RS * 16 + 4096) = c;
        *reinterpret_cast<uint4*>(o + i * RS * 16 + 6144) = d;
      }
    };
    auto known = [&](int j) { pga_wait(&i_full[j % kPtInfo], (unsigned)(j / kPtInfo) & 1u, dead, P.err); __syncwarp(); };
    auto done = [&](uint64_t* bar) { pt_fence_async(); __syncwarp(); if (lane == 0) mbar_arrive(bar); };
    if (total > 0) {
      known(0);
      fetch(P.k, info[0].k_page, info[0], kr);
      fetch(P.v, info[0].v_page, info[0], vr);
    }
#pragma unroll 1
    for (int j = 0; j < total; ++j) {
      const PtTile& T = info[j % kPtInfo];
      const PtTile& N = info[(j + 1) % kPtInfo];
      if (j > 1) { pga_wait(&k_empty[j & 1], (unsigned)((j >> 1) - 1) & 1u, dead, P.err); __syncwarp(); }
      if (T.first) {                              // the item's query rows (once all scores of the item before are done): a lane has every fourth 16-byte piece of 8 rows a
                                                  // step, so that four lanes read 64 bytes of a row
        if (j > 0) { pga_wait(&k_empty[(j - 1) & 1], (unsigned)((j - 1) >> 1) & 1u, dead, P.err); __syncwarp(); }
        ++item;
        const int nr = T.nq * grp;
#pragma unroll 1
        for (int step = 0; step < 2 * MT; ++step) {
          const int at = (step >> 1) * 128 + cw * 16 + (step & 1) * 8 + (lane & 7), r = (step >> 1) * 128 + (at & 127) % RP, row = T.rt * RB + r;
          const bool there = r < RB && row < nr;
          const int tok = there ? row / grp : 0, h = T.kvh * grp + (there ? row - tok * grp : 0), d0 = (lane >> 3) * 8;
          const __nv_bfloat16* p = reinterpret_cast<const __nv_bfloat16*>(A.q) + (long long)(T.q0 + tok) * A.q_stride + (long long)h * HD + d0;
          uint4 q[NP];
#pragma unroll
          for (int i = 0; i < NP; ++i) q[i] = make_uint4(0, 0, 0, 0);
          if (there) {
            if (vec) {
#pragma unroll
              for (int i = 0; i < NP; ++i) q[i] = *reinterpret_cast<const uint4*>(p + i * 32);
            } else {
              const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
              for (int i = 0; i < NP; ++i)
                q[i] = make_uint4(u[i * 32] | (uint32_t)u[i * 32 + 1] << 16, u[i * 32 + 2] | (uint32_t)u[i * 32 + 3] << 16,
                                  u[i * 32 + 4] | (uint32_t)u[i * 32 + 5] << 16, u[i * 32 + 6] | (uint32_t)u[i * 32 + 7] << 16);
            }
          }
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < NP; ++i)
            top = __vmaxu2(top, __vmaxu2(__vmaxu2(q[i].x & 0x7FFF7FFFu, q[i].y & 0x7FFF7FFFu), __vmaxu2(q[i].z & 0x7FFF7FFFu, q[i].w & 0x7FFF7FFFu)));
          top = max(top & 0xFFFFu, top >> 16);
          top = max(top, __shfl_xor_sync(FULL, top, 8));
          top = max(top, __shfl_xor_sync(FULL, top, 16));
          // the largest value to 2^14 .. 2^15
          const int ex = min(max((int)(top >> 7) - 127, -100), 127);
          const float up = __uint_as_float((uint32_t)(127 + 14 - ex) << 23);
          if (lane < 8) s_cr[item & 3][at] = __uint_as_float((uint32_t)(127 - 14 + ex) << 23) * 256.0f;
          // (dims whose codes are shifted: 2^8 more; they are the second 16 of every 32, lanes 16 on)
          const float u = lane >= 16 ? up : up * (1.0f / 256.0f);
          auto half2 = [&](uint32_t v) { return pack_f16(__uint_as_float(v << 16) * u, __uint_as_float(v & 0xFFFF0000u) * u); };
          unsigned char* dst = sm + L::kQOff + (step >> 1) * L::kOp + (d0 >> 3) * 2048 + (at & 127) * 16;
#pragma unroll
          for (int i = 0; i < NP; ++i) *reinterpret_cast<uint4*>(dst + i * 4 * 2048) = make_uint4(half2(q[i].x), half2(q[i].y), half2(q[i].z), half2(q[i].w));
        }
      }
      put(sm + L::kKOff + (j & 1) * L::kOp, kr);
      done(&k_full[j & 1]);
      if (j + 1 < total) { known(j + 1); fetch(P.k, N.k_page, N, kr); }
      if (j > 1) { pga_wait(&v_empty[j & 1], (unsigned)((j >> 1) - 1) & 1u, dead, P.err); __syncwarp(); }
      put(sm + L::kVOff + (j & 1) * L::kOp, vr);
      done(&v_full[j & 1]);
      if (j + 1 < total) fetch(P.v, N.v_page, N, vr);
    }
  } else if (warp < W_CONV) {
    // ---- softmax ----
    const int m = MT == 2 ? warp >> 2 : 0, half = MT == 2 ? 0 : warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, t_o = tm_o + m * 128 + lanes;
    constexpr int COLS = 64 * MT / COPIES;        // the positions of a chunk that this thread takes, from col0 on
    const int part = COPIES == 1 ? 0 : row / RP, col0 = (part * (MT == 2 ? 1 : 2) + half) * COLS;
    constexpr int DIMS = MT == 2 ? HD : HD / 2;   // the dims of O that it rescales and writes, from dim0 on
    const int dim0 = half * DIMS;
    float M = kPgaFloor, l = 0.0f, cr = 0.0f, slope = 0.0f;
    int lim = 0, pos = 0, item = -1;
    unsigned long long bits = 0;
#pragma unroll 1
    for (int j = 0; j < total; ++j) {
      const PtTile& T = info[j % kPtInfo];
      const int b = MT == 2 ? m : (j & 1);
      const uint32_t t_s = tmem + b * 128 + lanes, t_p = MT == 2 ? t_s : tmem + 384 + b * 64 + lanes;
      pga_wait(&s_full[b], (unsigned)(MT == 2 ? j : (j >> 1)) & 1u, dead, P.err);
      __syncwarp();
      pt_fence_after();
      const bool first = T.first;
      if (first) {
        ++item;
        const int rr = T.rt * RB + m * 128 + row % RP, base = T.len - T.nq;
        const bool there = m * 128 + row % RP < RB && rr < T.nq * grp;
        const int i = there ? rr / grp : 0, h = T.kvh * grp + (there ? rr - i * grp : 0);
        M = kPgaFloor; l = 0.0f;
        cr = s_cr[item & 3][m * 128 + row] * (cap ? A.scale / A.softcap : A.scale * log2e);
        pos = base + i;
        lim = there ? max(0, max(A.tree ? base : min(T.len, base + i + 1), T.pre)) : 0;
        slope = there && A.slopes ? A.slopes[h] * log2e : 0.0f;
        bits = there && A.tree ? A.tree[T.q0 + i] : 0ull;
      }
      // Caps, biases and masks first, in place (16 columns, one page's, at a time); then every chunk is alike.
      const bool pre = cap || A.slopes || T.j0 + kPtChunk > T.lim_min || T.gaps;
      if (pre) {
#pragma unroll 1
        for (int c = col0; c < col0 + COLS; c += 16) {
          float x[16];
          pt_ld16(t_s + c, x);
          const float4 mt = T.meta[c >> 4];
          const float a = cr * mt.x;
          pt_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; i += 2) { const float2 y = mul2(make_float2(x[i], x[i + 1]), make_float2(a, a)); x[i] = y.x; x[i + 1] = y.y; }
          if (cap) {
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; i += 2) top = max3(top, fabsf(x[i]), fabsf(x[i + 1]));
            const float c2 = A.softcap * log2e;
            if (!__any_sync(FULL, !(top <= 0.5f))) {      // tanh y = y (1 - y^2 / 3 + ...): the next term is 9e-8
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                const float2 y = make_float2(x[i], x[i + 1]), z = mul2(y, y);
                float2 s = make_float2(0.0035921280f, 0.0035921280f);
                s = fma2(s, z, make_float2(-0.0088632355f, -0.0088632355f));
                s = fma2(s, z, make_float2(0.0218694885f, 0.0218694885f));
                s = fma2(s, z, make_float2(-0.0539682540f, -0.0539682540f));
                s = fma2(s, z, make_float2(0.1333333333f, 0.1333333333f));
                s = fma2(s, z, make_float2(-0.3333333333f, -0.3333333333f));
                s = mul2(fma2(mul2(s, z), y, y), make_float2(c2, c2));
                x[i] = s.x; x[i + 1] = s.y;
              }
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) x[i] = c2 * pga_tanh(x[i], ex2_approx(x[i] * (2.0f * log2e)));
            }
          }
          if (A.slopes) {
            const float d0 = (float)(pos - T.j0 - c);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = fmaf(-slope, fabsf(d0 - (float)i), x[i]);
          }
          if (T.j0 + c + 16 > T.lim_min || mt.y == -INFINITY) {
            uint32_t seen = 0;                    // of 16 positions
            if (mt.y != -INFINITY) {
              const int n = lim - T.j0 - c, d = T.j0 + c - (T.len - T.nq);
              seen = n >= 16 ? 0xFFFFu : (n > 0 ? (1u << n) - 1u : 0u);
              if (A.tree && d > -16 && d < 64) {
                uint32_t t = (uint32_t)(d >= 0 ? bits >> d : bits << -d);
                const int behind = T.nq - d;      // rows of the entry from here on
                seen |= t & (behind >= 16 ? 0xFFFFu : (behind > 0 ? (1u << behind) - 1u : 0u));
              }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) if (!((seen >> i) & 1u)) x[i] = -INFINITY;
          }
          pt_st16(t_s + c, reinterpret_cast<const uint32_t*>(x));
        }
        pt_wait_st();
      }
      // The largest exponent: of 16 raw scores, then scaled (the next ones are on their way meanwhile).
      float top = -INFINITY;
      {
        float x[2][16];
        pt_ld16(t_s + col0, x[0]);
#pragma unroll 1
        for (int c = 0; c < COLS; c += 32) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float4 mt = T.meta[(col0 + c + 16 * h) >> 4];
            const float a = pre ? 1.0f : cr * mt.x, *y = x[h];
            pt_wait_ld();
            pt_ld16(t_s + ((col0 + c + 16 * h + 16) & 127), x[h ^ 1]);
            float t = max3(y[0], y[1], y[2]);
#pragma unroll
            for (int i = 3; i < 15; i += 2) t = max3(t, y[i], y[i + 1]);
            top = max3(top, fmaf(fmaxf(t, y[15]), a, mt.y), top);
          }
        }
        pt_wait_ld();
      }
      if (MT == 1) {                              // both halves of the row's positions have one maximum
        s_top[j & 1][half][row] = top;
        pt_sync<1, 256>();
        top = fmaxf(top, s_top[j & 1][half ^ 1][row]);
      }
      const bool grow = top > M + kPgaSlack;
      if (__any_sync(FULL, grow)) {
        const float now = grow ? top : M, f = ex2_approx(M - now);
        M = now; l *= f;
        if (!first) {
          pga_wait(&o_done[m], (unsigned)(j - 1) & 1u, dead, P.err);
          __syncwarp();
          pt_fence_after();
#pragma unroll 1
          for (int c = dim0; c < dim0 + DIMS; c += 16) {
            float o[16];
            pt_ld16(t_o + c, o);
            pt_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= f;
            pt_st16(t_o + c, reinterpret_cast<const uint32_t*>(o));
          }
          pt_wait_st();
        }
      }
      // The weights: those of 32 positions take 16 columns (over scores that have been read); the positions of the other copy are zeros.
      {
        const float Mo = M - kPgaLift;
        float x[2][16];
        pt_ld16(t_s + col0, x[0]);
#pragma unroll 1
        for (int c = 0; c < COLS; c += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float4 mt = T.meta[(col0 + c + 16 * h) >> 4];
            const float a = pre ? 1.0f : cr * mt.x, bb = mt.y - Mo, *y = x[h];
            pt_wait_ld();
            pt_ld16(t_s + ((col0 + c + 16 * h + 16) & 127), x[h ^ 1]);
            float2 s0 = make_float2(0.0f, 0.0f), s1 = s0;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              float2 y0 = fma2(make_float2(y[i], y[i + 1]), make_float2(a, a), make_float2(bb, bb)), y1 = fma2(make_float2(y[i + 2], y[i + 3]), make_float2(a, a), make_float2(bb, bb));
              y0.x = ex2_approx(y0.x); y0.y = ex2_approx(y0.y); y1.x = ex2_approx(y1.x); y1.y = ex2_approx(y1.y);
              s0 = add2(s0, y0); s1 = add2(s1, y1);
              pk[8 * h + i / 2] = pack_f16(y0.x, y0.y);
              pk[8 * h + i / 2 + 1] = pack_f16(y1.x, y1.y);
            }
            s0 = add2(s0, s1);
            l = fmaf(s0.x + s0.y, mt.z, l);
          }
          pt_st16(t_p + ((col0 + c) >> 1), pk);
        }
        pt_wait_ld();
        if (COPIES == 2) {                        // (32 columns of zeros between the two threads of the row)
          uint32_t none[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) none[i] = 0;
          pt_st16(t_p + (part ^ 1) * 32 + half * 16, none);
        }
      }
      pt_wait_st();
      pt_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[b]);
      if (T.ends) {
        // the rows of O: the result, or this CTA's part of it
        pga_wait(&o_done[m], (unsigned)j & 1u, dead, P.err);
        __syncwarp();
        pt_fence_after();
        const int rows = min(RB, T.nq * grp - T.rt * RB), r = m * 128 + row % RP;
        float sum = l, top2 = M, f = 1.0f;
        if (MT == 1) {                            // the row's sums: of both halves of the positions, and of its copies
          s_ml[half][row] = make_float2(M, l);
          pt_sync<1, 256>();
          sum = 0.0f;
#pragma unroll
          for (int k = 0; k < COPIES; ++k) top2 = fmaxf(top2, s_ml[0][k * RP + row % RP].x);
#pragma unroll
          for (int k = 0; k < COPIES; ++k) {
            const float2 y = s_ml[0][k * RP + row % RP], z = s_ml[1][k * RP + row % RP];
            sum += (y.y + z.y) * ex2_approx(y.x - top2);
          }
          f = ex2_approx(M - top2);
        }
        const bool whole = T.whole, mine = r < rows && part == 0;
        const int rr = T.rt * RB + r, tok = rr / grp, h = T.kvh * grp + rr - tok * grp;
        const size_t slot = (size_t)(cta * 2 + T.slot) * A.part_rows + r;
        // (a row that saw nothing is 0; a sum that is not a number leaves its row that way)
        const float norm = whole ? (sum > 0.0f ? f / sum : (sum == 0.0f ? 0.0f : sum)) : f;
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(A.out) + (long long)(T.q0 + tok) * A.out_stride + (long long)h * HD;
        const bool vec32 = A.vec_q && (reinterpret_cast<uintptr_t>(out) & 31) == 0;
        float* buf = reinterpret_cast<float*>(sm + L::kEnd) + half * 64 * 17;      // MT = 1: [64][17] a block of 16 dims of the second copies
#pragma unroll 1
        for (int c = dim0; c < dim0 + DIMS; c += 16) {
          float o[16];
          pt_ld16(t_o + c, o);
          pt_wait_ld();
          const float g = c & 16 ? norm * 256.0f : norm;          // (the shifted dims)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] *= g;
          if (COPIES == 2) {
            if (part == 1)
#pragma unroll
              for (int i = 0; i < 16; ++i) buf[(row - RP) * 17 + i] = o[i];
            if (half == 0) pt_sync<2, 128>(); else pt_sync<3, 128>();
            if (part == 0)
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] += buf[row * 17 + i];
            if (half == 0) pt_sync<2, 128>(); else pt_sync<3, 128>();
          }
          if (mine) {
            if (whole) {
              if (vec32) {
                uint32_t u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = pack_bf16(o[2 * i], o[2 * i + 1]);
                stg32(out + c, u);
              } else {
                store8(out + c, A.vec_q, *reinterpret_cast<float (*)[8]>(o));
                store8(out + c + 8, A.vec_q, *reinterpret_cast<float (*)[8]>(o + 8));
              }
            } else {
              uint32_t* d = reinterpret_cast<uint32_t*>(A.part + slot * HD + c);
              stg32(d, reinterpret_cast<const uint32_t*>(o));
              stg32(d + 8, reinterpret_cast<const uint32_t*>(o) + 8);
            }
          }
        }
        if (mine && !whole && half == 0) *reinterpret_cast<float2*>(A.part_ml + slot * 2) = make_float2(top2, sum);
        if (tid == 0 && !whole) A.desc[cta * 2 + T.slot] = make_int4(1 | (T.to_end ? 2 : 0), T.e, T.kvh, T.rt);
        pt_fence_before();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&i_empty[j % kPtInfo]);
    }
  }
  __syncwarp();
  pt_fence_before();
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

}  // namespace tabed
