// Attention over a paged 8-bit cache for few query rows a KV head (decoding steps, short blocks), and for fp32 rows; more bf16 rows
// go to pages_attn_tc.cuh.
//
//   out_i = sum_j softmax_j(s_ij) v_j,   s_ij = cap(scale q_i k_j) - slope |pos_i - j|,   k = codes * scale of their page
//
// The bytes of the cache bound it (2 hd bytes and 4 hd flops per position and query row), so:
//   * the chunks (CH positions of one KV head) of all (entry, KV head, tile of rows) lie in one list, of which every CTA of a fixed grid
//     walks a contiguous part of equal cost: ragged batches and single long sequences split alike;
//   * a producer warp looks pages up (32 blocks of the table at a time) and brings a chunk's pages into a ring of stages with one bulk copy
//     per page, KV head and K or V, completing on an mbarrier; the scales travel beside them;
//   * four consumer warps take the codes from shared memory as they lie (no swizzle: a row of codes is 32 - 128 bytes) and turn
//     them into fp16 (exact) on the way into the fragments of mma.sync m16n8k16: scores with the query rows as A and positions as
//     columns, whose accumulators are then the A fragments of P V.  The summed indices of both products (dims of q k, positions of P V) and the
//     output columns are dealt so that a lane reads 4 - 16 neighbouring bytes: position pairs of V are interleaved with prmt;
//   * a warp has 16 rows (8 of them live where there are no more) and a slice of the chunk, or a tile of rows of its own
//     (WR = 1, 2 or 4 tiles of rows a CTA): with up to 16 rows the warps share them and meet at the end of a segment.
// Numbers.  q is scaled by a power of two per row and rounded to fp16: exact for bf16 values; fp32 rows take a second term (22 bits).
// With v's scale inside the exponent, w_j = 2^(s_j log2 e + log2 vs_j - M), the sum of w V needs no scale and the sum of
// weights is that of w_j / vs_j (a page of zeros has vs = 2^-126: kPgaLeastV).  w is rounded to fp16 (11 bits; a second term for fp32 rows), at up to 2^15 so that small ones keep them.  Sums are fp32.
// M only moves when a score exceeds it by more than 6, so the sums are rarely rescaled (all rows of a warp with one that needs it).
// Sequences that span CTAs are put together by k_pages_attn_join from the partial results, in fixed order.
//
// Measured (B200, replayed from a graph): 96 sequences of 256 - 4096 tokens, 12 heads of 64, one row: 72 us with the join for 321 MB, 4.45 TB/s,
// 0.68 of the measured copy rate; 8 KV heads of 128, 4 rows each, 114 us for 429 MB, 3.8 TB/s (168 registers: two CTAs an SM).  fp32 rows in
// number, 2 x 1024 against 2111 - 4096 tokens, 32 / 8 heads of 128: 956 us, 83 TFLOP/s (tiles of 64 rows, two terms of q and of the weights).  Four sequences of 65537 - 262144 tokens, 14 / 2 heads: 44 us for 168 MB (25.6 at the copy rate).  Parts of equal length instead of
// equal cost, at an earlier state: 110 and 77 us against 105 and 49 (the parallel join came with it).
#pragma once
#include "pages_kernels.cuh"

namespace tabed {

constexpr int kPgaWarps = 4;                     // consumers
constexpr int kPgaThreads = 32 * (kPgaWarps + 1);
constexpr int kPgaMaxCtas = 512;                 // of kPgaMaxRows query rows each, or kPtMaxCtas of kPtMaxRows (pages_attn_tc.cuh)
constexpr int kPgaStart = 3;                     // chunks that an item's beginning and end cost
constexpr int kPgaMaxRows = 16 * kPgaWarps;      // query rows of a CTA
template <int HD> __host__ __device__ constexpr int pga_chunk() { return HD == 128 ? 64 : 128; }
template <int HD> __host__ __device__ constexpr int pga_stages() { return 4; }
template <int HD> __host__ __device__ constexpr int pga_stage_bytes() { return 2 * pga_chunk<HD>() * HD; }
// stages, and the states of the warps at a segment's end: 64 rows (4 slices of 16, 2 of 32, 1 of 64), or 4 slices of 8
template <int HD, bool R8> __host__ __device__ constexpr int pga_state_rows() { return R8 ? 8 * kPgaWarps : kPgaMaxRows; }
template <int HD, bool R8> __host__ __device__ constexpr size_t pga_smem() { return (size_t)pga_stages<HD>() * pga_stage_bytes<HD>() + (size_t)pga_state_rows<HD, R8>() * (HD + 2) * 4; }

struct PagesAttnArgs {
  PagesDev P;
  int layer, n, n_tokens, max_new, H, WR, RB, vec_q;     // WR tiles of rows by warp; rows of a CTA: 16 WR, or 8
  const int *seq, *first, *length;
  const void* q;
  void* out;
  long long q_stride, out_stride;
  float scale, softcap;
  const float* slopes;
  const int* prefix;
  const unsigned long long* tree;
  float* part;                        // [CTAs][2][part_rows][hd] partial outputs, then [..][rows][2] maxima and sums
  float* part_ml;
  int part_rows;                      // rows of a part
  int4* desc;                         // [CTAs][2] {valid | finished << 1, entry, KV head, tile of rows}
};

struct PgaEntry { int seq, q0, nq, len, pre, bad; };

// What an entry asks for, with its lengths brought into range; CTA 0 records `bad`.
__device__ __forceinline__ PgaEntry pga_entry(const PagesAttnArgs& A, int e) {
  PgaEntry E;
  const int f0 = A.first[e], f1 = A.first[e + 1];
  E.seq = A.seq ? A.seq[e] : e;
  E.len = A.length[e];
  E.pre = A.prefix ? A.prefix[e] : 0;
  E.bad = 0;
  if (f0 < 0 || f1 < f0 || f1 > A.n_tokens) { E.q0 = 0; E.nq = 0; E.len = 0; E.pre = 0; E.bad = PGERR_INVALID; return E; }
  E.q0 = f0; E.nq = f1 - f0;
  if (E.seq < 0 || E.seq >= A.P.n_seqs || E.len < 0 || E.nq > A.max_new || (A.tree && E.nq > 64)) { E.seq = 0; E.len = 0; E.bad = PGERR_INVALID; }
  if ((long long)E.len > (long long)A.P.max_pages * A.P.ps) { E.len = 0; E.bad = PERR_KV; }
  E.pre = min(max(E.pre, 0), E.len);
  return E;
}
// positions below this one are seen by query row r of an entry (with a tree: and those of its mask)
__device__ __forceinline__ int pga_limit(const PagesAttnArgs& A, const PgaEntry& E, int r, int grp) {
  const int base = E.len - E.nq;
  return max(0, max(A.tree ? base : min(E.len, base + r / grp + 1), E.pre));
}

// The list of all chunks of CH positions: (entry, KV head, tile of RB query rows, chunk); a tile has the chunks up to the last position that one of
// its rows sees (one at least, which writes the zeros of rows that see nothing).
template <int CH>
struct PgaWalk {
  int e, kvh, rt, ch, nrt, nch, last;
  PgaEntry E;
  __device__ __forceinline__ void tile(const PagesAttnArgs& A, int grp) {
    last = A.tree ? E.len : pga_limit(A, E, min(E.nq * grp, (rt + 1) * A.RB) - 1, grp);
    nch = max(1, (last + CH - 1) / CH);
  }
  __device__ __forceinline__ void entry(const PagesAttnArgs& A, int grp) {
    E = pga_entry(A, e);
    nrt = (int)(((long long)E.nq * grp + A.RB - 1) / A.RB);
  }
  __device__ __forceinline__ long long head_chunks(const PagesAttnArgs& A, int grp) {      // of one KV head of the entry
    long long n = 0;
    rt = 0;
    if (nrt == 1) { tile(A, grp); return nch; }
#pragma unroll 1
    for (; rt < nrt; ++rt) { tile(A, grp); n += nch; }
    return n;
  }
  __device__ __forceinline__ void step(const PagesAttnArgs& A, int grp) {                   // to the next chunk; there is one
    if (++ch < nch) return;
    ch = 0;
    if (++rt >= nrt) {
      rt = 0;
      if (++kvh >= A.P.Hkv) {
        kvh = 0;
#pragma unroll 1
        do { ++e; entry(A, grp); } while (nrt == 0 && e + 1 < A.n);
      }
    }
    tile(A, grp);
  }
};

struct PgaShare { long long part[16][2]; int e, kvh, rt, ch, chunk[2]; };

// The CTA's part of the list: where it begins, and its chunks (0: none).  Beginning and ending an item costs about START chunks, so the list
// is cut into equal parts of chunks and that many more per item: a part of short sequences has fewer chunks.  All THREADS threads take part,
// each summing a strip of entries.  (A list of 2^31 chunks, 10^11 positions, is refused.)
template <int CH, int START, int THREADS>
__device__ __forceinline__ int pga_begin(const PagesAttnArgs& A, PgaShare& S, PgaWalk<CH>& w) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x, grp = A.H / A.P.Hkv, Hkv = A.P.Hkv;
  const int per = (A.n + THREADS - 1) / THREADS, e0 = min(A.n, tid * per), e1 = min(A.n, e0 + per);
  long long mine = 0, chunks = 0;                // cost, chunks of the strip
#pragma unroll 1
  for (w.e = e0; w.e < e1; ++w.e) {
    w.entry(A, grp);
    if (w.E.bad && cta == 0) atomicOr(A.P.err, w.E.bad);
    const long long c = w.head_chunks(A, grp) * Hkv;
    chunks += c;
    mine += c + (long long)w.nrt * START * Hkv;
  }
  long long x = mine, y = chunks;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long a = __shfl_up_sync(0xffffffffu, x, o), b = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) { x += a; y += b; }
  }
  if (lane == 31) { S.part[warp][0] = x; S.part[warp][1] = y; }
  if (tid < 2) S.chunk[tid] = 0;
  __syncthreads();
  long long before = x - mine, chunks_before = y - chunks, all64 = 0, all_chunks = 0;
#pragma unroll 1
  for (int i = 0; i < THREADS / 32; ++i) {
    if (i < warp) { before += S.part[i][0]; chunks_before += S.part[i][1]; }
    all64 += S.part[i][0]; all_chunks += S.part[i][1];
  }
  if (all64 > 0x7FFFFFFFll) { if (tid == 0) atomicOr(A.P.err, PGERR_INVALID); return 0; }
  const int all = (int)all64, nc = min((int)all_chunks, (int)gridDim.x), each = nc > 0 ? all / nc : 0, extra = all - each * nc;
  // both ends of the part in the list
#pragma unroll 1
  for (int end = 0; end < 2; ++end) {
    const int c = cta + end, at = c >= nc ? all : c * each + min(c, extra);
    if (at >= all) { if (tid == 0) S.chunk[end] = (int)all_chunks; continue; }
    if ((int)before <= at && at < (int)(before + mine)) {
      int left = at - (int)before, done = (int)chunks_before, per_head = 0, cost = 0;
#pragma unroll 1
      for (w.e = e0;; ++w.e) {
        w.entry(A, grp);
        per_head = (int)w.head_chunks(A, grp);
        cost = per_head + w.nrt * START;
        if (left < cost * Hkv) break;
        left -= cost * Hkv;
        done += per_head * Hkv;
      }
      const int kvh = left / cost;
      left -= kvh * cost;
      done += kvh * per_head;
#pragma unroll 1
      for (w.rt = 0;; ++w.rt) { w.tile(A, grp); if (left < w.nch + START) break; left -= w.nch + START; done += w.nch; }
      // (an item's start is not divided: whoever is cut in it has the item's first chunk first)
      const int ch = max(0, left - START);
      S.chunk[end] = done + ch;
      if (end == 0) { S.e = w.e; S.kvh = kvh; S.rt = w.rt; S.ch = ch; }
    }
  }
  __syncthreads();
  const int count = S.chunk[1] - S.chunk[0];
  if (count > 0) {
    w.e = S.e; w.kvh = S.kvh; w.rt = S.rt;
    w.entry(A, grp);
    w.tile(A, grp);
    w.ch = S.ch;
  }
  return count;
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// tanh to 2^-21 of its value: the quotient loses what is small against 1, and a cap far above the scores would multiply that; below 0.3 its
// Taylor series (the term left out is 5e-8 of it there).
__device__ __forceinline__ float pga_tanh(float y, float ex2_of_2y) {
  const float z = y * y;
  const float s = fmaf(fmaf(fmaf(0.0218694885f, z, -0.0539682540f), z, 0.1333333333f), z, -0.3333333333f);
  return fabsf(y) < 0.3f ? fmaf(s * z, y, y) : 1.0f - 2.0f * rcp_approx(1.0f + ex2_of_2y);
}
// bounded wait of a warp; false if it ran out (recorded)
__device__ __forceinline__ bool pga_wait(uint64_t* bar, unsigned parity, volatile int* dead, int* err) {
  unsigned spins = 0;
  while (!mbar_try_wait(bar, parity)) {
    if (*dead) return false;
    if (++spins > (1u << 20)) { atomicOr(err, PERR_COPY); *dead = 1; return false; }
    if (spins > 4096) __nanosleep(64);
  }
  return true;
}

template <int N> struct PgaBytes;
template <> struct PgaBytes<4> { uint32_t w[1]; __device__ __forceinline__ void load(const uint8_t* p) { w[0] = *reinterpret_cast<const uint32_t*>(p); } };
template <> struct PgaBytes<8> { uint32_t w[2]; __device__ __forceinline__ void load(const uint8_t* p) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; } };
template <> struct PgaBytes<16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const uint8_t* p) { const uint4 v = *reinterpret_cast<const uint4*>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
};

// V of a scale below this counts as zero, and log2 of the scale in the exponents stops here.  With s the least scale there and S the largest that a
// row sees, the sum of weights is 2^15 / s a position at most (2^31 of them: 2^118), and what ex2 flushes in it is below 2^-135 S / s of the
// largest weight (2^-63 S): with s = 2^-126, a page of zeros, the one was infinite and the other as large as the weights.
constexpr float kPgaLeastV = 0x1p-72f, kPgaLeastLog = -72.0f;
// of 16 positions: scale of k, log2 of v's scale, 1 / it
__device__ __forceinline__ float4 pga_meta(float ks, float vs, bool there) {
  const float lv = fmaxf(lg2_approx(vs), kPgaLeastLog);
  return there ? make_float4(ks, lv, ex2_approx(-lv), 0.0f) : make_float4(0.0f, -INFINITY, 0.0f, 0.0f);
}

constexpr float kPgaFloor = -1e30f;              // the running maximum of a row that has seen nothing
constexpr float kPgaSlack = 6.0f, kPgaLift = 9.0f;       // weights are at most 2^(slack + lift) = 2^15

// TWO: fp32 rows (two fp16 terms of q and of the weights).  R8: no entry has more than 8 rows a KV head.
template <int HD, bool TWO, bool R8>
__global__ void __launch_bounds__(kPgaThreads) k_pages_attn(const PagesAttnArgs A) {
  constexpr int CH = pga_chunk<HD>(), NS = pga_stages<HD>(), STAGE = pga_stage_bytes<HD>(), KS = HD / 16, NO = HD / 8;
  constexpr int NG = HD == 128 ? 1 : 2, SB = 16 * NG;         // positions that a warp takes at once
  constexpr unsigned FULL = 0xffffffffu;
  extern __shared__ __align__(128) unsigned char pga_smem_raw[];
  unsigned char* ring = pga_smem_raw;
  float* so = reinterpret_cast<float*>(pga_smem_raw + NS * STAGE);        // [slices][rows][HD] states of the warps at a segment's end
  float* sml = so + pga_state_rows<HD, R8>() * HD;                                      // [slices][rows][2]
  __shared__ uint64_t full[NS], empty[NS];
  __shared__ float4 meta[NS][CH / 16];           // (pga_meta)
  __shared__ PgaShare s_share;
  __shared__ int s_dead;
  const PagesDev& P = A.P;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
  const int H = A.H, Hkv = P.Hkv, grp = H / Hkv, ps = P.ps, WR = A.WR, WT = kPgaWarps / WR, RB = R8 ? 8 : 16 * WR;
  if (tid == 0) {
    for (int i = 0; i < NS; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], kPgaWarps); }
    s_dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_trigger();
  pdl_wait();
  if (tid < 2) A.desc[cta * 2 + tid] = make_int4(0, 0, 0, 0);
  PgaWalk<CH> w;
  const int total = pga_begin<CH, kPgaStart, kPgaThreads>(A, s_share, w);
  if (total == 0) return;
  PgaEntry& E = w.E;

  if (warp == kPgaWarps) {
    // ---- producer ----
    int cb = -1, ce = -1, ck = -1;               // block that lane 0 has looked up, entry, KV head
    int pg = -1;
    float pks = 1.0f, pvs = 1.0f;
    unsigned none = 0;                           // blocks from cb on whose V is not there or counts as zero
    const int ppc = ps < CH ? CH / ps : 1;       // pages of a chunk
    const int rows = ps < CH ? ps : CH;          // positions that it takes of each
    bool ok = true;
    int c = 0;
    for (; c < total; ++c) {
      const int st = c % NS;
      if (c >= NS) { ok = pga_wait(&empty[st], (unsigned)(c / NS - 1) & 1u, &s_dead, P.err); ok = __all_sync(FULL, ok); if (!ok) break; }
      const int p0 = w.ch * CH, blk0 = p0 >> P.ls, nblk = (E.len + ps - 1) >> P.ls;
      if (w.e != ce || blk0 < cb || blk0 + ppc > cb + 32) {
        cb = blk0; ce = w.e; ck = -1;
        const int b = cb + lane;
        pg = b < nblk ? P.table[(size_t)E.seq * P.max_pages + b] : -1;
        if (b < nblk && (pg < 0 || pg >= P.NP)) { atomicOr(P.err, PGERR_INVALID); pg = -2; }
      }
      if (w.kvh != ck) {
        ck = w.kvh;
        if (pg >= 0) {
          const size_t at = ((size_t)A.layer * P.NP + pg) * Hkv + w.kvh;
          pks = P.k_scale[at]; pvs = P.v_scale[at];
        }
        none = __ballot_sync(FULL, pg == -2 || (pg >= 0 && pvs < kPgaLeastV));
      }
      const int mypg = __shfl_sync(FULL, pg, min(blk0 + lane - cb, 31) & 31);
      const bool inside = lane < ppc && blk0 + lane < nblk, no_v = inside && ((none >> ((blk0 + lane - cb) & 31)) & 1u);
      const bool has = inside && mypg >= 0, has_v = has && !no_v;
      const unsigned bytes = (unsigned)rows * HD, copies = __popc(__ballot_sync(FULL, has)) + __popc(__ballot_sync(FULL, has_v));
      unsigned char* sk = ring + st * STAGE;
      {
        const int src = (((p0 + lane * 16) >> P.ls) - cb) & 31;       // (lanes beyond the chunk's groups read something and drop it)
        const float ks = __shfl_sync(FULL, pks, src), vs = __shfl_sync(FULL, pvs, src);
        const int gp = __shfl_sync(FULL, pg, src);
        if (lane < CH / 16) meta[st][lane] = pga_meta(ks, vs, gp >= 0);
      }
      if (none) {                                // zeros where no copy comes (K too, where there is no page: nothing stale)
        for (unsigned left = __ballot_sync(FULL, no_v); left; left &= left - 1) {
          const unsigned b = __ffs(left) - 1;
          for (unsigned i = lane * 16; i < bytes; i += 512) *reinterpret_cast<uint4*>(sk + CH * HD + b * bytes + i) = make_uint4(0, 0, 0, 0);
        }
        for (unsigned left = __ballot_sync(FULL, inside && mypg < 0); left; left &= left - 1) {
          const unsigned b = __ffs(left) - 1;
          for (unsigned i = lane * 16; i < bytes; i += 512) *reinterpret_cast<uint4*>(sk + b * bytes + i) = make_uint4(0, 0, 0, 0);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      __syncwarp();
      if (lane == 0) { if (copies) mbar_expect_tx(&full[st], copies * bytes); else mbar_arrive(&full[st]); }
      __syncwarp();
      if (has) {
        const size_t at = (((size_t)A.layer * P.NP + mypg) * Hkv + w.kvh) * ps * HD + (size_t)(ps > CH ? p0 & (ps - 1) : 0) * HD;
        bulk_g2s(sk + lane * bytes, P.k + at, bytes, &full[st]);
        if (has_v) bulk_g2s(sk + CH * HD + lane * bytes, P.v + at, bytes, &full[st]);
      }
      if (c + 1 < total) w.step(A, grp);
    }
    if (lane == 0) {                             // the last copies land before the shared memory goes, whatever the consumers did
      for (int i = max(0, c - NS); i < c; ++i) {
        unsigned spins = 0;
        while (!mbar_try_wait(&full[i % NS], (unsigned)(i / NS) & 1u) && ++spins < (1u << 16)) __nanosleep(64);
      }
    }
    return;
  }

  // ---- consumers ----
  const int g = lane >> 2, t = lane & 3, wr = warp % WR, wt = warp / WR, TS = CH / WT;
  const int perm = (g & ~1) + ((g & 1) ^ ((g >> 1) & 1));      // position of column g among 8, and of a lane's two columns:
  const int c0 = 2 * t + (t & 1), c1 = 2 * t + 1 - (t & 1);
  const float log2e = 1.4426950408889634f;
  const bool cap = A.softcap > 0.0f, slow = cap || A.slopes != nullptr;
  uint32_t qf[TWO ? 2 : 1][KS][4];
  float o[NO][4], M[2], l[2], cr[2], slope[2];
  int lim[2], pos[2], lim_min = 0, lim_max = 0, base = 0;
  unsigned long long bits[2] = {0, 0};
  bool whole_from = false, live = true;
  int nr = 0;

  auto load_q = [&]() {
    nr = E.nq * grp;
    base = E.len - E.nq;
    const int r_lo = w.rt * RB + wr * 16, r_hi = min(nr, r_lo + 16) - 1;
    live = r_lo < nr;
    lim_min = live ? pga_limit(A, E, r_lo, grp) : 0;
    lim_max = !live ? 0 : (A.tree ? E.len : pga_limit(A, E, r_hi, grp));
#pragma unroll
    for (int x = 0; x < (R8 ? 1 : 2); ++x) {
      const int r = r_lo + g + 8 * x;
      const bool there = r < nr;
      const int i = there ? r / grp : 0, h = w.kvh * grp + (there ? r - i * grp : 0);
      pos[x] = base + i;
      lim[x] = there ? pga_limit(A, E, r, grp) : 0;
      bits[x] = there && A.tree ? A.tree[E.q0 + i] : 0ull;
      slope[x] = there && A.slopes ? A.slopes[h] * log2e : 0.0f;
      float v[HD / 4];
      const long long at = (long long)(E.q0 + i) * A.q_stride + (long long)h * HD;
#pragma unroll
      for (int k = 0; k < HD / 32; ++k) {        // the dims of a lane: the 8 or 16 bytes of a row of codes that it reads
        const int d = HD == 32 ? t * 8 : (k >> 1) * 64 + t * 16 + (k & 1) * 8;
        float f[8];
        if (!there) {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = 0.0f;
        } else if (TWO) load8(reinterpret_cast<const float*>(A.q) + at + d, A.vec_q, f);
        else load8(reinterpret_cast<const __nv_bfloat16*>(A.q) + at + d, A.vec_q, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[k * 8 + j] = f[j];
      }
      float amax = 0.0f;
#pragma unroll
      for (int j = 0; j < HD / 4; ++j) amax = fmaxf(amax, fabsf(v[j]));
      amax = fmaxf(amax, __shfl_xor_sync(FULL, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(FULL, amax, 2));
      // largest value of the row to 2^14 .. 2^15
      const int ex = min(max((int)(__float_as_uint(amax) >> 23) - 127, -100), 127);
      const float up = __uint_as_float((uint32_t)(127 + 14 - ex) << 23), down = __uint_as_float((uint32_t)(127 - 14 + ex) << 23);
      cr[x] = cap ? A.scale / A.softcap * down : A.scale * log2e * down;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const float a = v[4 * ks] * up, b = v[4 * ks + 1] * up, cc = v[4 * ks + 2] * up, d = v[4 * ks + 3] * up;
        qf[0][ks][x] = pack_f16(a, b);
        qf[0][ks][2 + x] = pack_f16(cc, d);
        if (TWO) {
          const float2 h0 = f16x2_to_float2(qf[0][ks][x]), h1 = f16x2_to_float2(qf[0][ks][2 + x]);
          qf[TWO ? 1 : 0][ks][x] = pack_f16(a - h0.x, b - h0.y);
          qf[TWO ? 1 : 0][ks][2 + x] = pack_f16(cc - h1.x, d - h1.y);
        }
      }
      M[x] = kPgaFloor; l[x] = 0.0f;
    }
    if (R8) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) { qf[0][ks][1] = 0; qf[0][ks][3] = 0; if (TWO) { qf[TWO ? 1 : 0][ks][1] = 0; qf[TWO ? 1 : 0][ks][3] = 0; } }
    }
#pragma unroll
    for (int i = 0; i < NO; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
  };

  // SB positions from `j0` of the sequence, `in` of the chunk
  auto attend = [&](const unsigned char* sk, const float4* mt, int in, int j0) {
    constexpr int NX = R8 ? 2 : 4;
    float s[NG][2][4];
#pragma unroll
    for (int gg = 0; gg < NG; ++gg)
#pragma unroll
      for (int a = 0; a < 2; ++a) {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[gg][a][j] = 0.0f;
        const unsigned char* row = sk + (in + 16 * gg + 8 * a + perm) * HD;
#pragma unroll
        for (int b = 0; b < (HD == 128 ? 2 : 1); ++b) {
          PgaBytes<HD == 32 ? 8 : 16> kb;
          kb.load(row + b * 64 + t * (HD == 32 ? 8 : 16));
#pragma unroll
          for (int k = 0; k < (HD == 32 ? 2 : 4); ++k) {
            uint32_t b0, b1;
            e4m3x4_to_f16x4(kb.w[k], b0, b1);
            const int ks = b * 4 + k;
            mma_f16(s[gg][a], qf[0][ks][0], qf[0][ks][1], qf[0][ks][2], qf[0][ks][3], b0, b1);
            if (TWO) mma_f16(s[gg][a], qf[TWO ? 1 : 0][ks][0], qf[TWO ? 1 : 0][ks][1], qf[TWO ? 1 : 0][ks][2], qf[TWO ? 1 : 0][ks][3], b0, b1);
          }
        }
      }
    const bool edge = j0 + SB > lim_min;         // some row does not see all of these positions
    // scores in base 2, v's scale included
#pragma unroll
    for (int gg = 0; gg < NG; ++gg) {
      const float4 m = mt[(in >> 4) + gg];
      if (!slow) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int j = 0; j < NX; ++j) s[gg][a][j] = fmaf(s[gg][a][j], cr[j >> 1] * m.x, m.y);
      } else {
        const int jg = j0 + 16 * gg;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int j = 0; j < NX; ++j) {
            float z = s[gg][a][j] * (cr[j >> 1] * m.x);
            if (cap) z = (A.softcap * log2e) * pga_tanh(z, ex2_approx(z * (2.0f * log2e)));
            z -= slope[j >> 1] * fabsf((float)(pos[j >> 1] - (jg + 8 * a + ((j & 1) ? c1 : c0))));
            s[gg][a][j] = z + m.y;
          }
      }
    }
    if (edge) {
#pragma unroll
      for (int gg = 0; gg < NG; ++gg)
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int j = 0; j < NX; ++j) {
            const int jp = j0 + 16 * gg + 8 * a + ((j & 1) ? c1 : c0), d = jp - base;
            bool seen = jp < lim[j >> 1];
            if (A.tree) seen = seen || (jp < E.len && d >= 0 && d < 64 && ((bits[j >> 1] >> (d & 63)) & 1ull));
            if (!seen) s[gg][a][j] = -INFINITY;
          }
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int gg = 0; gg < NG; ++gg)
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int j = 0; j < NX; ++j) top[j >> 1] = fmaxf(top[j >> 1], s[gg][a][j]);
    const bool grow = top[0] > M[0] + kPgaSlack || (!R8 && top[1] > M[1] + kPgaSlack);
    if (__any_sync(FULL, grow)) {
#pragma unroll
      for (int x = 0; x < (R8 ? 1 : 2); ++x) {
        float n = top[x];
        n = fmaxf(n, __shfl_xor_sync(FULL, n, 1));
        n = fmaxf(n, __shfl_xor_sync(FULL, n, 2));
        n = fmaxf(n, M[x]);
        const float f = ex2_approx(M[x] - n);
        M[x] = n; l[x] *= f;
#pragma unroll
        for (int i = 0; i < NO; ++i) { o[i][2 * x] *= f; o[i][2 * x + 1] *= f; }
      }
    }
#pragma unroll
    for (int gg = 0; gg < NG; ++gg) {
      const float inv = mt[(in >> 4) + gg].z;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int j = 0; j < NX; ++j) {
          const float p = ex2_approx(s[gg][a][j] - (M[j >> 1] - kPgaLift));
          l[j >> 1] = fmaf(p, inv, l[j >> 1]);
          s[gg][a][j] = p;
        }
      uint32_t ph[4], pl[4];
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (R8 && x == 1) { ph[2 * a + 1] = 0; pl[2 * a + 1] = 0; continue; }
          ph[2 * a + x] = pack_f16(s[gg][a][2 * x], s[gg][a][2 * x + 1]);
          if (TWO) {
            const float2 h = f16x2_to_float2(ph[2 * a + x]);
            pl[2 * a + x] = pack_f16(s[gg][a][2 * x] - h.x, s[gg][a][2 * x + 1] - h.y);
          }
        }
      // the lane's four positions of V: pairs (c0, c1) of the group's two halves, NO neighbouring dims
      const unsigned char* vr = sk + CH * HD + (in + 16 * gg) * HD + g * NO;
      PgaBytes<NO> v[4];
      v[0].load(vr + c0 * HD); v[1].load(vr + c1 * HD); v[2].load(vr + (8 + c0) * HD); v[3].load(vr + (8 + c1) * HD);
      if (edge) {                                // what lies behind the last position seen may be anything, and 0 * NaN is not 0
        const int jg = j0 + 16 * gg;
        const uint32_t k0 = jg + c0 < lim_max ? ~0u : 0u, k1 = jg + c1 < lim_max ? ~0u : 0u, k2 = jg + 8 + c0 < lim_max ? ~0u : 0u, k3 = jg + 8 + c1 < lim_max ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < NO / 4; ++i) { v[0].w[i] &= k0; v[1].w[i] &= k1; v[2].w[i] &= k2; v[3].w[i] &= k3; }
      }
#pragma unroll
      for (int i = 0; i < NO / 4; ++i) {
        uint32_t b[4][2];
        e4m3x4_to_f16x4(__byte_perm(v[0].w[i], v[1].w[i], 0x5140), b[0][0], b[1][0]);
        e4m3x4_to_f16x4(__byte_perm(v[0].w[i], v[1].w[i], 0x7362), b[2][0], b[3][0]);
        e4m3x4_to_f16x4(__byte_perm(v[2].w[i], v[3].w[i], 0x5140), b[0][1], b[1][1]);
        e4m3x4_to_f16x4(__byte_perm(v[2].w[i], v[3].w[i], 0x7362), b[2][1], b[3][1]);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          mma_f16(o[4 * i + d], ph[0], ph[1], ph[2], ph[3], b[d][0], b[d][1]);
          if (TWO) mma_f16(o[4 * i + d], pl[0], pl[1], pl[2], pl[3], b[d][0], b[d][1]);
        }
      }
    }
  };

  // one row's dims d .. d + 3 of the result
  auto put = [&](int r, int d, float4 v) {
    const int i = r / grp, h = w.kvh * grp + r - i * grp;
    const long long at = (long long)(E.q0 + i) * A.out_stride + (long long)h * HD + d;
    if (TWO) {
      float* p = reinterpret_cast<float*>(A.out) + at;
      if (A.vec_q) *reinterpret_cast<float4*>(p) = v;
      else { p[0] = v.x; p[1] = v.y; p[2] = v.z; p[3] = v.w; }
    } else {
      __nv_bfloat16* p = reinterpret_cast<__nv_bfloat16*>(A.out) + at;
      if (A.vec_q) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
      else { p[0] = __float2bfloat16_rn(v.x); p[1] = __float2bfloat16_rn(v.y); p[2] = __float2bfloat16_rn(v.z); p[3] = __float2bfloat16_rn(v.w); }
    }
  };

  // The segment's states to shared memory; all consumers put them together and write the result or the part.
  auto finish = [&](bool from_start, bool to_end) {
    const int slices = WT;
#pragma unroll
    for (int x = 0; x < (R8 ? 1 : 2); ++x) {
      float sum = l[x];
      sum += __shfl_xor_sync(FULL, sum, 1);
      sum += __shfl_xor_sync(FULL, sum, 2);
      const int rr = wr * 16 + g + 8 * x;
      if (w.rt * RB + rr < nr) {
        float* p = so + ((size_t)wt * RB + rr) * HD + 2 * t * NO;
#pragma unroll
        for (int i = 0; i < NO; i += 4) {
          *reinterpret_cast<float4*>(p + i) = make_float4(o[i][2 * x], o[i + 1][2 * x], o[i + 2][2 * x], o[i + 3][2 * x]);
          *reinterpret_cast<float4*>(p + NO + i) = make_float4(o[i][2 * x + 1], o[i + 1][2 * x + 1], o[i + 2][2 * x + 1], o[i + 3][2 * x + 1]);
        }
        if (t == 0) *reinterpret_cast<float2*>(sml + ((size_t)wt * RB + rr) * 2) = make_float2(M[x], sum);
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kPgaWarps) : "memory");
    const int rows = min(RB, nr - w.rt * RB);
    const bool whole = from_start && to_end;
    const int slot = cta * 2 + (from_start ? 1 : 0);
    for (int x = tid; x < rows * (HD / 4); x += 32 * kPgaWarps) {
      const int r = x / (HD / 4), d = (x - r * (HD / 4)) * 4;
      float m = kPgaFloor, sum = 0.0f;
      for (int k = 0; k < slices; ++k) m = fmaxf(m, sml[(k * RB + r) * 2]);
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int k = 0; k < slices; ++k) {
        const float f = ex2_approx(sml[(k * RB + r) * 2] - m);
        const float4 u = *reinterpret_cast<const float4*>(so + ((size_t)k * RB + r) * HD + d);
        sum += sml[(k * RB + r) * 2 + 1] * f;
        v.x += u.x * f; v.y += u.y * f; v.z += u.z * f; v.w += u.w * f;
      }
      if (whole) {
        const float f = sum > 0.0f ? 1.0f / sum : 0.0f;
        // (a sum that is not a number leaves its row that way)
        const bool none = sum == 0.0f;
        put(w.rt * RB + r, d, none ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : (sum > 0.0f ? make_float4(v.x * f, v.y * f, v.z * f, v.w * f) : make_float4(sum, sum, sum, sum)));
      } else {
        *reinterpret_cast<float4*>(A.part + ((size_t)slot * A.part_rows + r) * HD + d) = v;
        if (d == 0) *reinterpret_cast<float2*>(A.part_ml + ((size_t)slot * A.part_rows + r) * 2) = make_float2(m, sum);
      }
    }
    if (!whole && tid == 0) A.desc[slot] = make_int4(1 | (to_end ? 2 : 0), w.e, w.kvh, w.rt);
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kPgaWarps) : "memory");
  };

  // (a wait that ran out is recorded, and all others then return at once: the warps meet at every segment's end, so they run through)
  bool fresh = true;
  for (int c = 0; c < total; ++c) {
    const int st = c % NS;
    if (fresh) { whole_from = w.ch == 0; load_q(); fresh = false; }
    pga_wait(&full[st], (unsigned)(c / NS) & 1u, &s_dead, P.err);
    __syncwarp();
    const unsigned char* sk = ring + st * STAGE;
    const int j0 = w.ch * CH + wt * TS;
#pragma unroll 1
    for (int i = 0; i < TS; i += SB)
      if (j0 + i < lim_max) attend(sk, meta[st], wt * TS + i, j0 + i);
    __syncwarp();
    if (lane == 0) mbar_arrive(&empty[st]);
    if (w.ch == w.nch - 1 || c == total - 1) { finish(whole_from, w.ch == w.nch - 1); fresh = true; }
    if (c + 1 < total) w.step(A, grp);
  }
}

// Puts the parts of the items that span CTAs together: block (c, y) takes ROWS rows of the item that begins in CTA c and goes on behind
// it.  The weights of all parts come first (their loads are independent), then the parts' outputs, split over the threads that the rows leave.
constexpr int kJoinThreads = 256;

template <int HD, bool TWO, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) k_pages_attn_join(const PagesAttnArgs A) {
  constexpr int ITEMS = ROWS * HD / 4, SPLIT = kJoinThreads / ITEMS, PER_ROW = kJoinThreads / ROWS;
  __shared__ float s_f[ROWS][kPgaMaxCtas + 1], s_red[ROWS][2][PER_ROW / 32], s_sum[ROWS];
  __shared__ float4 s_v[SPLIT > 1 ? SPLIT - 1 : 1][ITEMS];
  __shared__ int s_n;
  const int c = blockIdx.x, tid = threadIdx.x, lane = tid & 31, grp = A.H / A.P.Hkv, RB = A.RB, r0 = blockIdx.y * ROWS;
  pdl_wait();
  pdl_trigger();
  const int4 d = A.desc[c * 2 + 1];
  if (!(d.x & 1)) return;
  const int e = d.y, kvh = d.z, rt = d.w;
  const PgaEntry E = pga_entry(A, e);
  const int rows = min(RB, E.nq * grp - rt * RB) - r0;
  if (rows <= 0) return;
  if (tid < 32) {                                // CTAs that have a part: up to the first that has its end
    int n = 1;
    for (int k = 1;; k += 32) {
      const int x = c + k + lane < (int)gridDim.x ? A.desc[(c + k + lane) * 2].x : 0;
      const unsigned stop = __ballot_sync(0xffffffffu, !(x & 1) || (x & 2)), ends = __ballot_sync(0xffffffffu, (x & 3) == 3);
      if (stop) { const int at = __ffs(stop) - 1; n += at + ((ends >> at) & 1); break; }
      n += 32;
    }
    if (lane == 0) s_n = n;
  }
  __syncthreads();
  const int n = s_n;
  auto slot = [&](int k) { return (size_t)(k == 0 ? c * 2 + 1 : (c + k) * 2) * A.part_rows + r0; };
  {
    const int r = tid / PER_ROW, t = tid - r * PER_ROW, w = t >> 5;
    float m = kPgaFloor, sum = 0.0f;
    if (r < rows)
      for (int k = t; k < n; k += PER_ROW) { const float x = A.part_ml[(slot(k) + r) * 2]; s_f[r][k] = x; m = fmaxf(m, x); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) s_red[r][0][w] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER_ROW / 32; ++i) m = fmaxf(m, s_red[r][0][i]);
    if (r < rows)
      for (int k = t; k < n; k += PER_ROW) {
        const float f = ex2_approx(s_f[r][k] - m);
        s_f[r][k] = f;
        sum += A.part_ml[(slot(k) + r) * 2 + 1] * f;
      }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_red[r][1][w] = sum;
    __syncthreads();
    if (tid < ROWS) {
      float x = 0.0f;
#pragma unroll
      for (int i = 0; i < PER_ROW / 32; ++i) x += s_red[tid][1][i];
      s_sum[tid] = x;
    }
    __syncthreads();
  }
  const int item = tid % ITEMS, part = tid / ITEMS, r = item / (HD / 4), dd = (item - r * (HD / 4)) * 4;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (r < rows) {
#pragma unroll 8
    for (int k = part; k < n; k += SPLIT) {
      const float4 u = *reinterpret_cast<const float4*>(A.part + (slot(k) + r) * HD + dd);
      const float f = s_f[r][k];
      v.x += u.x * f; v.y += u.y * f; v.z += u.z * f; v.w += u.w * f;
    }
  }
  if (part > 0) s_v[part - 1][item] = v;
  __syncthreads();
  if (part > 0 || r >= rows) return;
#pragma unroll
  for (int k = 0; k < SPLIT - 1; ++k) { const float4 u = s_v[k][item]; v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w; }
  const float sum = s_sum[r], f = sum > 0.0f ? 1.0f / sum : 0.0f;
  const int row = rt * RB + r0 + r, i = row / grp, h = kvh * grp + row - i * grp;
  const long long at = (long long)(E.q0 + i) * A.out_stride + (long long)h * HD + dd;
  v = sum == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : (sum > 0.0f ? make_float4(v.x * f, v.y * f, v.z * f, v.w * f) : make_float4(sum, sum, sum, sum));
  if (TWO) {
    float* p = reinterpret_cast<float*>(A.out) + at;
    if (A.vec_q) *reinterpret_cast<float4*>(p) = v;
    else { p[0] = v.x; p[1] = v.y; p[2] = v.z; p[3] = v.w; }
  } else {
    __nv_bfloat16* p = reinterpret_cast<__nv_bfloat16*>(A.out) + at;
    if (A.vec_q) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    else { p[0] = __float2bfloat16_rn(v.x); p[1] = __float2bfloat16_rn(v.y); p[2] = __float2bfloat16_rn(v.z); p[3] = __float2bfloat16_rn(v.w); }
  }
}

}  // namespace tabed
