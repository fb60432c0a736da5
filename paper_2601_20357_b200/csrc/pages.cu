// C boundary of the paged 8-bit caches.  See include/tabed.h for the contract of every entry point; the kernels live in
// pages_kernels.cuh / pages_attn.cuh.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/tabed.h"
#include "pages.h"
#include "pages_attn.cuh"
#include "pages_attn_tc.cuh"
#include "pages_kernels.cuh"

using namespace tabed;

namespace {

constexpr int kMaxDevices = 64;
constexpr int kMaxPageSeqs = 32767;       // counts of references and of entries share a word of `ref` while a fork runs

struct OnDevice {
  int prev = -1; bool ok = true;
  explicit OnDevice(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
  }
  ~OnDevice() { if (prev >= 0) cudaSetDevice(prev); }
};

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check(const tabed_pages* p) {
  if (!p) return TABED_ERR_NULL_PTR;
  if (!p->k || !p->v || !p->k_scale || !p->v_scale || !p->table || !p->ref || !p->err || !p->workspace) return TABED_ERR_NULL_PTR;
  if (p->n_layers < 1 || p->n_pages < 1 || p->n_kv_heads < 1 || p->n_seqs < 1 || p->n_seqs > kMaxPageSeqs || p->max_pages < 1 ||
      (p->page_tokens != 16 && p->page_tokens != 32 && p->page_tokens != 64 && p->page_tokens != 128) ||
      (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) || p->device < 0 || p->device >= kMaxDevices ||
      (long long)p->max_pages * p->page_tokens > 0x7FFFFF00ll || (long long)p->n_seqs * p->max_pages > 0x7FFFFFFFll || p->n_kv_heads > 1024 || p->n_layers > 32767)
    return TABED_ERR_INVALID_ARG;
  if (!aligned(p->k, 32) || !aligned(p->v, 32) || !aligned(p->workspace, 32)) return TABED_ERR_INVALID_ARG;
  return TABED_OK;
}

PagesDev on_device(const tabed_pages* p) {
  PagesDev d;
  d.k = static_cast<uint8_t*>(p->k); d.v = static_cast<uint8_t*>(p->v);
  d.k_scale = p->k_scale; d.v_scale = p->v_scale; d.table = p->table; d.ref = p->ref; d.err = p->err;
  d.L = p->n_layers; d.NP = p->n_pages; d.Hkv = p->n_kv_heads; d.ps = p->page_tokens; d.ls = p->page_tokens == 16 ? 4 : (p->page_tokens == 32 ? 5 : (p->page_tokens == 64 ? 6 : 7)); d.hd = p->head_dim;
  d.n_seqs = p->n_seqs; d.max_pages = p->max_pages;
  return d;
}

size_t round16(size_t x) { return (x + 15) & ~size_t(15); }

// the fork's scratch: entries, counters, the kept blocks of every entry, the free pages
size_t fork_free_pages(const tabed_pages* p) { return std::min((size_t)p->n_pages, (size_t)p->n_seqs * p->max_pages); }
size_t fork_bytes(const tabed_pages* p) {
  return round16((size_t)p->n_seqs * sizeof(ForkEntry)) + 16 + round16((size_t)p->n_seqs * p->max_pages * 4) + round16(fork_free_pages(p) * 4);
}
// the attention's: partial results of the segments at both ends of a CTA's part, their maxima and sums, what they belong to
constexpr size_t kPartRows = 2 * (size_t)std::max(kPgaMaxCtas * kPgaMaxRows, kPtMaxCtas * kPtMaxRows);
size_t attn_part_bytes(const tabed_pages* p) { return kPartRows * p->head_dim * 4; }
size_t attn_bytes(const tabed_pages* p) {
  return attn_part_bytes(p) + kPartRows * 2 * 4 + (size_t)kPgaMaxCtas * 2 * sizeof(int4);
}

// As a programmatic dependent of the kernel before it in the stream: every kernel here waits before it touches memory.
// early = false: when that kernel has ended (the joins: as dependents they slow the next attention's launch down, 96 sequences
// of 256 - 4096 tokens back to back 103 us, 71 so).
template <typename ArgT>
int launch(const tabed_pages* p, void (*kern)(ArgT), dim3 grid, int block, size_t smem, const ArgT& args, bool early = true) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = reinterpret_cast<cudaStream_t>(p->stream);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = early ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, kern, args) != cudaSuccess) { cudaGetLastError(); return TABED_ERR_CUDA; }
  return TABED_OK;
}

int sm_count(int dev) {
  static int n[kMaxDevices] = {0};
  if (n[dev] == 0) {
    int v = 0;
    if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v < 1) { cudaGetLastError(); return 148; }
    n[dev] = v;
  }
  return n[dev];
}

// rows of `heads` heads of `hd` values of `esz` bytes, `stride` values apart, start on 16-byte boundaries
bool rows_aligned(const void* p, long long stride, size_t esz) { return aligned(p, 16) && (stride * (long long)esz) % 16 == 0; }

template <typename T, int THREADS, int MAXI>
int launch_append_long(const tabed_pages* p, const AppendArgs& a, dim3 grid, size_t smem) {
  auto kern = k_pages_append<T, THREADS, MAXI>;
  static bool set[kMaxDevices] = {false};
  if (!set[p->device]) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MAXI * THREADS * 4 * (int)sizeof(float4)) != cudaSuccess) { cudaGetLastError(); return TABED_ERR_CUDA; }
    set[p->device] = true;
  }
  return launch(p, kern, grid, THREADS, smem, a);
}

// items: of 8 rotated pairs, that a head's tokens of a block are at most
template <typename T>
int launch_append(const tabed_pages* p, const AppendArgs& a, dim3 grid, int items, size_t smem) {
  if (items <= 32) return launch(p, k_pages_append<T, 32, 1>, grid, kAppendThreads, smem, a);
  if (items <= 256) return launch_append_long<T, 256, 1>(p, a, grid, smem);
  return items <= 512 ? launch_append_long<T, 512, 1>(p, a, grid, smem) : launch_append_long<T, 512, 2>(p, a, grid, smem);
}

// the launch of an append whose arguments are in place but for its geometry
int run_append(const tabed_pages* p, AppendArgs& a, bool f32) {
  const int ps = p->page_tokens, most = std::min(a.max_new, ps);      // tokens of a block
  a.nblk = (a.max_new + ps - 2) / ps + 1;
  // Units of a warp where a head's tokens of a block are one item a lane (a token of 128 values has 8 of them)
  const int items = most * (p->head_dim / 16);
  const bool small = items <= 32;
  const int heads = 2 * p->n_kv_heads + (a.has_q ? a.n_heads : 0);
  const long long blocks = (long long)a.n * a.nblk;
  if (blocks > 0x7FFFFFFFll) return TABED_ERR_UNSUPPORTED;
  // heads of a CTA: the cosines serve all of them, as long as the grid keeps some CTAs for every SM
  const int per = small ? kAppendThreads / 32 : 1;
  int groups = (int)std::min<long long>((heads + per - 1) / per, std::max<long long>(1, (8ll * sm_count(p->device) + blocks - 1) / blocks));
  a.hpc = ((heads + groups - 1) / groups + per - 1) / per * per;
  groups = (heads + a.hpc - 1) / a.hpc;
  const size_t smem = a.n_axes > 0 ? (size_t)items * 4 * sizeof(float4) : 0;
  const dim3 grid((unsigned)blocks, (unsigned)groups);
  return f32 ? launch_append<float>(p, a, grid, items, smem) : launch_append<__nv_bfloat16>(p, a, grid, items, smem);
}

constexpr int kJoinFew = 2, kJoinMany = 4;      // rows of a join's block

template <int HD, bool TWO, bool R8>
int launch_attn(const tabed_pages* p, const PagesAttnArgs& a) {
  auto kern = k_pages_attn<HD, TWO, R8>;
  static int per_sm[kMaxDevices] = {0};
  if (per_sm[p->device] == 0) {
    int n = 0;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pga_smem<HD, R8>()) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, kPgaThreads, pga_smem<HD, R8>()) != cudaSuccess || n < 1) {
      cudaGetLastError();
      return TABED_ERR_CUDA;
    }
    per_sm[p->device] = n;
  }
  const int ctas = std::min(kPgaMaxCtas, per_sm[p->device] * sm_count(p->device));
  const int rc = launch(p, kern, dim3(ctas), kPgaThreads, pga_smem<HD, R8>(), a);
  return rc != TABED_OK ? rc : launch(p, k_pages_attn_join<HD, TWO, kJoinFew>, dim3(ctas, (a.RB + kJoinFew - 1) / kJoinFew), kJoinThreads, 0, a, false);
}

template <int HD, int MT, int COPIES>
int launch_attn_tc(const tabed_pages* p, const PagesAttnArgs& a) {
  auto kern = k_pages_attn_tc<HD, MT, COPIES>;
  static bool set[kMaxDevices] = {false};
  if (!set[p->device]) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPtSmem) != cudaSuccess) { cudaGetLastError(); return TABED_ERR_CUDA; }
    set[p->device] = true;
  }
  const int ctas = std::min(kPtMaxCtas, sm_count(p->device));
  const int rc = launch(p, kern, dim3(ctas), Pt<HD, MT>::kThreads, kPtSmem, a);
  return rc != TABED_OK ? rc : launch(p, k_pages_attn_join<HD, false, kJoinMany>, dim3(ctas, (a.RB + kJoinMany - 1) / kJoinMany), kJoinThreads, 0, a, false);
}

template <int HD>
int launch_attn_hd(const tabed_pages* p, const PagesAttnArgs& a, bool f32) {
  if (a.part_rows == kPtMaxRows)
    return a.RB == 256 ? launch_attn_tc<HD, 2, 1>(p, a) : (a.RB == 128 ? launch_attn_tc<HD, 1, 1>(p, a) : launch_attn_tc<HD, 1, 2>(p, a));
  if (a.RB == 8) return f32 ? launch_attn<HD, true, true>(p, a) : launch_attn<HD, false, true>(p, a);
  return f32 ? launch_attn<HD, true, false>(p, a) : launch_attn<HD, false, false>(p, a);
}

}  // namespace

namespace tabed {

int pages_match(const tabed_pages* p, int L, int Hkv, int hd, int device) {
  const int rc = check(p);
  if (rc != TABED_OK) return rc;
  return p->n_layers == L && p->n_kv_heads == Hkv && p->head_dim == hd && p->device == device ? TABED_OK : TABED_ERR_INVALID_ARG;
}

// (a launch a layer: 4 layers of 12 heads of 64, 704 tokens 18 us, 8192 80 us; 12 layers of 2 heads, 4096 tokens 47 us)
int pages_store_row(const tabed_pages* p, cudaStream_t stream, const DenseRow& r, int seq, int start, int len, int64_t* launches) {
  tabed_pages here = *p;
  here.stream = stream;
  const int hd = p->head_dim;
  const size_t esz = r.f32 ? 4 : 2;
  AppendArgs a = {};
  a.P = on_device(p); a.n = 1; a.n_tokens = len; a.max_new = len; a.seq0 = seq; a.start0 = start; a.held = r.len;
  a.kv_stride = hd; a.kv_head = (long long)r.cap * hd; a.vec_kv = 1;
  for (a.layer = 0; a.layer < p->n_layers; ++a.layer) {
    const size_t at = ((size_t)a.layer * p->n_kv_heads * r.cap + start) * hd * esz;
    a.k = static_cast<const char*>(r.k) + at; a.v = static_cast<const char*>(r.v) + at;
    const int rc = run_append(&here, a, r.f32);
    if (rc != TABED_OK) return rc;
    ++*launches;
  }
  return TABED_OK;
}

int pages_load_row(const tabed_pages* p, cudaStream_t stream, const DenseRow& r, int seq, int len, int64_t* launches) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((len + p->page_tokens - 1) / p->page_tokens, 2 * p->n_kv_heads, p->n_layers); cfg.blockDim = dim3(128); cfg.stream = stream;
  const PagesDev d = on_device(p);
  const cudaError_t rc = r.f32 ? cudaLaunchKernelEx(&cfg, k_pages_load_row<float>, d, seq, len, static_cast<float*>(r.k), static_cast<float*>(r.v), r.cap, r.len)
                               : cudaLaunchKernelEx(&cfg, k_pages_load_row<__nv_bfloat16>, d, seq, len, static_cast<__nv_bfloat16*>(r.k), static_cast<__nv_bfloat16*>(r.v), r.cap, r.len);
  if (rc != cudaSuccess) { cudaGetLastError(); return TABED_ERR_CUDA; }
  ++*launches;
  return TABED_OK;
}

}  // namespace tabed

extern "C" {

int tabed_pages_workspace(const tabed_pages* p, size_t* bytes) {
  if (!p || !bytes) return TABED_ERR_NULL_PTR;
  if (p->n_pages < 1 || p->n_seqs < 1 || p->max_pages < 1 || p->head_dim < 1) return TABED_ERR_INVALID_ARG;
  *bytes = std::max(fork_bytes(p), attn_bytes(p));
  return TABED_OK;
}

int tabed_pages_fork(const tabed_pages* p, const int32_t* src, const int32_t* dst, const int32_t* keep, const int32_t* len, int32_t n) {
  const int rc0 = check(p);
  if (rc0 != TABED_OK) return rc0;
  if (n < 0 || n > p->n_seqs) return TABED_ERR_INVALID_ARG;
  if (n == 0) return TABED_OK;                    // (arrays of no elements may be null, here and below)
  if (!src || !dst || !keep || !len) return TABED_ERR_NULL_PTR;
  OnDevice guard(p->device);
  if (!guard.ok) return TABED_ERR_CUDA;
  ForkArgs a;
  a.P = on_device(p); a.n = n; a.src = src; a.dst = dst; a.keep = keep; a.len = len;
  unsigned char* ws = static_cast<unsigned char*>(p->workspace);
  a.ent = reinterpret_cast<ForkEntry*>(ws); ws += round16((size_t)p->n_seqs * sizeof(ForkEntry));
  a.found = reinterpret_cast<int*>(ws); ws += 16;
  a.rows = reinterpret_cast<int*>(ws); ws += round16((size_t)p->n_seqs * p->max_pages * 4);
  a.free_list = reinterpret_cast<int*>(ws);
  a.vec_ref = aligned(p->ref, 16);
  int rc;
  if (n <= kPlanEntries && (long long)n * p->max_pages <= kPlanBlocks) {      // (15 blocks 9.8 us against 10.6 in three launches, 624 12.0 and 12.6, 1152 13.1 and 12.7, 6336 21.5 and 15.1)
    rc = launch(p, k_pages_plan, dim3(1), kForkAllocThreads, 0, a);
  } else {
    rc = launch(p, k_pages_share, dim3(n), kForkThreads, 0, a);
    if (rc == TABED_OK) rc = launch(p, k_pages_alloc, dim3(1), kForkAllocThreads, 0, a);
  }
  if (rc == TABED_OK) rc = launch(p, k_pages_settle, dim3(n, 1 + 2 * p->n_layers), kForkThreads, 0, a);
  return rc;
}

int tabed_pages_append(const tabed_pages* p, const tabed_pages_new* t) {
  const int rc0 = check(p);
  if (rc0 != TABED_OK) return rc0;
  if (!t) return TABED_ERR_NULL_PTR;
  const bool nothing = t->n == 0 || t->n_tokens == 0 || t->max_new == 0;
  if (!nothing && (!t->first || !t->start || !t->k || !t->v)) return TABED_ERR_NULL_PTR;
  const int hd = p->head_dim, half = hd / 2;
  if (t->layer < 0 || t->layer >= p->n_layers || t->n < 0 || t->n > p->n_seqs || t->n_tokens < 0 || t->max_new < 0 ||
      t->max_new > p->max_pages * p->page_tokens || (t->dtype != TABED_DTYPE_FP32 && t->dtype != TABED_DTYPE_BF16) ||
      t->kv_stride < (long long)p->n_kv_heads * hd || t->n_axes < 0 || t->n_axes > 4)
    return TABED_ERR_INVALID_ARG;
  const bool with_q = t->n_axes > 0 && t->q;
  const size_t esz = t->dtype == TABED_DTYPE_FP32 ? 4 : 2;
  if (!aligned(t->k, esz) || !aligned(t->v, esz)) return TABED_ERR_INVALID_ARG;
  if (t->n_axes > 0) {
    if (!nothing && !t->positions) return TABED_ERR_NULL_PTR;
    if (!(t->theta > 0.0f) || !std::isfinite(t->theta)) return TABED_ERR_INVALID_ARG;
    int sum = 0;
    for (int i = 0; i < t->n_axes; ++i) { if (t->sections[i] < 0 || t->sections[i] > half) return TABED_ERR_INVALID_ARG; sum += t->sections[i]; }
    if (sum != half) return TABED_ERR_INVALID_ARG;
  }
  if (with_q) {
    if (!nothing && !t->q_out) return TABED_ERR_NULL_PTR;
    if (t->n_heads < 1 || t->n_heads > 4096 || t->q_stride < (long long)t->n_heads * hd || t->q_out_stride < (long long)t->n_heads * hd ||
        !aligned(t->q, esz) || !aligned(t->q_out, esz))
      return TABED_ERR_INVALID_ARG;
  }
  if (nothing) return TABED_OK;
  OnDevice guard(p->device);
  if (!guard.ok) return TABED_ERR_CUDA;
  AppendArgs a = {};
  a.P = on_device(p); a.layer = t->layer; a.n = t->n; a.n_tokens = t->n_tokens; a.max_new = t->max_new; a.n_heads = t->n_heads;
  a.seq = t->seq; a.first = t->first; a.start = t->start; a.positions = t->positions; a.k = t->k; a.v = t->v; a.q = t->q; a.q_out = t->q_out;
  a.kv_stride = t->kv_stride; a.kv_head = hd; a.q_stride = t->q_stride; a.q_out_stride = t->q_out_stride; a.n_axes = t->n_axes; a.has_q = with_q;
  a.vec_kv = rows_aligned(t->k, t->kv_stride, esz) && aligned(t->v, 16);
  a.vec_q = with_q && rows_aligned(t->q, t->q_stride, esz) && rows_aligned(t->q_out, t->q_out_stride, esz);
  for (int i = 0; i < t->n_axes; ++i) a.sections[i] = t->sections[i];
  if (t->n_axes > 0)
    for (int i = 0; i < half; ++i) a.turns[i] = pow((double)t->theta, -2.0 * i / hd) / 6.283185307179586476925;
  return run_append(p, a, t->dtype == TABED_DTYPE_FP32);
}

int tabed_pages_attention(const tabed_pages* p, const tabed_pages_query* t) {
  const int rc0 = check(p);
  if (rc0 != TABED_OK) return rc0;
  if (!t) return TABED_ERR_NULL_PTR;
  const bool nothing = t->n == 0 || t->n_tokens == 0 || t->max_new == 0;
  if (!nothing && (!t->first || !t->length || !t->q || !t->out)) return TABED_ERR_NULL_PTR;
  const int hd = p->head_dim;
  const size_t esz = t->dtype == TABED_DTYPE_FP32 ? 4 : 2;
  if (t->layer < 0 || t->layer >= p->n_layers || t->n < 0 || t->n_tokens < 0 || t->max_new < 0 ||
      (t->dtype != TABED_DTYPE_FP32 && t->dtype != TABED_DTYPE_BF16) || t->n_heads < 1 || t->n_heads > 65536 || t->n_heads % p->n_kv_heads ||
      t->q_stride < (long long)t->n_heads * hd || t->out_stride < (long long)t->n_heads * hd || !(t->scale > 0.0f) || !std::isfinite(t->scale) ||
      !(t->softcap >= 0.0f) || !std::isfinite(t->softcap) || !aligned(t->q, esz) || !aligned(t->out, esz) || (t->tree && t->slopes) ||
      (t->tree && t->max_new > 64) || !aligned(t->tree, 8))
    return TABED_ERR_INVALID_ARG;
  if (nothing) return TABED_OK;
  PagesAttnArgs a = {};
  a.P = on_device(p); a.layer = t->layer; a.n = t->n; a.n_tokens = t->n_tokens; a.max_new = t->max_new; a.H = t->n_heads;
  a.seq = t->seq; a.first = t->first; a.length = t->length; a.q = t->q; a.out = t->out; a.q_stride = t->q_stride; a.out_stride = t->out_stride;
  a.scale = t->scale; a.softcap = t->softcap; a.slopes = t->slopes; a.prefix = t->prefix; a.tree = reinterpret_cast<const unsigned long long*>(t->tree);
  a.vec_q = rows_aligned(t->q, t->q_stride, esz) && rows_aligned(t->out, t->out_stride, esz);
  // Up to 16 rows a KV head (32 of head sizes 32 and 64), and fp32 rows, multiply from registers (8 rows a tile, or 16 a warp in 1 - 4 warps); more
  // bf16 rows go through tensor memory in tiles of 64, 128 or 256 rows.  Registers and tensor memory, us: 32 sequences of 500 - 8192 tokens, 8 KV
  // heads of 128, 16 rows 142 and 138, 20 rows 188 and 138, 64 rows 321 and 145; 12 KV heads of 64, 96 sequences of 256 - 4096, 16 rows 113 and
  // 211, 32 rows 158 and 214, 40 rows 254 and 215; 4 KV heads of 32, 64 sequences, 32 rows 49 and 63, 40 rows 60 and 65; prompt chunks of
  // 2048 tokens 1514 and 267.  Tiles of 64, 128 and 256 (heads of 128): 64 rows 145, 154, 221, 72 rows 232, 155, 224, 128 rows 259, 162, 228, 136 rows 342, 248, 230.
  const long long rows = (long long)t->max_new * (t->n_heads / p->n_kv_heads);
  a.WR = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
  a.RB = rows <= 8 ? 8 : 16 * a.WR;
  if ((long long)t->n_tokens * (t->n_heads / p->n_kv_heads) > 0x7FFFFF00ll) return TABED_ERR_UNSUPPORTED;      // (an entry's rows, up to the end of a tile of 256, are counted in 31 bits)
  a.part_rows = kPgaMaxRows;
  if (t->dtype == TABED_DTYPE_BF16 && rows > (hd == 128 ? 16 : 32)) {
    a.RB = rows <= 64 ? 64 : (rows <= 128 ? 128 : 256);
    a.part_rows = kPtMaxRows;
  }
  unsigned char* ws = static_cast<unsigned char*>(p->workspace);
  a.part = reinterpret_cast<float*>(ws); ws += attn_part_bytes(p);
  a.part_ml = reinterpret_cast<float*>(ws); ws += kPartRows * 2 * 4;
  a.desc = reinterpret_cast<int4*>(ws);
  OnDevice guard(p->device);
  if (!guard.ok) return TABED_ERR_CUDA;
  const bool f32 = t->dtype == TABED_DTYPE_FP32;
  return hd == 32 ? launch_attn_hd<32>(p, a, f32) : (hd == 64 ? launch_attn_hd<64>(p, a, f32) : launch_attn_hd<128>(p, a, f32));
}

int tabed_pages_compact(const tabed_pages* p, const int32_t* seq, const int32_t* start, const int32_t* count, const int32_t* index,
                        int32_t n, int32_t width) {
  const int rc0 = check(p);
  if (rc0 != TABED_OK) return rc0;
  if (n < 0 || n > p->n_seqs || width < 0) return TABED_ERR_INVALID_ARG;
  if (n == 0 || width == 0) return TABED_OK;
  if (!seq || !start || !count || !index) return TABED_ERR_NULL_PTR;
  OnDevice guard(p->device);
  if (!guard.ok) return TABED_ERR_CUDA;
  CompactArgs a;
  a.P = on_device(p); a.seq = seq; a.start = start; a.count = count; a.index = index; a.n = n; a.width = width;
  // A warp a unit where fewer tokens than a page move, else four; blocks of more than 4 KB take four.  Pages of 64 tokens of 64 values, 12 KV
  // heads, one warp against four: 768 units (sequences, layers, heads, K and V) of 32 tokens 6.0 and 6.6 us, of 128 9.4 and 8.9, of 1024 55 and 40; 5760
  // units of 512 127 and 102, 9600 of 256 113 and 102.  With few KV heads a CTA's eight warps are not all there, and four are faster
  // at any number: 1536 units of 2 KV heads, 6 tokens 10.2 and 8.8 (left: the call is bound by its launch and dependent trips).
  const int bytes = p->page_tokens * p->head_dim;
  const bool one = bytes <= 4096 && width < p->page_tokens;
  const int per = kCompactThreads / 32 / (one ? 1 : 4);
  const dim3 grid(n, p->n_layers, (2 * p->n_kv_heads + per - 1) / per);
  if (one) return launch(p, k_pages_compact<1, 8>, grid, kCompactThreads, 0, a);
  if (bytes <= 4096) return launch(p, k_pages_compact<4, 2>, grid, kCompactThreads, 0, a);
  return bytes <= 8192 ? launch(p, k_pages_compact<4, 4>, grid, kCompactThreads, 0, a) : launch(p, k_pages_compact<4, 8>, grid, kCompactThreads, 0, a);
}

int tabed_pages_last_error(const tabed_pages* p) {
  if (!p || !p->err) return TABED_ERR_NULL_PTR;
  if (p->device < 0 || p->device >= kMaxDevices) return TABED_ERR_INVALID_ARG;
  OnDevice guard(p->device);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  int bits = 0;
  if (!guard.ok || cudaMemcpyAsync(&bits, p->err, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaMemsetAsync(p->err, 0, sizeof(int), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) {
    cudaGetLastError();
    return TABED_ERR_CUDA;
  }
  if (bits & (PERR_BARRIER | PERR_COPY)) return TABED_ERR_TIMEOUT;
  if (bits & PGERR_INVALID) return TABED_ERR_INVALID_ARG;
  if (bits & PERR_KV) return TABED_ERR_KV_OVERFLOW;
  return bits & PGERR_NUMERIC ? TABED_ERR_NUMERIC : (bits ? TABED_ERR_CUDA : TABED_OK);
}

}  // extern "C"
