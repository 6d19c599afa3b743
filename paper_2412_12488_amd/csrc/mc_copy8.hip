// The 8-bit KV cache's writers and movers for gfx950: append (with rounding), conversion of page ranges
// between a 16-bit and an 8-bit pool, transfer of whole 8-bit pages.
//
// All of them are bound by bytes.  The unit of work of the rounding kernels is a block - one page's K or V
// of one kv head, 16 tokens x 128, 4 KiB in 16 bits and 2 KiB of codes - because a block has one scale, and
// a wavefront takes it: 64 values a lane, so the block's largest magnitude is one reduction across the
// wavefront and every value is read once.  A K block is [slot][128]: lanes hold 8 neighbouring d of a row.  A V block
// is [128][slot], what the attention kernel's V operand wants: a lane holds two d of all 16 tokens, loads
// them as 16 coalesced rows and writes its two columns as 32 contiguous bytes, so the transposition costs
// no exchange between lanes.
#include "mc_fp8.h"

namespace {

using mc::kBlockBytes;
using mc::kHeadPageBytes;
using mc::kPage;
using mc::kRowBytes;
using mc::ScaleLimits;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float low_half(uint32_t w) {
  return (float)__builtin_bit_cast(T, (uint16_t)w);
}
template <typename T>
__device__ __forceinline__ float high_half(uint32_t w) {
  return (float)__builtin_bit_cast(T, (uint16_t)(w >> 16));
}

// largest of all 64 lanes' values, by data-parallel moves (rows of 16 lanes, then the rows' last ones)
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  auto step = [&](uint32_t y) __attribute__((always_inline)) { x = max(x, y); };
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));   // row_shr:1
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));   // row_bcast:15
  step((uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));   // row_bcast:31
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// A block's new tokens, of slots [lo, hi), as one wavefront holds them: 32 values a lane, K 4 rows x 8, V 16 rows x 2.
// src: the row of slot lo; rows are row_stride bytes apart.
struct Rows {
  uint32_t w[16];
};
template <bool kV>
__device__ __forceinline__ Rows load_rows(const char* src, int64_t row_stride, int lo, int hi) {
  const int lane = threadIdx.x & 63;
  Rows r;
  // (a slot without a new token reads the nearest one's row: no load under a condition)
  if (kV) {
#pragma unroll
    for (int s = 0; s < kPage; ++s)
      r.w[s] = *reinterpret_cast<const uint32_t*>(src + (min(max(s, lo), hi - 1) - lo) * row_stride + lane * 4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = 4 * i + (lane >> 4);
      const u32x4 v = *reinterpret_cast<const u32x4*>(src + (min(max(s, lo), hi - 1) - lo) * row_stride + (lane & 15) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) r.w[4 * i + j] = v[j];
    }
  }
  return r;
}

// What a block holds that its new tokens do not replace: its scale, and of a V block this lane's columns 2 lane and
// 2 lane + 1, 16 codes each.
struct Held {
  float scale;
  u32x4 a, b;
};
template <bool kV>
__device__ __forceinline__ Held load_held(const char* block, const float* scale, int lo, int hi) {
  Held h = {0.f, {0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
  if (lo > 0) h.scale = *scale;
  if (kV && (lo > 0 || hi < kPage)) {
    const u32x4* columns = reinterpret_cast<const u32x4*>(block + (threadIdx.x & 63) * 32);
    h.a = columns[0];
    h.b = columns[1];
  }
  return h;
}

// One block by one wavefront: the new tokens become codes; slots [0, lo) hold codes already, at *scale, and move to the
// new scale where the new tokens need a larger one; slots from hi on keep their bytes.
template <typename T, bool kV>
__device__ __forceinline__ void encode_block(const Rows& rows, const Held& held, int lo, int hi, char* block, float* scale,
                                             ScaleLimits lim) {
  const int lane = threadIdx.x & 63;
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int s = kV ? i : (i & ~3) + (lane >> 4);
    w[i] = s < lo || s >= hi ? 0u : rows.w[i];
  }
  u32x4 a = held.a, b = held.b;
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    big = max(big, max(mc::magnitude(low_half<T>(w[i])), mc::magnitude(high_half<T>(w[i]))));
  int k = mc::scale_exponent(wave_max(big), lim);
  float by = 1.f;                      // old codes' factor
  if (lo > 0) {
    const int old = mc::exponent_of(held.scale, lim);
    k = max(k, old);
    by = mc::power_of_two(max(old - k, -126));
  }
  const float inv = mc::power_of_two(-k), most = k == lim.hi ? 240.f : 448.f;
  if (kV) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x[4], y[4];
      uint32_t fresh = 0;              // bytes of new tokens
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = 4 * j + i;
        x[i] = mc::before_code(low_half<T>(w[s]), inv, most);
        y[i] = mc::before_code(high_half<T>(w[s]), inv, most);
        if (s >= lo && s < hi) fresh |= 0xffu << (8 * i);
      }
      const uint32_t na = mc::four_codes(x[0], x[1], x[2], x[3]), nb = mc::four_codes(y[0], y[1], y[2], y[3]);
      uint32_t oa = a[j], ob = b[j];
      if (by != 1.f) {
        const int kept = min(max(lo - 4 * j, 0), 4);     // bytes of this word that hold earlier tokens
        const uint32_t earlier = kept == 4 ? 0xffffffffu : (1u << (8 * kept)) - 1u;
        oa = (mc::move_codes(oa, by) & earlier) | (oa & ~earlier);
        ob = (mc::move_codes(ob, by) & earlier) | (ob & ~earlier);
      }
      a[j] = (na & fresh) | (oa & ~fresh);
      b[j] = (nb & fresh) | (ob & ~fresh);
    }
    u32x4* columns = reinterpret_cast<u32x4*>(block + lane * 32);
    columns[0] = a;
    columns[1] = b;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = 4 * i + (lane >> 4);
      u32x2* to = reinterpret_cast<u32x2*>(block + s * mc::kHeadDim + (lane & 15) * 8);
      if (s >= lo && s < hi) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[2 * j] = mc::before_code(low_half<T>(w[4 * i + j]), inv, most);
          x[2 * j + 1] = mc::before_code(high_half<T>(w[4 * i + j]), inv, most);
        }
        *to = u32x2{mc::four_codes(x[0], x[1], x[2], x[3]), mc::four_codes(x[4], x[5], x[6], x[7])};
      } else if (s < lo && by != 1.f) {
        const u32x2 old = *to;
        *to = u32x2{mc::move_codes(old[0], by), mc::move_codes(old[1], by)};
      }
    }
  }
  if (lane == 0) *scale = mc::power_of_two(k);
}

// ---------------------------------------------------------------- append ----
struct Append8Args {
  char* codes;             // of the layer
  float* scales;
  const char* k_new;
  const char* v_new;
  const int32_t* cu_q;
  const int32_t* begin;
  const int32_t* page_table;
  const int32_t* cu_pages;
  int64_t page_stride;
  int32_t num_pages, batch, total_q, hkv;
  ScaleLimits lim;
  int32_t* skipped;
};

// What a new token is for its page.
struct NewToken {
  int first;     // the page's slot of this token if it is the page's first new one, else -1
  int count;     // new tokens of the page from this one on
  int page;      // -1: left out
};

__device__ __forceinline__ NewToken look_up(const Append8Args& a, int g, int s) {
  const int q0 = a.cu_q[s], q1 = min(a.cu_q[s + 1], a.total_q), b = a.begin[s];
  const int p0 = a.cu_pages[s], p1 = a.cu_pages[s + 1];
  NewToken t = {-1, 0, -1};
  if (g < q0 || g >= q1 || b < 0 || p0 < 0) return t;
  const int64_t pos = (int64_t)b + (g - q0);
  if (pos / kPage >= (int64_t)p1 - p0) return t;
  const int page = a.page_table[p0 + (int)(pos / kPage)], slot = (int)(pos % kPage);
  if (page < 0 || page >= a.num_pages) return t;
  t.page = page;
  if (g == q0 || slot == 0) {
    t.first = slot;
    t.count = min(kPage - slot, q1 - g);
  }
  return t;
}

// One workgroup: kTokens neighbouring new tokens, of which those that open a page stand for the page.  Even wavefronts
// take K, odd ones V.
// kTokens == 1: every token looks for itself, every block has a wavefront at once; blockIdx.y is a pair of heads.
// kTokens > 1: blockIdx.y is one head, and the two wavefronts of K (V) take the pages in turns, the next one's memory
// requested ahead of the present one's arithmetic.  The look-ups, five memory accesses one after the other, then serve several
// blocks, but pages that get one token each are taken at a memory access's time, 2.3 us, apiece.
template <typename T, bool kV, int kTokens>
__device__ __forceinline__ void append_pages(const Append8Args& a, const NewToken& t, int g0, int head, int part);

template <typename T, int kTokens>
__global__ __launch_bounds__(kThreads) void append8_kernel(Append8Args a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kv = wave & 1, part = wave >> 1;
  const int head = kTokens == 1 ? 2 * blockIdx.y + part : blockIdx.y;
  if (head >= a.hkv) return;
  const int g0 = blockIdx.x * kTokens;
  // the sequence of token g0: the last s with cu_q[s] <= g0, 64 offsets a round
  int s0 = 0, cnt = a.batch;
  while (cnt > 1) {
    const int step = (cnt + 63) / 64, end = s0 + cnt, i = s0 + lane * step;
    const unsigned long long m = __ballot(i < end && a.cu_q[i] <= g0);
    s0 += max((int)__popcll(m) - 1, 0) * step;
    cnt = min(step, end - s0);
  }
  // Lane i looks token g0 + i up.  The sequences behind s0 begin at the next 64 offsets, as far as these tokens are concerned,
  // unless there are many without tokens among them.
  const int later = kTokens > 1 && s0 + 1 + lane < a.batch ? a.cu_q[s0 + 1 + lane] : INT32_MAX;
  NewToken t = {-1, 0, -1};
  int s = s0;
  if (kTokens > 1)
    for (int i = 0; i < 64 && __builtin_amdgcn_readlane(later, i) < g0 + kTokens; ++i)
      s += __builtin_amdgcn_readlane(later, i) <= g0 + lane ? 1 : 0;
  if (lane < kTokens && g0 + lane < a.total_q) {
    if (kTokens > 1 && s == s0 + 64) {         // from there on by halves
      int n = a.batch - s;
      while (n > 1) {
        const int h = n / 2;
        if (a.cu_q[s + h] <= g0 + lane) { s += h; n -= h; } else { n = h; }
      }
    }
    t = look_up(a, g0 + lane, s);
    if (t.page < 0 && a.skipped && kv == 0 && part == 0 && head == 0) atomicAdd(a.skipped, 1);
  }
  if (kv)
    append_pages<T, true, kTokens>(a, t, g0, head, part);
  else
    append_pages<T, false, kTokens>(a, t, g0, head, part);
}

template <typename T, bool kV, int kTokens>
__device__ __forceinline__ void append_pages(const Append8Args& a, const NewToken& t, int g0, int head, int part) {
  struct Job {
    int lo, hi;
    char* block;
    float* scale;
    Rows rows;
    Held held;
  };
  const char* from = (kV ? a.v_new : a.k_new) + ((int64_t)g0 * a.hkv + head) * kRowBytes;
  const int64_t stride = (int64_t)a.hkv * kRowBytes;
  unsigned long long open = __ballot(t.first >= 0);
  auto take = [&](Job& j) __attribute__((always_inline)) {      // the next page's; false: there is none
    if (!open) return false;
    const int i = __builtin_ctzll(open);
    open &= open - 1;
    if (kTokens > 1) open &= open - 1;         // (that one is the other wavefront's)
    const int page = __builtin_amdgcn_readlane(t.page, i);
    j.lo = __builtin_amdgcn_readlane(t.first, i);
    j.hi = j.lo + __builtin_amdgcn_readlane(t.count, i);
    j.block = a.codes + page * a.page_stride + (int64_t)(kV * a.hkv + head) * kBlockBytes;
    j.scale = a.scales + ((int64_t)page * a.hkv + head) * 2 + kV;
    j.rows = load_rows<kV>(from + i * stride, stride, j.lo, j.hi);
    j.held = load_held<kV>(j.block, j.scale, j.lo, j.hi);
    return true;
  };
  if (kTokens > 1 && part) open &= open - 1;
  Job job, next;
  bool more = take(job);
  while (more) {
    more = take(next);
    encode_block<T, kV>(job.rows, job.held, job.lo, job.hi, job.block, job.scale, a.lim);
    job = next;
  }
}

// ------------------------------------------- 16-bit pool <-> 8-bit pool ------
struct Range8Args {
  char* pool;              // 16-bit pool
  char* codes;
  float* scales;
  const int32_t* pages;    // one sequence's table in the 16-bit pool
  const int32_t* pages8;   // ... and in the 8-bit one
  int64_t layer_stride, page_stride, layer_codes, page_codes, layer_scales;
  int32_t num_pages, num_pages8;
  int32_t layer_begin, s0, s1, hkv;
  ScaleLimits lim;
  int32_t *skipped, *skipped8;
};

// One lane of a range's first block reports a page that one of the pools does not have.
__device__ __forceinline__ bool both_pages(const Range8Args& a, int tp, int32_t* counter, int& page, int& page8) {
  page = a.pages[tp];
  page8 = a.pages8[tp];
  if (page >= 0 && page < a.num_pages && page8 >= 0 && page8 < a.num_pages8) return true;
  if (counter && blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) atomicAdd(counter, 1);
  return false;
}

// grid.x: page of the range, grid.y: pair of heads, grid.z: layer; wavefronts as in append8_kernel
template <typename T>
__global__ __launch_bounds__(kThreads) void compress_kernel(Range8Args a) {
  const int wave = threadIdx.x >> 6, kv = wave & 1, head = 2 * blockIdx.y + (wave >> 1);
  const int tp = a.s0 / kPage + blockIdx.x;
  int page, page8;
  if (!both_pages(a, tp, a.skipped8, page, page8) || head >= a.hkv) return;
  const int64_t layer = a.layer_begin + blockIdx.z, unit = (int64_t)kv * a.hkv + head;
  const char* src = a.pool + layer * a.layer_stride + page * a.page_stride + unit * kHeadPageBytes;
  char* block = a.codes + layer * a.layer_codes + page8 * a.page_codes + unit * kBlockBytes;
  float* scale = a.scales + layer * a.layer_scales + ((int64_t)page8 * a.hkv + head) * 2 + kv;
  const int hi = min(kPage, a.s1 - tp * kPage);
  if (kv)
    encode_block<T, true>(load_rows<true>(src, kRowBytes, 0, hi), load_held<true>(block, scale, 0, hi), 0, hi, block, scale, a.lim);
  else
    encode_block<T, false>(load_rows<false>(src, kRowBytes, 0, hi), load_held<false>(block, scale, 0, hi), 0, hi, block, scale, a.lim);
}

template <typename T>
__device__ __forceinline__ uint32_t two_values(uint32_t word, float scale, int pair);
template <>
__device__ __forceinline__ uint32_t two_values<_Float16>(uint32_t word, float scale, int pair) {
  return pair ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, scale, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, scale, false));
}
template <>
__device__ __forceinline__ uint32_t two_values<__bf16>(uint32_t word, float scale, int pair) {
  return pair ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, false));
}

template <typename T>
__global__ __launch_bounds__(kThreads) void restore_kernel(Range8Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kv = wave & 1, head = 2 * blockIdx.y + (wave >> 1);
  const int tp = a.s0 / kPage + blockIdx.x;
  int page, page8;
  if (!both_pages(a, tp, a.skipped, page, page8) || head >= a.hkv) return;
  const int64_t layer = a.layer_begin + blockIdx.z, unit = (int64_t)kv * a.hkv + head;
  char* dst = a.pool + layer * a.layer_stride + page * a.page_stride + unit * kHeadPageBytes;
  const char* block = a.codes + layer * a.layer_codes + page8 * a.page_codes + unit * kBlockBytes;
  const float scale = mc::power_of_two(mc::exponent_of(
      a.scales[layer * a.layer_scales + ((int64_t)page8 * a.hkv + head) * 2 + kv], a.lim));
  const int lo = max(0, a.s0 - tp * kPage), hi = min(kPage, a.s1 - tp * kPage);
  if (kv) {
    // columns 2 lane, 2 lane + 1 of the block: a dword of every row
    const u32x4* from = reinterpret_cast<const u32x4*>(block + lane * 32);
    const u32x4 x = from[0], y = from[1];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint32_t u = two_values<T>(x[j], scale, p), v = two_values<T>(y[j], scale, p);
        const int s = 4 * j + 2 * p;
        if (s >= lo && s < hi)
          *reinterpret_cast<uint32_t*>(dst + s * kRowBytes + lane * 4) = (u & 0xffffu) | (v << 16);
        if (s + 1 >= lo && s + 1 < hi)
          *reinterpret_cast<uint32_t*>(dst + (s + 1) * kRowBytes + lane * 4) = (u >> 16) | (v & 0xffff0000u);
      }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = 4 * i + (lane >> 4);
      if (s < lo || s >= hi) continue;
      const u32x2 x = *reinterpret_cast<const u32x2*>(block + s * mc::kHeadDim + (lane & 15) * 8);
      *reinterpret_cast<u32x4*>(dst + s * kRowBytes + (lane & 15) * 16) =
          u32x4{two_values<T>(x[0], scale, 0), two_values<T>(x[0], scale, 1), two_values<T>(x[1], scale, 0),
                two_values<T>(x[1], scale, 1)};
    }
  }
}

// ------------------------------------------------- whole 8-bit pages ---------
struct Move8Args {
  char* codes;
  float* scales;
  char* buf;               // codes of all pages moved, layer by layer, then their scales
  const int32_t* pages;
  int64_t layer_codes, page_codes, layer_scales;
  int32_t num_pages, layer_begin, hkv;
  int32_t* skipped;
};

// One workgroup: one page of one layer, K and V of all heads (hkv x 4 KiB contiguous on both sides), and its scales.
template <bool kPack>
__global__ __launch_bounds__(kThreads) void move8_kernel(Move8Args a) {
  const int page = a.pages[blockIdx.x];
  if (page < 0 || page >= a.num_pages) {
    if (a.skipped && blockIdx.y == 0 && threadIdx.x == 0) atomicAdd(a.skipped, 1);
    return;
  }
  const int64_t layer = a.layer_begin + (int64_t)blockIdx.y;
  const int64_t nth = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, total = (int64_t)gridDim.x * gridDim.y;
  char* in_pool = a.codes + layer * a.layer_codes + page * a.page_codes + threadIdx.x * 16;
  char* in_buf = a.buf + nth * a.page_codes + threadIdx.x * 16;
  for (int h0 = 0; h0 < a.hkv; h0 += 8) {
    u32x4 r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (h0 + i < a.hkv)
        r[i] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>((kPack ? in_pool : in_buf) + (int64_t)(h0 + i) * 2 * kBlockBytes));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (h0 + i < a.hkv)
        __builtin_nontemporal_store(
            r[i], reinterpret_cast<u32x4*>((kPack ? in_buf : in_pool) + (int64_t)(h0 + i) * 2 * kBlockBytes));
  }
  float* scale_pool = a.scales + layer * a.layer_scales + (int64_t)page * a.hkv * 2;
  float* scale_buf = reinterpret_cast<float*>(a.buf + total * a.page_codes) + nth * a.hkv * 2;
  for (int i = threadIdx.x; i < 2 * a.hkv; i += kThreads)
    *((kPack ? scale_buf : scale_pool) + i) = *((kPack ? scale_pool : scale_buf) + i);
}

// grid.x: layer - layer_begin
__global__ __launch_bounds__(kThreads) void page_copy8_kernel(Move8Args a, int src_page, int dst_page) {
  const int64_t layer = a.layer_begin + (int64_t)blockIdx.x;
  const char* src = a.codes + layer * a.layer_codes + src_page * a.page_codes + threadIdx.x * 16;
  char* dst = a.codes + layer * a.layer_codes + dst_page * a.page_codes + threadIdx.x * 16;
  for (int h = 0; h < a.hkv; ++h)
    *reinterpret_cast<u32x4*>(dst + (int64_t)h * 2 * kBlockBytes) =
        *reinterpret_cast<const u32x4*>(src + (int64_t)h * 2 * kBlockBytes);
  float* scales = a.scales + layer * a.layer_scales;
  for (int i = threadIdx.x; i < 2 * a.hkv; i += kThreads)
    scales[(int64_t)dst_page * a.hkv * 2 + i] = scales[(int64_t)src_page * a.hkv * 2 + i];
}

// ------------------------------------------------------------------ host -----
mc_status check_layers(const mc_pool8_desc* pool, int32_t layer_begin, int32_t layer_end) {
  return layer_begin < 0 || layer_end < layer_begin || layer_end > pool->num_layers ? MC_ERR_RANGE : MC_OK;
}

Move8Args move_args(const mc_pool8_desc* pool, int32_t layer_begin) {
  Move8Args a;
  a.codes = static_cast<char*>(pool->codes);
  a.scales = pool->scales;
  a.buf = nullptr;
  a.pages = nullptr;
  a.layer_codes = mc::layer8_stride(pool);
  a.page_codes = mc::page8_stride(pool);
  a.layer_scales = mc::layer8_scales(pool);
  a.num_pages = pool->num_pages;
  a.layer_begin = layer_begin;
  a.hkv = pool->num_kv_heads;
  a.skipped = pool->skipped;
  return a;
}

mc_status move_range(bool pack, const mc_pool8_desc* pool, int32_t layer_begin, int32_t layer_end,
                     const int32_t* pages, int32_t n_table_pages, int32_t s0, int32_t s1, void* sendbuf,
                     void* stream) {
  mc_status st = mc::check_pool8(pool);
  if (st != MC_OK) return st;
  if ((st = check_layers(pool, layer_begin, layer_end)) != MC_OK) return st;
  if (s0 < 0 || s1 < s0 || n_table_pages < 0 || s0 % kPage != 0) return MC_ERR_RANGE;
  if (s0 == s1 || layer_begin == layer_end) return MC_OK;
  if (!pages || !sendbuf || !mc::aligned16(sendbuf)) return MC_ERR_INVALID;
  if (((int64_t)s1 + kPage - 1) / kPage > n_table_pages) return MC_ERR_RANGE;
  if (layer_end - layer_begin > 65535) return MC_ERR_UNSUPPORTED;
  Move8Args a = move_args(pool, layer_begin);
  a.buf = static_cast<char*>(sendbuf);
  a.pages = pages + s0 / kPage;
  const dim3 grid((unsigned)((s1 - 1) / kPage - s0 / kPage + 1), (unsigned)(layer_end - layer_begin));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (pack)
    hipLaunchKernelGGL(move8_kernel<true>, grid, dim3(kThreads), 0, hs, a);
  else
    hipLaunchKernelGGL(move8_kernel<false>, grid, dim3(kThreads), 0, hs, a);
  return mc::launch_status();
}

mc_status convert_range(bool compress, const mc_pool_desc* pool, const mc_pool8_desc* pool8, int32_t layer_begin,
                        int32_t layer_end, const int32_t* pages, int32_t n_pages, const int32_t* pages8,
                        int32_t n_pages8, int32_t s0, int32_t s1, void* stream) {
  mc_status st = mc::check_pool(pool);
  if (st != MC_OK) return st;
  if ((st = mc::check_pool8(pool8)) != MC_OK) return st;
  if (pool->dtype != pool8->dtype || pool->num_kv_heads != pool8->num_kv_heads) return MC_ERR_UNSUPPORTED;
  if ((st = check_layers(pool8, layer_begin, layer_end)) != MC_OK) return st;
  if (layer_end > pool->num_layers) return MC_ERR_RANGE;
  if (s0 < 0 || s1 < s0 || n_pages < 0 || n_pages8 < 0 || (compress && s0 % kPage != 0)) return MC_ERR_RANGE;
  if (s0 == s1 || layer_begin == layer_end) return MC_OK;
  if (!pages || !pages8) return MC_ERR_INVALID;
  const int64_t need = ((int64_t)s1 + kPage - 1) / kPage;
  if (need > n_pages || need > n_pages8) return MC_ERR_RANGE;
  if (layer_end - layer_begin > 65535 || pool->num_kv_heads > 131070) return MC_ERR_UNSUPPORTED;
  Range8Args a;
  a.pool = static_cast<char*>(pool->base);
  a.codes = static_cast<char*>(pool8->codes);
  a.scales = pool8->scales;
  a.pages = pages;
  a.pages8 = pages8;
  a.layer_stride = mc::layer_stride_bytes(pool);
  a.page_stride = mc::page_stride_bytes(pool);
  a.layer_codes = mc::layer8_stride(pool8);
  a.page_codes = mc::page8_stride(pool8);
  a.layer_scales = mc::layer8_scales(pool8);
  a.num_pages = pool->num_pages;
  a.num_pages8 = pool8->num_pages;
  a.layer_begin = layer_begin;
  a.s0 = s0;
  a.s1 = s1;
  a.hkv = pool->num_kv_heads;
  a.lim = mc::scale_limits(pool->dtype);
  a.skipped = pool->skipped;
  a.skipped8 = pool8->skipped;
  const dim3 grid((unsigned)((s1 - 1) / kPage - s0 / kPage + 1), (unsigned)((a.hkv + 1) / 2),
                  (unsigned)(layer_end - layer_begin));
  auto* kernel = compress ? (pool->dtype == MC_F16 ? compress_kernel<_Float16> : compress_kernel<__bf16>)
                          : (pool->dtype == MC_F16 ? restore_kernel<_Float16> : restore_kernel<__bf16>);
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return mc::launch_status();
}

// How many neighbouring tokens a workgroup of the append looks at.  What counts is how many open a page: in a decode batch all,
// in a prompt one in 16.  Measured with 8 heads, in us, with 1 / 16 / 32 tokens a workgroup:
//   64 decode rows 5.1 / 21 / 40; 2048 of them 33 / 37 / 49; 64 sequences x 4 tokens 7.2 / 7.4 / 12, x 8 11 / 5.2 / 7.4;
//   8 decode rows and a prompt's 100 5.2 / 14 / 14; 256 and 2048 36 / 23 / 41;
//   prompts of 128 5.0 / 4.6 / 5.1, 512 10 / 4.8 / 5.3, 2048 31 / 5.7 / 5.8, 4096 58 / 8.7 / 7.8, 16384 219 / 26 / 21
// The host knows the totals alone: below 4 tokens a sequence, or few altogether, one; from 32768 rows of
// K, where the look-ups' number costs more than a decode batch among a prompt's tokens does, 32.
int tokens_per_workgroup(int32_t batch, int32_t total_q, int32_t hkv) {
  if (total_q <= 128 || total_q <= (int64_t)batch * 4) return 1;
  return (int64_t)total_q * hkv <= 32768 ? 16 : 32;
}

}  // namespace

extern "C" {

mc_status mc_kv8_append(const mc_pool8_desc* pool, int32_t layer, const void* k_new, const void* v_new,
                        int32_t batch, int32_t total_q, const int32_t* cu_q, const int32_t* begin,
                        const int32_t* page_table, const int32_t* cu_pages, void* stream) {
  mc_status st = mc::check_pool8(pool);
  if (st != MC_OK) return st;
  if (layer < 0 || layer >= pool->num_layers) return MC_ERR_RANGE;
  if (batch < 0 || total_q < 0) return MC_ERR_INVALID;
  if (batch == 0 || total_q == 0) return MC_OK;
  if (!k_new || !v_new || !cu_q || !begin || !page_table || !cu_pages) return MC_ERR_INVALID;
  if (!mc::aligned16(k_new) || !mc::aligned16(v_new)) return MC_ERR_INVALID;
  if (pool->num_kv_heads > 65535) return MC_ERR_UNSUPPORTED;
  Append8Args a;
  a.codes = static_cast<char*>(pool->codes) + layer * mc::layer8_stride(pool);
  a.scales = pool->scales + layer * mc::layer8_scales(pool);
  a.k_new = static_cast<const char*>(k_new);
  a.v_new = static_cast<const char*>(v_new);
  a.cu_q = cu_q;
  a.begin = begin;
  a.page_table = page_table;
  a.cu_pages = cu_pages;
  a.page_stride = mc::page8_stride(pool);
  a.num_pages = pool->num_pages;
  a.batch = batch;
  a.total_q = total_q;
  a.hkv = pool->num_kv_heads;
  a.lim = mc::scale_limits(pool->dtype);
  a.skipped = pool->skipped;
  const bool half = pool->dtype == MC_F16;
  const int tokens = tokens_per_workgroup(batch, total_q, a.hkv);
  const dim3 grid((unsigned)(((int64_t)total_q + tokens - 1) / tokens), tokens == 1 ? (a.hkv + 1) / 2 : a.hkv);
  auto* kernel = tokens == 1    ? (half ? append8_kernel<_Float16, 1> : append8_kernel<__bf16, 1>)
                 : tokens == 16 ? (half ? append8_kernel<_Float16, 16> : append8_kernel<__bf16, 16>)
                                : (half ? append8_kernel<_Float16, 32> : append8_kernel<__bf16, 32>);
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return mc::launch_status();
}

mc_status mc_kv8_copy_check(const mc_pool8_desc* pool, int32_t* skipped_out, void* stream) {
  if (!pool) return MC_ERR_INVALID;
  mc_pool_desc counter = {};
  counter.skipped = pool->skipped;
  return mc_kv_copy_check(&counter, skipped_out, stream);
}

mc_status mc_kv8_compress_range(const mc_pool_desc* pool, const mc_pool8_desc* pool8, int32_t layer_begin,
                                int32_t layer_end, const int32_t* pages, int32_t n_pages, const int32_t* pages8,
                                int32_t n_pages8, int32_t s0, int32_t s1, void* stream) {
  return convert_range(true, pool, pool8, layer_begin, layer_end, pages, n_pages, pages8, n_pages8, s0, s1, stream);
}

mc_status mc_kv8_restore_range(const mc_pool8_desc* pool8, const mc_pool_desc* pool, int32_t layer_begin,
                               int32_t layer_end, const int32_t* pages8, int32_t n_pages8, const int32_t* pages,
                               int32_t n_pages, int32_t s0, int32_t s1, void* stream) {
  return convert_range(false, pool, pool8, layer_begin, layer_end, pages, n_pages, pages8, n_pages8, s0, s1, stream);
}

mc_status mc_kv8_pack_range(const mc_pool8_desc* pool, int32_t layer_begin, int32_t layer_end,
                            const int32_t* pages, int32_t n_table_pages, int32_t s0, int32_t s1, void* sendbuf,
                            void* stream) {
  return move_range(true, pool, layer_begin, layer_end, pages, n_table_pages, s0, s1, sendbuf, stream);
}

mc_status mc_kv8_unpack_range(const mc_pool8_desc* pool, int32_t layer_begin, int32_t layer_end,
                              const int32_t* pages, int32_t n_table_pages, int32_t s0, int32_t s1,
                              const void* sendbuf, void* stream) {
  return move_range(false, pool, layer_begin, layer_end, pages, n_table_pages, s0, s1, const_cast<void*>(sendbuf),
                    stream);
}

mc_status mc_kv8_copy_page(const mc_pool8_desc* pool, int32_t layer_begin, int32_t layer_end, int32_t src_page,
                           int32_t dst_page, void* stream) {
  mc_status st = mc::check_pool8(pool);
  if (st != MC_OK) return st;
  if ((st = check_layers(pool, layer_begin, layer_end)) != MC_OK) return st;
  if (src_page < 0 || src_page >= pool->num_pages || dst_page < 0 || dst_page >= pool->num_pages)
    return MC_ERR_RANGE;
  if (src_page == dst_page) return MC_ERR_ALIAS;
  if (layer_begin == layer_end) return MC_OK;
  const Move8Args a = move_args(pool, layer_begin);
  hipLaunchKernelGGL(page_copy8_kernel, dim3((unsigned)(layer_end - layer_begin)), dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), a, src_page, dst_page);
  return mc::launch_status();
}

}  // extern "C"
