// Attention of the new token range over a paged KV cache held in 8 bits (see mc_fp8.h for the codes), for gfx950.
//
// Work
//   * A q tile is 128 rows (TOK = 128 / G tokens x the G query heads of one kv head) of one sequence, or all of its
//     rows where those are at most 16 (decode steps).  A tile walks the 64-key KV tiles that its rows may see.
//   * All visits of KV tiles by q tiles, kv head after kv head, form one line of units, each q tile's behind some that
//     stand for what it takes beside them; plan8_kernel writes down how many units lie before each
//     sequence, and the attention launch cuts the line into as many equal spans as workgroups run at a time.  A span is any mixture of whole q tiles and parts of some; a part's rows (O, maximum, sum)
//     go to the workspace, and the last workgroup to finish a part of a q tile combines them, in their order.
//   * Codes become 16-bit numbers in registers, by the instructions that convert two at a time and multiply by the
//     block's scale (exactly: it is a power of two), and go into the 16-bit matrix instructions.
#include <math.h>

#include <type_traits>

#include "mc_fp8.h"

namespace {

using mc::kBlockBytes;
using mc::kHeadDim;
using mc::kPage;
using mc::kRowBytes;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;     // 4 wavefronts
constexpr int kPlanThreads = 512; // of the plan, whose first workgroup looks every span's beginning up
constexpr int kTileRows = 128, kFewRows = 16;
constexpr int kBN = 64;           // keys per KV tile: 4 pages
constexpr int kSpans = 512;       // workgroups of an attention launch at most: two for each of 256 compute units
constexpr int kXcds = 8;
constexpr int kMinSpan = 4;       // units a span has at least (no fewer than a visit's) ...
// ... and what a q tile takes beside its visits, in visits: looking it up, its Q, its first copies, its rows at the end.
// (8 prompts of 1024..4096 tokens, with 2 / 4 / 7 / 12: 432 / 419 / 419 / 424 us; 8 decode rows, a layer, 4 / 7: 20.7 / 19.7.)
constexpr int kTileCost = 7;
constexpr int kMostTokens = 1 << 30;   // of a sequence: positions stay far inside 32 bits
constexpr int32_t kPlanMagic = 0x6d63706d;

struct Plan8Header {
  int32_t magic;
  int32_t heads;       // kv heads and group size of the plan, as in mc_attn.hip
  int32_t batch;
  int32_t total_q;
  int64_t units;       // of all q tiles of one kv head
  int64_t span;        // units per workgroup
  int32_t tile_rows;   // rows of a q tile at most: kTileRows, or kFewRows
  int32_t pad[7];
};
static_assert(sizeof(Plan8Header) == 64, "header is 64 bytes");

// A q tile of more than 16 rows that the spans from one on cut: which merge8_kernel combines.
struct MergeRec8 {
  int32_t q_first, ntok, hk, count;   // count: its parts, 0: none
};

// A sequence as the plan saw it.
struct PlanSeq {
  int32_t begin, q_first, q, table_off;
};

// Where a span begins: the kv head, the sequence, its q tile and that tile's place on the line.  (The plan looks it up once for
// all layers; in each launch that is a chain of three or four memory accesses before the first code.)
struct SpanStart {
  int32_t hk, seq;
  int64_t tile, tile_at;
  PlanSeq of;
};

struct Workspace8 {
  size_t cum, seqs, verdict, arrivals, starts, merges, part_ml, part_o, total;
  int32_t part_rows, spans;
  bool few;
};

inline bool few_rows_only(int32_t batch, int32_t total_q, int G);
inline size_t round64(size_t x) { return (x + 63) & ~size_t(63); }

// Every span has at most two parts of q tiles: the end of one that began in an earlier span (or a piece out of
// the middle of one), and the beginning of one that goes on behind it.
inline Workspace8 workspace8(int32_t batch, int32_t total_q, int G) {
  Workspace8 w;
  w.few = few_rows_only(batch, total_q, G);
  w.spans = kSpans;
  w.part_rows = w.few ? kFewRows : kTileRows;
  w.cum = sizeof(Plan8Header);
  w.seqs = w.cum + round64(sizeof(int64_t) * ((size_t)batch + 1));
  w.verdict = w.seqs + round64(sizeof(PlanSeq) * (size_t)batch);
  w.arrivals = w.verdict + round64(sizeof(int32_t) * (size_t)batch);
  w.starts = w.arrivals + round64(sizeof(uint32_t) * kSpans);
  w.merges = w.starts + round64(sizeof(SpanStart) * kSpans);
  w.part_ml = w.merges + sizeof(MergeRec8) * kSpans;
  w.part_o = w.part_ml + sizeof(float) * 2 * 2 * (size_t)w.spans * w.part_rows;
  w.total = w.part_o + sizeof(float) * kHeadDim * 2 * (size_t)w.spans * w.part_rows;
  return w;
}

// ---- q tiles of a sequence -----------------------------------------------------------------
// Two kinds of plan, by the batch's sizes alone.  Batches of no more new tokens than sequences (decode steps), and those
// of at most 256 rows a kv head, have q tiles of at most 16 rows, whatever the sequences have, and a kernel that knows no
// others, with its parts combined in the launch.  In other batches sequences of at most 16 rows have one such tile and others
// tiles of 128 rows.  Plan and attention, us, of either kind (32 / 8 heads; few rows alone / both kinds):
//   8 x 8 tokens over 4096 27 / 33, 1 x 16 over 8192 23 / 38, 1 x 32 29 / 42, 1 x 64 43 / 40, 1 x 64 over 512 22 / 25,
//   16 decode rows and 8 tokens over 1024 20 / 25, over 8192 60 / 64; 64 x 5 over 2048 87 / 56, 64 x 16 162 / 68
inline bool few_rows_only(int32_t batch, int32_t total_q, int G) {
  return total_q <= batch || (int64_t)total_q * G <= 16 * kFewRows;
}
__device__ __forceinline__ int rows_of_tiles(int q, int G, int tile_rows) {
  return (int64_t)q * G <= kFewRows ? kFewRows : tile_rows;
}
// A visit by a q tile of 128 rows takes a workgroup about 1.5 us, one by a tile of few rows, which its wavefronts share,
// 0.6: two units and one.  (24 decode rows of 700..2500 keys beside a range of 1066 tokens, 64 / 8 heads, fp16: one unit each
// 94 us, so 78.)
__device__ __forceinline__ int unit_shift(int rows) { return rows == kFewRows ? 0 : 1; }
__device__ __forceinline__ int64_t tiles64(int64_t keys) { return (keys + kBN - 1) >> 6; }
static_assert(kBN == 64, "shifts by 6");

// Visits, and kTileCost for each tile, of a sequence's first i q tiles, of `tok` tokens each (a power of two): tile j visits
// the tiles of the keys before b + min((j + 1) tok, q).
__device__ __forceinline__ int64_t visits_before(int64_t b, int64_t q, int tok, int64_t i) {
  int64_t n = i, sum = i * kTileCost;
  if (i * tok > q) {                 // the last tile is short
    n = i - 1;
    sum += tiles64(b + q);
  }
  if (tok >= kBN) return sum + n * tiles64(b) + (n * (n + 1) >> 1) * (tok >> 6);
  // one more KV tile is seen after every `per` q tiles
  const int shift = __builtin_ctz(kBN) - __builtin_ctz(tok), per = 1 << shift;
  for (int res = 1; res <= per && res <= n; ++res) {
    const int64_t cnt = ((n - res) >> shift) + 1;
    sum += cnt * tiles64(b + res * tok) + (cnt * (cnt - 1) >> 1);
  }
  return sum;
}

__device__ __forceinline__ int64_t units_before(const PlanSeq& s, int G, int rows, int64_t i) {
  return visits_before(s.begin, s.q, rows / G, i) << unit_shift(rows);
}

struct Plan8Args {
  const int32_t* cu_q;
  const int32_t* begin;
  const int32_t* page_table;
  const int32_t* cu_pages;
  Plan8Header* hdr;
  int64_t* cum;
  PlanSeq* seqs;
  int32_t* verdict;
  uint32_t* arrivals;
  SpanStart* starts;
  int32_t batch, total_q, num_pages, hkv, G, ahead;
  int32_t tile_rows, spans;
};

// New tokens of sequence s, 0 if its offsets are malformed or its table too short.
__device__ __forceinline__ int checked_tokens(const Plan8Args& a, int s, bool* bad) {
  const int q0 = a.cu_q[s], q1 = a.cu_q[s + 1], b = a.begin[s], p0 = a.cu_pages[s], p1 = a.cu_pages[s + 1];
  *bad = q0 < 0 || q1 < q0 || q1 > a.total_q || b < 0 || p0 < 0 || p1 < p0 ||
         (q1 > q0 && (int64_t)b + (q1 - q0) + a.ahead > min(((int64_t)p1 - p0) * kPage, (int64_t)kMostTokens));
  return *bad ? 0 : q1 - q0;
}

// Workgroup 0 sums the units; workgroup 1 + s looks at the page ids of sequence s.
__global__ __launch_bounds__(kPlanThreads) void plan8_kernel(Plan8Args a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (blockIdx.x > 0) {
    const int s = blockIdx.x - 1;
    bool bad;
    const int q = checked_tokens(a, s, &bad);
    if (!bad && q > 0) {
      const int32_t* table = a.page_table + a.cu_pages[s];
      const int n = (int)(((int64_t)a.begin[s] + q + a.ahead + kPage - 1) / kPage);
      for (int i = tid; i < n; i += kPlanThreads) bad |= (unsigned)table[i] >= (unsigned)a.num_pages;
    }
    const int any = __syncthreads_or(bad);
    if (tid == 0) a.verdict[s] = any ? MC_ERR_RANGE : MC_OK;
    return;
  }
  for (int i = tid; i < kSpans; i += kPlanThreads) a.arrivals[i] = 0;
  __shared__ int64_t s_wave[kPlanThreads / 64];
  int64_t before = 0;
  for (int s0 = 0; s0 < a.batch; s0 += kPlanThreads) {
    const int s = s0 + tid;
    int64_t v = 0;
    if (s < a.batch) {
      bool bad;
      const int q = checked_tokens(a, s, &bad);
      const PlanSeq of = {a.begin[s], a.cu_q[s], q, a.cu_pages[s]};
      if (q > 0) {
        const int rows = rows_of_tiles(q, a.G, a.tile_rows), tok = rows / a.G;
        v = units_before(of, a.G, rows, (q + tok - 1) / tok);
      }
      a.seqs[s] = of;
    }
    int64_t incl = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    int64_t base = before;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      if (w < wave) base += s_wave[w];
      before += s_wave[w];
    }
    if (s < a.batch) a.cum[s] = base + incl - v;
    __syncthreads();
  }
  const int64_t span = max((before * a.hkv + a.spans - 1) / a.spans, (int64_t)kMinSpan);
  if (tid == 0) {
    a.cum[a.batch] = before;
    Plan8Header h = {};
    h.magic = kPlanMagic;
    h.heads = a.hkv * 16 + a.G;
    h.batch = a.batch;
    h.total_q = a.total_q;
    h.units = before;
    h.span = span;
    h.tile_rows = a.tile_rows;
    *a.hdr = h;
  }
  __syncthreads();                 // (cum and seqs, of this workgroup's own writing)
  for (int w = tid; w < a.spans; w += kPlanThreads) {
    const int64_t at = w * span;
    if (at >= before * a.hkv) continue;
    SpanStart r = {};
    r.hk = (int)((double)at / (double)before);          // (to one too many or few: 64-bit division takes as long as all else)
    if (r.hk * before > at) --r.hk;
    if ((r.hk + 1) * before <= at) ++r.hk;
    const int64_t in_head = at - r.hk * before;
    // the sequence: the last s with cum[s] <= in_head (of equal ones the last, which is not empty)
    int s = 0;
    for (int cnt = a.batch; cnt > 1;) {
      const int half = cnt / 2;
      if (a.cum[s + half] <= in_head) {
        s += half;
        cnt -= half;
      } else {
        cnt = half;
      }
    }
    r.seq = s;
    r.of = a.seqs[s];
    // the q tile: the last i with units_before(i) <= what is left
    const int64_t left = in_head - a.cum[s];
    const int rows = rows_of_tiles(r.of.q, a.G, a.tile_rows), tok = rows / a.G;
    for (int64_t cnt = (r.of.q + tok - 1) / tok; cnt > 1;) {
      const int64_t half = cnt / 2;
      if (units_before(r.of, a.G, rows, r.tile + half) <= left) {
        r.tile += half;
        cnt -= half;
      } else {
        cnt = half;
      }
    }
    r.tile_at = at - left + units_before(r.of, a.G, rows, r.tile);
    a.starts[w] = r;
  }
}

// ---------------------------------------------------------------- attention --
template <typename T> struct Num;
template <> struct Num<_Float16> {
  typedef f16x8 vec8;
  static __device__ __forceinline__ f32x16 mfma32(vec8 a, vec8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(vec8 a, vec8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  template <bool kHigh>
  static __device__ __forceinline__ uint32_t from_codes(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, kHigh));
  }
};
template <> struct Num<__bf16> {
  typedef bf16x8 vec8;
  static __device__ __forceinline__ f32x16 mfma32(vec8 a, vec8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(vec8 a, vec8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  template <bool kHigh>
  static __device__ __forceinline__ uint32_t from_codes(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, kHigh));
  }
};
// two fp32 to the 16-bit type (to nearest even), the first in the low half
template <typename T>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  typedef T t2 __attribute__((ext_vector_type(2)));
  t2 v;
  v[0] = (T)x;
  v[1] = (T)y;
  return __builtin_bit_cast(uint32_t, v);
}
// eight codes -> eight numbers of the 16-bit type
template <typename T>
__device__ __forceinline__ typename Num<T>::vec8 numbers(uint32_t lo, uint32_t hi, float scale) {
  const u32x4 v = {Num<T>::template from_codes<false>(lo, scale), Num<T>::template from_codes<true>(lo, scale),
                   Num<T>::template from_codes<false>(hi, scale), Num<T>::template from_codes<true>(hi, scale)};
  return __builtin_bit_cast(typename Num<T>::vec8, v);
}
// The largest of three, a NaN if one is, in one instruction (fmaxf quiets each operand by another).  What follows from a
// NaN maximum: the reference stays, and the row's sum is a NaN anyway.
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
// x's upper 32 lanes <-> y's lower 32 lanes.  (The builtin of this hands out its first result twice where both operands are
// one value; the s_nop is the distance to the vector instructions that wrote them.)
__device__ __forceinline__ void swap_halves(uint32_t& x, uint32_t& y) {
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
}
// top bits of the bytes that are NaN codes (0x7f, 0xff)
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// A NaN in V counts for the rows that see its key, and for no other, but P is 0 for those and 0 x NaN is NaN.  So in
// KV tiles that not all rows see whole, NaN codes are taken out of V, and their places, as 2^126, go through a product
// with the keys that each row sees, as 2^126 or 0: that adds an infinity where both are, and a second
// one of the other sign makes it a NaN.  (In bf16, whatever the pool's type: fp16 has no such numbers.)
__device__ __forceinline__ u32x4 take_nan_codes(u32x4& v) {
  u32x4 at;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t b = nan_codes(v[j]) >> 7;
    at[j] = b * 0x38u;                   // the code of 1
    v[j] &= ~(b * 0xffu);
  }
  return at;
}
__device__ __forceinline__ bf16x8 huge(u32x4 at, int half, bool positive) {
  u32x4 w = __builtin_bit_cast(u32x4, numbers<__bf16>(at[2 * half], at[2 * half + 1], 0x1p126f));
  if (!positive) w ^= 0x80008000u;
  return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ bf16x8 keys_seen(int key, int pos) {
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = (key + 2 * j <= pos ? 0x7e80u : 0u) | (key + 2 * j + 1 <= pos ? 0x7e800000u : 0u);
  return __builtin_bit_cast(bf16x8, w);
}

struct Attn8Args {
  const char* codes;       // of the layer
  const float* scales;
  const char* q;
  char* out;
  float* lse;
  const int32_t* begin;
  const int32_t* page_table;
  const int32_t* cu_pages;
  const Plan8Header* hdr;
  const int64_t* cum;
  const PlanSeq* seqs;
  const int32_t* verdict;
  uint32_t* arrivals;
  const SpanStart* starts;
  MergeRec8* merges;
  float* part_ml;          // [part][row]: maximum (of the exponents, base 2), sum
  float* part_o;           // [part][row][D], relative to the part's maximum
  int32_t num_pages, hkv, hq, batch, total_q, part_rows;
  int32_t spans;           // workgroups
  float scale_log2;        // softmax scale x log2(e)
};

typedef __attribute__((address_space(3))) void* lds_void_ptr;
__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(size_t)(lds_void_ptr)(p); }

// Asynchronous copies from global memory into LDS: lane L's 16 (4) bytes land at lds_base + 16 (4) L.
// As assembly so that the compiler does not wait for them before LDS reads of other buffers; they are waited for
// by count before the barrier that publishes them.  (The s_nop: five wait states between a vector instruction that
// writes a scalar register, which the address may come from, and a memory instruction that reads it.)
// (The first: 2 KiB, a block, the instruction's offset moving both addresses.)
__device__ __forceinline__ void copy_block_to_lds(const char* base, uint32_t lane_off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1\n\t"
               "global_load_lds_dwordx4 %0, %1 offset:1024"
               :: "v"(lane_off), "s"(base), "s"(lds_base) : "memory", "m0");
}
__device__ __forceinline__ void copy4_to_lds(const void* base, uint32_t lane_off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dword %0, %1"
               :: "v"(lane_off), "s"(base), "s"(lds_base) : "memory", "m0");
}

// What a workgroup works on: KV tiles [t0, t1) of the q tile of ntok tokens from q_first on, of kv head hk.
struct Piece {
  int hk, q_first, ntok, first_pos;  // first_pos: position of the first token
  int t0, t1;
  int table_off, last_entry;         // last entry of the page table that holds a key the tile sees
  int kv_len;                        // keys the tile's last token sees
};

constexpr int kStages = 4;
constexpr int kTileBytes = 4 * 2 * kBlockBytes;         // codes of a KV tile: page by page, K then V
constexpr int kScaleBytes = 4 * 256;                    // its scales: page by page, K and V in turns (256 bytes land)
constexpr int kStageBytes = kTileBytes + kScaleBytes;
constexpr int kOStride = kHeadDim + 4;                  // floats between rows of O in LDS (few rows)
constexpr int kFewBytes = 4 * kFewRows * kOStride * 4 + 4 * kFewRows * 8;
constexpr int kLdsBytes = kStages * kStageBytes;
static_assert(kLdsBytes >= kFewBytes && (kStages & (kStages - 1)) == 0, "areas that share the LDS; a ring by masks");

// Address of a page's codes of one kv head's K; V lies hkv blocks behind
__device__ __forceinline__ int64_t page_offset(const Attn8Args& a, int page, int hk) {
  page = min(max(page, 0), a.num_pages - 1);            // (the plan has looked at them)
  return ((int64_t)page * 2 * a.hkv + hk) * kBlockBytes;
}

// Where a piece's rows go: the result, or a part in the workspace.
struct Target {
  int part;            // < 0: out and lse
};

// Parts of a q tile are written by one workgroup and read by another of the same launch, on any XCD: through
// buffer instructions of device scope (sc1), which go to the level that all XCDs share, so that no L2 has to be
// written back or invalidated as a whole (with fences of device scope instead, 256 decode rows took 485 us a
// layer).  What merge8_kernel reads goes by plain ones.
typedef __amdgpu_buffer_rsrc_t buffer_rsrc;
constexpr int kDeviceScope = 16, kLaunchScope = 0;
__device__ __forceinline__ buffer_rsrc make_rsrc(void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(p, 0, (uint32_t)bytes, 0x00020000);   // raw, 32-bit; bounds checked
}
struct Parts {
  buffer_rsrc o, ml;
  int rows;
  __device__ __forceinline__ explicit Parts(const Attn8Args& a)
      : o(make_rsrc(a.part_o, 2ll * a.spans * a.part_rows * kHeadDim * 4)),
        ml(make_rsrc(a.part_ml, 2ll * a.spans * a.part_rows * 8)), rows(a.part_rows) {}
  __device__ __forceinline__ uint32_t at(int part, int row) const { return (uint32_t)(part * rows + row); }
  // Rows of q tiles of 128 lie as a wavefront's registers do: vector (i, j) of all its lanes together.
  __device__ __forceinline__ uint32_t vector_at(int part, int wave, int i, int j) const {
    return (uint32_t)((((part * 4 + wave) * 4 + i) * 4 + j) * 64 + (threadIdx.x & 63)) * 16;
  }
  __device__ __forceinline__ void put_vector(uint32_t at, f32x4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), o, at, 0, kLaunchScope);
  }
  __device__ __forceinline__ f32x4 get_vector(uint32_t at) const {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(o, at, 0, kLaunchScope));
  }
  template <int kScope>
  __device__ __forceinline__ void put(uint32_t i, int d, f32x4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), o, (i * kHeadDim + d) * 4, 0, kScope);
  }
  template <int kScope>
  __device__ __forceinline__ void put_ml(uint32_t i, float m, float l) const {
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{__builtin_bit_cast(uint32_t, m), __builtin_bit_cast(uint32_t, l)}, ml,
                                          i * 8, 0, kScope);
  }
  template <int kScope>
  __device__ __forceinline__ f32x4 get(uint32_t i, int d) const {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(o, (i * kHeadDim + d) * 4, 0, kScope));
  }
  template <int kScope>
  __device__ __forceinline__ f32x2 get_ml(uint32_t i) const {
    return __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(ml, i * 8, 0, kScope));
  }
};

template <int G>
__device__ __forceinline__ int64_t out_row(const Attn8Args& a, const Piece& p, int row) {
  return (int64_t)(p.q_first + row / G) * a.hq + p.hk * G + row % G;
}

// ---- at most 16 rows ------------------------------------------------------------------------
// Bound by reading the codes.  The four wavefronts take KV tiles in turns, each straight from memory into
// registers, on v_mfma_f32_16x16x32.  Lane l, c = l % 16, g = l / 16: for S^T = K Q^T the matrix rows are keys,
// and row m of product x is slot 4 x + m % 4 of page m / 4, so that a lane ends up with the 16 scores of page g
// and query row c, P^T is the second product's operand as it lies, and that product's other operand, V^T, is
// 16 contiguous bytes of page g's V block: no exchange between lanes but the maximum's.
template <typename T, int G>
__device__ __forceinline__ void few_rows_piece(const Attn8Args& a, const Piece& p, const Target& to, char* lds) {
  typedef typename Num<T>::vec8 vec8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const int tok = min(c / G, p.ntok - 1);
  const int my_pos = p.first_pos + tok;
  const float c2 = a.scale_log2;
  // Q^T operand: step 2 j + e of the d axis holds d = 64 j + 16 g + 8 e + [0, 8)
  vec8 q[4];
  {
    const char* row = a.q + ((int64_t)(p.q_first + tok) * a.hq + p.hk * G + c % G) * kRowBytes;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      q[u] = *reinterpret_cast<const vec8*>(row + ((u >> 1) * 64 + g * 16 + (u & 1) * 8) * 2);
  }
  f32x4 o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  u32x4 kc[8], vc[8];
  float ks, vs;
  const int32_t* table = a.page_table + p.table_off;
  auto entry = [&](int t, int i) __attribute__((always_inline)) { return table[min(4 * t + i, p.last_entry)]; };
  // K of tile t: page c / 4, slots c % 4 + 4 x
  auto load_k = [&](int page) __attribute__((always_inline)) {
    const char* at = a.codes + page_offset(a, page, p.hk) + (c & 3) * kHeadDim + g * 16;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      kc[i] = *reinterpret_cast<const u32x4*>(at + (i >> 1) * 4 * kHeadDim + (i & 1) * 64);
    ks = a.scales[((int64_t)min(max(page, 0), a.num_pages - 1) * a.hkv + p.hk) * 2];
  };
  auto load_v = [&](int page) __attribute__((always_inline)) {
    const char* at = a.codes + page_offset(a, page, p.hk) + (int64_t)a.hkv * kBlockBytes + c * kPage;
#pragma unroll
    for (int i = 0; i < 8; ++i) vc[i] = *reinterpret_cast<const u32x4*>(at + i * 16 * kPage);
    vs = a.scales[((int64_t)min(max(page, 0), a.num_pages - 1) * a.hkv + p.hk) * 2 + 1];
  };
  int t = p.t0 + wave;
  if (t < p.t1) {
    load_k(entry(t, c >> 2));
    load_v(entry(t, g));
  }
  for (; t < p.t1; t += 4) {
    const bool more = t + 4 < p.t1;
    const int next_k = entry(more ? t + 4 : t, c >> 2), next_v = entry(more ? t + 4 : t, g);
    f32x4 s[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x4 w = kc[2 * x + j];
        s[x] = Num<T>::mfma16(numbers<T>(w[0], w[1], ks), q[2 * j], s[x]);
        s[x] = Num<T>::mfma16(numbers<T>(w[2], w[3], ks), q[2 * j + 1], s[x]);
      }
    }
    if (more) load_k(next_k);
    // lane: scores of keys 64 t + 16 g + 4 x + r
    const int key0 = t * kBN + 16 * g;
    const bool masked = t * kBN + kBN - 1 > p.first_pos;
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (key0 + i > my_pos) s[i >> 2][i & 3] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int i = 1; i < 15; i += 2) mx = max3(mx, s[i >> 2][i & 3], s[(i + 1) >> 2][(i + 1) & 3]);
    mx = max3(mx, mx, s[3][3]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * c2;
    if (__builtin_amdgcn_ballot_w64(mx > m + 8.f) != 0) {
      const float m_new = fmaxf(m, mx);
      const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    uint32_t pk[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][(2 * i) & 3], c2, -ref));
      const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][(2 * i + 1) & 3], c2, -ref));
      l += p0 + p1;
      pk[i] = pack2<T>(p0, p1);
    }
    vec8 pt[2];
    pt[0] = __builtin_bit_cast(vec8, u32x4{pk[0], pk[1], pk[2], pk[3]});
    pt[1] = __builtin_bit_cast(vec8, u32x4{pk[4], pk[5], pk[6], pk[7]});
    if (masked) {
      // slots behind the last key hold anything: no code of theirs counts
      const int n = min(max(p.kv_len - key0, 0), 16);
      uint32_t some = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int kept = min(max(n - 4 * j, 0), 4);
          vc[i][j] &= kept == 4 ? 0xffffffffu : (1u << (8 * kept)) - 1u;
          some |= nan_codes(vc[i][j]);
        }
      if (__builtin_amdgcn_ballot_w64(some != 0) != 0) {
        bf16x8 seen[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) seen[e] = keys_seen(key0 + 8 * e, my_pos);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const u32x4 at = take_nan_codes(vc[i]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[i] = Num<__bf16>::mfma16(huge(at, e & 1, e < 2), seen[e & 1], o[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      o[i] = Num<T>::mfma16(numbers<T>(vc[i][0], vc[i][1], vs), pt[0], o[i]);
      o[i] = Num<T>::mfma16(numbers<T>(vc[i][2], vc[i][3], vs), pt[1], o[i]);
    }
    if (more) load_v(next_v);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  // the four wavefronts' rows, through LDS
  float* so = reinterpret_cast<float*>(lds);
  float* sml = so + 4 * kFewRows * kOStride;
  __syncthreads();                       // (earlier readers of the LDS are done)
#pragma unroll
  for (int i = 0; i < 8; ++i)
    *reinterpret_cast<f32x4*>(so + (wave * kFewRows + c) * kOStride + 16 * i + 4 * g) = o[i];
  if (g == 0) {
    sml[(wave * kFewRows + c) * 2] = m;
    sml[(wave * kFewRows + c) * 2 + 1] = l;
  }
  __syncthreads();
  const int row = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;
  float mm = -INFINITY, ll = 0.f, acc[8];
#pragma unroll
  for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sml[(w * kFewRows + row) * 2]);
  const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(sml[(w * kFewRows + row) * 2] - ref);
    ll += f * sml[(w * kFewRows + row) * 2 + 1];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += f * so[(w * kFewRows + row) * kOStride + d + j];
  }
  if (row >= p.ntok * G) return;
  if (to.part >= 0) {
    const Parts parts(a);
    const uint32_t at = parts.at(to.part, row);
    parts.put<kDeviceScope>(at, d, f32x4{acc[0], acc[1], acc[2], acc[3]});
    parts.put<kDeviceScope>(at, d + 4, f32x4{acc[4], acc[5], acc[6], acc[7]});
    if (d == 0) parts.put_ml<kDeviceScope>(at, mm, ll);
  } else {
    const int64_t at = out_row<G>(a, p, row);
    const float inv = 1.f / ll;
    *reinterpret_cast<u32x4*>(a.out + at * kRowBytes + d * 2) =
        u32x4{pack2<T>(acc[0] * inv, acc[1] * inv), pack2<T>(acc[2] * inv, acc[3] * inv),
              pack2<T>(acc[4] * inv, acc[5] * inv), pack2<T>(acc[6] * inv, acc[7] * inv)};
    if (d == 0) a.lse[at] = (mm + __builtin_amdgcn_logf(ll)) * 0.6931471805599453f;
  }
}

// 32 d of a row, of which lane h (and its neighbour h ^ 1, 32 lanes away) holds 8 j + 4 h + [0, 4): 16 bytes a store, of j for
// the lane with h = 0, of j + 1 for the other.
template <typename T>
__device__ __forceinline__ void store_block(char* to, int h, const f32x4 (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; j += 2) {
    uint32_t x0 = pack2<T>(v[j][0], v[j][1]), x1 = pack2<T>(v[j][2], v[j][3]);
    uint32_t y0 = pack2<T>(v[j + 1][0], v[j + 1][1]), y1 = pack2<T>(v[j + 1][2], v[j + 1][3]);
    swap_halves(x0, y0);
    swap_halves(x1, y1);
    *reinterpret_cast<u32x4*>(to + 16 * (j + h)) = u32x4{x0, x1, y0, y1};
  }
}

// ---- 128 rows ---------------------------------------------------------------------------------
// Bound by the matrix and the vector pipes.  Each wavefront has 32 rows and walks all keys of the piece, a half tile (32 keys,
// two pages) at a time, on v_mfma_f32_32x32x16; two workgroups share a compute unit.  KV tiles are copied as
// they lie into a ring of LDS buffers, and every wavefront converts what it reads.  Lane l, n = l % 32, h = l / 32:
// matrix row i of S^T is slot (i / 8) * 4 + i % 4 of page (i / 4) % 2 of the half tile, so a lane ends up with the 16 scores
// of page h and query row n, P^T is the second product's operand as it lies, and V^T is 16 contiguous bytes of page h.
// K rows are 128 bytes, 8 chunks of 16; chunk c of slot s of page g lies at c ^ (s % 4 + 4 (g % 2)): any 8
// neighbouring lanes of a K read then hit 8 different chunks, so all banks.  V reads are contiguous.
//   half step  phase 1: S of the next half on the matrix pipe; beside it K's conversion and half of this one's exponentials
//              phase 2: O^T += V^T P^T; beside it the other half, the row maxima of the next S, V's conversion
// K's codes could enter the matrix pipe as they are, with Q in two rows of codes, 8 % faster at 32k over 0; but the
// instructions for scaled 8-bit numbers drop what lies 2^-13 below the largest of the 64 products they add, and the scores
// would not be sums in 32 bits (lse off by 1e-4 instead of 1e-6).
// The order within a phase is pinned: a matrix instruction, then what fits beside it.  Phase 2 has priority: of the two wavefronts
// of a SIMD the one that came first is otherwise served first throughout, runs ahead, and the other ends alone (16k over
// 16k tokens: 6.66 ms; with it 5.92).
template <typename T, int G>
__device__ __forceinline__ void tile_piece(const Attn8Args& a, const Piece& p, const Target& to, char* lds) {
  typedef typename Num<T>::vec8 vec8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int row = wave * 32 + n, tok = min(row / G, p.ntok - 1), my_pos = p.first_pos + tok;
  const bool active = wave * 32 < p.ntok * G;
  const float c2 = a.scale_log2;
  const uint32_t lds0 = lds_addr(lds);

  // this wavefront copies page `wave` of every tile
  const int32_t* table = a.page_table + p.table_off;
  auto look_up_pages = [&](int t) __attribute__((always_inline)) { return table[min(4 * (t + lane) + wave, p.last_entry)]; };
  int ids = look_up_pages(p.t0), ids_t = p.t0;     // lane i holds the page id of tile ids_t + i
  // Q^T operand: step 2 cc + e of the d axis holds d = 32 cc + 16 h + 8 e + [0, 8)
  u32x4 q_raw[8];
  {
    const char* from = a.q + ((int64_t)(p.q_first + tok) * a.hq + p.hk * G + row % G) * kRowBytes;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      q_raw[u] = *reinterpret_cast<const u32x4*>(from + ((u >> 1) * 32 + h * 16 + (u & 1) * 8) * 2);
  }
  // where in the page a lane's 16 bytes of the K (V) block's halves come from
  const uint32_t k_from = (lane >> 3) * kHeadDim + (((lane & 7) ^ ((lane >> 3 & 3) | (wave & 1) << 2)) << 4);
  const uint32_t v_from = a.hkv * kBlockBytes + lane * 16;
  const char* codes = a.codes + (int64_t)p.hk * kBlockBytes;
  const float* scales = a.scales + 2 * p.hk;
  const uint32_t page_stride = 2u * a.hkv * kBlockBytes;
  const uint32_t lds_wave = lds0 + wave * 2 * kBlockBytes, lds_scales = lds0 + kTileBytes + wave * 256;
  auto stage_at = [&](int t) __attribute__((always_inline)) { return (uint32_t)((t - p.t0) & (kStages - 1)) * kStageBytes; };
  auto copy_tile = [&](int t) __attribute__((always_inline)) {
    if (t >= ids_t + 64) {
      ids_t = t;
      ids = look_up_pages(t);
    }
    const int page = min(max(__builtin_amdgcn_readlane(ids, t - ids_t), 0), a.num_pages - 1);
    const char* from = codes + (uint64_t)(uint32_t)page * page_stride;
    const uint32_t stage = stage_at(t);
    copy_block_to_lds(from, k_from, lds_wave + stage);
    copy_block_to_lds(from, v_from, lds_wave + stage + kBlockBytes);
    copy4_to_lds(scales + (uint64_t)(uint32_t)page * (2u * a.hkv), (lane & 1) * 4, lds_scales + stage);
  };
  constexpr int kCopies = 5;             // of a wavefront and tile

  auto first_copies = [&]() __attribute__((always_inline)) {
    __syncthreads();                     // (earlier readers of the LDS are done)
    if (ids_t != p.t0) ids = look_up_pages(ids_t = p.t0);
    for (int i = 0; i < kStages - 1; ++i)
      if (p.t0 + i < p.t1) copy_tile(p.t0 + i);
  };
  first_copies();
  vec8 q[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) q[u] = __builtin_bit_cast(vec8, q_raw[u]);
  f32x16 o[4], s_a, s_b;
  const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  float m, l, mx;

  // LDS offsets of this lane's fragments within a stage, of half tile 0; half tile 1 lies two pages behind
  const int k_page = n >> 2 & 1, k_slot = (n >> 3) * 4 + (n & 3);
  const uint32_t k_off = k_page * 2 * kBlockBytes + k_slot * kHeadDim + ((h ^ ((k_slot & 3) | k_page << 2)) << 4);
  const uint32_t v_off = h * 2 * kBlockBytes + kBlockBytes + n * kPage;
  const uint32_t ks_off = kTileBytes + k_page * 256, vs_off = kTileBytes + h * 256 + 4;
  u32x4 kc[4], vc[4];                    // raw codes: of the next half's K, of this half's V
  float ks;
  auto load_k = [&](uint32_t stage, int half, int cc) __attribute__((always_inline)) {
    kc[cc] = *reinterpret_cast<const u32x4*>(lds + stage + (k_off ^ (cc << 5)) + half * 4 * kBlockBytes);
  };
  auto load_v = [&](uint32_t stage, int half, int i) __attribute__((always_inline)) {
    vc[i] = *reinterpret_cast<const u32x4*>(lds + stage + v_off + half * 4 * kBlockBytes + i * 32 * kPage);
  };
  auto load_ks = [&](uint32_t stage, int half) __attribute__((always_inline)) {
    ks = *reinterpret_cast<const float*>(lds + stage + ks_off + half * 512);
  };
  // lane: scores of keys key0 + 16 h + r
  auto mask = [&](int key0, f32x16& s) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (key0 + 16 * h + r > my_pos) s[r] = -INFINITY;
  };
  auto across = [&](float x) __attribute__((always_inline)) {
    uint32_t lo = __builtin_bit_cast(uint32_t, x), hi = lo;
    swap_halves(lo, hi);
    return fmaxf(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)) * c2;
  };
  // codes of keys behind the last one go; NaN codes count for the rows that see their key (take_nan_codes)
  auto mend_v = [&](int key0) __attribute__((always_inline)) {
    const int first = key0 + 16 * h, valid = min(max(p.kv_len - first, 0), 16);
    uint32_t some = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int kept = min(max(valid - 4 * j, 0), 4);
        vc[i][j] &= kept == 4 ? 0xffffffffu : (1u << (8 * kept)) - 1u;
        some |= nan_codes(vc[i][j]);
      }
    if (__builtin_amdgcn_ballot_w64(some != 0) == 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 at = take_nan_codes(vc[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o[i] = Num<__bf16>::mfma32(huge(at, e & 1, e < 2), keys_seen(first + 8 * (e & 1), my_pos), o[i]);
    }
  };

  // Tile t + 1 is there, for every wavefront, and none reads tile t - 1 any more.
  auto turn = [&](int t) __attribute__((always_inline)) {
    if (t + 2 < p.t1)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kCopies) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (t + kStages - 1 < p.t1) copy_tile(t + kStages - 1);
  };

  // s: scores of keys key0 .. key0 + 31, s_next: of the 32 behind them, whose codes are in kc
  // kFixed: the rows' reference stays where the first half put it (see run)
  auto half_step = [&](auto fixed, int t, auto which, f32x16& s, f32x16& s_next) __attribute__((always_inline)) {
    constexpr bool kFixed = decltype(fixed)::value;
    constexpr int kHalf = decltype(which)::value;
    const int key0 = t * kBN + 32 * kHalf;
    const uint32_t stage = stage_at(t), next = stage_at(t + 1);   // (behind the last tile: stale, and not used)
    // the rows' reference moves when a maximum has risen by more than 2^8
    if (!kFixed && __builtin_amdgcn_ballot_w64(mx > m + 8.f) != 0) {
      const float m_new = fmaxf(m, mx);
      const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= f;
    }
    const float ref = !kFixed && m == -INFINITY ? 0.f : m;
    const float vs = *reinterpret_cast<const float*>(lds + stage + vs_off + kHalf * 512);
    uint32_t pk[8];
    float e0, e1;
    auto soft_exp = [&](int i) __attribute__((always_inline)) {
      e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * i], c2, -ref));
      e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * i + 1], c2, -ref));
    };
    auto soft_sum = [&](int i) __attribute__((always_inline)) {
      l += e0 + e1;
      pk[i] = pack2<T>(e0, e1);
      asm volatile("" : "+v"(l), "+v"(pk[i]));     // (stays in this phase)
    };
    vec8 op;
    // ---- phase 1: words 0..3 of P are made on the way
    __builtin_amdgcn_s_setprio(0);
    op = numbers<T>(kc[0][0], kc[0][1], ks);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      s_next = Num<T>::mfma32(op, q[u], u == 0 ? zero : s_next);
      if (u & 1) soft_sum(u >> 1);
      else soft_exp(u >> 1);
      if (u < 7) {
        const u32x4& w = kc[(u + 1) >> 1];
        op = numbers<T>(w[2 * ((u + 1) & 1)], w[2 * ((u + 1) & 1) + 1], ks);
      }
      if (u >= 2 && u < 6) load_v(stage, kHalf, u - 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (kHalf == 0) turn(t);
    // (the empty statements keep the compiler from doing either always, by selects)
    if (key0 + 63 > p.first_pos) {
      asm volatile("");
      mask(key0 + 32, s_next);
    }
    if (key0 + 31 > p.first_pos) {
      asm volatile("");
      mend_v(key0);
    }
    // ---- phase 2: V's d blocks with keys 0..7 of the page, then with keys 8..15
    __builtin_amdgcn_s_setprio(1);
    load_ks(next, kHalf);
    op = numbers<T>(vc[0][0], vc[0][1], vs);
    float x = -INFINITY;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int e = u >> 2;
      const u32x4 pw = {pk[4 * e], pk[4 * e + 1], pk[4 * e + 2], pk[4 * e + 3]};
      o[u & 3] = Num<T>::mfma32(op, __builtin_bit_cast(vec8, pw), o[u & 3]);
      if (u < 4) {
        soft_exp(4 + u);
        soft_sum(4 + u);
        // the half behind the next: of this tile's successor
        if constexpr (kHalf == 0) load_k(next, 0, u);
        else load_k(next, 1, u);
      } else if (!kFixed) {
        x = max3(x, s_next[4 * (u - 4)], s_next[4 * (u - 4) + 1]);
        x = max3(x, s_next[4 * (u - 4) + 2], s_next[4 * (u - 4) + 3]);
      }
      if (u < 7) {
        const u32x4& w = vc[(u + 1) & 3];
        op = numbers<T>(w[2 * ((u + 1) >> 2)], w[2 * ((u + 1) >> 2) + 1], vs);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!kFixed) mx = across(x);
  };
  // One pass over the piece.  Any reference gives the same O and sum as long as nothing leaves P's range, and a reference
  // that stays at the first half tile's maximum spares the others theirs, their comparison and the exchange
  // between lanes, a ninth of the vector instructions (16k over 16k tokens 5.92 ms, with one that moves 6.22; 8 prompts 419 and
  // 439 us).  The caller looks at the sums and accumulators afterwards, and
  // repeats the pass with a reference that moves where something was lost.  (bf16 P has fp32's range; fp16 P ends at 2^16
  // above the reference, beyond which it is an infinity, and has full precision down to 2^-14 below it, as
  // with a reference that moves: that one lies at most 2^8 below the row's maximum.)
  auto run = [&](bool may_fix) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = zero;
    m = mx = -INFINITY;
    l = 0.f;
    if (!active || p.t0 >= p.t1) {
      for (int t = p.t0; t < p.t1; ++t) turn(t);
      return;
    }
    const uint32_t stage = stage_at(p.t0);
    load_ks(stage, 0);
#pragma unroll
    for (int cc = 0; cc < 4; ++cc) load_k(stage, 0, cc);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      s_a = Num<T>::mfma32(numbers<T>(kc[u >> 1][2 * (u & 1)], kc[u >> 1][2 * (u & 1) + 1], ks), q[u], u == 0 ? zero : s_a);
    if (p.t0 * kBN + 31 > p.first_pos) mask(p.t0 * kBN, s_a);
    float x = s_a[0];
#pragma unroll
    for (int i = 1; i < 15; i += 2) x = max3(x, s_a[i], s_a[i + 1]);
    mx = across(max3(x, x, s_a[15]));
    load_ks(stage, 1);
#pragma unroll
    for (int cc = 0; cc < 4; ++cc) load_k(stage, 1, cc);
    auto loop = [&](auto fixed) __attribute__((always_inline)) {
      for (int t = p.t0; t < p.t1; ++t) {
        half_step(fixed, t, std::integral_constant<int, 0>(), s_a, s_b);
        half_step(fixed, t, std::integral_constant<int, 1>(), s_b, s_a);
      }
    };
    // (a row that sees no key of the first half has no reference there)
    if (may_fix && __builtin_amdgcn_ballot_w64(mx == -INFINITY) == 0) {
      m = mx;
      loop(std::true_type());
    } else {
      loop(std::false_type());
    }
  };
  // (the repeat has a copy of the loop to itself: as a second turn of a loop around one it cost the first 26 spilled
  // registers, and 8 prompts 2 %)
  run(true);
  {
    // A sum below 2^60 proves that no exponential was lost; an accumulator that is infinite or not a number shows here.
    float ends = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) ends = __builtin_fmaf(o[i][r], 0.f, ends);
    if (__syncthreads_or(!(l < 0x1p60f) || ends != 0.f)) {
      first_copies();
      run(false);
    }
  }
  l += __shfl_xor(l, 32);
  // lane: d = 32 i + 8 j + 4 h + [0, 4) of its row
  if (to.part >= 0) {
    const Parts parts(a);
    if (!active) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        parts.put_vector(parts.vector_at(to.part, wave, i, j),
                         f32x4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]});
    if (h == 0) parts.put_ml<kLaunchScope>(parts.at(to.part, row), m, l);
  } else if (row < p.ntok * G) {
    const int64_t at = out_row<G>(a, p, row);
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = f32x4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]} * inv;
      store_block<T>(a.out + at * kRowBytes + 64 * i, h, v);
    }
    if (h == 0) a.lse[at] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  }
}

// Part i of a q tile that spans from w0 on have written: the tile's beginning lies at the end of its span, the others at the
// beginning of theirs.
__device__ __forceinline__ int part_of(int w0, int i) { return 2 * (w0 + i) + (i == 0 ? 1 : 0); }

// The next kAhead parts' maxima and sums of a row, joined to what is there: factors of each part's O, and of the one so far.
template <int kAhead>
__device__ __forceinline__ float join(const f32x2 (&ml)[kAhead], int live, float& m, float& l, float (&f)[kAhead]) {
  float mx = m;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) mx = i < live ? fmaxf(mx, ml[i][0]) : mx;
  const float ref = mx == -INFINITY ? 0.f : mx, f0 = __builtin_amdgcn_exp2f(m - ref);
  m = mx;
  l *= f0;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    f[i] = i < live ? __builtin_amdgcn_exp2f(ml[i][0] - ref) : 0.f;
    l += i < live ? f[i] * ml[i][1] : 0.f;
  }
  return f0;
}

// The parts of a q tile of at most 16 rows, combined in their order: 16 threads a row.
template <typename T, int G>
__device__ __forceinline__ void combine_few(const Attn8Args& a, const Piece& p, int w0, int count) {
  constexpr int kAhead = 8;
  const Parts parts(a);
  const int row = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;
  if (row >= p.ntok * G) return;
  float m = -INFINITY, l = 0.f;
  f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  for (int i0 = 0; i0 < count; i0 += kAhead) {
    f32x2 ml[kAhead];
    f32x4 o[kAhead][2];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ml[i] = parts.get_ml<kDeviceScope>(parts.at(part_of(w0, min(i0 + i, count - 1)), row));
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        o[i][j] = parts.get<kDeviceScope>(parts.at(part_of(w0, min(i0 + i, count - 1)), row), d + 4 * j);
    float f[kAhead];
    const float f0 = join(ml, count - i0, m, l, f);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      acc[j] *= f0;
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i0 + i < count) acc[j] += f[i] * o[i][j];
    }
  }
  const int64_t to = out_row<G>(a, p, row);
  const float inv = 1.f / l;
  *reinterpret_cast<u32x4*>(a.out + to * kRowBytes + d * 2) =
      u32x4{pack2<T>(acc[0][0] * inv, acc[0][1] * inv), pack2<T>(acc[0][2] * inv, acc[0][3] * inv),
            pack2<T>(acc[1][0] * inv, acc[1][1] * inv), pack2<T>(acc[1][2] * inv, acc[1][3] * inv)};
  if (d == 0) a.lse[to] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// The parts of q tiles of 128 rows, in a launch of its own, bound by reading them: a workgroup takes 32 d of all rows of the
// tile that begins in span w and goes on behind it, if there is one, on the XCD that wrote its first part.  (500 new
// tokens over 4500, plan, attention and this: 66.5 us; on any XCD with 6 parts requested at a time instead of 4 64.1, on
// this one 64.5, both 60.8.)
constexpr int kMergeBlocks = 4;
template <typename T, int G>
__global__ __launch_bounds__(kThreads) void merge8_kernel(Attn8Args a) {
  constexpr int kAhead = 6;
  const int w = blockIdx.x % kXcds * (a.spans / kXcds) + blockIdx.x / kXcds / kMergeBlocks,
            i32 = blockIdx.x / kXcds % kMergeBlocks;
  const MergeRec8 r = a.merges[w];
  const Plan8Header hdr = *a.hdr;
  if (hdr.magic != kPlanMagic || hdr.heads != a.hkv * 16 + G || hdr.batch != a.batch || hdr.total_q != a.total_q)
    return;
  if (r.count < 2 || w + r.count > a.spans) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, row = wave * 32 + (lane & 31);
  if (wave * 32 >= r.ntok * G) return;
  const Parts parts(a);
  float m = -INFINITY, l = 0.f;
  f32x4 acc[4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  for (int i0 = 0; i0 < r.count; i0 += kAhead) {
    f32x2 ml[kAhead];
    f32x4 o[kAhead][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ml[i] = parts.get_ml<kLaunchScope>(parts.at(part_of(w, min(i0 + i, r.count - 1)), row));
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        o[i][j] = parts.get_vector(parts.vector_at(part_of(w, min(i0 + i, r.count - 1)), wave, i32, j));
    float f[kAhead];
    const float f0 = join(ml, r.count - i0, m, l, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[j] *= f0;
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i0 + i < r.count) acc[j] += f[i] * o[i][j];
    }
  }
  if (row >= r.ntok * G) return;       // (both lanes of a row)
  Piece p = {};
  p.hk = r.hk;
  p.q_first = r.q_first;
  const int64_t to = out_row<G>(a, p, row);
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] *= 1.f / l;
  store_block<T>(a.out + to * kRowBytes + 64 * i32, h, acc);
  if (i32 == 0 && h == 0) a.lse[to] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int G, bool kFewOnly>
__global__ __launch_bounds__(kThreads, 2) void attn8_kernel(Attn8Args a) {
  __shared__ __attribute__((aligned(1024))) char lds[kFewOnly ? kFewBytes : kLdsBytes];
  __shared__ int s_last;
  constexpr int kRows = kFewOnly ? kFewRows : kTileRows;
  const Plan8Header hdr = *a.hdr;
  // the plan must be one of this very batch
  if (hdr.magic != kPlanMagic || hdr.heads != a.hkv * 16 + G || hdr.batch != a.batch || hdr.total_q != a.total_q ||
      hdr.tile_rows != kRows)
    return;
  const int64_t units = hdr.units, span = hdr.span;
  // neighbouring spans, which share K and V, on one XCD (workgroups go to the XCDs in turns)
  const int w = blockIdx.x % kXcds * (gridDim.x / kXcds) + blockIdx.x / kXcds;
  static_assert(kSpans % kXcds == 0, "every span is some workgroup's");
  if (!kFewOnly && threadIdx.x == 0) a.merges[w].count = 0;
  int64_t at = w * span;
  const int64_t end = min(at + span, units * a.hkv);
  if (at >= end) return;
  const SpanStart start = a.starts[w];
  int hk = start.hk, s = start.seq;
  int64_t tile = start.tile, tile_at = start.tile_at;
  PlanSeq sq = start.of;
  int now = a.begin[s];
  bool usable = a.verdict[s] == MC_OK;
  int entries = a.cu_pages[s + 1] - sq.table_off;
  while (at < end) {
    const int q0 = sq.q_first, q = sq.q, rows = rows_of_tiles(q, G, kRows), tok = rows / G, b = sq.begin;
    const bool few = kFewOnly || rows == kFewRows;
    const int shift = kFewOnly ? 0 : unit_shift(rows), weight = 1 << shift;
    const int row0 = (int)tile * tok, ntok = min(tok, q - row0);
    const int planned = (int)tiles64((int64_t)b + row0 + ntok);     // KV tiles of this q tile, by the plan
    // the visits whose first unit lies in this span (every span has at least kMinSpan units, so a visit's beginning)
    const int64_t first = tile_at + (kTileCost << shift), tile_end = first + ((int64_t)planned << shift);
    const int64_t stop = min(tile_end, end);
    const int t0 = (int)(max(at - first + weight - 1, (int64_t)0) >> shift), t1 = (int)(max(stop - first + weight - 1, (int64_t)0) >> shift);
    if (at < tile_at || at >= tile_end) return;     // (never of a plan: a workspace written over)
    Piece p;
    p.hk = hk;
    p.q_first = q0 + row0;
    p.ntok = ntok;
    p.first_pos = now + row0;
    p.kv_len = p.first_pos + ntok;
    const int actual = (int)tiles64(p.kv_len);           // begin may have grown since the plan
    p.t0 = t0;
    p.t1 = t1 == planned ? actual : min(t1, actual);
    p.table_off = sq.table_off;
    p.last_entry = (p.kv_len - 1) / kPage;
    // what a table of the length that the plan saw cannot hold is not read
    const bool ok = usable && now >= 0 && now <= kMostTokens && p.last_entry < entries;
    const bool whole = t0 == 0 && t1 == planned;
    if (ok && t0 < t1) {
      Target to;
      to.part = whole ? -1 : 2 * w + (t0 == 0 ? 1 : 0);
      if (few)
        few_rows_piece<T, G>(a, p, to, lds);
      else if constexpr (!kFewOnly)
        tile_piece<T, G>(a, p, to, lds);
      if (!whole) {
        const int w0 = (int)(first / span), count = (int)((tile_end - weight) / span) - w0 + 1;
        if (!few) {
          if (t0 == 0 && threadIdx.x == 0) a.merges[w] = MergeRec8{p.q_first, p.ntok, p.hk, count};
        } else {
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // this wavefront's rows have been written
          __syncthreads();
          if (threadIdx.x == 0)
            s_last = __hip_atomic_fetch_add(a.arrivals + w0, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                     (unsigned)(count - 1);
          __syncthreads();
          if (s_last) {
            if (threadIdx.x == 0)      // for the next layer
              __hip_atomic_store(a.arrivals + w0, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            combine_few<T, G>(a, p, w0, count);
          }
        }
      }
    }
    at = stop;
    tile_at = tile_end;
    if ((tile + 1) * tok < q) {
      ++tile;
    } else {
      tile = 0;
      // the next sequence with new tokens, of this kv head or the next
      const int64_t done = a.cum[s + 1];
      if (done == units) {
        ++hk;
        s = 0;
        while (s + 1 < a.batch && a.cum[s + 1] == 0) ++s;
      } else {
        ++s;
        while (s + 1 < a.batch && a.cum[s + 1] == done) ++s;
      }
      sq = a.seqs[s];
      now = a.begin[s];
      usable = a.verdict[s] == MC_OK;
      entries = a.cu_pages[s + 1] - sq.table_off;
    }
  }
}

mc_status check_shape8(const mc_pool8_desc* pool, int32_t num_q_heads, int32_t batch, int32_t total_q, int* G_out) {
  mc_status st = mc::check_pool8(pool);
  if (st != MC_OK) return st;
  if (num_q_heads <= 0 || batch < 0 || total_q < 0) return MC_ERR_INVALID;
  if (num_q_heads % pool->num_kv_heads != 0) return MC_ERR_UNSUPPORTED;
  const int G = num_q_heads / pool->num_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8) return MC_ERR_UNSUPPORTED;
  *G_out = G;
  return MC_OK;
}

template <typename T>
mc_status launch_attn8(int G, bool few, hipStream_t hs, const Attn8Args& a) {
  auto* kernel = few ? (G == 1   ? attn8_kernel<T, 1, true>
                        : G == 2 ? attn8_kernel<T, 2, true>
                        : G == 4 ? attn8_kernel<T, 4, true>
                                 : attn8_kernel<T, 8, true>)
                     : (G == 1   ? attn8_kernel<T, 1, false>
                        : G == 2 ? attn8_kernel<T, 2, false>
                        : G == 4 ? attn8_kernel<T, 4, false>
                                 : attn8_kernel<T, 8, false>);
  hipLaunchKernelGGL(kernel, dim3(a.spans), dim3(kThreads), 0, hs, a);
  const mc_status st = mc::launch_status();
  if (st != MC_OK || few) return st;
  auto* merge = G == 1   ? merge8_kernel<T, 1>
                : G == 2 ? merge8_kernel<T, 2>
                : G == 4 ? merge8_kernel<T, 4>
                         : merge8_kernel<T, 8>;
  hipLaunchKernelGGL(merge, dim3(a.spans * kMergeBlocks), dim3(kThreads), 0, hs, a);
  return mc::launch_status();
}

}  // namespace

extern "C" {

size_t mc_attn8_workspace_size(int32_t batch, int32_t total_q, int32_t num_q_heads, int32_t num_kv_heads) {
  if (batch < 0 || total_q < 0 || num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads != 0) return 0;
  const int G = num_q_heads / num_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8) return 0;
  return workspace8(batch, total_q, G).total;
}

mc_status mc_attn8_plan_ahead(const mc_pool8_desc* pool, int32_t num_q_heads, int32_t batch, int32_t total_q,
                              const int32_t* cu_q, const int32_t* begin, const int32_t* page_table,
                              const int32_t* cu_pages, int32_t ahead_tokens, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (ahead_tokens < 0 || ahead_tokens > (1 << 20)) return MC_ERR_RANGE;
  int G = 0;
  const mc_status st = check_shape8(pool, num_q_heads, batch, total_q, &G);
  if (st != MC_OK) return st;
  if (!workspace || !mc::aligned16(workspace)) return MC_ERR_INVALID;
  const Workspace8 w = workspace8(batch, total_q, G);
  if (workspace_bytes < w.total) return MC_ERR_INVALID;
  if (!cu_q || !cu_pages || (batch > 0 && (!begin || !page_table))) return MC_ERR_INVALID;
  char* ws = static_cast<char*>(workspace);
  Plan8Args a;
  a.cu_q = cu_q;
  a.begin = begin;
  a.page_table = page_table;
  a.cu_pages = cu_pages;
  a.hdr = reinterpret_cast<Plan8Header*>(ws);
  a.cum = reinterpret_cast<int64_t*>(ws + w.cum);
  a.seqs = reinterpret_cast<PlanSeq*>(ws + w.seqs);
  a.verdict = reinterpret_cast<int32_t*>(ws + w.verdict);
  a.arrivals = reinterpret_cast<uint32_t*>(ws + w.arrivals);
  a.starts = reinterpret_cast<SpanStart*>(ws + w.starts);
  a.batch = batch;
  a.total_q = total_q;
  a.num_pages = pool->num_pages;
  a.hkv = pool->num_kv_heads;
  a.G = G;
  a.ahead = ahead_tokens;
  a.tile_rows = w.few ? kFewRows : kTileRows;
  a.spans = w.spans;
  hipLaunchKernelGGL(plan8_kernel, dim3(1 + (unsigned)batch), dim3(kPlanThreads), 0, static_cast<hipStream_t>(stream), a);
  return mc::launch_status();
}

mc_status mc_attn8_plan_check(const void* workspace, void* stream) {
  if (!workspace) return MC_ERR_INVALID;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  auto read = [&](void* to, size_t from, size_t bytes) {
    return hipMemcpyAsync(to, static_cast<const char*>(workspace) + from, bytes, hipMemcpyDeviceToHost, hs) ==
               hipSuccess &&
           hipStreamSynchronize(hs) == hipSuccess;
  };
  Plan8Header h;
  if (!read(&h, 0, sizeof(h))) return MC_ERR_HIP;
  if (h.magic != kPlanMagic) return MC_ERR_INVALID;
  const size_t verdicts = workspace8(h.batch, 0, 1).verdict;
  int32_t some[1024];
  for (int32_t s = 0; s < h.batch; s += 1024) {
    const int32_t n = h.batch - s < 1024 ? h.batch - s : 1024;
    if (!read(some, verdicts + sizeof(int32_t) * (size_t)s, sizeof(int32_t) * (size_t)n)) return MC_ERR_HIP;
    for (int32_t i = 0; i < n; ++i)
      if (some[i] != MC_OK) return static_cast<mc_status>(some[i]);
  }
  return MC_OK;
}

mc_status mc_attn8_plan(const mc_pool8_desc* pool, int32_t num_q_heads, int32_t batch, int32_t total_q,
                        const int32_t* cu_q, const int32_t* begin, const int32_t* page_table,
                        const int32_t* cu_pages, void* workspace, size_t workspace_bytes, void* stream) {
  return mc_attn8_plan_ahead(pool, num_q_heads, batch, total_q, cu_q, begin, page_table, cu_pages, 0, workspace,
                             workspace_bytes, stream);
}

mc_status mc_prefix_prefill_attn8(const mc_pool8_desc* pool, int32_t layer, const void* q, int32_t num_q_heads,
                                  int32_t batch, int32_t total_q, const int32_t* cu_q, const int32_t* begin,
                                  const int32_t* page_table, const int32_t* cu_pages, float sm_scale, void* out,
                                  float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  int G = 0;
  const mc_status st = check_shape8(pool, num_q_heads, batch, total_q, &G);
  if (st != MC_OK) return st;
  if (layer < 0 || layer >= pool->num_layers) return MC_ERR_RANGE;
  if (!(sm_scale >= 0.f) || !isfinite(sm_scale)) return MC_ERR_INVALID;
  if (batch == 0 || total_q == 0) return MC_OK;
  if (!q || !out || !lse || !cu_q || !begin || !page_table || !cu_pages || !workspace) return MC_ERR_INVALID;
  if (!mc::aligned16(q) || !mc::aligned16(out) || !mc::aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u))
    return MC_ERR_INVALID;
  const Workspace8 w = workspace8(batch, total_q, G);
  if (workspace_bytes < w.total) return MC_ERR_INVALID;
  char* ws = static_cast<char*>(workspace);
  Attn8Args a;
  a.codes = static_cast<const char*>(pool->codes) + layer * mc::layer8_stride(pool);
  a.scales = pool->scales + layer * mc::layer8_scales(pool);
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.begin = begin;
  a.page_table = page_table;
  a.cu_pages = cu_pages;
  a.hdr = reinterpret_cast<const Plan8Header*>(ws);
  a.cum = reinterpret_cast<const int64_t*>(ws + w.cum);
  a.seqs = reinterpret_cast<const PlanSeq*>(ws + w.seqs);
  a.verdict = reinterpret_cast<const int32_t*>(ws + w.verdict);
  a.arrivals = reinterpret_cast<uint32_t*>(ws + w.arrivals);
  a.starts = reinterpret_cast<const SpanStart*>(ws + w.starts);
  a.merges = reinterpret_cast<MergeRec8*>(ws + w.merges);
  a.part_ml = reinterpret_cast<float*>(ws + w.part_ml);
  a.part_o = reinterpret_cast<float*>(ws + w.part_o);
  a.num_pages = pool->num_pages;
  a.hkv = pool->num_kv_heads;
  a.hq = num_q_heads;
  a.batch = batch;
  a.total_q = total_q;
  a.part_rows = w.part_rows;
  a.spans = w.spans;
  const float scale = sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)kHeadDim);
  a.scale_log2 = scale * 1.4426950408889634f;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  return pool->dtype == MC_F16 ? launch_attn8<_Float16>(G, w.few, hs, a) : launch_attn8<__bf16>(G, w.few, hs, a);
}

}  // extern "C"
