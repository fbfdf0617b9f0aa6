// Attention of chunks of new tokens over a paged KV cache on tcgen05 (bf16 storage, head dims 64 and 128).
//
// Rows of a score tile are packed: token x head of one KV head's group, heads inside, floor(128 / G) tokens to a tile of 128 rows, so one
// drafted token or a long chunk fill as much of a tile as they can and K and V are read once for the whole group.  A unit of work is
// (sequence, KV head, one tile of tokens or two neighbouring ones); its cost is the number of 128-row blocks of the cache that its last token
// sees.  All units laid end to end make a line of blocks, which is cut into as many equal pieces as there are CTAs (one per SM): every
// CTA has the same number of blocks, whatever the batch.  A unit that several CTAs work on leaves shares (O, maximum, sum) in the
// workspace, joined by paged_attn_join_kernel.  Lengths and starts are read on the device; nothing depends on the host's view.
//
//   warp 0      TMA producer: Q tiles (boxes of G heads x tokens), then the blocks of K and V in the order in which they are needed, page
//               by page, into a ring of five tiles
//   warp 1      TMEM owner and single-thread MMA issuer; columns S_0 | S_1 | O_0 | O_1
//   warp 2      clears, in shared memory, the rows of V behind a sequence's last one (they may hold anything, and 0 * NaN is NaN)
//   warps 4-7   softmax of slot 0, warps 8-11 of slot 1, one row per thread
// The two slots are the unit's two tiles, which share every block of K and V, or, where it has one tile, two neighbouring blocks of the cache
// (joined at the end of the unit): either way the tensor core has the other slot's products while one slot's softmax runs.
// P V reads V as it lies in the pages (row = token): its operand is the transposed one, 128-byte swizzled with the head dims along the row.
#include <climits>

#include "paged_common.cuh"
#include "tc_ptx.cuh"

namespace spts {

namespace {

using namespace paged;
using namespace ptx;

constexpr int BLOCK = 128;                     // rows of the cache to a block, rows of a score tile
constexpr int SLAB = BLOCK * 128;              // a tile of Q: [128 rows x 64 bf16] for each 64 dims, 128-byte swizzle
constexpr int RING = 5;                        // tiles of K or V in flight
constexpr int PA_THREADS = 384;
constexpr int PA_COLS = 512;
constexpr int REGS_LIGHT = 72, REGS_SOFTMAX = 216;   // 128 * 72 + 256 * 216 = 384 * 168, the launch's total
constexpr int SOLO_ROWS = 16;                  // rows of a unit, on average, up to which it is joined within the kernel
constexpr float RESCALE = 8.0f;                // log2 units the running maximum may lag behind
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <int D> constexpr int tile_bytes() { return D / 64 * SLAB; }
template <int D> constexpr int pa_smem() { return 1024 + (2 + RING) * tile_bytes<D>() + 512 + 1024 + 128; }
// A share: O as [D / 8][128 rows][8], so that a warp's rows are written without gaps, then (maximum, sum) of each row.
template <int D> constexpr int share_floats() { return BLOCK * (D + 2); }
__device__ __forceinline__ int share_at(int row, int col) { return ((col >> 3) * BLOCK + row) * 8 + (col & 7); }
// 32 bytes: whole sectors where a warp's lanes write different rows
__device__ __forceinline__ void store32(void* p, uint4 x, uint4 y) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w), "r"(y.x), "r"(y.y),
               "r"(y.z), "r"(y.w)
               : "memory");
}

struct AttnArgs {
  Cache c;
  const int32_t* row_start; int n_rows;
  int H, Hkv, G;
  int tile_tokens, unit_tokens;                // floor(128 / G); that or twice that
  int extra;                                   // blocks that a unit costs beside its own
  const bf16* Q; int64_t ldq;
  bf16* O; int64_t ldo; float* lse;
  int wide;                                    // rows of O begin on 32 bytes
  float* share; int* arrived;
  struct OpenUnit* open;                       // [CTAs]
  int solo;                                    // units are joined by the CTA that is done last instead of a second kernel
  int* status;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// Tiles of K and V in shared memory: [128 / 8 groups of rows][D / 64][8 rows][64 bf16], so that one box brings in all dims of the rows of a
// page, 128-byte swizzled.  As K-major operand (rows = N or M): the next eight rows are a group further.  As the operand of P V (rows
// along K, dims along N): the next eight of K are a group further, the next 64 of N 1024 bytes.
// A descriptor's low word holds the address / 16, so it moves by additions; its high word is constant.
template <int D> constexpr int group_bytes() { return D / 64 * 1024; }
constexpr uint32_t desc_high(int stride_bytes) { return (uint32_t)(stride_bytes >> 4) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, int leading_bytes) { return ((saddr & 0x3FFFFu) >> 4) | ((uint32_t)(leading_bytes >> 4) << 16); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b64 da, db;\n"
      "mov.b64 da, {%1, %2};\n"
      "mov.b64 db, {%3, %4};\n"
      "setp.ne.b32 p, %6, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n"
      "}\n" ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      ".reg .b64 db;\n"
      "mov.b64 db, {%2, %3};\n"
      "setp.ne.b32 p, %5, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n"
      "}\n" ::"r"(d), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
constexpr uint32_t B_ALONG_N = 1u << 16;       // instruction descriptor: B is stored N-contiguous

__device__ __forceinline__ bool elect_lane() {
  uint32_t mine;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "elect.sync _|p, 0xffffffff;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(mine));
  return mine != 0;
}

// A wait whose limit counts from its own beginning or from the CTA's last sign of life.  `flags`: [0] somebody gave up; [1] grows with every
// block of the cache that is asked for and while rows are computed again (plain_row): the warp that clears the rows behind a sequence's last one
// may have nothing to do until the end of a piece that takes many seconds.
constexpr int ABORT = 0, BUSY = 1;
__device__ __forceinline__ void sign_of_life(volatile int* busy) { atomicAdd(const_cast<int*>(busy), 1); }
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* flags) {
  if (mbar_test_wait(bar, parity)) return true;
  uint64_t t0 = 0;
  int busy = 0;
  for (uint32_t it = 0;; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 0xFFu) == 0xFFu) {
      if (flags[ABORT]) return false;
      const uint64_t now = globaltimer_ns();
      if (t0 == 0 || flags[BUSY] != busy) {
        t0 = now;
        busy = flags[BUSY];
      } else if (now - t0 > WAIT_LIMIT_NS) {
        flags[ABORT] = 1;
        return false;
      }
    }
  }
}

// The same for a whole warp: all lanes or none go on.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* flags) {
  return __all_sync(0xffffffffu, wait(bar, parity, flags));
}

// ------------------------------------------------------------------------------------------------ the line of blocks
// sum of floor((a i + b) / m), i < n, by the well-known recursion of such sums that follows Euclid's algorithm on (m, a); a, b and m stay small, so 32 bits hold a n + b for all
// but the longest lines
__device__ unsigned long long floor_sum(uint32_t n, uint32_t m, uint32_t a, uint32_t b) {
  unsigned long long sum = 0;
  while (true) {
    if (a >= m) { sum += (unsigned long long)n * (n - 1) / 2 * (a / m); a %= m; }
    if (b >= m) { sum += (unsigned long long)n * (b / m); b %= m; }
    if (n < 1u << 23) {                        // (a, b < 2^9)
      const uint32_t y = a * n + b;
      if (y < m) return sum;
      n = y / m;
      b = y % m;
    } else {
      const unsigned long long y = (unsigned long long)a * n + b;
      if (y < m) return sum;
      n = (uint32_t)(y / m);
      b = (uint32_t)(y % m);
    }
    const uint32_t t = m;
    m = a;
    a = t;
  }
}
// Blocks of unit g of a sequence whose n queries see off + 1, off + 2, ... rows: one at least (the unit's rows are written even where
// they see nothing).
__device__ __forceinline__ int unit_blocks(int n, int off, int R, int g) {
  const int seen = off + min(n, (g + 1) * R);
  return max(1, (seen + BLOCK - 1) / BLOCK);
}
// of the units before g, each with `extra` places behind its blocks at which there is nothing to do: what a unit costs beside its blocks (its
// first products, reading out O), in blocks
__device__ long long blocks_before(int n, int off, int R, int extra, int g) {
  const int whole = min(g, n / R);
  const int blind = off < 0 ? min(whole, -off / R) : 0;            // units that see nothing
  long long sum = blind + (long long)extra * g;
  if (whole > blind) sum += (long long)floor_sum(whole - blind, BLOCK, R, off + (blind + 1) * R + BLOCK - 1);
  if (g > whole) sum += unit_blocks(n, off, R, whole);
  return sum;
}
// The largest g in [0, count) with before(g) <= x, by a warp: 32 guesses at a time.
template <typename F> __device__ __forceinline__ int warp_find(int count, long long x, F before) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = count;                      // before(lo) <= x, and not at hi
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, g = lo + lane * step;
    const uint32_t below = __ballot_sync(0xffffffffu, g < hi && (lane == 0 || before(g) <= x));
    lo += (31 - __clz(below)) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// Where the piece of CTA `cta` begins.  Fewer pieces than CTAs: one to each of the first, so that no CTA between two others is without.
// (Divisions of 64 bits cost a microsecond together: lines of ordinary length are cut in 32.)
__device__ __forceinline__ long long cut_line(long long total, int cta, int ctas) {
  if (total < ctas) return min((long long)cta, total);
  if (total < 1 << 23) return (uint32_t)total * (uint32_t)cta / (uint32_t)ctas;
  return total * cta / ctas;
}
// The CTA whose piece holds block x: the largest c with cut_line(c) <= x, that is total c / ctas < x + 1.
__device__ __forceinline__ int cta_of(long long total, long long x, int ctas) {
  if (total < ctas) return (int)x;
  if (total < 1 << 23) return (int)((((uint32_t)x + 1) * (uint32_t)ctas - 1) / (uint32_t)total);
  return (int)(((x + 1) * ctas - 1) / total);
}

struct Place { int b, h, g, j; };              // block j of unit (b, h, g)

struct Line {
  long long* pre;                              // [n_seq + 1] blocks before each sequence
  long long total;
  template <int NT> __device__ __forceinline__ void make(const AttnArgs& a, long long* scratch, bool check) {
    pre = scratch + 32;
    total = block_prefix<NT>(a.c.n_seq, pre, scratch, [&](int b) {
      int first, n;
      call_rows(a.row_start, a.n_rows, b, first, n);
      if (check) check_starts(a.row_start, a.n_rows, b, a.status);
      const int R = a.unit_tokens;
      return n == 0 ? 0LL : a.Hkv * blocks_before(n, held_rows(a.c, b) - n, R, a.extra, (n + R - 1) / R);
    });
  }
  __device__ __forceinline__ long long cut(int cta, int ctas) const { return cut_line(total, cta, ctas); }
  // (by a warp)
  __device__ __forceinline__ Place find(const AttnArgs& a, long long x) const {
    Place p;
    p.b = find_share(pre, a.c.n_seq, x);
    int first, n;
    call_rows(a.row_start, a.n_rows, p.b, first, n);
    const int off = held_rows(a.c, p.b) - n, R = a.unit_tokens;
    const long long all = pre[p.b + 1] - pre[p.b];
    x -= pre[p.b];
    long long head;
    if (all < 1LL << 31) {
      head = (uint32_t)all / (uint32_t)a.Hkv;
      p.h = (int)((uint32_t)x / (uint32_t)head);
    } else {
      head = all / a.Hkv;
      p.h = (int)(x / head);
    }
    x -= p.h * head;
    p.g = warp_find((n + R - 1) / R, x, [&](int g) { return blocks_before(n, off, R, a.extra, g); });
    p.j = (int)(p.g == 0 ? x : x - blocks_before(n, off, R, a.extra, p.g));
    return p;
  }
};

// A CTA's share of one unit: blocks [j0, j1) of `cost`.
struct Segment {
  int b, h, j0, j1, cost;
  int held, off;                               // the sequence's rows, rows before its first query
  long long begin;                             // of the unit on the line
  int token, tokens;                           // first token of the unit (in its sequence), how many
  int row;                                     // first row of the unit in Q and O
  bool two;                                    // two tiles
};

// Each role of a CTA walks over the CTA's segments by itself.
struct Walk {
  Place p;
  long long at, left;                          // place on the line, what is left of the piece
  int first, n, off, held;
  __device__ __forceinline__ void sequence(const AttnArgs& a) {
    call_rows(a.row_start, a.n_rows, p.b, first, n);
    held = held_rows(a.c, p.b);
    off = held - n;
  }
  __device__ __forceinline__ bool next(const AttnArgs& a, Segment& s) {
    const int R = a.unit_tokens;
    while (left > 0) {
      s.cost = unit_blocks(n, off, R, p.g);
      s.j0 = p.j;
      const int j1 = (int)min((long long)s.cost + a.extra, p.j + left);
      s.j1 = min(j1, s.cost);
      s.b = p.b; s.h = p.h; s.held = held;
      s.token = p.g * R;
      s.tokens = min(R, n - s.token);
      s.off = off;
      s.row = first + s.token;
      s.two = s.tokens > a.tile_tokens;
      s.begin = at - p.j;
      left -= j1 - p.j;
      at += j1 - p.j;
      p.j = 0;
      if ((p.g + 1) * R < n) {
        ++p.g;
      } else {
        p.g = 0;
        if (++p.h == a.Hkv) {
          p.h = 0;
          while (left > 0 && ++p.b < a.c.n_seq) {
            sequence(a);
            if (n > 0) break;
          }
        }
      }
      if (s.j0 < s.j1) return true;
    }
    return false;
  }
};

// ------------------------------------------------------------------------------------------------ rows that came out not finite
// A weight of zero does not keep an infinity or NaN of V out of a product of matrices.  A row with a finite sum of weights that came out not
// finite, of a segment that holds rows it does not see, is computed again, by its warp, over the rows [k0, k1) of the cache that it sees:
// D / 32 dims to a lane, eight rows at a time.  (m in log2 units; o not divided by l.)
template <int D>
__device__ __noinline__ void plain_row(const AttnArgs& a, int b, int kvh, const bf16* q, int k0, int k1, volatile int* busy, float& m_out, float& l_out,
                                       float* o_out) {
  constexpr int PER = D / 32, STEP = 8;
  const int lane = threadIdx.x & 31;
  const auto load = [&](const char* x, int64_t slot, float (&to)[PER]) {
    const __nv_bfloat162* at = reinterpret_cast<const __nv_bfloat162*>(reinterpret_cast<const bf16*>(x) + (max(slot, (int64_t)0) * a.Hkv + kvh) * D + lane * PER);
#pragma unroll
    for (int e = 0; e < PER / 2; ++e) {
      const float2 y = __bfloat1622float2(__ldg(at + e));
      to[2 * e] = slot < 0 ? 0.f : y.x;
      to[2 * e + 1] = slot < 0 ? 0.f : y.y;
    }
  };
  float qf[PER], m = -INFINITY, l = 0.f, o[PER];
  const float sc = LOG2E * rsqrtf((float)D);
#pragma unroll
  for (int e = 0; e < PER; ++e) { qf[e] = __bfloat162float(q[lane * PER + e]) * sc; o[e] = 0.f; }
  for (int j0 = k0; j0 < k1; j0 += 32) {
    if (lane == 0) sign_of_life(busy);
    const int64_t slots = j0 + lane < k1 ? slot_of(a.c, b, j0 + lane) : -1;
    for (int u0 = 0; u0 < 32 && j0 + u0 < k1; u0 += STEP) {
      float s[STEP], v[STEP][PER];
#pragma unroll
      for (int u = 0; u < STEP; ++u) {
        const int64_t slot = __shfl_sync(0xffffffffu, slots, u0 + u);
        float kf[PER];
        load(a.c.k, slot, kf);
        load(a.c.v, slot, v[u]);
        s[u] = 0.f;
#pragma unroll
        for (int e = 0; e < PER; ++e) s[u] = fmaf(qf[e], kf[e], s[u]);
      }
      float now = m;
#pragma unroll
      for (int u = 0; u < STEP; ++u) {
        s[u] = warp_sum(s[u]);
        if (j0 + u0 + u >= k1) s[u] = -INFINITY;
        now = fmaxf(now, s[u]);
      }
      const float base = now == -INFINITY ? 0.f : now, alpha = m == -INFINITY ? 0.f : ex2(m - base);
      l *= alpha;
#pragma unroll
      for (int e = 0; e < PER; ++e) o[e] *= alpha;
#pragma unroll
      for (int u = 0; u < STEP; ++u) {
        const float p = ex2(s[u] - base);
        l += p;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = p == 0.f ? o[e] : fmaf(p, v[u][e], o[e]);
      }
      m = now;
    }
  }
  m_out = m;
  l_out = l;
#pragma unroll
  for (int e = 0; e < PER; ++e) o_out[e] = o[e];
}

// ------------------------------------------------------------------------------------------------ joining shares
constexpr int JOIN_AT_ONCE = 10;
struct OpenUnit { int last, row, h, tokens; };   // the unit that begins in a CTA and goes on, up to CTA `last` (-1: there is none)

// Row `row` of a tile of a unit that CTAs first .. last worked on, by one warp: the shares in the order of the line (of the first CTA its last
// segment, of the others their first).
template <int D>
__device__ __forceinline__ void join_row(const AttnArgs& a, int unit_row, int h, int first, int last, int tile, int row) {
  constexpr int PER = D / 32;
  const int lane = threadIdx.x & 31, parts = last - first + 1;
  const auto share = [&](int i) { return a.share + ((int64_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * 2 + tile) * share_floats<D>(); };
  float m = -INFINITY, l = 0.f, o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = 0.f;
  for (int i0 = 0; i0 < parts; i0 += JOIN_AT_ONCE) {
    // the loads of some shares are all on their way before the first is used; O is carried on to a larger maximum as in the kernel
    const int n = min(JOIN_AT_ONCE, parts - i0);
    float2 x = make_float2(-INFINITY, 0.f);
    if (lane < n) x = __ldcg(reinterpret_cast<const float2*>(share(i0 + lane) + BLOCK * D + 2 * row));
    float v[JOIN_AT_ONCE][PER];
#pragma unroll
    for (int i = 0; i < JOIN_AT_ONCE; ++i) {
      const float* y = share(i0 + min(i, n - 1)) + share_at(row, lane * PER);
      if (PER == 4) {
        const float4 z = __ldcg(reinterpret_cast<const float4*>(y));
        v[i][0] = z.x; v[i][1] = z.y; v[i][PER - 2] = z.z; v[i][PER - 1] = z.w;
      } else {
        const float2 z = __ldcg(reinterpret_cast<const float2*>(y));
        v[i][0] = z.x; v[i][1] = z.y;
      }
    }
    const float now = fmaxf(m, warp_max(x.x)), b = now == -INFINITY ? 0.f : now;
    const float alpha = m == -INFINITY ? 0.f : ex2(m - b), f = ex2(x.x - b);
    // (a share without a maximum: nothing was seen, l = 0; or NaN alone)
    l = l * alpha + warp_sum(x.x == -INFINITY ? x.y : x.y * f);
    m = now;
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = alpha == 0.f ? 0.f : o[e] * alpha;
#pragma unroll
    for (int i = 0; i < JOIN_AT_ONCE; ++i) {
      const float fi = __shfl_sync(0xffffffffu, f, i);
#pragma unroll
      for (int e = 0; e < PER; ++e) o[e] = i >= n || fi == 0.f ? o[e] : fmaf(v[i][e], fi, o[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  const int64_t out_row = (int64_t)unit_row + tile * a.tile_tokens + row / a.G;
  const int head = h * a.G + row % a.G;
  uint32_t* to_o = reinterpret_cast<uint32_t*>(a.O + out_row * a.ldo + (int64_t)head * D) + lane * (PER / 2);
#pragma unroll
  for (int e = 0; e < PER / 2; ++e) to_o[e] = l == 0.f ? 0u : pack2(o[2 * e] * inv, o[2 * e + 1] * inv);
  if (lane == 0 && a.lse != nullptr) a.lse[out_row * a.H + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

// ------------------------------------------------------------------------------------------------ the kernel
// Long chunks fill no unit (2048 tokens over 34816 rows, 32 heads of 128 dims, replayed: 0.96 to 1.07 ms, 1060 to 1180 TFLOP/s; tensor pipe busy
// 64 %, issue slots 38 %, and 2.27 GB read where K and V hold 143 MB, which the L2 does not): what is left is the two softmax warpgroups' chain of
// loads, maxima, exponentials and stores beside the products, and blocks that miss the L2 (16384 fresh tokens, whose K and V fit it: 1225 to 1279
// TFLOP/s).  With a quarter of the exponentials as polynomials of degree five 7 % slower.  Decode steps are bound by memory (64 sequences of up to
// 16384 rows: 280 us, 6.2 TB/s; 48 of up to nine drafted tokens 129 us, 5.0 TB/s), single short ones by their chain of latencies (777
// rows: 11.9 us).  Sixteen softmax warps instead of eight were slower (64 single tokens 188 us against 147; 2048 tokens 1064
// against 964).
struct Start { Walk walk; long long total; };      // a CTA's piece, the line's length

template <int D>
__global__ void __launch_bounds__(PA_THREADS, 1)
paged_attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ AttnArgs a) {
  constexpr int TILE = tile_bytes<D>(), SLABS = D / 64;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sQ = base, sR = sQ + 2 * TILE, bars = sR + RING * TILE;
  const uint32_t q_full = bars, q_free = bars + 16;            // [2]
  const uint32_t s_full = bars + 32, o_full = bars + 48;       // [2] slots
  const uint32_t p_full = bars + 64;                           // [2 slots][2 halves]
  const uint32_t full = bars + 96, free_ = full + 8 * RING;    // [RING]
  // [RING] a tile of V with rows behind the last one was asked for; is cleared.  One for each place, since several short segments' tails may
  // be in the ring at a time
  const uint32_t v_tail = free_ + 8 * RING, v_clean = v_tail + 8 * RING;
  const uint32_t x_full = v_clean + 8 * RING, x_free = x_full + 8;   // slot 1's maximum and sum are there; its O has been read
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + (bars - base) + 384);
  volatile int* flags = reinterpret_cast<volatile int*>(tmem_slot + 1);        // [2]
  float2* ml = reinterpret_cast<float2*>(gen + (bars - base) + 512);
  const uint32_t g_done = x_free + 8;          // [2 slots] the slot's threads are at the same point
  volatile int* g_last = flags + 2;            // [2 slots] the slot's share was the last of its unit
  Start* start = reinterpret_cast<Start*>(gen + (bars - base) + 512 + 1024);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    flags[ABORT] = flags[BUSY] = 0;
    for (int s = 0; s < 2; ++s) {
      mbar_init(q_full + 8 * s, 1); mbar_init(q_free + 8 * s, 1);
      mbar_init(s_full + 8 * s, 1); mbar_init(o_full + 8 * s, 1);
      for (int h = 0; h < 2; ++h) mbar_init(p_full + 8 * (2 * s + h), 128);
    }
    for (int s = 0; s < RING; ++s) {
      mbar_init(full + 8 * s, 1); mbar_init(free_ + 8 * s, 1);
      mbar_init(v_tail + 8 * s, 1); mbar_init(v_clean + 8 * s, 32);
    }
    mbar_init(x_full, 128); mbar_init(x_free, 128); mbar_init(g_done, 128); mbar_init(g_done + 8, 128);
    fence_mbar_init();
    prefetch_tensormap(&tmQ); prefetch_tensormap(&tmK); prefetch_tensormap(&tmV);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32((const void*)tmem_slot), PA_COLS);
    tmem_relinquish();
  }
  // this CTA's piece of the line; the prefix sums lie where K and V will
  dep_wait();
  {
    Line line;
    line.make<PA_THREADS>(a, reinterpret_cast<long long*>(gen + (sR - base)), blockIdx.x == 0);
    if (warp == 0) {
      Walk w;
      w.at = line.cut(blockIdx.x, gridDim.x);
      w.left = line.cut(blockIdx.x + 1, gridDim.x) - w.at;
      if (w.left > 0) { w.p = line.find(a, w.at); w.sequence(a); }
      if (lane == 0) *start = {w, line.total};
    }
    fence_proxy_async_smem();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  Walk walk = start->walk;
  Segment s;

  // The order of the ring's tiles within a segment of nb blocks: with two tiles K_0, V_0, K_1, V_1, ...; with one (slots on neighbouring
  // blocks) K_0, K_1, V_0, K_2, V_1, ...: `ahead` tiles of K before the first of V, then V_i and K_{i + ahead} in turn, V last.
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_LIGHT));
    if (warp == 0) {
      const int shift = a.c.shift, page = 1 << shift, box = min(page, BLOCK);     // rows of a box
      const uint32_t q_bytes = (uint32_t)(a.G * a.tile_tokens * 128 * SLABS);
      uint32_t slot = 0, phase = 1, q_phase = 3, q_next = 0;     // (q_phase: a bit for each place)
      bool ok = true;
      while (ok && walk.next(a, s)) {
        const int nb = s.j1 - s.j0, ahead = s.two ? 1 : 2;
        // where this lane's box of block j lies; rows behind the last one and entries that name no page: a place behind the last page
        const int32_t* table = a.c.table + (int64_t)s.b * a.c.max_pages;
        const int nowhere = a.c.n_pages << shift;
        auto place = [&](int j) {
          const int row = j * BLOCK + lane * box;
          if (j >= s.j1 || lane * box >= BLOCK || row >= s.held) return -1;
          const int p = __ldg(table + (row >> shift));
          if (p < 0 || p >= a.c.n_pages) { set_status(a.status, SPTS_ERR_INDEX); return nowhere; }
          return (p << shift) + (row & (page - 1));
        };
        int y0 = place(s.j0), y1 = place(s.j0 + 1), y2 = place(s.j0 + 2);
        for (int t = 0; t < (s.two ? 2 : 1); ++t) {
          const int buf = s.two ? t : (int)q_next;
          ok = ok && wait_warp(q_free + 8 * buf, (q_phase >> buf) & 1, flags);
          q_phase ^= 1u << buf;
          if (ok && lane == 0) {
            mbar_expect_tx(q_full + 8 * buf, q_bytes);
            for (int h = 0; h < SLABS; ++h)
              tma_load_3d(sQ + buf * TILE + h * SLAB, &tmQ, q_full + 8 * buf, 64 * h, s.h * a.G, s.row + t * a.tile_tokens);
          }
        }
        if (!s.two) q_next ^= 1;
        auto load = [&](bool is_v, int j, int y) {
          ok = ok && wait_warp(free_ + 8 * slot, phase, flags);
          if (!ok) return;
          const int rows = max(0, min(BLOCK, s.held - j * BLOCK)), boxes = (rows + box - 1) / box;
          const uint32_t bar = full + 8 * slot;
          if (lane == 0) {
            if (boxes > 0) mbar_expect_tx(bar, (uint32_t)(boxes * box * 128 * SLABS));
            else mbar_arrive(bar);
            if (is_v && rows < BLOCK) mbar_arrive(v_tail + 8 * slot);
          }
          __syncwarp();
          if (y >= 0) tma_load_4d(sR + slot * TILE + lane * box * 128 * SLABS, is_v ? &tmV : &tmK, bar, 0, 0, s.h * SLABS, y >> 3);
          if (++slot == RING) { slot = 0; phase ^= 1; }
        };
        load(false, s.j0, y0);
        if (ahead == 2 && nb > 1) load(false, s.j0 + 1, y1);
        for (int j = s.j0; j < s.j1 && ok; ++j) {
          if (lane == 0) sign_of_life(flags + BUSY);
          load(true, j, y0);
          if (j + ahead < s.j1) load(false, j + ahead, ahead == 1 ? y1 : y2);
          y0 = y1; y1 = y2; y2 = place(j + 3);
        }
      }
    } else if (warp == 1) {
      {
        // The instructions around the products are what bounds long chunks.  The whole warp runs this role, on values that are the same for
        // all its lanes (and known to be: shuffles and votes), so that descriptors live in uniform registers; one lane issues.  Descriptors
        // advance by additions, phases are bits.
        const bool leader = elect_lane();
        constexpr uint32_t idesc_s = idesc_bf16(BLOCK, BLOCK), idesc_o = idesc_bf16(BLOCK, D) | B_ALONG_N;
        constexpr uint32_t q_hi = desc_high(1024), k_hi = desc_high(group_bytes<D>());
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem_base, 0);
        const uint32_t q_lo = desc_low(__shfl_sync(0xffffffffu, sQ, 0), 0), k_lo = desc_low(__shfl_sync(0xffffffffu, sR, 0), 0), v_lo = k_lo | (1024 >> 4 << 16);
        uint32_t slot = 0, phase = 0, clean = 0;         // the ring's place; phases of v_clean
        uint32_t bits = 0;                               // phases: 0, 1 of p_full; 2, 3 of q_full
        uint32_t turn = 0, q_next = 0;
        bool ok = true;
        const auto next_slot = [&]() {
          if (++slot == RING) { slot = 0; phase ^= 1; }
        };
        // the ring's next tile has come (a tail of V: has been cleared)
        const auto wait_tile = [&]() { ok = ok && wait_warp(full + 8 * slot, phase, flags); };
        const auto wait_v = [&](bool tail) {
          if (tail) {
            ok = ok && wait_warp(v_clean + 8 * slot, (clean >> slot) & 1, flags);
            clean ^= 1u << slot;
          } else {
            wait_tile();
          }
        };
        const auto commit = [&](uint32_t bar) {
          if (leader) mma_commit(bar);
        };
        const auto qk = [&](int t, uint32_t q, uint32_t k) {
          if (!leader) return;
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
            mma_ss(tm + t * BLOCK, q + (((i >> 2) * SLAB + (i & 3) * 32) >> 4), q_hi, k + (((i >> 2) * 1024 + (i & 3) * 32) >> 4), k_hi, idesc_s, i > 0);
          mma_commit(s_full + 8 * t);
        };
        // O_t += P_t V, P_t read from the columns of S_t, in the halves in which the softmax warps hand it over
        const auto pv = [&](int t, uint32_t v, bool first) {
          const uint32_t ph = (bits >> t) & 1;
          bits ^= 1u << t;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            ok = ok && wait_warp(p_full + 8 * (2 * t + half), ph, flags);
            if (!ok) return;
            tc_fence_after();
            if (leader) {
#pragma unroll
              for (int i = 4 * half; i < 4 * half + 4; ++i)
                mma_ts(tm + 2 * BLOCK + t * BLOCK, tm + t * BLOCK + 8 * i, v + i * (2 * group_bytes<D>() >> 4), k_hi, idesc_o, !first || i > 0);
            }
          }
        };
        while (ok && __any_sync(0xffffffffu, walk.next(a, s))) {
          const int nb = __shfl_sync(0xffffffffu, s.j1 - s.j0, 0);
          const bool tail = __any_sync(0xffffffffu, s.j1 * BLOCK > s.held);
          if (__any_sync(0xffffffffu, s.two)) {
            ok = ok && wait_warp(q_full, (bits >> 2) & 1, flags) && wait_warp(q_full + 8, (bits >> 3) & 1, flags);
            bits ^= 12;
            wait_tile();
            if (!ok) break;
            tc_fence_after();
            const uint32_t k0 = k_lo + slot * (TILE >> 4);
            qk(0, q_lo, k0);
            qk(1, q_lo + (TILE >> 4), k0);
            commit(free_ + 8 * slot);
            next_slot();
            for (int i = 0; i + 1 < nb; ++i) {
              wait_v(false);
              const uint32_t v = v_lo + slot * (TILE >> 4), v_free = free_ + 8 * slot;
              next_slot();
              wait_tile();
              const uint32_t k = k_lo + slot * (TILE >> 4), k_free = free_ + 8 * slot;
              next_slot();
              if (!ok) break;
              pv(0, v, i == 0);
              if (!ok) break;
              qk(0, q_lo, k);                    // (its commit also covers P_t V: O_t rests when S_t arrives)
              pv(1, v, i == 0);
              if (!ok) break;
              qk(1, q_lo + (TILE >> 4), k);
              commit(v_free);
              commit(k_free);
            }
            if (!ok) break;
            commit(q_free);
            commit(q_free + 8);
            wait_v(tail);
            const uint32_t v = v_lo + slot * (TILE >> 4);
            if (!ok) break;
            pv(0, v, nb == 1);
            commit(o_full);
            if (!ok) break;
            pv(1, v, nb == 1);
            commit(o_full + 8);
            commit(free_ + 8 * slot);
            next_slot();
          } else {
            const uint32_t q = q_lo + q_next * (TILE >> 4), qf = q_free + 8 * q_next;
            ok = ok && wait_warp(q_full + 8 * q_next, (bits >> (2 + q_next)) & 1, flags);
            bits ^= 4u << q_next;
            q_next ^= 1;
            for (int i = 0; i < 2 && i < nb; ++i) {
              wait_tile();
              if (!ok) break;
              tc_fence_after();
              qk((i + turn) & 1, q, k_lo + slot * (TILE >> 4));
              commit(free_ + 8 * slot);
              next_slot();
            }
            if (!ok) break;
            if (nb <= 2) commit(qf);
            for (int i = 0; i < nb; ++i) {
              const int t = (i + turn) & 1;
              wait_v(tail && i + 1 == nb);
              if (!ok) break;
              pv(t, v_lo + slot * (TILE >> 4), i < 2);
              if (!ok) break;
              commit(free_ + 8 * slot);
              next_slot();
              if (i + 2 < nb) {
                wait_tile();
                if (!ok) break;
                tc_fence_after();
                qk(t, q, k_lo + slot * (TILE >> 4));
                commit(free_ + 8 * slot);
                next_slot();
                if (i + 3 == nb) commit(qf);
              } else {
                commit(o_full + 8 * t);
              }
            }
            turn = (turn + nb) & 1;
          }
        }
      }
    } else if (warp == 2) {
      uint32_t at = 0, tails = 0;                // tiles of the ring up to this segment's end; a phase for each place
      bool ok = true;
      while (ok && walk.next(a, s)) {
        at += 2 * (s.j1 - s.j0);
        if (s.j1 * BLOCK <= s.held) continue;
        // the tile was asked for: the one that was in its place before has been used, and it will stay until it is clear
        const uint32_t slot = (at - 1) % RING;
        ok = wait_warp(v_tail + 8 * slot, (tails >> slot) & 1, flags) && wait_warp(full + 8 * slot, ((at - 1) / RING) & 1, flags);
        tails ^= 1u << slot;
        if (!ok) break;
        const int rows = max(0, s.held - (s.j1 - 1) * BLOCK);
        for (int h = 0; h < SLABS; ++h)
          for (int i = rows * 8 + lane; i < BLOCK * 8; i += 32)      // 16 bytes of row i / 8
            *reinterpret_cast<uint4*>(gen + (sR - base) + slot * TILE + (i >> 6) * group_bytes<D>() + h * 1024 + (i & 63) * 16) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
        mbar_arrive(v_clean + 8 * slot);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
    const int t = (warp - 4) >> 2;                     // slot
    const int quarter = warp & 3;                      // TMEM lanes this warp may access
    const int row = quarter * 32 + lane;
    const int row_token = row / a.G, row_head = row % a.G;
    const uint32_t lane_off = (uint32_t)(quarter * 32) << 16;
    const uint32_t tS = tmem_base + t * BLOCK + lane_off, tO = tmem_base + 2 * BLOCK + t * BLOCK + lane_off;
    const float sc = LOG2E / (D == 128 ? 11.313708498984761f : 8.0f);
    const float2 sc2 = make_float2(sc, sc);
    uint32_t n_s = 0, n_o = 0, n_x = 0, n_g = 0, turn = 0;
    bool open = false;                                 // the last segment's unit begins here and goes on in other CTAs
    bool ok = true;
    while (ok && walk.next(a, s)) {
      open = s.j0 == 0 && s.j1 < s.cost;
      const int nb = s.j1 - s.j0, tile = s.two ? t : 0;
      const int tokens = min(a.tile_tokens, s.tokens - tile * a.tile_tokens);
      const int token = s.token + tile * a.tile_tokens + row_token;        // in the sequence
      const bool live = row_token < tokens;
      const bool any_live = quarter * 32 < tokens * a.G;                   // of this warp
      // rows that this query sees (a row of no query is not masked: nothing of it is used, and its warp need not look)
      const int limit = live ? max(0, s.off + token + 1) : INT_MAX;
      float m_used = -INFINITY, l = 0.f;
      int done = 0;
      for (int i = s.two ? 0 : ((t + turn) & 1); i < nb && ok; i += s.two ? 1 : 2) {
        ok = wait_warp(s_full + 8 * t, n_s & 1, flags);
        ++n_s;
        if (!ok) break;
        if (!any_live) {                                                   // rows of no query: whatever P holds stays in them
          mbar_arrive(p_full + 16 * t);
          mbar_arrive(p_full + 16 * t + 8);
          continue;
        }
        tc_fence_after();
        const int key0 = (s.j0 + i) * BLOCK;
        uint32_t r[BLOCK];
#pragma unroll
        for (int c = 0; c < BLOCK; c += 32) tmem_ld32(tS + c, r + c);
        tmem_ld_wait();
        if (__any_sync(0xffffffffu, limit < key0 + BLOCK)) {
#pragma unroll
          for (int e = 0; e < BLOCK; ++e)
            if (key0 + e >= limit) r[e] = 0xFF800000u;                     // -inf
        }
        float bm[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < BLOCK; e += 8) {
#pragma unroll
          for (int u = 0; u < 4; ++u) bm[u] = max3(bm[u], __uint_as_float(r[e + 2 * u]), __uint_as_float(r[e + 2 * u + 1]));
        }
        const float bmax = fmaxf(fmaxf(bm[0], bm[1]), fmaxf(bm[2], bm[3])) * sc;
        float alpha = 1.0f;                            // for O and l where the running maximum is replaced
        if (bmax > m_used + RESCALE || m_used == -INFINITY) {
          alpha = m_used == -INFINITY ? 0.0f : ex2(m_used - bmax);
          m_used = bmax;
        }
        // S_t complete means that the last P_t V has completed, too, and the next cannot start before this thread's P arrives
        if (done > 0 && __any_sync(0xffffffffu, alpha != 1.0f)) {
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            tmem_ld32(tO + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st32(tO + c, o);
          }
        }
        const float shift = m_used == -INFINITY ? 0.f : -m_used;
        const float2 nm2 = make_float2(shift, shift);
        float2 ps[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) ps[u] = make_float2(0.f, 0.f);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t pk[32];
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            const int e0 = 64 * half + e;
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(r[e0]), __uint_as_float(r[e0 + 1])), sc2, nm2);
            const float2 p = make_float2(ex2(x.x), ex2(x.y));
            ps[(e >> 1) & 3] = __fadd2_rn(ps[(e >> 1) & 3], p);
            // rounded to bf16 once, since the product takes both operands in V's type; the sum takes it unrounded.  That adds as much to
            // the error as the result's own rounding (0.0017 -> 0.0022 to 0.0024 of the RMS); a second product for what the rounding
            // leaves would double P V.
            pk[e >> 1] = pack2(p.x, p.y);
          }
#pragma unroll
          for (int c = 0; c < 32; c += 16) tmem_st16(tS + 32 * half + c, pk + c);
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(p_full + 8 * (2 * t + half));
        }
        const float2 ps0 = __fadd2_rn(ps[0], ps[1]), ps1 = __fadd2_rn(ps[2], ps[3]);
        l = l * alpha + ((ps0.x + ps0.y) + (ps1.x + ps1.y));
        ++done;
      }
      if (!ok) break;
      // ---- the end of a segment
      const bool merge = !s.two && nb > 1, mine = s.two || (merge ? t == 0 : (int)(turn & 1) == t);
      if (!s.two) turn = (turn + nb) & 1;
      if (mine || merge) {
        ok = wait_warp(o_full + 8 * t, n_o & 1, flags);
        ++n_o;
        if (!ok) break;
        tc_fence_after();
      }
      float f0 = 1.f, f1 = 0.f;                        // factors of this slot's and of slot 1's O
      if (merge && t == 1) {
        ml[row] = make_float2(m_used, l);
        tc_fence_before();
        mbar_arrive(x_full);
        ok = wait_warp(x_free, n_x & 1, flags);
        ++n_x;
        continue;
      }
      if (!mine) continue;
      if (merge) {
        ok = wait_warp(x_full, n_x & 1, flags);
        ++n_x;
        if (!ok) break;
        tc_fence_after();
        const float2 other = ml[row];
        const float m = fmaxf(m_used, other.x), b = m == -INFINITY ? 0.f : m;
        f0 = ex2(m_used - b);
        f1 = ex2(other.x - b);
        l = l * f0 + other.y * f1;
        m_used = m;
      }
      const bool direct = s.j0 == 0 && s.j1 == s.cost;
      const int64_t out_row = (int64_t)s.row + tile * a.tile_tokens + row_token;
      const int head = s.h * a.G + row_head;
      bf16* orow = a.O + out_row * a.ldo + (int64_t)head * D;
      float* share = a.share + ((int64_t)(2 * blockIdx.x + (s.j0 == 0 ? 1 : 0)) * 2 + tile) * share_floats<D>();
      const float inv = direct ? (l == 0.f ? 0.f : 1.0f / l) : 1.0f;
      float odd = 0.f;                                 // becomes NaN with a value that is not finite
      if (any_live) {
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          tmem_ld32(tO + c, o);
          tmem_ld_wait();
          if (merge) {
            uint32_t o1[32];
            tmem_ld32(tO + BLOCK + c, o1);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float x0 = f0 == 0.f ? 0.f : __uint_as_float(o[e]) * f0, x1 = f1 == 0.f ? 0.f : __uint_as_float(o1[e]) * f1;
              o[e] = __float_as_uint(x0 + x1);
            }
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float x = l == 0.f ? 0.f : __uint_as_float(o[e]) * inv;
            odd = fmaf(x, 0.f, odd);
            o[e] = __float_as_uint(x);
          }
          if (live && direct) {
            uint4 w[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              w[g].x = pack2(__uint_as_float(o[g * 8 + 0]), __uint_as_float(o[g * 8 + 1]));
              w[g].y = pack2(__uint_as_float(o[g * 8 + 2]), __uint_as_float(o[g * 8 + 3]));
              w[g].z = pack2(__uint_as_float(o[g * 8 + 4]), __uint_as_float(o[g * 8 + 5]));
              w[g].w = pack2(__uint_as_float(o[g * 8 + 6]), __uint_as_float(o[g * 8 + 7]));
            }
            if (a.wide) {
              store32(orow + c, w[0], w[1]);
              store32(orow + c + 16, w[2], w[3]);
            } else {
#pragma unroll
              for (int g = 0; g < 4; ++g) *reinterpret_cast<uint4*>(orow + c + g * 8) = w[g];
            }
          } else if (live) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
              store32(share + share_at(row, c + g * 8), make_uint4(o[g * 8], o[g * 8 + 1], o[g * 8 + 2], o[g * 8 + 3]),
                      make_uint4(o[g * 8 + 4], o[g * 8 + 5], o[g * 8 + 6], o[g * 8 + 7]));
          }
        }
        if (live && direct && a.lse != nullptr) a.lse[out_row * a.H + head] = l == 0.f ? -INFINITY : (m_used + log2f(l)) * LN2;
        if (live && !direct) *reinterpret_cast<float2*>(share + BLOCK * D + 2 * row) = make_float2(m_used, l);
      }
      if (merge) {
        tc_fence_before();
        mbar_arrive(x_free);
      }
      uint32_t again = __ballot_sync(0xffffffffu, live && odd != odd && l == l && limit < s.j1 * BLOCK);
      while (again) {
        const int who = __ffs(again) - 1;
        again &= again - 1;
        const int w_token = __shfl_sync(0xffffffffu, row_token, who), w_head = __shfl_sync(0xffffffffu, head, who), w_row = quarter * 32 + who;
        const int w_limit = __shfl_sync(0xffffffffu, limit, who);
        const int64_t w_out = (int64_t)s.row + tile * a.tile_tokens + w_token;
        float m, sum, o[D / 32];
        plain_row<D>(a, s.b, s.h, a.Q + w_out * a.ldq + (int64_t)w_head * D, s.j0 * BLOCK, min(s.j1 * BLOCK, w_limit), flags + BUSY, m, sum, o);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
          const int col = lane * (D / 32) + e;
          if (direct) a.O[w_out * a.ldo + (int64_t)w_head * D + col] = __float2bfloat16_rn(sum == 0.f ? 0.f : o[e] / sum);
          else share[share_at(w_row, col)] = o[e];
        }
        if (lane == 0) {
          if (direct && a.lse != nullptr) a.lse[w_out * a.H + w_head] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * LN2;
          if (!direct) *reinterpret_cast<float2*>(share + BLOCK * D + 2 * w_row) = make_float2(m, sum);
        }
        __syncwarp();
      }
      if (!direct && a.solo) {
        // the CTA that leaves the unit's last share joins it, a warp to a row
        const long long total = start->total;
        const int ctas = gridDim.x, first = cta_of(total, s.begin, ctas), last = cta_of(total, s.begin + s.cost - 1, ctas);
        mbar_arrive(g_done + 8 * t);
        ok = wait_warp(g_done + 8 * t, n_g & 1, flags);
        ++n_g;
        if (!ok) break;
        if (row == 0) {
          const bool is_last = count_arrival(a.arrived + 8 * first) == last - first;
          if (is_last) a.arrived[8 * first] = 0;
          g_last[t] = is_last;
        }
        mbar_arrive(g_done + 8 * t);
        ok = wait_warp(g_done + 8 * t, n_g & 1, flags);
        ++n_g;
        if (!ok) break;
        if (g_last[t]) {
          for (int r = quarter; r < s.tokens * a.G; r += 4) join_row<D>(a, s.row, s.h, first, last, 0, r);
        }
      }
    }
    if (threadIdx.x == 128 && !a.solo)
      a.open[blockIdx.x] = {open && ok ? cta_of(start->total, s.begin + s.cost - 1, gridDim.x) : -1, s.row, s.h, s.tokens};
  }

  tc_fence_before();
  __syncthreads();
  if (flags[ABORT]) {
    if (threadIdx.x == 0) set_status(a.status, SPTS_ERR_TIMEOUT);
    const uint64_t t1 = globaltimer_ns();
    while (globaltimer_ns() - t1 < 200000ull) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, PA_COLS);
  }
}

// Joins the shares of units that several CTAs worked on: blockIdx.x = the CTA in which such a unit begins (its last one), blockIdx.y = which of
// its rows; a warp per row, the shares in the order of the line.
constexpr int JOIN_THREADS = 256, JOIN_SPLIT = 16;     // a unit's 256 rows: two to a warp
template <int D>
__global__ void __launch_bounds__(JOIN_THREADS)
paged_attn_join_kernel(const __grid_constant__ AttnArgs a) {
  dep_wait();
  const int4 raw = __ldcg(reinterpret_cast<const int4*>(a.open + blockIdx.x));
  const OpenUnit u = {raw.x, raw.y, raw.z, raw.w};
  if (u.last < 0) return;
  const int rows0 = min(a.tile_tokens, u.tokens) * a.G, rows = u.tokens * a.G, warp = threadIdx.x >> 5;
  for (int r = blockIdx.y * (JOIN_THREADS / 32) + warp; r < rows; r += JOIN_SPLIT * (JOIN_THREADS / 32))
    join_row<D>(a, u.row, u.h, blockIdx.x, u.last, r >= rows0 ? 1 : 0, r >= rows0 ? r - rows0 : r);
}

// ------------------------------------------------------------------------------------------------ gathered weights
// The weight that rows of the cache get needs every query's sum of exponentials first, so it is a second pass over K: S^T = K Q^T with the
// cache's rows along the 128 lanes of the accumulator, so that a thread owns a row and adds up its exponentials over the columns (queries) without
// meeting another one.  A unit is two blocks of 128 rows of a sequence, its cost the number of (KV head, tile of queries) that see any of
// them; all units end to end are cut into equal pieces as in the attention.  The warps of a unit that several CTAs work on leave their sums
// in the workspace; of each 32 rows the warp that comes last adds them up in the order of the line.
//   warp 0      TMA producer: for every KV head the two blocks of K (two pairs in flight), for every tile of queries its Q (two)
//   warp 1      TMEM owner and MMA issuer: two accumulators for each of the two blocks
//   warps 2-3   -lse log2(e) of a tile's queries into shared memory
//   warps 4-11  the exponentials of every second item, warps 12-19 of the others; of the first block warps 4-7 and 12-15
// Bound by memory where queries are few (16 single tokens over up to 8192 rows: 26.3 us, 4.2 TB/s with the launch and the line's ends), by the
// exponential unit where they are many: 512 tokens over 32768 rows take 193 us (290 with two warps on each of its quarters instead of four),
// 64 tokens 33 us (37; with all 128 columns of a row in registers at once 46).
constexpr int PW_THREADS = 640;
constexpr int PW_Q = 2, PW_E = 4;              // tiles of queries in flight, of their lse
template <int D> constexpr int pw_smem() { return 1024 + (4 + PW_Q) * tile_bytes<D>() + 256 + (PW_E + 2) * BLOCK * 4 + 64; }

static_assert(pw_smem<128>() <= 232448 && pa_smem<128>() <= 232448, "shared memory of a block");

struct WeightArgs {
  Cache c;
  const int32_t* row_start; int n_rows;
  int H, Hkv, G, tile_tokens;
  const float* lse;
  float decay;
  float* share; int* arrived;                  // [2 * CTAs, 256] sums; [CTAs, 8] warps that left theirs, zero between calls
  int* status;
};

// Items of the first u units of a sequence: for each KV head, the tiles of queries that see any of its rows; one for each unit where there are
// no queries (its weights fade).
__device__ long long items_before(int n, int off, int tt, int Hkv, int u) {
  if (n == 0) return u;
  const int tiles = (n + tt - 1) / tt, u0 = off > 0 ? min(u, (off + 2 * BLOCK - 1) / (2 * BLOCK)) : 0;
  long long sum = (long long)u * tiles;
  if (u > u0) sum -= (long long)floor_sum(u - u0, tt, 2 * BLOCK, 2 * BLOCK * u0 - off);
  return sum * Hkv;
}
__device__ __forceinline__ int first_tile(int off, int tt, int u) { return max(0, 2 * BLOCK * u - off) / tt; }

struct Unit {
  int b, u, i0, i1, cost;                      // items [i0, i1) of `cost`
  int held, n, off, row;                       // the sequence's rows, its queries, rows before the first query, first query in Q
  int tile0, tiles;                            // tiles of queries that see the unit's rows, for each head (0: no queries)
  bool two;                                    // it has a second block
};

struct UnitWalk {
  int b, u, i, row, n, off, held;
  long long left, at, total;                   // left of the piece; where it begins, and the line's length
  __device__ __forceinline__ void sequence(const WeightArgs& a) {
    call_rows(a.row_start, a.n_rows, b, row, n);
    held = held_rows(a.c, b);
    off = held - n;
  }
  __device__ __forceinline__ bool next(const WeightArgs& a, Unit& s) {
    if (left <= 0) return false;
    s.b = b; s.u = u; s.held = held; s.n = n; s.off = off; s.row = row;
    s.tile0 = n == 0 ? 0 : first_tile(off, a.tile_tokens, u);
    s.tiles = n == 0 ? 0 : (n + a.tile_tokens - 1) / a.tile_tokens - s.tile0;
    s.cost = n == 0 ? 1 : s.tiles * a.Hkv;
    s.i0 = i;
    s.i1 = (int)min((long long)s.cost, i + left);
    s.two = held - 2 * BLOCK * u > BLOCK;
    left -= s.i1 - s.i0;
    i = 0;
    if (2 * BLOCK * (u + 1) < held) { ++u; return true; }
    u = 0;
    while (left > 0 && ++b < a.c.n_seq) {
      sequence(a);
      if (held > 0) break;
    }
    return true;
  }
};

template <int D>
__global__ void __launch_bounds__(PW_THREADS, 1)
paged_weights_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ WeightArgs a) {
  constexpr int TILE = tile_bytes<D>(), SLABS = D / 64;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t sK = base, sQ = sK + 4 * TILE, bars = sQ + PW_Q * TILE;
  const uint32_t k_full = bars, k_free = bars + 16;            // [2] pairs of blocks
  const uint32_t q_full = bars + 32, q_free = q_full + 8 * PW_Q;
  const uint32_t e_full = q_free + 8 * PW_Q, e_free = e_full + 8 * PW_E;      // lse of a tile
  const uint32_t s_full = e_free + 8 * PW_E, s_free = s_full + 32;            // [2 blocks][2 accumulators]
  const uint32_t x_full = s_free + 32, x_free = x_full + 16;                  // [2 blocks] the second warps' sums are there; have been taken
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + (bars - base) + 240);
  volatile int* flags = reinterpret_cast<volatile int*>(tmem_slot + 1);        // [2]
  float* s_lse = reinterpret_cast<float*>(gen + (bars - base) + 256);
  float* s_sum = s_lse + PW_E * BLOCK;         // [2 blocks][128]
  UnitWalk* start = reinterpret_cast<UnitWalk*>(gen + (bars - base) + 256 + (PW_E + 2) * BLOCK * 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    flags[ABORT] = flags[BUSY] = 0;
    for (int s = 0; s < 2; ++s) { mbar_init(k_full + 8 * s, 1); mbar_init(k_free + 8 * s, 1); }
    for (int s = 0; s < PW_Q; ++s) {
      mbar_init(q_full + 8 * s, 1); mbar_init(q_free + 8 * s, 1);
    }
    for (int s = 0; s < PW_E; ++s) { mbar_init(e_full + 8 * s, 64); mbar_init(e_free + 8 * s, 256); }
    for (int s = 0; s < 4; ++s) { mbar_init(s_full + 8 * s, 1); mbar_init(s_free + 8 * s, 128); }
    for (int s = 0; s < 2; ++s) { mbar_init(x_full + 8 * s, 128); mbar_init(x_free + 8 * s, 128); }
    fence_mbar_init();
    prefetch_tensormap(&tmQ); prefetch_tensormap(&tmK);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32((const void*)tmem_slot), PA_COLS);
    tmem_relinquish();
  }
  dep_wait();
  {
    long long* scratch = reinterpret_cast<long long*>(gen);
    long long* pre = scratch + 32;
    const long long total = block_prefix<PW_THREADS>(a.c.n_seq, pre, scratch, [&](int b) {
      int row, n;
      call_rows(a.row_start, a.n_rows, b, row, n);
      if (blockIdx.x == 0) check_starts(a.row_start, a.n_rows, b, a.status);
      const int held = held_rows(a.c, b);
      return held == 0 ? 0LL : items_before(n, held - n, a.tile_tokens, a.Hkv, (held + 2 * BLOCK - 1) / (2 * BLOCK));
    });
    if (warp == 0) {
      const long long from = cut_line(total, blockIdx.x, gridDim.x);
      UnitWalk w;
      w.at = from;
      w.total = total;
      w.left = cut_line(total, blockIdx.x + 1, gridDim.x) - from;
      if (w.left > 0) {
        w.b = find_share(pre, a.c.n_seq, from);
        w.sequence(a);
        const long long x = from - pre[w.b];
        const auto before = [&](int u) { return items_before(w.n, w.off, a.tile_tokens, a.Hkv, u); };
        w.u = warp_find((w.held + 2 * BLOCK - 1) / (2 * BLOCK), x, before);
        w.i = (int)(x - before(w.u));
      }
      if (lane == 0) *start = w;
    }
    fence_proxy_async_smem();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  UnitWalk walk = *start;
  Unit s;
  bool ok = true;

  if (warp == 0) {
    const int shift = a.c.shift, page = 1 << shift, box = min(page, BLOCK);
    const uint32_t q_bytes = (uint32_t)(a.G * a.tile_tokens * 128 * SLABS);
    uint32_t n_k = 0, n_q = 0;
    while (ok && walk.next(a, s)) {
      const int32_t* table = a.c.table + (int64_t)s.b * a.c.max_pages;
      // this lane's boxes of the two blocks
      int y[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int row = (2 * s.u + t) * BLOCK + lane * box;
        y[t] = -1;
        if (lane * box < BLOCK && row < s.held) {
          const int p = __ldg(table + (row >> shift));
          if (p < 0 || p >= a.c.n_pages) { set_status(a.status, SPTS_ERR_INDEX); y[t] = a.c.n_pages << shift; }
          else y[t] = (p << shift) + (row & (page - 1));
        }
      }
      if (s.tiles == 0) continue;
      const int rows = min(2 * BLOCK, s.held - 2 * BLOCK * s.u), boxes = (rows + box - 1) / box;
      for (int i = s.i0; i < s.i1 && ok; ++i) {
        const int h = i / s.tiles, q = s.tile0 + i % s.tiles;
        if (i == s.i0 || q == s.tile0) {
          const uint32_t st = n_k & 1, bar = k_full + 8 * st;
          ok = wait_warp(k_free + 8 * st, ((n_k >> 1) & 1) ^ 1, flags);
          ++n_k;
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(bar, (uint32_t)(boxes * box * 128 * SLABS));
          __syncwarp();
#pragma unroll
          for (int t = 0; t < 2; ++t)
            if (y[t] >= 0) tma_load_4d(sK + (2 * st + t) * TILE + lane * box * 128 * SLABS, &tmK, bar, 0, 0, h * SLABS, y[t] >> 3);
        }
        const uint32_t st = n_q % PW_Q;
        ok = wait_warp(q_free + 8 * st, ((n_q / PW_Q) & 1) ^ 1, flags);
        ++n_q;
        if (ok && lane == 0) {
          mbar_expect_tx(q_full + 8 * st, q_bytes);
          for (int l = 0; l < SLABS; ++l)
            tma_load_3d(sQ + st * TILE + l * SLAB, &tmQ, q_full + 8 * st, 64 * l, h * a.G, s.row + q * a.tile_tokens);
        }
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    // (as in the attention: the whole warp, on uniform values, one lane issues)
    const bool leader = elect_lane();
    constexpr uint32_t k_hi = desc_high(group_bytes<D>()), q_hi = desc_high(1024);
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem_base, 0);
    const uint32_t k_lo = desc_low(__shfl_sync(0xffffffffu, sK, 0), 0), q_lo = desc_low(__shfl_sync(0xffffffffu, sQ, 0), 0);
    uint32_t n_k = 0, n_q = 0, used = 0;       // (used: a phase for each accumulator)
    while (ok && __any_sync(0xffffffffu, walk.next(a, s))) {
      const int tiles = __shfl_sync(0xffffffffu, s.tiles, 0), i0 = __shfl_sync(0xffffffffu, s.i0, 0), i1 = __shfl_sync(0xffffffffu, s.i1, 0);
      const int left = __shfl_sync(0xffffffffu, s.n - s.tile0 * a.tile_tokens, 0);      // queries from the first tile on
      const bool two = __any_sync(0xffffffffu, s.two);
      if (tiles == 0) continue;
      int q = i0 % tiles;                      // tile of queries, counted from the first
      for (int i = i0; i < i1 && ok; ++i) {
        if (i == i0 || q == 0) { ok = wait_warp(k_full + 8 * (n_k & 1), (n_k >> 1) & 1, flags); ++n_k; }
        const uint32_t kst = (n_k - 1) & 1, qst = n_q % PW_Q, buf = n_q & 1;      // items alternate between the accumulators
        ok = ok && wait_warp(q_full + 8 * qst, (n_q / PW_Q) & 1, flags);
        ++n_q;
        const int cols = (min(a.tile_tokens, left - q * a.tile_tokens) * a.G + 15) & ~15;
        const uint32_t idesc = idesc_bf16(BLOCK, 0) | ((uint32_t)(cols >> 3) << 17), qd = q_lo + qst * (TILE >> 4);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (!ok || (t == 1 && !two)) break;
          ok = wait_warp(s_free + 8 * (2 * t + buf), ((used >> (2 * t + buf)) & 1) ^ 1, flags);
          used ^= 1u << (2 * t + buf);
          if (!ok) break;
          tc_fence_after();
          const uint32_t k = k_lo + (2 * kst + t) * (TILE >> 4);
          if (leader) {
#pragma unroll
            for (int e = 0; e < D / 16; ++e)
              mma_ss(tm + (2 * t + buf) * BLOCK, k + (((e >> 2) * 1024 + (e & 3) * 32) >> 4), k_hi, qd + (((e >> 2) * SLAB + (e & 3) * 32) >> 4), q_hi, idesc,
                     e > 0);
            mma_commit(s_full + 8 * (2 * t + buf));
          }
        }
        if (!ok) break;
        if (leader) mma_commit(q_free + 8 * qst);
        if (++q == tiles) q = 0;
        if (leader && (i + 1 == i1 || q == 0)) mma_commit(k_free + 8 * kst);
      }
    }
  } else if (warp < 4) {
    uint32_t n_q = 0;
    while (ok && walk.next(a, s)) {
      if (s.tiles == 0) continue;
      for (int i = s.i0; i < s.i1 && ok; ++i) {
        const int h = i / s.tiles, q = s.tile0 + i % s.tiles, tokens = min(a.tile_tokens, s.n - q * a.tile_tokens);
        const uint32_t st = n_q % PW_E;
        const int64_t row = (int64_t)s.row + q * a.tile_tokens;
        float e[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int c = (warp - 2) * 32 + lane + 64 * u;
          e[u] = c < tokens * a.G ? -__ldg(a.lse + (row + c / a.G) * a.H + h * a.G + c % a.G) * LOG2E : 0.f;
          if (e[u] == INFINITY) e[u] = 0.f;    // a query that sees nothing: all its scores become -inf, and stay
        }
        ok = wait_warp(e_free + 8 * st, ((n_q / PW_E) & 1) ^ 1, flags);
        ++n_q;
        if (!ok) break;
#pragma unroll
        for (int u = 0; u < 2; ++u) s_lse[st * BLOCK + (warp - 2) * 32 + lane + 64 * u] = e[u];
        mbar_arrive(e_full + 8 * st);
      }
    }
  } else {
    const int t = ((warp - 4) >> 2) & 1, group = warp >= 12 ? 1 : 0, quarter = warp & 3;
    const uint32_t src = tmem_base + (2 * t + group) * BLOCK + ((uint32_t)(quarter * 32) << 16);
    const float sc = LOG2E / (D == 128 ? 11.313708498984761f : 8.0f);
    const float2 sc2 = make_float2(sc, sc);
    uint32_t n_q = 0, n_s = 0, n_x = 0;
    long long at = walk.at;                    // the line's item at which the segment begins
    const long long total = walk.total;
    while (ok && walk.next(a, s)) {
      const int key = (2 * s.u + t) * BLOCK + quarter * 32 + lane;
      const bool work = t == 0 || s.two;
      float2 sum[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) sum[u] = make_float2(0.f, 0.f);
      for (int i = s.i0; i < s.i1 && s.tiles > 0 && ok; ++i, ++n_q) {
        if ((int)(n_q & 1) != group) continue;
        const int q = s.tile0 + i % s.tiles, tokens = min(a.tile_tokens, s.n - q * a.tile_tokens), cols = tokens * a.G;
        const uint32_t st = n_q % PW_E;
        ok = wait_warp(e_full + 8 * st, (n_q / PW_E) & 1, flags);
        if (!ok) break;
        if (work) {
          ok = wait_warp(s_full + 8 * (2 * t + group), n_s & 1, flags);
          ++n_s;
          if (!ok) break;
          tc_fence_after();
          // column c is query q tile_tokens + c / G, which sees key if key <= off + query
          const int from_col = min(max(0, key - s.off - q * a.tile_tokens), BLOCK) * a.G;
          const bool all = !__any_sync(0xffffffffu, from_col > 0);
          const float4* lse4 = reinterpret_cast<const float4*>(s_lse + st * BLOCK);
#pragma unroll 1
          for (int c0 = 0; c0 < cols; c0 += 32) {
            uint32_t r[32];
            tmem_ld32(src + c0, r);
            tmem_ld_wait();
            if (!all || c0 + 32 > cols) {
#pragma unroll
              for (int c = 0; c < 32; ++c)
                if (c0 + c < from_col || c0 + c >= cols) r[c] = 0xFF800000u;      // -inf
            }
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              const float4 e = lse4[(c0 + c) >> 2];
              const float2 x = __ffma2_rn(make_float2(__uint_as_float(r[c]), __uint_as_float(r[c + 1])), sc2, make_float2(e.x, e.y));
              const float2 y = __ffma2_rn(make_float2(__uint_as_float(r[c + 2]), __uint_as_float(r[c + 3])), sc2, make_float2(e.z, e.w));
              sum[(c >> 1) & 3] = __fadd2_rn(sum[(c >> 1) & 3], make_float2(ex2(x.x), ex2(x.y)));
              sum[((c >> 1) + 1) & 3] = __fadd2_rn(sum[((c >> 1) + 1) & 3], make_float2(ex2(y.x), ex2(y.y)));
            }
          }
          tc_fence_before();
          mbar_arrive(s_free + 8 * (2 * t + group));
        }
        mbar_arrive(e_free + 8 * st);
      }
      if (!ok) break;
      const float2 s01 = __fadd2_rn(sum[0], sum[1]), s23 = __fadd2_rn(sum[2], sum[3]);
      float w = (s01.x + s01.y) + (s23.x + s23.y);
      const long long begin = at - s.i0, end = begin + s.cost;
      at += s.i1 - s.i0;
      // the second group hands its sums to the first
      float* mine = s_sum + t * BLOCK + quarter * 32 + lane;
      if (group == 1) {
        ok = wait_warp(x_free + 8 * t, (n_x & 1) ^ 1, flags);
        ++n_x;
        if (!ok) break;
        *mine = w;
        mbar_arrive(x_full + 8 * t);
        continue;
      }
      ok = wait_warp(x_full + 8 * t, n_x & 1, flags);
      ++n_x;
      if (!ok) break;
      w += *mine;
      mbar_arrive(x_free + 8 * t);
      bool write = true;
      if (s.i0 > 0 || s.i1 < s.cost) {
        // CTAs whose pieces reach into the unit: the first one's share is its last, the others' their first
        const int cta = blockIdx.x, ctas = gridDim.x;
        const int first = cta_of(total, begin, ctas), last = cta_of(total, end - 1, ctas);
        float* share = a.share + (size_t)(2 * cta + (s.i0 == 0 ? 1 : 0)) * 2 * BLOCK;
        __stcg(share + t * BLOCK + quarter * 32 + lane, w);
        __syncwarp();
        int seen = 0;
        int* arrived = a.arrived + first * 8 + (warp - 4);
        if (lane == 0) seen = count_arrival(arrived);
        __syncwarp();
        seen = __shfl_sync(0xffffffffu, seen, 0);
        write = seen == last - first;
        if (write) {
          if (lane == 0) *arrived = 0;
          w = 0.f;
          for (int c = first; c <= last; ++c)
            w += __ldcg(a.share + (size_t)(2 * c + (c == first ? 1 : 0)) * 2 * BLOCK + t * BLOCK + quarter * 32 + lane);
        }
      }
      if (write && key < s.held) {
        const int64_t slot = slot_of(a.c, s.b, key);
        if (slot >= 0) a.c.weight[slot] = (a.decay == 0.f ? 0.f : a.decay * a.c.weight[slot]) + w / (float)a.H;
        else set_status(a.status, SPTS_ERR_INDEX);
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (flags[ABORT]) {
    if (threadIdx.x == 0) set_status(a.status, SPTS_ERR_TIMEOUT);
    const uint64_t t1 = globaltimer_ns();
    while (globaltimer_ns() - t1 < 200000ull) { }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, PA_COLS);
  }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode(spts_ctx* ctx, CUtensorMap* tm, const void* p, int rank, const cuuint64_t* dim, const cuuint64_t* stride, const cuuint32_t* box) {
  const cuuint32_t step[4] = {1, 1, 1, 1};
  return reinterpret_cast<EncodeTiledFn>(ctx->paged_encode)(
             tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(p), dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// K or V of all pages as [rows / 8][Hkv * d / 64][8 rows][64]; a box is one head's dims of the rows of a page (of half a page of 256), in
// the order in which they lie in a tile
bool map_pages(spts_ctx* ctx, CUtensorMap* tm, const void* p, const spts_paged_kv* c) {
  const cuuint64_t width = (cuuint64_t)ctx->desc.n_kv_heads * ctx->desc.head_dim;
  const cuuint64_t dim[4] = {64, 8, width / 64, (cuuint64_t)c->n_pages * c->page_size / 8}, stride[3] = {width * 2, 128, width * 16};
  const cuuint32_t box[4] = {64, 8, (cuuint32_t)(ctx->desc.head_dim / 64), (cuuint32_t)((c->page_size < BLOCK ? c->page_size : BLOCK) / 8)};
  return encode(ctx, tm, p, 4, dim, stride, box);
}
// Q as [rows, H, d]; a box is 64 dims of `heads` heads of `tokens` rows
bool map_queries(spts_ctx* ctx, CUtensorMap* tm, const void* p, int64_t ld, int n_rows, int heads, int tokens) {
  const cuuint64_t H = ctx->desc.n_q_heads, d = ctx->desc.head_dim;
  const cuuint64_t dim[3] = {d, H, (cuuint64_t)n_rows}, stride[2] = {d * 2, (cuuint64_t)(n_rows == 1 ? H * d : ld) * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)tokens};
  return encode(ctx, tm, p, 3, dim, stride, box);
}

// As a dependent of what runs before: a CTA sets up its barriers and tensor memory before it waits for that.
template <typename... KArgs, typename... Args>
cudaError_t launch_big(spts_ctx* ctx, void (*kernel)(KArgs...), int ctas, int threads, int smem, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D>
spts_status attention_t(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start, int n_rows, void* O,
                        int64_t ldo, float* lse) {
  AttnArgs a;
  a.c = make_cache(cache); a.row_start = row_start; a.n_rows = n_rows;
  a.H = ctx->desc.n_q_heads; a.Hkv = ctx->desc.n_kv_heads; a.G = a.H / a.Hkv;
  a.tile_tokens = BLOCK / a.G;
  // two tiles to a unit where sequences have more tokens than one holds, on average (63 single tokens and a chunk of 512, 8192 rows each,
  // which take one: 410 us together, 327 and 86 by themselves)
  a.unit_tokens = n_rows > (int64_t)cache->n_seq * a.tile_tokens ? 2 * a.tile_tokens : a.tile_tokens;
  // (measured: with 1, 2, 3 blocks 64 single tokens over up to 8192 rows take 151, 144, 145 us, 8192 fresh tokens 495, 461, 456 us)
  a.extra = a.unit_tokens > a.tile_tokens ? 3 : 2;
  a.Q = (const bf16*)Q; a.ldq = ldq; a.O = (bf16*)O; a.ldo = ldo; a.lse = lse;
  a.wide = (reinterpret_cast<uintptr_t>(O) & 31) == 0 && (ldo * 2) % 32 == 0;
  a.share = ctx->ws.paged_part; a.arrived = ctx->ws.paged_arrived + 64; a.status = ctx->ws.status;
  a.open = reinterpret_cast<OpenUnit*>(ctx->ws.paged_open);
  // a unit of a few rows is joined in the time that a launch takes; one of many rows wants more warps than one CTA's
  a.solo = ceil_div(n_rows, cache->n_seq) * a.G <= SOLO_ROWS;
  CUtensorMap tmQ, tmK, tmV;
  if (!map_queries(ctx, &tmQ, Q, ldq, n_rows, a.G, a.tile_tokens) || !map_pages(ctx, &tmK, cache->k, cache) || !map_pages(ctx, &tmV, cache->v, cache))
    return SPTS_ERR_CUDA;
  const int ctas = ctx->sm_count < PAGED_MAX_CTAS ? ctx->sm_count : PAGED_MAX_CTAS;
  if (launch_big(ctx, paged_attn_kernel<D>, ctas, PA_THREADS, pa_smem<D>(), tmQ, tmK, tmV, a) != cudaSuccess) return SPTS_ERR_CUDA;
  ctx->launches++;
  if (a.solo) return SPTS_OK;
  if (launch_dependent(paged_attn_join_kernel<D>, dim3(ctas, JOIN_SPLIT), dim3(JOIN_THREADS), ctx->stream, a) != cudaSuccess) return SPTS_ERR_CUDA;
  ctx->launches++;
  return SPTS_OK;
}

template <int D>
spts_status weights_t(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start, int n_rows,
                      const float* lse, float decay) {
  WeightArgs a;
  a.c = make_cache(cache); a.row_start = row_start; a.n_rows = n_rows;
  a.H = ctx->desc.n_q_heads; a.Hkv = ctx->desc.n_kv_heads; a.G = a.H / a.Hkv;
  // tiles of queries as long as the sequences' chunks on average: a box brings in no more queries than that.  (Chunks far from the average pay
  // for it: 63 single tokens and a chunk of 512, 8192 rows each, take 270 us together, 171 and 61 by themselves.)
  const int most = BLOCK / a.G, mean = ceil_div(n_rows, cache->n_seq);
  a.tile_tokens = mean < 1 ? 1 : mean < most ? mean : most;
  a.lse = lse; a.decay = decay;
  a.share = ctx->ws.paged_part; a.arrived = ctx->ws.paged_arrived + 64; a.status = ctx->ws.status;
  CUtensorMap tmQ, tmK;
  // (without a query no box is read; the map still wants a place)
  if (!map_queries(ctx, &tmQ, n_rows > 0 ? Q : cache->k, ldq, n_rows > 0 ? n_rows : 1, a.G, a.tile_tokens) || !map_pages(ctx, &tmK, cache->k, cache))
    return SPTS_ERR_CUDA;
  const int ctas = ctx->sm_count < PAGED_MAX_CTAS ? ctx->sm_count : PAGED_MAX_CTAS;
  if (launch_big(ctx, paged_weights_kernel<D>, ctas, PW_THREADS, pw_smem<D>(), tmQ, tmK, a) != cudaSuccess) return SPTS_ERR_CUDA;
  ctx->launches++;
  return SPTS_OK;
}

}  // namespace

size_t paged_part_floats(const spts_model_desc& d) {
  if (d.dtype != SPTS_BF16) return 64;
  return (size_t)4 * PAGED_MAX_CTAS * BLOCK * (d.head_dim + 2);
}

spts_status paged_tc_init(spts_ctx* ctx) {
  cudaDriverEntryPointQueryResult q;
  ctx->paged_encode = nullptr;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ctx->paged_encode, cudaEnableDefault, &q) != cudaSuccess || ctx->paged_encode == nullptr)
    return SPTS_ERR_CUDA;
  const bool ok = cudaFuncSetAttribute(paged_attn_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, pa_smem<64>()) == cudaSuccess &&
                  cudaFuncSetAttribute(paged_attn_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, pa_smem<128>()) == cudaSuccess &&
                  cudaFuncSetAttribute(paged_weights_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, pw_smem<64>()) == cudaSuccess &&
                  cudaFuncSetAttribute(paged_weights_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, pw_smem<128>()) == cudaSuccess;
  return ok ? SPTS_OK : SPTS_ERR_CUDA;
}

spts_status launch_paged_attention_tc(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start, int n_rows,
                                      void* O, int64_t ldo, float* lse) {
  return ctx->desc.head_dim == 64 ? attention_t<64>(ctx, cache, Q, ldq, row_start, n_rows, O, ldo, lse)
                                  : attention_t<128>(ctx, cache, Q, ldq, row_start, n_rows, O, ldo, lse);
}

spts_status launch_paged_weights_tc(spts_ctx* ctx, const spts_paged_kv* cache, const void* Q, int64_t ldq, const int32_t* row_start, int n_rows,
                                    const float* lse, float decay) {
  return ctx->desc.head_dim == 64 ? weights_t<64>(ctx, cache, Q, ldq, row_start, n_rows, lse, decay)
                                  : weights_t<128>(ctx, cache, Q, ldq, row_start, n_rows, lse, decay);
}

}  // namespace spts
