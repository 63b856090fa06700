// Attention for many query rows a KV head (trees of drafted tokens, chunks): both products on tcgen05.
//
// A CTA streams 128 keys of one KV head at a time past its query rows.  S[128 rows x 128 keys] = Q K^T goes to tensor memory;
// a warpgroup reads it (a thread is a row: maximum and sum need no shuffle), writes the probabilities back over it in 16
// bits, and O[128 x channels] += P V takes them from there.  K and V lie in shared memory as they are in the cache, rows of
// 128 bytes swizzled: K is the right operand with its channels along k, V the right operand with its keys along k, so
// one layout serves both and nothing is transposed.
//
// Two such jobs run at a time, a warpgroup each, so that the products of one run under the exponentials of the other.  TWO: up to
// 256 rows, a job for each 128 of them and every K and V tile used twice.  Otherwise (up to 128 rows, bound by the stream): the
// jobs take alternate key tiles of the same rows and join their sums at the end of a piece.  Tensor memory: 2 x O and 2 x S, 128
// columns each.  One warp issues both jobs' products in turn, which keeps the warpgroups half a tile apart: in step (a warp for
// each job) they would share the exponential units and then both wait for the products (249 against 293 us).
//
// Exponentials do not wait for their tile's maximum: they are taken, 64 keys at a time, against the maximum known before; only
// a row whose new maximum is more than 2^kLazy higher (rare after the first tile) makes its warp rescale what it has and take them again.
//
// Loading: warps of their own bring the tiles in turn.  Where blocks are a multiple of 8 tokens a tile is a few TMA boxes (rows of
// one head out of a block, swizzled on the way); the ragged end of a request, new tokens whose V has to be looked through, and
// other block sizes go through 16-byte asynchronous copies.  8-bit codes land in a staging area that belongs to the warp, which
// widens them to f16 into the ring, exactly (three pairs of such warps, against three).  Scales multiply scores and probabilities as in
// the row kernel.
//
// Measured, 8 KV heads of 128, 256 rows (TWO), 16 requests of 8k, bf16: 169 to 191 us by the GPU and its clock, for 581 MB and 144 GFLOP
// (3.4 to 3.0 TB/s, 850 to 755 TFLOP/s; either alone would take 89 us); over an e4m3 cache 289 to 303, over a 4-bit one 287 to 300 (its records of 80 bytes come
// whole, scales among them; without the widening 254, without the multiplications by scales too 193).  In the fast case a tile of 128 keys takes 2.0 us, in which a warpgroup is busy for 1.3 with its exponentials and waits 0.7
// for its products, whose scores cannot be asked for before the probabilities in the same place are used up.  Around the stream:
// 7 us until Q is in and the first scores are there, 5 for each epilogue, 12 to 15 for a join.  104 rows of an int8 cache, 2 KV heads, 32
// requests of 8k: 121 to 124 us for 152 MB: 2.5 us a tile, of which a widening warp takes 1.4 for its half of K or V.
//
// Prompts and chunks run here too, but nothing is made for them: each tile of rows streams all keys, those behind its last row
// included, and past the context every tile is masked and (16 bits) its V looked through.  One prompt of 8k, 32 query heads: 1.8 ms
// (bf16), 2.3 ms (e4m3), against 0.34 ms for the causal half of the products; 2k over a context of 32k: 1.1 to 1.3 and 1.9 against 0.69.
//
// Every wait on a barrier is bounded (the allocation of tensor memory is not: it waits until other kernels on the SM have given theirs
// back).  One that runs out sets a flag which all roles see, and the kernel ends in the ordinary way (copies
// drained, products drained, tensor memory freed) with the status word set.
#pragma once
#include "kvr_attend_common.cuh"

namespace kvr {
namespace {

constexpr int kTileKeys = 128;
constexpr int kSoftmax = 256;

// ---- barriers, fences, tensor memory
// A warp's wait.  All lanes ask and meet again behind it: what follows are instructions of the whole warp (tcgen05.ld, .mma, .commit) with
// operands in uniform registers, and a loop that one lane ran while the others waited ahead of them led to wild addresses (it
// was also slower, 170 clocks on a barrier that is complete against 95).  A wait that runs out (after `polls`), here or in another role,
// sets the flag and goes on like one that did not, on whatever is there: all addresses stay in bounds, later waits give up at
// once, and the roles look at the flag once a step.
__device__ __forceinline__ void bar_wait(unsigned bar, unsigned parity, volatile int *gave_up, unsigned polls) {
  unsigned spin = 0;
  while (!bar_try(bar, parity)) {
    if (++spin == polls) *gave_up = 1;
    if ((spin & 15) == 0 && *gave_up) break;
  }
  __syncwarp();
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The issuing warp runs in step, so that addresses stay in uniform registers; `leader` (one lane) is a predicate of the
// instruction itself.
__device__ __forceinline__ unsigned elect_one() {
  unsigned r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r;
}
__device__ __forceinline__ void tc_commit(unsigned bar, unsigned leader) {
  asm volatile("{\n\t.reg .pred l;\n\tsetp.ne.u32 l, %1, 0;\n\t"
               "@l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader) : "memory");
}
// Shared-memory operand: rows of 128 bytes, 16-byte columns xor-ed with the row's number mod 8, 1024-byte groups of 8 rows
// one after the other; `stride` bytes from one group of 64 elements of the other dimension to the next (unused along k).
// The high word is the same for all: 1024 bytes between groups, descriptor version 1, 128-byte swizzle.
constexpr unsigned kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ unsigned operand(unsigned addr, unsigned stride) { return (addr & 0x3ffffu) >> 4 | (stride >> 4) << 16; }

// operands in shared memory are given by the low words of their descriptors
__device__ __forceinline__ void tc_product_ss(unsigned d, unsigned a, unsigned b, unsigned desc, unsigned add, unsigned leader) {
  asm volatile("{\n\t.reg .pred p, l;\n\t.reg .b64 x, y;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 l, %6, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
               "@l tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "r"(desc), "r"(add), "n"(kOperandHigh), "r"(leader) : "memory");
}
__device__ __forceinline__ void tc_product_ts(unsigned d, unsigned a, unsigned b, unsigned desc, unsigned add, unsigned leader) {
  asm volatile("{\n\t.reg .pred p, l;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 l, %6, 0;\n\tmov.b64 y, {%2, %5};\n\t"
               "@l tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
               ::"r"(d), "r"(a), "r"(b), "r"(desc), "r"(add), "n"(kOperandHigh), "r"(leader) : "memory");
}
#define KVR_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define KVR_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
__device__ __forceinline__ void tm_load32(unsigned (&x)[32], unsigned at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : KVR_R8(x, 0), KVR_R8(x, 8), KVR_R8(x, 16), KVR_R8(x, 24) : "r"(at));
}
__device__ __forceinline__ void tm_store32(unsigned at, const unsigned (&x)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
               ::KVR_W8(x, 0), KVR_W8(x, 8), KVR_W8(x, 16), KVR_W8(x, 24), "r"(at) : "memory");
}
__device__ __forceinline__ unsigned tm_load1(unsigned at) {
  unsigned x;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(x) : "r"(at));
  return x;
}
__device__ __forceinline__ void tm_store1(unsigned at, unsigned x) { asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%1], {%0};" ::"r"(x), "r"(at) : "memory"); }
__device__ __forceinline__ void tm_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void box_load(unsigned dst, const CUtensorMap *map, unsigned bar, int x, int head, int row, int block, int plane) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(head), "r"(row), "r"(block), "r"(plane) : "memory");
}

template <int FMT, int DP, bool TWO>
struct TileShape {
  static constexpr bool kQuant = quantised(FMT), kFour = four_bit(FMT);
  static constexpr int kBlocks = DP / 64;                                // 128-byte columns of a row
  // Warps: 0..7 softmax, 8 issues the products, the others load.  Whole warpgroups: registers are dealt to those.
  static constexpr int kSteps = 3, kPerStep = kQuant ? 2 : 1;         // steps loaded at a time, warps of a step
  static constexpr int kLoaders = kSteps * kPerStep, kSpan = kTileKeys / kPerStep; // a warp's keys of a step
  static constexpr int kThreads = kQuant ? 512 : 384;
  // Q, a tile or two of 128 rows.  At a piece's end the place holds what the warpgroups exchange, 32 channels each way, and the
  // weights of a join (16 pieces).
  static constexpr int kQBytes = TWO || DP < 128 ? 2 * 128 * DP * 2 : 128 * DP * 2;
  static_assert(kQBytes >= 2 * 32 * 128 * 4 && kQBytes >= kJoinAtOnce * 256 * 4, "");
  static constexpr int kBuffer = kTileKeys * DP * 2;                     // K or V of a tile, 16 bits
  // Buffers: what shared memory holds.  No fewer than the steps loaded at a time: a loader waits for step s - kRing to be used up
  // having filled step s - kSteps, and a barrier's parity is clear only if step s - 2 kRing is known to be over.
  static constexpr int kRing = (kQuant ? 3 : 5) + (kQuant && !TWO ? 1 : 0);
  static_assert(kRing >= kSteps, "");
  static constexpr int kRaw = kTileKeys * DP;                            // codes (4 bits: records, which are no longer) of K or V of a tile
  static_assert(!kFour || record_bytes(DP) <= DP, "");
  static constexpr int kScaleSlots = kQuant ? 4 : 0;                     // 128 scales of K, 128 of V
  static constexpr int kBytes = kQBytes + kRing * kBuffer + (kQuant ? kSteps * (kRaw + 2 * kTileKeys * 4) : 0) + kScaleSlots * 1024 + 1024;
};

struct TileBars {
  unsigned long long full[5], empty[5];
  unsigned long long s_full[2], p_full[2], pv_done[2], q_full, join, scale_full[4], drained;
  unsigned long long raw_full[6];
};

// The order in which tiles are loaded and used: of a piece of n tiles K 0 .. ahead-1, then V t, K t + ahead, ...
template <int AHEAD>
struct TileWalk {
  Piece p;
  int t0, n, k, v, step, tiles;          // step and tiles (of K): since the CTA's start
  bool more;
  __device__ __forceinline__ void open(const AttendArgs &a, int unit_tiles) {
    t0 = p.begin * unit_tiles;
    n = min(p.end * unit_tiles, (p.len.keys + kTileKeys - 1) / kTileKeys) - t0;
    k = v = 0;
  }
  __device__ __forceinline__ bool is_k() const { return k < n && k < v + AHEAD; }
  __device__ __forceinline__ int tile() const { return t0 + (is_k() ? k : v); }
  __device__ __forceinline__ int slot() const { return (is_k() ? tiles : tiles - (k - v)) & 3; }     // of the tile's scales
  __device__ __forceinline__ void advance(const AttendArgs &a, int unit_tiles, unsigned last) {
    ++step;
    if (is_k()) { ++k; ++tiles; } else ++v;
    if (v == n) {
      more = next_piece(a, p, last);
      if (more) open(a, unit_tiles);
    }
  }
};

// Which of the keys key0 .. key0 + 63 a row sees: bit i is key0 + i.  The context, then the row's own bits, nothing behind the
// request's last new token.
__device__ __forceinline__ unsigned long long visible(const AttendArgs &a, const Lengths &len, int key0, bool have, int t_row) {
  const int off = key0 - len.context;
  if (off <= -64) return ~0ull;
  unsigned long long vis = 0;
  if (off < 0) vis = ~0ull >> (64 + off);                       // -off low bits (off > -64)
  if (have) {
    unsigned long long fresh = 0;                                // bit i: new token off + i
    if (a.mask) {
      const unsigned long long *m = a.mask + (long long)(len.first + t_row) * a.mask_words;
      const int lo = off >> 6, sh = off & 63;                    // floor, also for negative off
      const unsigned long long w0 = lo >= 0 && lo < a.mask_words ? __ldg(m + lo) : 0ull;
      const unsigned long long w1 = lo + 1 >= 0 && lo + 1 < a.mask_words ? __ldg(m + lo + 1) : 0ull;
      fresh = sh ? w0 >> sh | w1 << (64 - sh) : w0;
    } else {
      const int upto = t_row - off + 1;                          // tokens off .. t_row
      fresh = upto <= 0 ? 0ull : upto >= 64 ? ~0ull : ~0ull >> (64 - upto);
    }
    const int room = len.fresh - off;                            // tokens there are from off on
    if (room <= 0) fresh = 0; else if (room < 64) fresh &= ~0ull >> (64 - room);
    vis |= off < 0 ? fresh & ~(~0ull >> (64 + off)) : fresh;
  }
  return vis;
}

// The largest of a tile's 128 scales among the keys that this thread's row sees.  Out of line, as it is seldom asked for.
__device__ __noinline__ float largest_seen(const AttendArgs &a, const Lengths &len, int key0, bool have, int t_row, const float *scales) {
  float big = 0.f;
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    const unsigned long long vis = visible(a, len, key0 + h * 64, have, t_row);
    if (vis == 0) continue;
#pragma unroll
    for (int i = 0; i < 64; i += 4) {
      const float4 x = *reinterpret_cast<const float4 *>(scales + h * 64 + i);
      if (vis >> i & 1) big = fmaxf(big, x.x);
      if (vis >> (i + 1) & 1) big = fmaxf(big, x.y);
      if (vis >> (i + 2) & 1) big = fmaxf(big, x.z);
      if (vis >> (i + 3) & 1) big = fmaxf(big, x.w);
    }
  }
  return big;
}

// The rows of a segment from its pieces of n CTAs c, c + step, ...: to the output, or (fold) to the first one's place.  256 threads.
// First, a thread a row, what each piece counts for (weights[piece][row]); then the sums, a thread four rows and 8 channels at a
// time: pieces lie channel by channel, and 16 loads of 16 bytes are under way for each thread (a row a thread, 4 bytes at a time, took
// 5 to 7 us longer for two or three pieces of 256 rows).
__device__ __noinline__ void join_weights(const AttendArgs &a, const Piece &p, const Cut &cut, int c, int step, int n, bool fold, int row, float *weights) {
  if (row >= a.row_tile || p.row0 + row >= p.len.fresh * (int)a.group.d) return;
  float2 ml[kJoinAtOnce];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int k = 0; k < kJoinAtOnce; ++k) {
    ml[k] = make_float2(-INFINITY, 0.f);
    if (k < n) ml[k] = __ldcg(a.part_ml + (long long)cut.piece(c + k * step) * a.row_tile + row);
    m = fmaxf(m, ml[k].x);
  }
#pragma unroll
  for (int k = 0; k < kJoinAtOnce; ++k) {
    ml[k].x = ml[k].x == m ? 1.f : exp2_fast(ml[k].x - m);      // both -infinity: a piece of an empty row
    l += ml[k].y * ml[k].x;
  }
  const float inv = fold ? 1.f : l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
#pragma unroll
  for (int k = 0; k < kJoinAtOnce; ++k) if (k < n) weights[k * 256 + row] = ml[k].x * inv;
  if (fold) {
    a.part_ml[(long long)cut.piece(c) * a.row_tile + row] = make_float2(m, l);
  } else if (a.lse) {
    const int t = (int)a.group.div(p.row0 + row), q_head = p.head_group * (int)a.group.d + (p.row0 + row - t * (int)a.group.d);
    a.lse[(long long)(p.len.first + t) * a.q_heads + q_head] = l == 0.f ? -INFINITY : m * 0.69314718f + logf(l);
  }
}
__device__ __noinline__ void join_rows(const AttendArgs &a, const Piece &p, const Cut &cut, int c, int step, int n, bool fold, int thread, const float *weights) {
  const int quads = a.row_tile / 4, row = (thread & (quads - 1)) * 4, rows = min(4, p.len.fresh * (int)a.group.d - p.row0 - row);
  if (rows <= 0) return;
#pragma unroll 1
  for (int d = (thread >> (a.row_shift - 2)) * 8; d < a.c.head_dim; d += 256 / quads * 8) {
    float4 o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int k = 0; k < n; k += 2) {
      float4 x[2][8];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float *src = a.part_o + ((long long)cut.piece(c + min(k + e, n - 1) * step) * a.c.head_dim + d) * a.row_tile + row;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[e][i] = __ldcg(reinterpret_cast<const float4 *>(src + i * a.row_tile));
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (k + e == n) break;
        const float4 f = *reinterpret_cast<const float4 *>(weights + (k + e) * 256 + row);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          o[i].x += f.x * x[e][i].x; o[i].y += f.y * x[e][i].y; o[i].z += f.z * x[e][i].z; o[i].w += f.w * x[e][i].w;
        }
      }
    }
    if (fold) {
#pragma unroll
      for (int i = 0; i < 8; ++i) *reinterpret_cast<float4 *>(a.part_o + ((long long)cut.piece(c) * a.c.head_dim + d + i) * a.row_tile + row) = o[i];
      continue;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e >= rows) break;
      const int t = (int)a.group.div(p.row0 + row + e), q_head = p.head_group * (int)a.group.d + (p.row0 + row + e - t * (int)a.group.d);
      char *dst = a.out.data + (long long)(p.len.first + t) * a.out.token_stride + (long long)q_head * a.out.head_stride + d * 2;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = e == 0 ? o[i].x : e == 1 ? o[i].y : e == 2 ? o[i].z : o[i].w;
      if (a.out.type == KVR_BF16) store8<KVR_BF16>(dst, y); else store8<KVR_F16>(dst, y);
    }
  }
}

// Codes that are NaN set to zero in KEYS rows of DP codes, by a warp; were there any?  Out of line: the callers'
// loops need the registers.
template <int DP, int KEYS>
__device__ __noinline__ bool clear_nan(unsigned char *rows, int lane) {
  unsigned found = 0;
#pragma unroll 8
  for (int i = lane; i < KEYS * DP / 16; i += 32) {
    const uint4 x = *reinterpret_cast<const uint4 *>(rows + i * 16);
    found |= nan_codes(x.x) | nan_codes(x.y) | nan_codes(x.z) | nan_codes(x.w);
  }
  if (!__any_sync(0xffffffffu, found != 0)) return false;
#pragma unroll 1
  for (int i = lane; i < KEYS * DP / 4; i += 32) {
    unsigned *w = reinterpret_cast<unsigned *>(rows) + i;
    *w &= ~(nan_codes(*w) / 0x80u * 0xffu);
  }
  __syncwarp();
  return true;
}

// Channels d .. d + 31 of V (bits) in which a key among key0 .. key0 + n - 1 that this thread's row sees is NaN, of an e4m3 cache.  (Of
// the tiles that the loaders look through: those that reach past the context.)
__device__ __noinline__ unsigned nan_channels(const AttendArgs &a, const Lengths &len, int r, int head, int key0, int n, bool have, int t_row, int d) {
  unsigned bits = 0;
#pragma unroll 1
  for (int j = max(key0, len.context / kTileKeys * kTileKeys); j < min(key0 + n, len.keys); ++j) {
    const long long off = token_offset(a.b, a.c, a.bs, r, j);
    if (off < 0 || !have || (j >= len.context && !sees(a, len.first, t_row, j - len.context))) continue;
    const char *v = a.c.base + a.c.v_offset + off + (long long)head * a.c.head_dim;
#pragma unroll 1
    for (int i = 0; i < min(32, a.c.head_dim - d); ++i) bits |= (unsigned)((v[d + i] & 0x7f) == 0x7f) << i;
  }
  return bits;
}

// 8 codes times their group's scale, as f16
__device__ __forceinline__ uint4 widen_group(unsigned w, unsigned scale) {
  auto times = [&](unsigned x) {
    const __half2 v = __hmul2(*reinterpret_cast<const __half2 *>(&x), *reinterpret_cast<const __half2 *>(&scale));
    return *reinterpret_cast<const unsigned *>(&v);
  };
  return make_uint4(times(widen_e2m1<0>(w)), times(widen_e2m1<1>(w)), times(widen_e2m1<2>(w)), times(widen_e2m1<3>(w)));
}

template <int FMT, int DP, bool TWO>
__global__ void __launch_bounds__(TileShape<FMT, DP, TWO>::kThreads, 1)
attend_tiles_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map) {
  using S = TileShape<FMT, DP, TWO>;
  constexpr bool kQuant = S::kQuant, kFour = S::kFour, kBf16 = FMT == KVR_CACHE_BF16;
  constexpr int kAhead = TWO ? 1 : 2;            // key tiles whose scores are made before the first is used
  constexpr float kLazy = kQuant ? 4.f : 8.f;    // 8-bit: leaves room for V's scale, see the row kernel
  extern __shared__ unsigned char raw_smem[];
  __shared__ unsigned scratch[39];
  __shared__ __align__(8) TileBars bars;
  __shared__ unsigned tm_slot;
  __shared__ int gave_up_word, last_in;
  __shared__ int brought[S::kSteps];             // 16-bit caches: a loader's last step
  __shared__ unsigned long long odd_keys[5][2];  // by ring slot: keys of a V tile with elements that are not finite
  __shared__ volatile int odd_codes;             // a loader has met codes of V that are NaN among a request's new tokens
  __shared__ float2 join_ml[2][128];
  __shared__ int box_ids[S::kLoaders][64];                 // by loader: block ids of the boxes around its step
  volatile int *gave_up = &gave_up_word;
  unsigned char *smem = reinterpret_cast<unsigned char *>(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
  unsigned char *q_tile = smem, *ring = q_tile + S::kQBytes, *raw = ring + S::kRing * S::kBuffer;
  float *scales = reinterpret_cast<float *>(raw + (kQuant ? S::kSteps : 0) * S::kRaw);
  float *scale_raw = scales + S::kScaleSlots * 256;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  Shares shares;
  Piece piece;
  if (!find_share(a, scratch, shares, piece.r, piece.base, piece.len)) return;
  const unsigned first = shares.first(blockIdx.x), last = shares.first(blockIdx.x + 1);
  piece.unit = first;
  if (!open_piece(a, piece, last)) return;     // an opening alone
  const int unit_tiles = (int)a.unit.d / kTileKeys;
  auto first_tile = [&](const Piece &p) { return p.begin * unit_tiles; };
  auto last_tile = [&](const Piece &p) { return min(p.end * unit_tiles, (p.len.keys + kTileKeys - 1) / kTileKeys); };

  if (threadIdx.x == 0) {
    gave_up_word = a.polls == 0;
    odd_codes = 0;
    for (int i = 0; i < S::kRing; ++i) { bar_init(shared_at(&bars.full[i]), S::kPerStep); bar_init(shared_at(&bars.empty[i]), 1); }
    for (int w = 0; w < 2; ++w) { bar_init(shared_at(&bars.s_full[w]), 1); bar_init(shared_at(&bars.p_full[w]), 4); bar_init(shared_at(&bars.pv_done[w]), 1); }
    bar_init(shared_at(&bars.q_full), 8);
    bar_init(shared_at(&bars.join), 8);
    bar_init(shared_at(&bars.drained), 1);
    for (int i = 0; i < 4; ++i) bar_init(shared_at(&bars.scale_full[i]), 2);       // brought with K by two warps
    for (int i = 0; i < 6; ++i) bar_init(shared_at(&bars.raw_full[i]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_at(&tm_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const unsigned tm = *reinterpret_cast<volatile unsigned *>(&tm_slot);
  const unsigned tm_o[2] = {tm, tm + 128};
  auto tm_s = [&](int w) { return tm + 256 + w * 128; };

  if (warp >= 9 && warp < 9 + S::kLoaders) {
    // ---- loaders: a step (K or V of a tile) for each, or for a pair
    const int me = warp - 9, group = me / S::kPerStep, span0 = (me % S::kPerStep) * S::kSpan;
    constexpr int kElement = kQuant ? 1 : 2, kChunks = DP * kElement / 16, kAtOnce = 32 / kChunks;
    const int chunk = lane % kChunks, sub = lane / kChunks;
    const int staged = kFour ? a.c.head_bytes : DP * kElement;   // of a key in the staging area
    const int used = a.c.head_bytes / 16;
    TileWalk<kAhead> at;
    at.p = piece; at.step = at.tiles = 0; at.more = true;
    at.open(a, unit_tiles);

    // Ids of the blocks that the boxes of a piece lie in, 32 boxes at a time, a batch ahead of its use: V's steps are at most one
    // tile (16 boxes of 8 tokens) behind K's, so both find theirs among the last 64.
    int *ids = box_ids[me];
    const int per_tile = a.box_rows ? kTileKeys / a.box_rows : 0;
    int box_next = 0, fetched = 0;       // first box of the batch in `fetched`
    unsigned at_unit = ~0u;
    auto fetch = [&]() {
      const int token = (box_next + lane) * a.box_rows;
      fetched = token < at.p.len.keys ? __ldg(a.b.tables + (long long)at.p.r * a.b.table_stride + a.bs.div(token)) : -1;
    };
    auto have_ids = [&](int tile) {
      if (at.p.unit != at_unit) {
        at_unit = at.p.unit;
        box_next = at.t0 * per_tile;
        fetch();
      }
      while (box_next < (tile + 1) * per_tile) {
        ids[(box_next + lane) & 63] = fetched;
        box_next += 32;
        fetch();
      }
      __syncwarp();
    };
    // This warp's keys of K or V of a tile, to dst (the tile's first row of them): boxes that complete on bar (true), or copies by this warp's lanes (false)
    auto bring = [&](unsigned char *dst, unsigned long long *bar, bool v, int tile, bool look) {
      const int key0 = tile * kTileKeys + span0;
      if (a.box_rows && !look && key0 + S::kSpan <= at.p.len.keys) {
        have_ids(tile);
        // a lane a box; 16-bit heads of 128 channels take two, side by side
        constexpr int kWide = kQuant ? 1 : S::kBlocks;
        const int box = lane / kWide, part = lane % kWide, boxes = per_tile / S::kPerStep;
        const int id = box < boxes ? ids[(key0 / a.box_rows + box) & 63] : 0;
        if (__all_sync(0xffffffffu, (unsigned)id < (unsigned)a.c.num_blocks)) {
          if (lane == 0) bar_expect(shared_at(bar), S::kSpan * staged);
          __syncwarp();
          if (box < boxes) {
            const int token = key0 + box * a.box_rows, row = token - (int)a.bs.div(token) * (int)a.bs.d;
            unsigned char *to = kQuant ? dst + box * a.box_rows * staged : dst + part * (kTileKeys * 128) + box * a.box_rows * 128;
            box_load(shared_at(to), &map, shared_at(bar), part * 64, at.p.head_group, row, id, v);
          }
          __syncwarp();
          return true;
        }
      }
      const char *base = a.c.base + (v ? a.c.v_offset : 0) + at.p.head_group * a.c.head_bytes;
#pragma unroll 1
      for (int k0 = 0; k0 < S::kSpan; k0 += 32) {
        // a lane finds a key; a wait for the table in every turn below came to 10 us a tile
        const int j = key0 + k0 + lane;
        const long long found = j < at.p.len.keys ? token_offset(a.b, a.c, a.bs, at.p.r, j) : -1;
        if (found < 0 && j < at.p.len.keys) report(a.b.status, KVR_DEV_BAD_BLOCK);
#pragma unroll 4
        for (int i = 0; i < 32 / kAtOnce; ++i) {
          const int key = k0 + i * kAtOnce + sub;
          const long long off = __shfl_sync(0xffffffffu, found, i * kAtOnce + sub);
          const bool got = off >= 0 && chunk < used;
          const char *src = got ? base + off + chunk * 16 : a.c.base;
          if constexpr (kFour) { if (chunk < used) copy16(shared_at(dst + key * staged + chunk * 16), src, got); }
          else if constexpr (kQuant) copy16(shared_at(dst + key * DP + chunk * 16), src, got);
          else copy16(shared_at(dst + (chunk >> 3) * (kTileKeys * 128) + key * 128 + (((chunk & 7) ^ (key & 7)) << 4)), src, got);
        }
      }
      return false;
    };
    bool ok = true;
    int done = -1;                       // this loader's last step
    auto slot_free = [&](int step) {     // has the buffer's previous tenant been used up?
      if (step >= S::kRing) bar_wait(shared_at(&bars.empty[step % S::kRing]), (step / S::kRing - 1) & 1, gave_up, a.polls);
      return __any_sync(0xffffffffu, *gave_up != 0) == 0;
    };
    auto mine = [&]() { while (at.more && at.step % S::kSteps != group) at.advance(a, unit_tiles, last); };
    mine();
    if constexpr (!kQuant) {
      while (at.more) {
        const int slot = at.step % S::kRing, tile = at.tile();
        const bool v = !at.is_k();
        const bool look = v && (tile + 1) * kTileKeys > at.p.len.context && (at.p.len.fresh > 1 || a.mask);
        if (!(ok = slot_free(at.step))) break;
        unsigned char *buf = ring + slot * S::kBuffer;
        if (!bring(buf, &bars.full[slot], v, tile, look)) {
          copy_commit();
          copy_wait<0>();
          if (look) {
            // Elements of V that are not finite must not meet the zero probabilities of rows that do not see their key: they
            // are set to zero here and added by the softmax threads, row by row.  A thread looks at what it copied (of new tokens:
            // all rows see the context).
            unsigned long long odd[2] = {0, 0};
            constexpr unsigned kExp = kBf16 ? 0x7f80u : 0x7c00u;
#pragma unroll 4
            for (int i = max(at.p.len.context - tile * kTileKeys, 0) / kAtOnce; i < kTileKeys / kAtOnce; ++i) {
              const int key = i * kAtOnce + sub;
              uint4 *x_at = reinterpret_cast<uint4 *>(buf + (chunk >> 3) * (kTileKeys * 128) + key * 128 + (((chunk & 7) ^ (key & 7)) << 4));
              uint4 x = *x_at;
              unsigned *e = reinterpret_cast<unsigned *>(&x);
              bool any = false;
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                if ((e[q] & kExp) == kExp) { e[q] &= 0xffff0000u; any = true; }
                if ((e[q] >> 16 & kExp) == kExp) { e[q] &= 0xffffu; any = true; }
              }
              if (any) { *x_at = x; if (key < 64) odd[0] |= 1ull << key; else odd[1] |= 1ull << (key - 64); }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const unsigned lo = __reduce_or_sync(0xffffffffu, (unsigned)odd[h]), hi = __reduce_or_sync(0xffffffffu, (unsigned)(odd[h] >> 32));
              if (lane == 0) odd_keys[slot][h] = (unsigned long long)hi << 32 | lo;
            }
          }
          fence_async();
          __syncwarp();
          if (lane == 0) bar_arrive(shared_at(&bars.full[slot]));
        }
        done = at.step;
        at.advance(a, unit_tiles, last);
        mine();
      }
      if (lane == 0) brought[group] = done;
    } else {
      // a step's codes and scales come to this warp's stage and are widened into the ring
      unsigned char *stage = raw + group * S::kRaw + span0 * DP;
      float *scale_stage = scale_raw + group * 2 * kTileKeys + span0;
      unsigned phase = 0;                // of raw_full
      while (at.more) {
        const bool v = !at.is_k();
        const int tile = at.tile(), slot = at.step % S::kRing, scale_slot = at.slot();
        const bool boxes = bring(stage, &bars.raw_full[me], v, tile, false);
        if (!v) {
          // the scales of K and of V: scores must not wait for V's codes to be widened
#pragma unroll
          for (int h = 0; h < S::kSpan; h += 32) {
            const int j = tile * kTileKeys + span0 + h + lane;
            long long off = -1;
            if (boxes) {                 // all keys are there, their blocks' ids at hand
              const int row = j - (int)a.bs.div(j) * (int)a.bs.d;
              off = (long long)ids[(a.box_rows == 16 ? j >> 4 : j >> 3) & 63] * a.c.block_stride + (long long)row * a.c.row_bytes;
            } else if (j < at.p.len.keys) {
              off = token_offset(a.b, a.c, a.bs, at.p.r, j);
            }
            const char *src = a.c.base + (off >= 0 ? off + a.c.scale_offset + (kFour ? a.c.head_bytes : 4) * at.p.head_group : 0);
            copy4(shared_at(scale_stage + h + lane), src, off >= 0);
            copy4(shared_at(scale_stage + kTileKeys + h + lane), src + (off >= 0 ? a.c.v_offset : 0), off >= 0);
          }
        }
        copy_commit();
        ok = slot_free(at.step);
        copy_wait<0>();
        if (boxes) {
          bar_wait(shared_at(&bars.raw_full[me]), phase, gave_up, a.polls);
          ok = __any_sync(0xffffffffu, *gave_up != 0) == 0 && ok;
          phase ^= 1;
        }
        __syncwarp();
        if (!ok) {                       // the boxes land all the same before the CTA ends
          if (boxes && !bar_settle(shared_at(&bars.raw_full[me]), phase ^ 1)) *gave_up = 1;
          break;
        }
        // 16 channels of a key are two neighbouring 16-byte columns.  Which goes first alternates with the half of the row and
        // with the key, so that 8-byte reads of 16 lanes and 16-byte writes of 8 lanes fall into different banks.
        const int c0 = (chunk & 3) * 2, swap = ((chunk >> 2) ^ sub) & 1;
        const unsigned char *src = stage + sub * DP + chunk * 16;
        unsigned char *row = ring + slot * S::kBuffer + (chunk >> 2) * (kTileKeys * 128) + (span0 + sub) * 128;
        if (FMT == KVR_CACHE_E4M3 && v && (tile + 1) * kTileKeys > at.p.len.context && (at.p.len.fresh > 1 || a.mask)) {
          // Codes of V that are NaN must not meet the zero probabilities of rows that do not see their key: set to zero, and the
          // softmax threads are told that there were some (append stores none).
          if (clear_nan<DP, S::kSpan>(stage, lane)) odd_codes = 1;
        }
        if constexpr (kFour) {
          // 16 channels are a group: 8 bytes of codes and one scale, which goes into the elements (exact)
          const unsigned char *record = stage + sub * staged;
#pragma unroll 4
          for (int i = 0; i < S::kSpan / kAtOnce; ++i) {
            const int key = i * kAtOnce + sub;
            const uint2 x = *reinterpret_cast<const uint2 *>(record + i * kAtOnce * staged + chunk * 8);
            const unsigned scale = group_scale(record[i * kAtOnce * staged + a.c.scale_offset + 4 + chunk]) * 0x10001u;
            unsigned char *to = row + i * (kAtOnce * 128);
            *reinterpret_cast<uint4 *>(to + (((c0 + swap) ^ (key & 7)) << 4)) = widen_group(swap ? x.y : x.x, scale);
            *reinterpret_cast<uint4 *>(to + (((c0 + 1 - swap) ^ (key & 7)) << 4)) = widen_group(swap ? x.x : x.y, scale);
          }
        } else {
#pragma unroll 4
        for (int i = 0; i < S::kSpan / kAtOnce; ++i) {
          const int key = i * kAtOnce + sub;             // kAtOnce is even: the key's parity is sub's
          const uint2 x = *reinterpret_cast<const uint2 *>(src + i * (kAtOnce * DP) + swap * 8), y = *reinterpret_cast<const uint2 *>(src + i * (kAtOnce * DP) + 8 - swap * 8);
          unsigned char *to = row + i * (kAtOnce * 128);
          *reinterpret_cast<uint4 *>(to + (((c0 + swap) ^ (key & 7)) << 4)) =
              make_uint4(widen<FMT, false>(x.x), widen<FMT, true>(x.x), widen<FMT, false>(x.y), widen<FMT, true>(x.y));
          *reinterpret_cast<uint4 *>(to + (((c0 + 1 - swap) ^ (key & 7)) << 4)) =
              make_uint4(widen<FMT, false>(y.x), widen<FMT, true>(y.x), widen<FMT, false>(y.y), widen<FMT, true>(y.y));
        }
        }
        if (!v) {
#pragma unroll
          for (int h = 0; h < S::kSpan; h += 32) {
            scales[scale_slot * 256 + span0 + h + lane] = scale_stage[h + lane] * (kFour ? kGroupUnit : 1.f);
            scales[scale_slot * 256 + 128 + span0 + h + lane] = scale_stage[kTileKeys + h + lane] * (kFour ? kGroupUnit : 1.f);
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) {
          bar_arrive(shared_at(&bars.full[slot]));
          if (!v) bar_arrive(shared_at(&bars.scale_full[scale_slot]));
        }
        at.advance(a, unit_tiles, last);
        mine();
      }
      copy_wait<0>();
    }
  } else if (warp == 8) {
    // ---- products: the warp runs in step, one lane issues
    const unsigned leader = elect_one();
    constexpr unsigned kType = kBf16 ? 1u : 0u;
    constexpr unsigned kS = 1u << 4 | kType << 7 | kType << 10 | (kTileKeys / 8) << 17 | (128 / 16) << 24;
    constexpr unsigned kO = 1u << 4 | kType << 7 | kType << 10 | 1u << 16 | (DP / 8) << 17 | (128 / 16) << 24;
    const unsigned q_low = operand(shared_at(q_tile), 16), k_low = operand(shared_at(ring), 16), v_low = operand(shared_at(ring), kTileKeys * 128);
    int used[2] = {0, 0}, pieces = 0, slot = 0, round = 0;     // jobs whose product with V is issued; the step's place in the ring
    bool again = true;
    auto take = [&]() {                        // the next step's buffer, when it is full
      bar_wait(shared_at(&bars.full[slot]), round & 1, gave_up, a.polls);
      const int s = slot;
      if (++slot == S::kRing) { slot = 0; ++round; }
      return s;
    };
    auto scores = [&](int w, int k_slot) {
      const unsigned k_at = k_low + k_slot * (S::kBuffer / 16), q = q_low + (TWO ? w : 0) * (128 * DP * 2 / 16);
#pragma unroll
      for (int k = 0; k < DP / 16; ++k)        // 16 channels: 32 bytes of a row; 64: the next 128-byte column
        tc_product_ss(tm_s(w), q + (k >> 2) * (128 * 128 / 16) + (k & 3) * 2, k_at + (k >> 2) * (kTileKeys * 128 / 16) + (k & 3) * 2, kS, k > 0, leader);
      tc_commit(shared_at(&bars.s_full[w]), leader);
    };
    while (again) {
      const int n = last_tile(piece) - first_tile(piece), head_start = min(kAhead, n);
      bar_wait(shared_at(&bars.q_full), pieces & 1, gave_up, a.polls);
      ++pieces;
      for (int t = 0; t < head_start; ++t) {
        const int k_slot = take();
        tc_after();
        scores(TWO ? 0 : t & 1, k_slot);
        if (TWO) scores(1, k_slot);
        tc_commit(shared_at(&bars.empty[k_slot]), leader);
      }
#pragma unroll 1
      for (int t = 0; t < n; ++t) {
        const bool next = t + kAhead < n;      // scores of tile t + kAhead follow (!TWO: kAhead is even, the same job's)
        const int v_slot = take(), k_slot = next ? take() : 0;
        const unsigned v_at = v_low + v_slot * (S::kBuffer / 16), old = t >= (TWO ? 1 : 2);    // a job's first product overwrites O
#pragma unroll 1
        for (int i = 0; i < (TWO ? 2 : 1); ++i) {
          const int w = TWO ? i : t & 1;
          bar_wait(shared_at(&bars.p_full[w]), (w ? used[1] : used[0]) & 1, gave_up, a.polls);
          tc_after();
#pragma unroll
          for (int s = 0; s < kTileKeys / 16; ++s)
            tc_product_ts(tm + w * 128, tm_s(w) + s * 8, v_at + s * (16 * 128 / 16), kO, s > 0 ? 1u : old, leader);
          used[0] += 1 - w;
          used[1] += w;
          if (next) scores(w, k_slot);
          tc_commit(shared_at(&bars.pv_done[w]), leader);      // (read at a piece's end and where V is not finite)
        }
        tc_commit(shared_at(&bars.empty[v_slot]), leader);
        if (next) tc_commit(shared_at(&bars.empty[k_slot]), leader);
        if (__any_sync(0xffffffffu, *gave_up != 0)) break;
      }
      again = next_piece(a, piece, last) && !__any_sync(0xffffffffu, *gave_up != 0);
    }
    // all products have ended before tensor memory is given back
    tc_commit(shared_at(&bars.drained), leader);
    if (!bar_settle(shared_at(&bars.drained), 0)) *gave_up = 1;
  } else if (warp < 8) {
    // ---- softmax: warpgroup w, thread = row
    const int w = warp >> 2, tid = threadIdx.x & 127;
    const unsigned lanes = (unsigned)(warp & 3) << 21;   // this warp's 32 lanes of tensor memory
    int jobs = 0, joins = 0, tiles_before = 0, steps_before = 0;
    bool ok = true, again = true;
    // A wait that runs out goes on like one that did not, on whatever is there; the flag is looked at once a tile.
    auto wait = [&](unsigned long long *bar, unsigned parity) { bar_wait(shared_at(bar), parity, gave_up, a.polls); };
    // The product of job j with V.  That of job j - 1 has ended when the scores of job j are there, which were issued behind it.
    auto wait_product = [&](int j) { wait(&bars.pv_done[w], j & 1); };
    auto join = [&]() {
      __syncwarp();
      if (lane == 0) bar_arrive(shared_at(&bars.join));
      wait(&bars.join, joins & 1);
      ++joins;
      return __all_sync(0xffffffffu, !*gave_up) != 0;
    };
    while (ok && again) {
      const Lengths len = piece.len;
      const int head = piece.head_group, t0 = first_tile(piece), n = last_tile(piece) - t0;
      const int row = piece.row0 + (TWO ? w * 128 : 0) + tid;
      const bool have = row < len.fresh * (int)a.group.d && (TWO ? w * 128 : 0) + tid < a.row_tile && head < a.c.kv_heads;
      const int t_row = have ? (int)a.group.div(row) : 0, q_head = head * (int)a.group.d + (have ? row - t_row * (int)a.group.d : 0);
      // Q to the operand layout.  The lanes of a warp stand side by side along a few of its 32 rows at a time.
      float scale = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);     // a scale of zero: Q is zero instead
      {
        constexpr int kLanes = DP / 8, kRows = 32 / kLanes;
        const int c = lane % kLanes, row_base = (TWO ? w * 128 : 0) + (warp & 3) * 32;
        const unsigned flip = a.scale_log2 < 0 ? 0x80008000u : 0u;       // a negative one: Q's sign
        uint4 x[kLanes];
#pragma unroll
        for (int i = 0; i < kLanes; ++i) {
          const int local = row_base + i * kRows + lane / kLanes, at = piece.row0 + local, t_at = (int)a.group.div(at);
          x[i] = make_uint4(0, 0, 0, 0);
          if (at < len.fresh * (int)a.group.d && local < a.row_tile && c * 8 < a.c.head_dim && a.scale_log2 != 0.f)
            x[i] = *reinterpret_cast<const uint4 *>(a.q.data + (long long)(len.first + t_at) * a.q.token_stride +
                                                    (long long)(head * (int)a.group.d + at - t_at * (int)a.group.d) * a.q.head_stride + c * 16);
        }
        if constexpr (kQuant) {
          // f16 of rows that have been brought to [1, 2) by a power of two, which goes to the row's scale
          const bool bf16 = a.q.type == KVR_BF16;
#pragma unroll
          for (int i = 0; i < kLanes; ++i) {
            float y[8], most = 0.f, down = 1.f;
            if (bf16) widen8<KVR_BF16>(x[i], y); else widen8<KVR_F16>(x[i], y);
#pragma unroll
            for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(y[k]));
#pragma unroll
            for (int d = kLanes / 2; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            const unsigned e = __float_as_uint(most) >> 23, up = e >= 1 && e <= 253 ? e << 23 : 127u << 23;
            if (e >= 1 && e <= 253) down = __uint_as_float((254u - e) << 23);
            const unsigned own = __shfl_sync(0xffffffffu, up, lane % kRows * kLanes);
            if (lane / kRows == i) scale *= __uint_as_float(own);        // this thread's own row
            x[i] = make_uint4(pack_f16(y[0] * down, y[1] * down), pack_f16(y[2] * down, y[3] * down), pack_f16(y[4] * down, y[5] * down), pack_f16(y[6] * down, y[7] * down));
          }
        }
        if (TWO || w == 0) {
          unsigned char *dst = q_tile + (TWO ? w : 0) * (128 * DP * 2) + (c >> 3) * (128 * 128);
#pragma unroll
          for (int i = 0; i < kLanes; ++i) {
            const int r = (warp & 3) * 32 + i * kRows + lane / kLanes;
            *reinterpret_cast<uint4 *>(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(x[i].x ^ flip, x[i].y ^ flip, x[i].z ^ flip, x[i].w ^ flip);
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) bar_arrive(shared_at(&bars.q_full));
      }
      float top = -INFINITY, sum = 0.f;  // top: of scaled scores
      float v_unit = unit_first(have);   // of V's scales
      int mine = 0;                      // jobs of this warpgroup in this piece
#pragma unroll 1
      for (int t = TWO ? 0 : w; t < n; t += TWO ? 1 : 2) {
        const int key0 = (t0 + t) * kTileKeys, tile = tiles_before + t;
        const float *ks = scales + (tile & 3) * 256;     // K's scales, then V's
        const unsigned s_at = tm_s(w) + lanes;
        wait(&bars.s_full[w], jobs & 1);
        tc_after();
        if constexpr (kQuant) wait(&bars.scale_full[tile & 3], (tile >> 2) & 1);
        const bool edge = key0 + kTileKeys > len.context;
        float s[64];
        auto load_scores = [&](int h) {          // keys 64 h .. 64 h + 63
          {
            unsigned x[32], y[32];
            tm_load32(x, s_at + h * 64);
            tm_load32(y, s_at + h * 64 + 32);
            tm_loaded();
#pragma unroll
            for (int i = 0; i < 32; ++i) { s[i] = __uint_as_float(x[i]); s[32 + i] = __uint_as_float(y[i]); }
          }
          if constexpr (kQuant) {
            const float *k_scale = ks + h * 64;
#pragma unroll
            for (int i = 0; i < 64; i += 4) {
              const ulonglong2 k4 = *reinterpret_cast<const ulonglong2 *>(k_scale + i);
              const float2 p = unpair(mul2(pair(s[i], s[i + 1]), k4.x)), q = unpair(mul2(pair(s[i + 2], s[i + 3]), k4.y));
              s[i] = p.x; s[i + 1] = p.y; s[i + 2] = q.x; s[i + 3] = q.y;
            }
          }
        };
        float f_unit = 1.f;                      // what a change of V's unit does to O
        if constexpr (kQuant) {
          const float *vs = ks + 128;
          float big = fmaxf(fmaxf(vs[lane], vs[lane + 32]), fmaxf(vs[lane + 64], vs[lane + 96]));
#pragma unroll
          for (int d = 16; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
          if (__any_sync(0xffffffffu, big * v_unit >= kUnitLimit)) {
            if (edge) {
              const Lengths copy = len;          // what the call is shown lies in memory
              big = largest_seen(a, copy, key0, have, t_row, vs);
            }
            if (big * v_unit >= kUnitLimit) {
              f_unit = unit_of(big) * unit_back(v_unit);
              v_unit = unit_of(big);
            }
            __syncwarp();
          }
        }
        const Pair scale2 = pair(scale, scale), unit2 = pair(v_unit, v_unit);
#pragma unroll 1
        for (int h = 0; h < 2;) {
          load_scores(h);
          unsigned long long vis = ~0ull;
          if (__builtin_expect(edge, 0)) {
            vis = visible(a, len, key0 + h * 64, have, t_row);
#pragma unroll
            for (int i = 0; i < 64; ++i) if (!(vis >> i & 1)) s[i] = -INFINITY;
          }
          float m0 = fmaxf(s[0], s[1]), m1 = fmaxf(s[2], s[3]);
#pragma unroll
          for (int i = 4; i < 64; i += 4) { m0 = max3(m0, s[i], s[i + 1]); m1 = max3(m1, s[i + 2], s[i + 3]); }
          m0 = fmaxf(m0, m1);
          const float base = top == -INFINITY ? 0.f : top;
          const Pair base2 = pair(-base, -base);
          Pair sum0 = 0, sum1 = 0;
#pragma unroll
          for (int i = 0; i < 64; i += 4) {
            const float2 p = unpair(fma2(pair(s[i], s[i + 1]), scale2, base2)), q = unpair(fma2(pair(s[i + 2], s[i + 3]), scale2, base2));
            s[i] = exp2_fast(p.x); s[i + 1] = exp2_fast(p.y); s[i + 2] = exp2_fast(q.x); s[i + 3] = exp2_fast(q.y);
            sum0 = add2(sum0, pair(s[i], s[i + 1]));
            sum1 = add2(sum1, pair(s[i + 2], s[i + 3]));
          }
          const float best = m0 == -INFINITY ? m0 : m0 * scale;
          const bool higher = best > top + kLazy;
          if (__builtin_expect(__any_sync(0xffffffffu, higher || f_unit != 1.f), 0)) {
            // O, the sum and the probabilities that are already there go down; then the same 64 keys again: their scores
            // have not been written over yet
            float f = 1.f;
            if (higher) {
              f = top == -INFINITY ? 0.f : exp2_fast(top - best);
              top = best;
            }
            sum *= f;
            const float f_o = f * f_unit;
            f_unit = 1.f;
            if (mine > 0) {              // the last product is over: these scores were issued behind it
#pragma unroll 1
              for (int c = 0; c < DP; c += 32) {
                unsigned x[32];
                tm_load32(x, tm_o[w] + lanes + c);
                tm_loaded();
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * f_o);
                tm_store32(tm_o[w] + lanes + c, x);
              }
              tm_stored();
            }
            if (h == 1) {                // (V's unit moves before the first half only: f alone)
              unsigned x[32];
              tm_load32(x, s_at);
              tm_loaded();
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                if constexpr (kBf16) {
                  x[i] = pack_bf16(__uint_as_float(x[i] << 16) * f, __uint_as_float(x[i] & 0xffff0000u) * f);
                } else {
                  const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&x[i]));
                  x[i] = pack_f16(p.x * f, p.y * f);
                }
              }
              tm_store32(s_at, x);
              tm_stored();
            }
            continue;
          }
          const float2 sums = unpair(add2(sum0, sum1));
          sum += sums.x + sums.y;
          if constexpr (kQuant) {
            const float *v_scale = ks + 128 + h * 64;
#pragma unroll
            for (int i = 0; i < 64; i += 4) {
              const ulonglong2 v4 = *reinterpret_cast<const ulonglong2 *>(v_scale + i);
              const float2 p = unpair(mul2(pair(s[i], s[i + 1]), mul2(v4.x, unit2))), q = unpair(mul2(pair(s[i + 2], s[i + 3]), mul2(v4.y, unit2)));
              s[i] = p.x; s[i + 1] = p.y; s[i + 2] = q.x; s[i + 3] = q.y;
            }
            if (__builtin_expect(edge, 0)) {     // a scale that is not finite, at a key that the row does not see
#pragma unroll
              for (int i = 0; i < 64; ++i) if (!(vis >> i & 1)) s[i] = 0.f;
            }
          }
          unsigned p[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) p[i] = kBf16 ? pack_bf16(s[2 * i], s[2 * i + 1]) : pack_f16(s[2 * i], s[2 * i + 1]);
          __syncwarp();
          tm_store32(s_at + h * 32, p);  // over the scores of keys that are done with
          tm_stored();
          ++h;
        }
        const bool look = !kQuant && edge && (len.fresh > 1 || a.mask);
        unsigned long long odd[2] = {0, 0};
        if (__builtin_expect(look, 0)) {
          // V's tile is in its buffer and stays there until this warpgroup has handed over its probabilities
          const int at = steps_before + min(kAhead, n) + t + min(t, max(n - kAhead, 0)), slot_v = at % S::kRing;
          wait(&bars.full[slot_v], (at / S::kRing) & 1);
          odd[0] = *reinterpret_cast<volatile unsigned long long *>(&odd_keys[slot_v][0]);
          odd[1] = *reinterpret_cast<volatile unsigned long long *>(&odd_keys[slot_v][1]);
        }
        tc_before();
        __syncwarp();
        if (lane == 0) bar_arrive(shared_at(&bars.p_full[w]));
        if (__builtin_expect((odd[0] | odd[1]) != 0, 0)) {
          // infinite or NaN elements of V: added as they are to the rows that see their key (the probability is positive)
          wait_product(jobs);
          tc_after();
#pragma unroll 1
          for (int i = 0; i < kTileKeys; ++i) {
            if (!((i < 64 ? odd[0] >> i : odd[1] >> (i - 64)) & 1)) continue;
            const bool sees_it = visible(a, len, key0 + (i & 64), have, t_row) >> (i & 63) & 1;
            const long long off = token_offset(a.b, a.c, a.bs, piece.r, key0 + i);
            if (off < 0) continue;
            const char *v = a.c.base + a.c.v_offset + off + (long long)head * a.c.head_dim * 2;
            for (int d = 0; d < a.c.head_dim; ++d) {
              const float x = load1<kBf16 ? KVR_BF16 : KVR_F16>(v + d * 2);
              if (!(fabsf(x) < INFINITY)) {
                __syncwarp();
                const float o = __uint_as_float(tm_load1(tm_o[w] + lanes + d));
                tm_loaded();
                tm_store1(tm_o[w] + lanes + d, __float_as_uint(sees_it ? o + x : o));
                tm_stored();
              }
            }
          }
        }
        ++jobs;
        ++mine;
        if (__any_sync(0xffffffffu, *gave_up != 0)) break;
      }
      if (mine > 0) wait_product(jobs - 1);
      if (!(ok = __all_sync(0xffffffffu, !*gave_up))) break;
      tc_after();
      tiles_before += n;
      steps_before += 2 * n;
      const float unit = kQuant ? unit_back(v_unit) : 1.f;
      // The row's sums, to the output or to the workspace.  Not TWO: the warpgroups have sums of the same rows.  Each takes half of
      // the channels, 32 at a time, and gives the other's half away.
      constexpr int kOwn = TWO ? DP : DP / 2;
      const int d_own = TWO ? 0 : w * kOwn, d_give = kOwn - d_own, local = (TWO ? w * 128 : 0) + tid;
      float *ex = reinterpret_cast<float *>(q_tile);     // [warpgroup][channel][row]
      float own = unit, other = 0.f;
      const bool whole = piece.begin == 0 && piece.end == len.units;
      const long long slot = (long long)blockIdx.x * 2 + (piece.unit == first ? 0 : 1);
      char *dst = a.out.data + (long long)(len.first + t_row) * a.out.token_stride + (long long)q_head * a.out.head_stride;
      if constexpr (!TWO) {
        join_ml[w][tid] = make_float2(top, sum);
        if (!(ok = join())) break;       // Q is used up
        const float2 theirs = join_ml[1 - w][tid];
        const float m = fmaxf(top, theirs.x), f = top == m ? 1.f : exp2_fast(top - m);
        other = theirs.x == -INFINITY ? 0.f : theirs.x == m ? 1.f : exp2_fast(theirs.x - m);
        own = mine > 0 ? unit * f : 0.f;
        sum = sum * f + theirs.y * other;
        top = m;
      }
      const float inv = !whole ? 1.f : sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : NAN;
#pragma unroll 1
      for (int c = 0; c < kOwn; c += 32) {
        unsigned x[32];
        if constexpr (!TWO) {
          if (mine > 0) {
            tm_load32(x, tm_o[w] + lanes + d_give + c);
            tm_loaded();
#pragma unroll
            for (int i = 0; i < 32; ++i) ex[(w * 32 + i) * 128 + tid] = __uint_as_float(x[i]) * unit;
          }
          if (!(ok = join())) break;
        }
        tm_load32(x, tm_o[w] + lanes + d_own + c);
        tm_loaded();
        float o[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = !TWO && mine == 0 ? 0.f : __uint_as_float(x[i]) * own;
        if constexpr (!TWO) {
          if (other != 0.f) {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] += ex[((1 - w) * 32 + i) * 128 + tid] * other;
          }
        }
        if constexpr (FMT == KVR_CACHE_E4M3) {
          if (__builtin_expect(odd_codes, 0)) {  // set before the products that are waited for above
            const Lengths copy = len;    // what the call is shown lies in memory
            const unsigned nan = nan_channels(a, copy, piece.r, head, t0 * kTileKeys, n * kTileKeys, have, t_row, d_own + c);
#pragma unroll
            for (int i = 0; i < 32; ++i) if (nan >> i & 1) o[i] = NAN;
          }
        }
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          const int d = d_own + c + i;
          if (!have || d >= a.c.head_dim) break;
          if (whole) {
            const float y[8] = {o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv, o[i + 4] * inv, o[i + 5] * inv, o[i + 6] * inv, o[i + 7] * inv};
            if (a.out.type == KVR_BF16) store8<KVR_BF16>(dst + d * 2, y); else store8<KVR_F16>(dst + d * 2, y);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) a.part_o[(slot * a.c.head_dim + d + e) * a.row_tile + local] = o[i + e];
          }
        }
        __syncwarp();
        if constexpr (!TWO) {
          if (!(ok = join())) break;     // read: may be written again, with Q too
        }
      }
      if (!ok) break;
      if (have && (TWO || w == 0)) {
        if (!whole) a.part_ml[slot * a.row_tile + local] = make_float2(top, sum);
        else if (a.lse) a.lse[(long long)(len.first + t_row) * a.q_heads + q_head] = sum == 0.f ? -INFINITY : top * 0.69314718f + logf(sum);
      }
      if (!whole)
        ok = hand_in(a, piece, shares, join, &last_in, warp, lane, [&](const Cut &cut, int c, int step, int n, bool fold) {
          const Piece copy = piece;      // what the call is shown lies in memory
          join_weights(a, copy, cut, c, step, n, fold, threadIdx.x, ex);
          join();
          join_rows(a, copy, cut, c, step, n, fold, threadIdx.x, ex);
          join();                        // the weights have been read
        });
      again = next_piece(a, piece, last);
    }
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (gave_up_word) {
    // Boxes under way when a wait ran out land before the CTA ends.  (Of 8-bit and 4-bit caches each loader has seen to its own.)  All roles have
    // stopped: the last step that went to a buffer is the only one that may not have landed, for each took the place of one that had been used up.
    if (!kQuant && threadIdx.x < S::kRing) {
      int step = -1;
      for (int g = 0; g < S::kSteps; ++g) {
        int mine = brought[g];
        while (mine >= 0 && mine % S::kRing != (int)threadIdx.x) mine -= S::kSteps;
        step = max(step, mine);
      }
      if (step >= 0) bar_settle(shared_at(&bars.full[threadIdx.x]), (step / S::kRing) & 1);
    }
    __syncthreads();
  }
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
  if (threadIdx.x == 0 && gave_up_word) report(a.b.status, KVR_DEV_GAVE_UP);
}

template <int FMT, int DP, bool TWO>
cudaError_t launch_tiles(const AttendArgs &a, const CUtensorMap &map, cudaStream_t s) {
  using S = TileShape<FMT, DP, TWO>;
  const auto kernel = attend_tiles_kernel<FMT, DP, TWO>;
  static OncePerDevice once;
  if (const cudaError_t e = allow_shared(once, kernel, S::kBytes)) return e;
  kernel<<<a.ctas, S::kThreads, S::kBytes, s>>>(a, map);
  return cudaGetLastError();
}
template <int FMT>
cudaError_t launch_tiles(const AttendArgs &a, const CUtensorMap &map, cudaStream_t s) {
  if (a.c.head_dim <= 64) return a.row_tile > 128 ? launch_tiles<FMT, 64, true>(a, map, s) : launch_tiles<FMT, 64, false>(a, map, s);
  return a.row_tile > 128 ? launch_tiles<FMT, 128, true>(a, map, s) : launch_tiles<FMT, 128, false>(a, map, s);
}

}  // namespace
}  // namespace kvr
