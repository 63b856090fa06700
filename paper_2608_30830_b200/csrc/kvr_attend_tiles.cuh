// Attention for many query rows a KV head (trees of drafted tokens, chunks): both products on tcgen05.
//
// A CTA streams 64 keys of one KV head at a time past its query rows.  S[128 rows x 64 keys] = Q K^T goes to tensor memory;
// a warpgroup reads it (a thread is a row: maximum and sum need no shuffle), writes the probabilities back over it in 16
// bits, and O[128 x channels] += P V takes them from there.  K and V lie in shared memory as they are in the cache, rows of
// 128 bytes swizzled: K is the right operand with its channels along k, V the right operand with its keys along k, so
// one layout serves both and nothing is transposed.
//
// Two warpgroups work at a time.  TWO: up to 256 rows, each warpgroup has 128 of them and every K and V tile is used twice.
// Otherwise (up to 128 rows, bound by the stream): the warpgroups take alternate key tiles of the same rows and join their
// sums at the end of a piece.  S is double-buffered for each warpgroup, so the products of the next tile run under the
// exponentials of this one.  Tensor memory: 2 x O (128 columns), 2 x 2 x S (64).
//
// 128 threads load.  16-bit caches: asynchronous copies into the ring, kLag tiles in flight.  8-bit caches: copies into
// a private staging area (a thread widens what it copied itself), then to f16 in the ring, exactly; scales multiply scores
// and probabilities as in the row kernel.
//
// Every wait is bounded.  One that runs out sets a flag which all roles see, and the kernel ends in the ordinary way (copies
// drained, products drained, tensor memory freed) with the status word set.
#pragma once
#include "kvr_attend_common.cuh"

namespace kvr {
namespace {

constexpr int kTileKeys = 64;
constexpr int kLoaders = 128, kSoftmax = 256, kTileThreads = kSoftmax + kLoaders + 32;
constexpr unsigned kTileSpin = 1u << 20, kTileNap = 1000;               // tries, and nanoseconds that one may sleep

// ---- barriers, fences, tensor memory
__device__ __forceinline__ void bar_init(unsigned bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(unsigned bar, unsigned parity) {
  unsigned ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity), "r"(kTileNap) : "memory");
  return ok != 0;
}
// false: the limit ran out here, or another role has given up
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity, volatile int *gave_up) {
  for (unsigned spin = 0; spin < kTileSpin; ++spin) {
    if (bar_try(bar, parity)) return true;
    if ((spin & 15) == 15 && *gave_up) return false;
  }
  *gave_up = 1;
  return false;
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(unsigned bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_product_ss(unsigned d, unsigned long long a, unsigned long long b, unsigned desc, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((unsigned)add) : "memory");
}
__device__ __forceinline__ void tc_product_ts(unsigned d, unsigned a, unsigned long long b, unsigned desc, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(desc), "r"((unsigned)add) : "memory");
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

// Shared-memory operand: rows of 128 bytes, 16-byte columns xor-ed with the row's number mod 8, 1024-byte groups of 8 rows
// one after the other; `stride` bytes from one group of 64 elements of the other dimension to the next (unused along k).
__device__ __forceinline__ unsigned long long operand(unsigned addr, unsigned stride) {
  return (unsigned long long)((addr & 0x3ffffu) >> 4) | (unsigned long long)(stride >> 4) << 16 | (unsigned long long)(1024 >> 4) << 32 |
         1ull << 46 | 2ull << 61;
}

template <int FMT, int DP>
struct TileShape {
  static constexpr bool kQuant = quantised(FMT);
  static constexpr int kBlocks = DP / 64;                                // 128-byte columns of a row
  static constexpr int kQBytes = 2 * 128 * DP * 2;                       // two tiles of 128 rows
  static constexpr int kBuffer = kTileKeys * DP * 2;                     // K or V of a tile, 16 bits
  static constexpr int kRing = kQuant ? 6 : 9;
  static constexpr int kLag = kQuant ? 6 : 5;                            // loads in flight, in buffers
  static constexpr int kRaw = kTileKeys * DP;                            // codes of K or V of a tile
  static constexpr int kRawRing = kQuant ? kLag + 1 : 0;
  static constexpr int kScaleSlots = kQuant ? 8 : 0;                     // 64 scales of K, 64 of V
  static constexpr int kScaleRaw = kQuant ? kRawRing * kLoaders * 4 : 0;
  static constexpr int kBytes = kQBytes + kRing * kBuffer + kRawRing * kRaw + kScaleSlots * 512 + kScaleRaw + 1024;
};

struct TileBars {
  unsigned long long full[9], empty[9];
  unsigned long long s_full[2][2], p_full[2][2], pv_done[2][2], q_full, join, scale_full[8], drained;
};

template <int FMT, int DP, bool TWO>
__global__ void __launch_bounds__(kTileThreads, 1) attend_tiles_kernel(const __grid_constant__ AttendArgs a) {
  using S = TileShape<FMT, DP>;
  constexpr bool kQuant = S::kQuant, kBf16 = FMT == KVR_CACHE_BF16;
  constexpr int kAhead = TWO ? 2 : 4;            // key tiles whose scores are made before the first is used
  constexpr float kLazy = 4.f;
  extern __shared__ unsigned char raw_smem[];
  __shared__ long long scratch[34];
  __shared__ __align__(8) TileBars bars;
  __shared__ unsigned tm_slot;
  __shared__ int gave_up_word;
  __shared__ unsigned long long odd_keys[9];     // by ring slot: keys of a V tile with elements that are not finite
  __shared__ float join_ml[128][2];
  volatile int *gave_up = &gave_up_word;
  unsigned char *smem = reinterpret_cast<unsigned char *>(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
  unsigned char *q_tile = smem, *ring = q_tile + S::kQBytes, *raw = ring + S::kRing * S::kBuffer;
  float *scales = reinterpret_cast<float *>(raw + S::kRawRing * S::kRaw);
  float *scale_raw = scales + S::kScaleSlots * 128;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  const long long total = total_units(a, scratch);
  const int ctas = (int)min((long long)a.ctas, total);
  if ((int)blockIdx.x >= ctas) return;
  const long long first = first_unit(total, ctas, blockIdx.x), last = first_unit(total, ctas, blockIdx.x + 1);
  Piece piece;
  find_unit(a, first, scratch, piece.r, piece.base);
  piece.unit = first;
  piece.len = attend_lengths(a, piece.r);
  open_piece(a, piece, last);
  const int unit_tiles = a.unit_keys / kTileKeys;
  auto first_tile = [&](const Piece &p) { return p.begin * unit_tiles; };
  auto last_tile = [&](const Piece &p) { return min(p.end * unit_tiles, (p.len.keys + kTileKeys - 1) / kTileKeys); };

  if (threadIdx.x == 0) {
    gave_up_word = 0;
    for (int i = 0; i < S::kRing; ++i) { bar_init(shared_at(&bars.full[i]), 4); bar_init(shared_at(&bars.empty[i]), 1); }
    for (int w = 0; w < 2; ++w) {
      for (int b = 0; b < 2; ++b) { bar_init(shared_at(&bars.s_full[w][b]), 1); bar_init(shared_at(&bars.p_full[w][b]), 4); bar_init(shared_at(&bars.pv_done[w][b]), 1); }
    }
    bar_init(shared_at(&bars.q_full), 8);
    bar_init(shared_at(&bars.join), 8);
    bar_init(shared_at(&bars.drained), 1);
    for (int i = 0; i < 8; ++i) bar_init(shared_at(&bars.scale_full[i]), 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_at(&tm_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const unsigned tm = *reinterpret_cast<volatile unsigned *>(&tm_slot);
  const unsigned tm_o[2] = {tm, tm + 128};
  auto tm_s = [&](int w, int b) { return tm + 256 + (w * 2 + b) * 64; };

  if (warp >= 8 && warp < 12) {
    // ---- loaders: 16 keys of a tile a warp; K and V tiles in the order in which the products take them
    const int w16 = (warp - 8) * 16, tid = threadIdx.x - kSoftmax;
    constexpr int kChunks = DP * (kQuant ? 1 : 2) / 16, kAtOnce = 32 / kChunks, kCopies = 16 / kAtOnce;
    const int chunk = lane % kChunks, sub = lane / kChunks;
    const int used = a.c.head_dim * (kQuant ? 1 : 2) / 16;
    const int element = kQuant ? 1 : 2;
    // the order within a piece of n tiles: K 0 .. ahead-1, then V t, K t + ahead, ...
    struct Step { Piece p; int t0, n, k, v; bool more; } st;
    st.p = piece; st.t0 = first_tile(piece); st.n = last_tile(piece) - st.t0; st.k = st.v = 0; st.more = true;
    auto is_k = [&]() { return st.k < st.n && st.k < st.v + kAhead; };
    auto advance = [&]() {
      if (is_k()) ++st.k; else ++st.v;
      if (st.v == st.n) {
        st.more = next_piece(a, st.p, last);
        if (st.more) { st.t0 = first_tile(st.p); st.n = last_tile(st.p) - st.t0; st.k = st.v = 0; }
      }
    };
    // what the next copies need, fetched one step ahead
    int next_id = 0, next_j = 0;
    bool next_in = false;
    auto fetch = [&]() {
      if (!st.more) return;
      next_j = (st.t0 + (is_k() ? st.k : st.v)) * kTileKeys + w16 + (lane & 15);
      next_in = next_j < st.p.len.keys;
      next_id = next_in ? __ldg(a.b.tables + (long long)st.p.r * a.b.table_stride + a.bs.div(next_j)) : 0;
    };
    // of a step whose copies are under way: is it V, the tile's number in the call's order, does it hold new tokens
    int issued = 0, done = 0, tiles_k = 0;
    unsigned char kind[8];               // by step mod 8: bit 0 V, bit 1 look for odd values, bits 2..4 scale slot
    bool ok = true;
    auto issue = [&]() {                 // copies of the next step, if there is one
      if (st.more) {
        const bool v = !is_k();
        const bool known = (unsigned)next_id < (unsigned)a.c.num_blocks, in = next_in && known;
        if (!known) report(a.b.status, KVR_DEV_BAD_BLOCK);
        const int within = next_j - (int)a.bs.div(next_j) * (int)a.bs.d;
        const long long offset = in ? (long long)next_id * a.c.block_stride + (long long)within * a.c.row_bytes : 0;
        const unsigned valid = __ballot_sync(0xffffffffu, in);
        const char *plane = a.c.base + (v ? a.c.v_offset : 0);
        const char *base = plane + st.p.head_group * a.c.head_dim * element;
        unsigned dst;
        if constexpr (kQuant) dst = shared_at(raw + (issued % S::kRawRing) * S::kRaw + tid * 16);
        else dst = shared_at(ring + (issued % S::kRing) * S::kBuffer);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int key = i * kAtOnce + sub;
          const long long off = __shfl_sync(0xffffffffu, offset, key);
          const bool got = (valid >> key & 1) && chunk < used;
          const char *src = base + off + (got ? chunk * 16 : 0);
          if constexpr (kQuant) copy16(dst + i * (kLoaders * 16), src, got);
          else copy16(dst + (chunk >> 3) * (kTileKeys * 128) + (w16 + key) * 128 + (((chunk & 7) ^ (key & 7)) << 4), src, got);
        }
        if constexpr (kQuant) {
          // lanes 0..15 of a warp bring its keys' scales
          if (lane < 16) copy4(shared_at(scale_raw + (issued % S::kRawRing) * kLoaders + w16 + lane), plane + offset + (in ? a.c.scale_offset + 4 * st.p.head_group : 0), in);
        }
        const int slot = (v ? tiles_k - (st.k - st.v) : tiles_k) & 7;
        const bool look = !kQuant && v && (st.t0 + st.v + 1) * kTileKeys > st.p.len.context && (st.p.len.fresh > 1 || a.mask);
        kind[issued & 7] = (unsigned char)((v ? 1 : 0) | (look ? 2 : 0) | slot << 2);
        if (!v) ++tiles_k;
        ++issued;
        advance();
        fetch();
      }
      copy_commit();
    };
    fetch();
    auto slot_free = [&](int step) {     // has the buffer's previous tenant been used up?
      if (step < S::kRing) return true;
      bool good = true;
      if (lane == 0) good = bar_wait(shared_at(&bars.empty[step % S::kRing]), (step / S::kRing - 1) & 1, gave_up);
      return __shfl_sync(0xffffffffu, (int)good, 0) != 0;
    };
    // kLag - 1 steps ahead
    for (int i = 0; i < S::kLag - 1; ++i) issue();       // kLag - 1 < kRing: these buffers are fresh
    while (ok && (st.more || done < issued)) {
      if constexpr (!kQuant) { if (st.more) ok = slot_free(issued); }
      if (!ok) break;
      issue();
      copy_wait<S::kLag - 1>();
      const int what = kind[done & 7];
      unsigned char *buf = ring + (done % S::kRing) * S::kBuffer;
      if constexpr (!kQuant) {
        if (what & 2) {
          // Elements of V that are not finite must not meet the zero probabilities of rows that do not see their key: they
          // are set to zero here and added by the softmax threads, row by row.  A thread looks at what it copied.
          unsigned odd = 0;
          constexpr unsigned kExp = kBf16 ? 0x7f80u : 0x7c00u;
#pragma unroll
          for (int i = 0; i < kCopies; ++i) {
            const int key = i * kAtOnce + sub;
            uint4 *at = reinterpret_cast<uint4 *>(buf + (chunk >> 3) * (kTileKeys * 128) + (w16 + key) * 128 + (((chunk & 7) ^ (key & 7)) << 4));
            uint4 x = *at;
            unsigned *e = reinterpret_cast<unsigned *>(&x);
            bool any = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if ((e[j] & kExp) == kExp) { e[j] &= 0xffff0000u; any = true; }
              if ((e[j] >> 16 & kExp) == kExp) { e[j] &= 0xffffu; any = true; }
            }
            if (any) { *at = x; odd |= 1u << key; }
          }
          odd = __reduce_or_sync(0xffffffffu, odd);
          if (lane == 0) reinterpret_cast<unsigned short *>(&odd_keys[done % S::kRing])[warp - 8] = (unsigned short)odd;
        } else if ((what & 1) && lane == 0) {
          reinterpret_cast<unsigned short *>(&odd_keys[done % S::kRing])[warp - 8] = 0;
        }
      } else {
        ok = slot_free(done);
        if (!ok) break;
        const unsigned char *mine = raw + (done % S::kRawRing) * S::kRaw + tid * 16;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int key = i * kAtOnce + sub;
          const uint4 x = *reinterpret_cast<const uint4 *>(mine + i * (kLoaders * 16));
          // 16 channels, 32 bytes: two neighbouring 16-byte columns
          unsigned char *row = buf + (chunk >> 2) * (kTileKeys * 128) + (w16 + key) * 128;
          const int c0 = (chunk & 3) * 2;
          *reinterpret_cast<uint4 *>(row + ((c0 ^ (key & 7)) << 4)) =
              make_uint4(widen<FMT, false>(x.x), widen<FMT, true>(x.x), widen<FMT, false>(x.y), widen<FMT, true>(x.y));
          *reinterpret_cast<uint4 *>(row + (((c0 + 1) ^ (key & 7)) << 4)) =
              make_uint4(widen<FMT, false>(x.z), widen<FMT, true>(x.z), widen<FMT, false>(x.w), widen<FMT, true>(x.w));
        }
        if (lane < 16) scales[(what >> 2) * 128 + (what & 1) * 64 + w16 + lane] = scale_raw[(done % S::kRawRing) * kLoaders + w16 + lane];
      }
      fence_async();
      __syncwarp();
      if (lane == 0) {
        bar_arrive(shared_at(&bars.full[done % S::kRing]));
        if (kQuant && (what & 1)) bar_arrive(shared_at(&bars.scale_full[what >> 2]));
      }
      ++done;
    }
    copy_wait<0>();
  } else if (warp == 12) {
    // ---- products, issued by one thread
    if (lane == 0) {
      constexpr unsigned kType = kBf16 ? 1u : 0u;
      constexpr unsigned kS = 1u << 4 | kType << 7 | kType << 10 | (kTileKeys / 8) << 17 | (128 / 16) << 24;
      constexpr unsigned kO = 1u << 4 | kType << 7 | kType << 10 | 1u << 16 | (DP / 8) << 17 | (128 / 16) << 24;
      const unsigned q_at = shared_at(q_tile), ring_at = shared_at(ring);
      int step = 0, jobs_s[2] = {0, 0}, jobs_p[2] = {0, 0}, pieces = 0;
      bool ok = true, again = true;
      auto take = [&]() { return bar_wait(shared_at(&bars.full[step % S::kRing]), (step / S::kRing) & 1, gave_up); };
      auto scores = [&](int w) {                 // of the K tile in the current step's buffer
        const unsigned k_at = ring_at + (step % S::kRing) * S::kBuffer, q = q_at + (TWO ? w : 0) * (128 * DP * 2);
        const unsigned d = tm_s(w, jobs_s[w] & 1);
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
          tc_product_ss(d, operand(q + (k >> 2) * (128 * 128) + (k & 3) * 32, 16), operand(k_at + (k >> 2) * (kTileKeys * 128) + (k & 3) * 32, 16), kS, k > 0);
        tc_commit(shared_at(&bars.s_full[w][jobs_s[w] & 1]));
        ++jobs_s[w];
      };
      while (ok && again) {
        const int n = last_tile(piece) - first_tile(piece);
        int fresh[2] = {1, 1};                   // the first product of a piece overwrites O
        ok = bar_wait(shared_at(&bars.q_full), pieces & 1, gave_up);
        ++pieces;
        tc_after();
        for (int t = 0; ok && t < min(kAhead, n); ++t) {
          if (!(ok = take())) break;
          tc_after();
          if (TWO) { scores(0); scores(1); } else scores(t & 1);
          tc_commit(shared_at(&bars.empty[step % S::kRing]));
          ++step;
        }
        for (int t = 0; ok && t < n; ++t) {
          if (!(ok = take())) break;             // V of tile t
          const unsigned v_at = ring_at + (step % S::kRing) * S::kBuffer;
          const int v_slot = step % S::kRing;
          ++step;
          const bool next = t + kAhead < n;
          bool have_next = false;
#pragma unroll
          for (int i = 0; i < (TWO ? 2 : 1); ++i) {
            const int w = TWO ? i : t & 1, b = jobs_p[w] & 1;
            if (!(ok = bar_wait(shared_at(&bars.p_full[w][b]), (jobs_p[w] >> 1) & 1, gave_up))) break;
            tc_after();
#pragma unroll
            for (int k = 0; k < kTileKeys / 16; ++k)
              tc_product_ts(tm_o[w], tm_s(w, b) + k * 8, operand(v_at + k * (16 * 128), kTileKeys * 128), kO, !fresh[w] || k > 0);
            fresh[w] = 0;
            tc_commit(shared_at(&bars.pv_done[w][b]));
            ++jobs_p[w];
            if (i == (TWO ? 1 : 0)) tc_commit(shared_at(&bars.empty[v_slot]));
            if (next) {
              if (!have_next) {
                if (!(ok = take())) break;
                tc_after();
                have_next = true;
              }
              scores(w);
            }
          }
          if (ok && next) {
            tc_commit(shared_at(&bars.empty[step % S::kRing]));
            ++step;
          }
        }
        again = next_piece(a, piece, last);
      }
      // all products have ended before tensor memory is given back
      tc_commit(shared_at(&bars.drained));
      for (unsigned spin = 0; spin < kTileSpin && !bar_try(shared_at(&bars.drained), 0); ++spin) {}
    }
    __syncwarp();
  } else {
    // ---- softmax: warpgroup w, thread = row
    const int w = warp >> 2, tid = threadIdx.x & 127;
    const unsigned lanes = (unsigned)(warp & 3) << 21;   // this warp's 32 lanes of tensor memory
    int jobs = 0, joins = 0, tiles_before = 0, steps_before = 0;
    bool ok = true, again = true;
    auto wait_all = [&](unsigned long long *bar, unsigned parity) {      // the same answer for the whole warp
      return __all_sync(0xffffffffu, bar_wait(shared_at(bar), parity, gave_up)) != 0;
    };
    // The product of job j with V.  One barrier for even and one for odd jobs: that of job j - 2 is known to have ended (the
    // scores of job j, which this warpgroup has seen, were issued behind it), so the parity tells job j from it.
    auto wait_product = [&](int j) { return wait_all(&bars.pv_done[w][j & 1], (j >> 1) & 1); };
    auto join = [&]() {
      __syncwarp();
      if (lane == 0) bar_arrive(shared_at(&bars.join));
      const bool r = wait_all(&bars.join, joins & 1);
      ++joins;
      return r;
    };
    while (ok && again) {
      const Lengths len = piece.len;
      const int head = piece.head_group, t0 = first_tile(piece), n = last_tile(piece) - t0;
      const int row = piece.row0 + (TWO ? w * 128 : 0) + tid;
      const bool have = row < len.fresh * (int)a.group.d && (TWO ? w * 128 : 0) + tid < a.row_tile;
      const int t_row = have ? (int)a.group.div(row) : 0, q_head = head * (int)a.group.d + (have ? row - t_row * (int)a.group.d : 0);
      // the row of Q, to the operand layout
      float scale = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);     // a scale of zero: Q is zero instead
      {
        const char *src = a.q.data + (long long)(len.first + t_row) * a.q.token_stride + (long long)q_head * a.q.head_stride;
        unsigned char *dst = q_tile + (TWO ? w : 0) * (128 * DP * 2) + tid * 128;
        const unsigned flip = a.scale_log2 < 0 ? 0x80008000u : 0u;       // a negative one: Q's sign
        float down = 1.f;
        if constexpr (kQuant) {
          float top = 0.f;
#pragma unroll 4
          for (int c = 0; c < DP / 8; ++c) {
            if (!have || c * 8 >= a.c.head_dim) break;
            float y[8];
            if (a.q.type == KVR_BF16) load8<KVR_BF16>(src + c * 16, y); else load8<KVR_F16>(src + c * 16, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(y[i]));
          }
          const unsigned e = __float_as_uint(top) >> 23;
          if (e >= 1 && e <= 253) { down = __uint_as_float((254u - e) << 23); scale *= __uint_as_float(e << 23); }
        }
        if (TWO || w == 0) {
#pragma unroll 4
          for (int c = 0; c < DP / 8; ++c) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (have && c * 8 < a.c.head_dim && a.scale_log2 != 0.f) {
              if constexpr (!kQuant) {
                x = *reinterpret_cast<const uint4 *>(src + c * 16);
              } else {
                float y[8];
                if (a.q.type == KVR_BF16) load8<KVR_BF16>(src + c * 16, y); else load8<KVR_F16>(src + c * 16, y);
                x = make_uint4(pack_f16(y[0] * down, y[1] * down), pack_f16(y[2] * down, y[3] * down), pack_f16(y[4] * down, y[5] * down), pack_f16(y[6] * down, y[7] * down));
              }
              x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
            }
            *reinterpret_cast<uint4 *>(dst + (c >> 3) * (128 * 128) + (((c & 7) ^ (tid & 7)) << 4)) = x;
          }
        }
        fence_async();
        __syncwarp();
        if (lane == 0) bar_arrive(shared_at(&bars.q_full));
      }
      float top = -INFINITY, sum = 0.f;  // top: of scaled scores
      int v_exp = -1000, mine = 0;       // mine: jobs of this warpgroup in this piece
      for (int t = TWO ? 0 : w; t < n; t += TWO ? 1 : 2) {
        const int b = jobs & 1, key0 = (t0 + t) * kTileKeys;
        if (!(ok = wait_all(&bars.s_full[w][b], (jobs >> 1) & 1))) break;
        tc_after();
        float s[64];
        {
          unsigned x[32], y[32];
          tm_load32(x, tm_s(w, b) + lanes);
          tm_load32(y, tm_s(w, b) + lanes + 32);
          tm_loaded();
#pragma unroll
          for (int i = 0; i < 32; ++i) { s[i] = __uint_as_float(x[i]); s[32 + i] = __uint_as_float(y[i]); }
        }
        const int tile = tiles_before + t, slot = tile & 7;
        const float *ks = scales + slot * 128, *vs = ks + 64;
        if constexpr (kQuant) {
          if (!(ok = wait_all(&bars.scale_full[slot], (tile >> 3) & 1))) break;
#pragma unroll
          for (int i = 0; i < 64; i += 4) {
            const float4 k4 = *reinterpret_cast<const float4 *>(ks + i);
            s[i] *= k4.x; s[i + 1] *= k4.y; s[i + 2] *= k4.z; s[i + 3] *= k4.w;
          }
        }
        const bool edge = key0 + kTileKeys > len.context;
        unsigned long long vis = ~0ull;
        if (edge) {
          // bit i: key0 + i.  Context below, then the row's own bits, nothing behind the last new token
          const int off = key0 - len.context;
          vis = 0;
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
#pragma unroll
          for (int i = 0; i < 64; ++i) if (!(vis >> i & 1)) s[i] = -INFINITY;
        }
        float m0 = s[0], m1 = s[1], m2 = s[2], m3 = s[3];
#pragma unroll
        for (int i = 4; i < 64; i += 4) { m0 = fmaxf(m0, s[i]); m1 = fmaxf(m1, s[i + 1]); m2 = fmaxf(m2, s[i + 2]); m3 = fmaxf(m3, s[i + 3]); }
        m0 = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
        const float best = m0 == -INFINITY ? m0 : m0 * scale;
        float f = 1.f, f_unit = 1.f;     // of the sum, and of O's unit
        if (best > top + kLazy) {
          f = top == -INFINITY ? 0.f : exp2_fast(top - best);
          top = best;
        }
        float v_unit = 1.f;
        if constexpr (kQuant) {
          // the row kernel's rule for V's scales
          float big = fmaxf(vs[lane], vs[lane + 32]);
#pragma unroll
          for (int d = 16; d > 0; d >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
          const int e = (int)(__float_as_uint(big) >> 23) - 127;
          if (big > 0.f && big < INFINITY && e - v_exp >= 11) {
            const int next = max(e - 7, -126);
            if (v_exp != -1000) f_unit = power2(v_exp - next);
            v_exp = next;
          }
          if (v_exp != -1000) v_unit = power2(-v_exp);
        }
        const float f_o = f * f_unit;
        if (mine > 0 && __any_sync(0xffffffffu, f_o != 1.f)) {
          if (!(ok = wait_product(jobs - 1))) break;
          tc_after();
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
        const float base = top == -INFINITY ? 0.f : top;
        float a0 = 0.f, a1 = 0.f, a2 = 0.f, a3 = 0.f;
#pragma unroll
        for (int i = 0; i < 64; i += 4) {
          s[i] = exp2_fast(fmaf(s[i], scale, -base)); s[i + 1] = exp2_fast(fmaf(s[i + 1], scale, -base));
          s[i + 2] = exp2_fast(fmaf(s[i + 2], scale, -base)); s[i + 3] = exp2_fast(fmaf(s[i + 3], scale, -base));
          a0 += s[i]; a1 += s[i + 1]; a2 += s[i + 2]; a3 += s[i + 3];
        }
        sum = sum * f + ((a0 + a1) + (a2 + a3));
        if constexpr (kQuant) {
#pragma unroll
          for (int i = 0; i < 64; i += 4) {
            const float4 v4 = *reinterpret_cast<const float4 *>(vs + i);
            s[i] *= v4.x * v_unit; s[i + 1] *= v4.y * v_unit; s[i + 2] *= v4.z * v_unit; s[i + 3] *= v4.w * v_unit;
          }
          if (edge) {                    // a scale that is not finite, at a key that the row does not see
#pragma unroll
            for (int i = 0; i < 64; ++i) if (!(vis >> i & 1)) s[i] = 0.f;
          }
        }
        const bool look = !kQuant && edge && (len.fresh > 1 || a.mask);
        unsigned long long odd = 0;
        if (look) {
          // V's tile is in its buffer and stays there until this warpgroup has handed over its probabilities
          const int at = steps_before + min(kAhead, n) + t + min(t, max(n - kAhead, 0)), slot_v = at % S::kRing;
          if (!(ok = wait_all(&bars.full[slot_v], (at / S::kRing) & 1))) break;
          odd = *reinterpret_cast<volatile unsigned long long *>(&odd_keys[slot_v]);
        }
        __syncwarp();
        {
          unsigned p[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) p[i] = kBf16 ? pack_bf16(s[2 * i], s[2 * i + 1]) : pack_f16(s[2 * i], s[2 * i + 1]);
          tm_store32(tm_s(w, b) + lanes, p);
        }
        tm_stored();
        tc_before();
        __syncwarp();
        if (lane == 0) bar_arrive(shared_at(&bars.p_full[w][b]));
        if (odd) {
          // infinite or NaN elements of V: added as they are to the rows that see their key (the probability is positive)
          if (!(ok = wait_product(jobs))) break;
          tc_after();
          while (odd) {
            const int i = __ffsll((long long)odd) - 1;
            odd &= odd - 1;
            const long long off = token_offset(a.b, a.c, a.bs, piece.r, key0 + i);
            if (off < 0) continue;
            const char *v = a.c.base + a.c.v_offset + off + (long long)head * a.c.head_dim * 2;
            for (int d = 0; d < a.c.head_dim; ++d) {
              const float x = load1<kBf16 ? KVR_BF16 : KVR_F16>(v + d * 2);
              if (!(fabsf(x) < INFINITY)) {
                const float o = __uint_as_float(tm_load1(tm_o[w] + lanes + d));
                tm_loaded();
                tm_store1(tm_o[w] + lanes + d, __float_as_uint(vis >> i & 1 ? o + x : o));
                tm_stored();
              }
            }
          }
        }
        ++jobs;
        ++mine;
      }
      if (ok && mine > 0) ok = wait_product(jobs - 1);
      if (!ok) break;
      tc_after();
      tiles_before += n;
      steps_before += 2 * n;
      float unit = kQuant && v_exp != -1000 ? power2(v_exp) : 1.f, other = 0.f;
      float *ex = reinterpret_cast<float *>(q_tile);     // [channel][row]: Q is used up when both warpgroups have joined
      if constexpr (!TWO) {
        if (!(ok = join())) break;
        if (w == 1 && mine > 0) {
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            unsigned x[32];
            tm_load32(x, tm_o[1] + lanes + c);
            tm_loaded();
#pragma unroll
            for (int i = 0; i < 32; ++i) ex[(c + i) * 128 + tid] = __uint_as_float(x[i]) * unit;
          }
        }
        if (w == 1) { join_ml[tid][0] = top; join_ml[tid][1] = sum; }
        if (!(ok = join())) break;
        if (w == 0 && n > 1) {
          const float m2 = join_ml[tid][0], m = fmaxf(top, m2);
          const float f = top == m ? 1.f : exp2_fast(top - m);
          other = m2 == -INFINITY ? 0.f : m2 == m ? 1.f : exp2_fast(m2 - m);
          sum = sum * f + join_ml[tid][1] * other;
          top = m;
          unit *= f;
        }
      }
      if (TWO || w == 0) {
        const bool whole = piece.begin == 0 && piece.end == len.units;
        const int local = (TWO ? w * 128 : 0) + tid;
        const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : NAN;
        const long long place = ((long long)blockIdx.x * 2 + (piece.unit == first ? 0 : 1)) * a.row_tile + local;
        char *dst = a.out.data + (long long)(len.first + t_row) * a.out.token_stride + (long long)q_head * a.out.head_stride;
        const bool joined = !TWO && n > 1;
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
          unsigned x[32];
          tm_load32(x, tm_o[w] + lanes + c);
          tm_loaded();
          float o[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(x[i]) * unit;
          if (joined && other != 0.f) {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] += ex[(c + i) * 128 + tid] * other;
          }
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (!have || c + i >= a.c.head_dim) break;
            if (whole) {
              const float y[8] = {o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv, o[i + 4] * inv, o[i + 5] * inv, o[i + 6] * inv, o[i + 7] * inv};
              if (a.out.type == KVR_BF16) store8<KVR_BF16>(dst + (c + i) * 2, y); else store8<KVR_F16>(dst + (c + i) * 2, y);
            } else {
              const float y[8] = {o[i], o[i + 1], o[i + 2], o[i + 3], o[i + 4], o[i + 5], o[i + 6], o[i + 7]};
              store8<KVR_F32>(reinterpret_cast<char *>(a.part_o + place * a.c.head_dim + c + i), y);
            }
          }
          __syncwarp();
        }
        if (have) {
          if (!whole) a.part_ml[place] = make_float2(top, sum);
          else if (a.lse) a.lse[(long long)(len.first + t_row) * a.q_heads + q_head] = sum == 0.f ? -INFINITY : top * 0.69314718f + logf(sum);
        }
      }
      if (!TWO) ok = join();             // the exchange has been read: Q's place may be written again
      again = next_piece(a, piece, last);
    }
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tm) : "memory");
  if (threadIdx.x == 0 && gave_up_word) report(a.b.status, KVR_DEV_GAVE_UP);
}

template <int FMT, int DP, bool TWO>
cudaError_t launch_tiles(const AttendArgs &a, cudaStream_t s) {
  static const cudaError_t set = cudaFuncSetAttribute(attend_tiles_kernel<FMT, DP, TWO>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileShape<FMT, DP>::kBytes);
  if (set != cudaSuccess) return set;
  attend_tiles_kernel<FMT, DP, TWO><<<a.ctas, kTileThreads, TileShape<FMT, DP>::kBytes, s>>>(a);
  return cudaGetLastError();
}
template <int FMT>
cudaError_t launch_tiles(const AttendArgs &a, cudaStream_t s) {
  if (a.c.head_dim <= 64) return a.row_tile > 128 ? launch_tiles<FMT, 64, true>(a, s) : launch_tiles<FMT, 64, false>(a, s);
  return a.row_tile > 128 ? launch_tiles<FMT, 128, true>(a, s) : launch_tiles<FMT, 128, false>(a, s);
}

}  // namespace
}  // namespace kvr
