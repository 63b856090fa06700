// Attention for few query rows a KV head over a 4-bit cache.  The products and the chunks of 16 keys are those of the row kernel
// (kvr_attend_rows.cuh): S^T = K Q^T and O^T = V^T P^T by mma.sync, the cache as the left operand.  What differs is how the cache gets to them, for 4 bits
// leave half as many cycles for a key.
//
// A warp of its own brings the keys of a stage for all heads of the CTA's group: TMA boxes of whole tokens (a group's records side by
// side, K and V), or, for block sizes that are no multiple of 8, a bulk copy for each token.  The warps of the heads spend nothing on addresses.  A
// stage's rows stand `stride` bytes apart, 32 more than a multiple of 128 where records are many (the boxes are wider than the rows):
// then the rows that a read looks at (four keys, 32 bytes of each) fall into different banks, with keys 4 to 7 of each 8 swapped in pairs.
//
// An element is widened to code times its group's scale, exactly: a conversion of two codes and a product of two f16.  The head's
// scale multiplies the score (K) or the probability (V).  Probability times scale is rounded to f16, for the matrix instructions take no more: by up to
// 2^-11 of it, which comes to 2.0e-4 of an output over 8k random keys, a twentieth of a bf16 step.  So one bf16 output in ten, the small ones most, falls on the
// other side of a rounding (8.6e-4 over all, against fp32 probabilities; from 64 bits 1.66e-3 instead of 1.65e-3).  Two products, with the upper and the
// lower half of the bits, would have them all at twice the instructions of the second product.  No pattern of bits is widened to NaN or infinity (a NaN lies in the head's scale
// alone), so what a row does not see needs no look at V.
//
// Eight warps share the heads, at 168 registers each (16 warps of 96 spill in the loop: 290 against 280 us, two tiles of rows 150 against 100), and take
// 48 keys a turn (32 of 128 channels: 300 us; 64: 287), so that the maximum, the votes and the barriers come once for three chunks.
//
// Measured, 8 KV heads of 128.  8 requests of 128k, one token of 4 query heads: 1.34 GB in 279 to 285 us, 4.7 TB/s (72 % of a copy; the algorithm's
// bytes without the padding 198 us).  The same loads and waits without the arithmetic take 244 us, the arithmetic over
// zeros with nothing brought 272: the arithmetic bounds it, and no pipe is full (ALU 43 %, 0.52 instructions a cycle and scheduler from two
// warps, 299 instructions for a chunk).  32 requests of 8k: 88 us, of which 20 to 25 are the start
// (lengths, table, first box: 5 us), pieces handed in and joined.  One request of 333 tokens from a cold cache: 14 us.
#pragma once
#include "kvr_attend_common.cuh"

namespace kvr {
namespace {

// ---- barriers and boxes
// A warp's wait.  One that runs out (after `polls`) sets the flag and goes on like one that did not, on whatever is there, as do all later
// ones at once: the heads' warps do not leave their loops early, so that barriers between them always meet.
__device__ __forceinline__ void bar4_wait(unsigned bar, unsigned parity, volatile int *gave_up, unsigned polls) {
  unsigned spin = 0;
  while (!bar_try(bar, parity)) {
    if (++spin >= polls) *gave_up = 1;
    if ((spin & 15) == 0 && *gave_up) break;
  }
  __syncwarp();
}
__device__ __forceinline__ void box4_load(unsigned dst, const CUtensorMap *map, unsigned bar, int x, int row, int block, int plane) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(row), "r"(block), "r"(plane) : "memory");
}
__device__ __forceinline__ void row4_load(unsigned dst, const char *src, int bytes, unsigned bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void product4(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ unsigned transpose4(unsigned v) {
  unsigned r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ unsigned times(unsigned x, unsigned scale) {
  unsigned r;
  asm("mul.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(scale));
  return r;
}
template <int BYTE>
__device__ __forceinline__ unsigned widen_times(unsigned w, unsigned scale) { return times(widen_e2m1<BYTE>(w), scale); }

// Reads of shared memory, by address; volatile, so that they stay between the barriers.
__device__ __forceinline__ unsigned lds1(unsigned at) { unsigned r; asm volatile("ld.shared.u8 %0, [%1];" : "=r"(r) : "r"(at)); return r; }
__device__ __forceinline__ unsigned lds4(unsigned at) { unsigned r; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(at)); return r; }
__device__ __forceinline__ uint2 lds8(unsigned at) { uint2 r; asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(at)); return r; }
__device__ __forceinline__ uint4 lds16(unsigned at) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at));
  return r;
}

constexpr int kMaxStages4 = 16;

// The rows of a segment from its pieces of n CTAs c, c + step, ...: to the output, or (fold) to the first one's place.  A thread 4 channels of
// a row, 8 pieces' loads under way at a time.  Out of line: the loop's registers are the products'.
__device__ __noinline__ void join4(const AttendArgs &a, const Piece &p, const Cut &cut, int c, int step, int n, bool fold, int rows, int heads, int threads) {
  constexpr int kAhead = 8;
  const int quads = a.c.head_dim >> 2, items = rows * heads * quads;
  const long long stride = (long long)step * 2 * a.group_heads * a.row_tile;     // rows from one piece to the next
  // the first CTA of a segment may hold it as its second piece, all others as their first
  const long long second = c == cut.c0 && cut.which0 ? (long long)a.group_heads * a.row_tile : 0;
#pragma unroll 1
  for (int i = threadIdx.x; i < items; i += threads) {
    const int both = i / quads, d = (i - both * quads) * 4, lh = both / rows, row = both - lh * rows;
    const long long at = ((long long)c * 2 * a.group_heads + lh) * a.row_tile + row;
    float m = -INFINITY, l = 0.f, o[4] = {};
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += kAhead) {
      float2 ml[kAhead];
      float4 x[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + k < n) {
          const long long from = at + (k0 + k) * stride + (k0 + k == 0 ? second : 0);
          ml[k] = __ldcg(a.part_ml + from);
          x[k] = __ldcg(reinterpret_cast<const float4 *>(a.part_o + from * a.c.head_dim + d));
        }
      }
      float best = m;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) best = fmaxf(best, ml[k].x);
      const float was = m == best ? 1.f : exp2_fast(m - best);             // both -infinity: pieces of an empty row
      l *= was;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= was;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float f = ml[k].x == best ? 1.f : exp2_fast(ml[k].x - best);
        l += ml[k].y * f;
        o[0] += x[k].x * f; o[1] += x[k].y * f; o[2] += x[k].z * f; o[3] += x[k].w * f;
      }
      m = best;
    }
    if (fold) {
      *reinterpret_cast<float4 *>(a.part_o + (at + second) * a.c.head_dim + d) = make_float4(o[0], o[1], o[2], o[3]);
      continue;                        // maximum and sum are read by other threads too: fold4
    }
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN;
    const int t = (int)a.group.div(p.row0 + row), q_head = (p.head_group * a.group_heads + lh) * (int)a.group.d + (p.row0 + row - t * (int)a.group.d);
    char *dst = a.out.data + (long long)(p.len.first + t) * a.out.token_stride + (long long)q_head * a.out.head_stride + d * 2;
    uint2 w;
    if (a.out.type == KVR_BF16) w = make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    else w = make_uint2(pack_f16(o[0] * inv, o[1] * inv), pack_f16(o[2] * inv, o[3] * inv));
    *reinterpret_cast<uint2 *>(dst) = w;
    if (a.lse && d == 0) a.lse[(long long)(p.len.first + t) * a.q_heads + q_head] = l == 0.f ? -INFINITY : m * 0.69314718f + logf(l);
  }
}

// Behind join4 (fold), when all its threads are through: the rows' maxima and sums.
__device__ __noinline__ void fold4(const AttendArgs &a, const Cut &cut, int c, int step, int n, int rows, int heads, int threads) {
  const long long stride = (long long)step * 2 * a.group_heads * a.row_tile;
  const long long second = c == cut.c0 && cut.which0 ? (long long)a.group_heads * a.row_tile : 0;
  for (int i = threadIdx.x; i < rows * heads; i += threads) {
    const int lh = i / rows;
    const long long at = ((long long)c * 2 * a.group_heads + lh) * a.row_tile + (i - lh * rows);
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int k = 0; k < n; ++k) {
      const float2 ml = __ldcg(a.part_ml + at + k * stride + (k == 0 ? second : 0));
      const float best = fmaxf(m, ml.x);
      l = l * (m == best ? 1.f : exp2_fast(m - best)) + ml.y * (ml.x == best ? 1.f : exp2_fast(ml.x - best));
      m = best;
    }
    a.part_ml[at + second] = make_float2(m, l);
  }
}

// EXACT: head_dim is DP, so that the scales' place is known.
template <int DP, int NT, bool EXACT>
__global__ void __launch_bounds__((kRows4Warps + 1) * 32, 1)
attend_rows4_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Rows4 r4, const __grid_constant__ CUtensorMap map) {
  constexpr int kTiles = DP / 16, kChunks = rows4_chunks(DP, NT), kWide = DP / 64, kTails = DP == 256 ? 2 : 1;
  constexpr float kLazy = 4.f;         // as in the row kernel
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ unsigned scratch[39];
  __shared__ __align__(8) unsigned long long full[kMaxStages4], empty[kMaxStages4];
  __shared__ int last_in, gave_up_word;
  __shared__ Piece pieces[kRows4Warps];     // of the heads' warps, whose registers are the products'
  volatile int *gave_up = &gave_up_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const int slices = r4.slices, stride = r4.stride, warps = a.group_heads * slices, stage_keys = 16 * kChunks * slices;
  const int plane_bytes = stage_keys * stride, stage_bytes = 2 * plane_bytes;

  Shares shares;
  Piece start;
  if (!find_share(a, scratch, shares, start.r, start.base, start.len)) return;
  const unsigned first = shares.first(blockIdx.x), last = shares.first(blockIdx.x + 1);
  start.unit = first;
  if (!open_piece(a, start, last)) return;     // an opening alone
  if (threadIdx.x == 0) {
    gave_up_word = a.polls == 0;
    for (int i = 0; i < r4.stages; ++i) { bar_init(shared_at(&full[i]), 1); bar_init(shared_at(&empty[i]), warps); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp < warps && lane == 0) pieces[warp] = start;
  __syncthreads();
  // stages of a piece
  const int unit_stages = (int)a.unit.d / stage_keys;
  auto stage_end = [&](const Piece &p) { return min(p.end * unit_stages, (p.len.keys + stage_keys - 1) / stage_keys); };

  if (warp == warps) {
    // ---- loads
    int stage = 0, t = start.begin * unit_stages, end = stage_end(start);
    unsigned round = 0;                // of the ring
    bool more = true;
    // Ids of the blocks that the boxes of a piece lie in, a lane a box: of boxes id_base .. + 31, and of the 32 behind them, on their way while
    // those are used.
    int id_base = 0, ids = 0, later_ids = 0;
    auto fetch_ids = [&](int box) {
      const int token = (box + lane) * r4.box_rows;
      return token < start.len.keys ? __ldg(a.b.tables + (long long)start.r * a.b.table_stride + a.bs.div((unsigned)token)) : 0;
    };
    auto first_ids = [&]() {
      id_base = t * stage_keys / r4.box_rows;
      ids = fetch_ids(id_base);
      later_ids = fetch_ids(id_base + 32);
    };
    if (r4.box_rows) first_ids();
    while (more) {
      const int key0 = t * stage_keys, keys = min(stage_keys, start.len.keys - key0), x0 = start.head_group * a.group_heads * a.c.head_bytes;
      unsigned char *st = smem + stage * stage_bytes;
      const unsigned bar = shared_at(&full[stage]);
      if (round) bar4_wait(shared_at(&empty[stage]), (round - 1) & 1, gave_up, a.polls);
      if (__any_sync(0xffffffffu, *gave_up != 0)) break;     // nothing more is brought into places that may be in use
      // K and V of up to 32 pieces of the stage, a lane a piece: brought by bring() where its block is known, zeros where not.  All of the stage's bytes
      // are expected by the one arrival, which comes with its last pieces.
      auto bring_all = [&](bool in, bool known, unsigned char *to, int bytes, bool last_ones, auto bring) {
        if (in && !known) {
          report(a.b.status, KVR_DEV_BAD_BLOCK);
          for (int i = 0; i < bytes; i += 16)
            *reinterpret_cast<uint4 *>(to + i) = *reinterpret_cast<uint4 *>(to + plane_bytes + i) = make_uint4(0, 0, 0, 0);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();                  // a vote orders no memory: the zeros go before lane 0's arrival
        const unsigned got = __popc(__ballot_sync(0xffffffffu, known));
        if (lane == 0) {
          if (last_ones) bar_expect(bar, got * 2 * bytes);
          else asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(got * 2 * bytes) : "memory");
        }
        __syncwarp();
        if (known) bring();
        __syncwarp();
      };
      if (r4.box_rows) {
        const int boxes = min(stage_keys, keys + r4.box_rows - 1) / r4.box_rows, box0 = key0 / r4.box_rows;
        for (int b0 = 0; b0 < boxes; b0 += 32) {
          if (box0 + b0 >= id_base + 32) {
            id_base += 32;
            ids = later_ids;
            later_ids = fetch_ids(id_base + 32);
          }
          const int box = b0 + lane, at = box0 + box - id_base, token = key0 + box * r4.box_rows;
          const int now = __shfl_sync(0xffffffffu, ids, at & 31), then = __shfl_sync(0xffffffffu, later_ids, at & 31), id = at < 32 ? now : then;
          unsigned char *to = st + box * r4.box_bytes;
          bring_all(box < boxes, box < boxes && (unsigned)id < (unsigned)a.c.num_blocks, to, r4.box_bytes, b0 + 32 >= boxes, [&] {
            const int row = token - (int)a.bs.div((unsigned)token) * (int)a.bs.d;
            box4_load(shared_at(to), &map, bar, x0 >> 3, row, id, 0);
            box4_load(shared_at(to + plane_bytes), &map, bar, x0 >> 3, row, id, 1);
          });
        }
      } else {
        const int bytes = min(a.group_heads * a.c.head_bytes, a.c.kv_heads * a.c.head_bytes - x0);
        for (int k0 = 0; k0 < keys; k0 += 32) {
          const int key = k0 + lane;
          const long long off = key < keys ? token_offset(a.b, a.c, a.bs, start.r, key0 + key) : -1;
          unsigned char *to = st + key * stride;
          bring_all(key < keys, off >= 0, to, bytes, k0 + 32 >= keys, [&] {
            row4_load(shared_at(to), a.c.base + off + x0, bytes, bar);
            row4_load(shared_at(to + plane_bytes), a.c.base + off + a.c.v_offset + x0, bytes, bar);
          });
        }
      }
      if (++stage == r4.stages) { stage = 0; ++round; }
      if (++t == end) {
        more = next_piece(a, start, last);
        t = start.begin * unit_stages;
        end = stage_end(start);
        if (more && r4.box_rows) first_ids();
      }
    }
    // What has been asked for lands before the CTA ends, also where a wait has run out.
    for (int i = 0; i < r4.stages; ++i) {
      const unsigned asked = round + (i < stage);
      if (asked && !bar_settle(shared_at(&full[i]), (asked - 1) & 1)) *gave_up = 1;
    }
  } else {
    // ---- products and softmax
    const Piece &piece = pieces[warp];
    int slot = 0;                      // of the ring
    unsigned round = 0;
    auto meet = [&]() { asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory"); return true; };
    const int local_head = warp / slices, slice = warp - local_head * slices;
    float *merge = reinterpret_cast<float *>(smem + r4.stages * stage_bytes);
    const int swapped = gid ^ (gid >> 2), first_key = (2 * tig) ^ (tig >> 1), codes = EXACT ? DP / 2 : a.c.scale_offset;
    // what a lane reads: K's rows of key `swapped` and + 8, V's of four keys
    const unsigned k_first = shared_at(smem) + (slice * 16 * kChunks + swapped) * stride + local_head * a.c.head_bytes;
    const unsigned v_first = shared_at(smem) + plane_bytes + (slice * 16 * kChunks + first_key) * stride + local_head * a.c.head_bytes;
    const int v_step = tig < 2 ? stride : -stride;
    for (bool again = true; again;) {
      const Lengths &len = piece.len;
      const int context = len.context, head = piece.head_group * a.group_heads + local_head;
      const int rows = min(a.row_tile, len.fresh * (int)a.group.d - piece.row0);     // of this tile
      const bool live = head < a.c.kv_heads;
      // Q^T fragments: k-step (group of 64 channels w, s) has channels 64 w + 16 tig + 4 s + 0..3
      uint2 q[NT][kTiles];
      Pair q_scale[NT];                // of the rows whose scores this lane holds (tig * 2, + 1)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int row = piece.row0 + n * 8 + gid;
        const bool have = live && n * 8 + gid < rows;
        const int t = have ? (int)a.group.div(row) : 0, g = have ? row - t * (int)a.group.d : 0;
        const char *src = a.q.data + (long long)(len.first + t) * a.q.token_stride + (long long)((live ? head : 0) * (int)a.group.d + g) * a.q.head_stride;
        float top = 0.f;
        float x[kWide][16];
#pragma unroll
        for (int w = 0; w < kWide; ++w) {
          const int d = w * 64 + tig * 16;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float y[8] = {};
            if (have && d < a.c.head_dim) {
              if (a.q.type == KVR_BF16) load8<KVR_BF16>(src + (d + h * 8) * 2, y);
              else load8<KVR_F16>(src + (d + h * 8) * 2, y);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) { x[w][h * 8 + i] = y[i]; top = fmaxf(top, fabsf(y[i])); }
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // The row's largest element is brought to [2^8, 2^9) by a power of two, 2^(8 - e), and 2^e goes to the scores: 2^-8 of it meets the
        // unit of K's groups.  (Not quite so far where 2^e is below 2^-118; rows of zeros, subnormals and infinities stay as they are.)
        const unsigned e = __float_as_uint(top) >> 23, field = e >= 1 && e <= 253 ? min(262u - e, 253u) : 127u;
        const float down = __uint_as_float(field << 23), up = __uint_as_float((262u - field) << 23);
#pragma unroll
        for (int w = 0; w < kWide; ++w)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            q[n][w * 4 + s] = make_uint2(pack_f16(x[w][4 * s] * down, x[w][4 * s + 1] * down), pack_f16(x[w][4 * s + 2] * down, x[w][4 * s + 3] * down));
          }
        q_scale[n] = pair(a.scale_log2 * __shfl_sync(0xffffffffu, up, tig * 8), a.scale_log2 * __shfl_sync(0xffffffffu, up, tig * 8 + 4));
      }
      float o[kTiles][NT][4] = {};
      float top[NT][2], unit[NT][2];   // unit: of V's scales
      Pair base[NT], sum[NT];          // base: -top, 0 where that is infinite
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        top[n][0] = top[n][1] = -INFINITY;
        base[n] = sum[n] = pair(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 2; ++e) unit[n][e] = unit_first(n * 8 + tig * 2 + e < rows);
      }

      const int end = stage_end(piece);
#pragma unroll 1
      for (int t = piece.begin * unit_stages; t < end; ++t) {
        bar4_wait(shared_at(&full[slot]), round & 1, gave_up, a.polls);
        unsigned k_at = k_first + slot * stage_bytes, v_at = v_first + slot * stage_bytes;
        const int key0 = (t * slices + slice) * (16 * kChunks);
        const bool edge = key0 + 16 * kChunks > context;

        // S^T = K Q^T
        float s[kChunks][NT][4] = {}, v_scale[kChunks][2];
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
          uint4 tail[2];               // of K's records: the head's scale, groups 0 to 11
          unsigned more[2] = {};       // groups 12 to 15
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const unsigned row = k_at + (u * 16 + e * 8) * stride + codes;
            tail[e] = lds16(row);
            if constexpr (kTails == 2) more[e] = lds4(row + 16);
            v_scale[u][e] = __uint_as_float(lds4(row + plane_bytes));
          }
#pragma unroll
          for (int w = 0; w < kWide; ++w) {
            uint2 x[2];
            unsigned scale[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              x[e] = lds8(k_at + (u * 16 + e * 8) * stride + tig * 8 + w * 32);
              const unsigned four = w == 0 ? tail[e].y : w == 1 ? tail[e].z : w == 2 ? tail[e].w : more[e];
              scale[e] = (four >> (tig * 8) & 0x7fu) * 0x00800080u;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const unsigned xa = k < 2 ? x[0].x : x[0].y, xb = k < 2 ? x[1].x : x[1].y;
              const unsigned f[4] = {k & 1 ? widen_times<2>(xa, scale[0]) : widen_times<0>(xa, scale[0]), k & 1 ? widen_times<2>(xb, scale[1]) : widen_times<0>(xb, scale[1]),
                                     k & 1 ? widen_times<3>(xa, scale[0]) : widen_times<1>(xa, scale[0]), k & 1 ? widen_times<3>(xb, scale[1]) : widen_times<1>(xb, scale[1])};
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                product4(s[u][n], f, q[n][w * 4 + k].x, q[n][w * 4 + k].y);
              }
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float k_scale = __uint_as_float(tail[i].x);
              const float2 v = unpair(mul2(pair(s[u][n][2 * i], s[u][n][2 * i + 1]), mul2(q_scale[n], pair(k_scale, k_scale))));
              s[u][n][2 * i] = v.x; s[u][n][2 * i + 1] = v.y;
            }
        }
        if (__builtin_expect(edge, 0)) {                     // what a row does not see
#pragma unroll
          for (int u = 0; u < kChunks; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int j = key0 + u * 16 + swapped + i * 8 - context;         // among the new tokens
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  const int row = n * 8 + tig * 2 + e;
                  const bool seen = j < 0 || (j < len.fresh && row < rows && sees(a, len.first, (int)a.group.div(piece.row0 + row), j));
                  if (!seen) s[u][n][i * 2 + e] = -INFINITY;
                }
            }
        }

        // running maximum of each row, over the 8 lanes that share it
        float best[NT][2];
        bool moved = false;
        float big = fmaxf(v_scale[0][0], v_scale[0][1]);
#pragma unroll
        for (int u = 1; u < kChunks; ++u) big = max3(big, v_scale[u][0], v_scale[u][1]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = fmaxf(s[0][n][e], s[0][n][2 + e]);
#pragma unroll
            for (int u = 1; u < kChunks; ++u) m = max3(m, s[u][n][e], s[u][n][2 + e]);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            best[n][e] = m;
            moved = moved || m > top[n][e] + kLazy || big * unit[n][e] >= kUnitLimit;      // from -infinity: any score moves it
          }
        if (__builtin_expect(__any_sync(0xffffffffu, moved), 0)) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float f[2], less[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // the largest of V's scales that the row sees
              float own = 0.f;
#pragma unroll
              for (int u = 0; u < kChunks; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  if (s[u][n][i * 2 + e] != -INFINITY) own = fmaxf(own, v_scale[u][i]);
              own = fmaxf(own, __shfl_xor_sync(0xffffffffu, own, 4));
              own = fmaxf(own, __shfl_xor_sync(0xffffffffu, own, 8));
              own = fmaxf(own, __shfl_xor_sync(0xffffffffu, own, 16));
              less[e] = 1.f;
              if (own * unit[n][e] >= kUnitLimit) {
                less[e] = unit_of(own) * unit_back(unit[n][e]);
                unit[n][e] = unit_of(own);
              }
              const float was = top[n][e];
              if (best[n][e] > was + kLazy) top[n][e] = best[n][e];
              f[e] = was == top[n][e] ? 1.f : exp2_fast(was - top[n][e]);      // was = -infinity: 0
              less[e] *= f[e];
            }
            base[n] = pair(top[n][0] == -INFINITY ? 0.f : -top[n][0], top[n][1] == -INFINITY ? 0.f : -top[n][1]);
            sum[n] = mul2(sum[n], pair(f[0], f[1]));
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[t][n][i] *= less[i & 1];
          }
        }
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
          // P^T, as the right operand of the second product
          unsigned p[NT][2];
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float2 x = unpair(add2(pair(s[u][n][2 * i], s[u][n][2 * i + 1]), base[n]));
              const Pair y = pair(exp2_fast(x.x), exp2_fast(x.y));
              sum[n] = add2(sum[n], y);
              float2 v = unpair(mul2(y, mul2(pair(unit[n][0], unit[n][1]), pair(v_scale[u][i], v_scale[u][i]))));
              if (__builtin_expect(edge, 0)) {               // a scale that is not finite, at a key that the row does not see
                if (s[u][n][2 * i] == -INFINITY) v.x = 0.f;
                if (s[u][n][2 * i + 1] == -INFINITY) v.y = 0.f;
              }
              p[n][i] = transpose4(pack_f16(v.x, v.y));
            }
          // O^T += V^T P^T.  The lane's keys are rows 2 tig, 2 tig + 1, + 8, + 9 of S^T, its channels gid * DP / 8 + 0 .. DP / 8 - 1.  Codes of two
          // keys at one channel are brought into one byte: those of even channels, then of odd ones.
          constexpr int kWords = DP / 64;
          unsigned w[4][kWords], scale[2][kTails];           // of keys 0 and 1, 2 and 3
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const unsigned row = v_at + (j & 1 ? v_step : 0) + (u * 16 + (j >> 1) * 8) * stride;
            if constexpr (DP == 64) {
              w[j][0] = lds4(row + gid * 4);
            } else if constexpr (DP == 128) {
              const uint2 x = lds8(row + gid * 8);
              w[j][0] = x.x; w[j][kWords - 1] = x.y;
            } else {
              const uint4 x = lds16(row + gid * 16);
              w[j][0] = x.x; w[j][1 % kWords] = x.y; w[j][2 % kWords] = x.z; w[j][3 % kWords] = x.w;
            }
#pragma unroll
            for (int g = 0; g < kTails; ++g) {
              const unsigned byte = lds1(row + (DP == 64 ? gid >> 1 : gid * kTails) + codes + 4 + g);
              if (j & 1) scale[j >> 1][g] = ((scale[j >> 1][g] | byte << 16) << 7) & 0x3f803f80u; else scale[j >> 1][g] = byte;
            }
          }
#pragma unroll
          for (int x = 0; x < kWords; ++x) {
            unsigned even[2], odd[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              even[h] = (w[2 * h][x] & 0x0f0f0f0fu) | (w[2 * h + 1][x] << 4 & 0xf0f0f0f0u);
              odd[h] = (w[2 * h][x] >> 4 & 0x0f0f0f0fu) | (w[2 * h + 1][x] & 0xf0f0f0f0u);
            }
            const unsigned s01 = scale[0][kTails == 2 ? x >> 1 & 1 : 0], s23 = scale[1][kTails == 2 ? x >> 1 & 1 : 0];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              auto of = [&](unsigned word) { return b == 0 ? widen_e2m1<0>(word) : b == 1 ? widen_e2m1<1>(word) : b == 2 ? widen_e2m1<2>(word) : widen_e2m1<3>(word); };
              const unsigned f[4] = {times(of(even[0]), s01), times(of(odd[0]), s01), times(of(even[1]), s23), times(of(odd[1]), s23)};
#pragma unroll
              for (int n = 0; n < NT; ++n) product4(o[x * 4 + b][n], f, p[n][0], p[n][1]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) bar_arrive(shared_at(&empty[slot]));
        if (++slot == r4.stages) { slot = 0; ++round; }
      }

      // ---- the piece's result
      float l[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 both = unpair(sum[n]);
        l[n][0] = both.x; l[n][1] = both.y;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 4);
          l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 8);
          l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 16);
        }
      }
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][n][i] = o[t][n][i] * unit_back(unit[n][i & 1]) * kGroupUnit;
      if (slices > 1) {
        // The slices of a head are joined through shared memory in slice order: first the maxima and sums of all, then the accumulators, a
        // quarter of one n-tile at a time, scaled to the common maximum.
        constexpr int kPart = kTiles / 4;
        float2 *ml = reinterpret_cast<float2 *>(merge);      // [head][slice][n-tile][8 rows]
        float *parts = merge + warps * NT * 16;              // [head][slice - 1][kPart * 4][32]
        if (gid == 0) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) ml[(warp * NT + n) * 8 + tig * 2 + e] = make_float2(top[n][e], l[n][e]);
        }
        meet();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            // a lane takes slices gid and gid + 8 (of 16 at most); lanes of the same rows put theirs together
            float2 x[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
              x[k] = gid + 8 * k < slices ? ml[((local_head * slices + gid + 8 * k) * NT + n) * 8 + tig * 2 + e] : make_float2(-INFINITY, 0.f);
            float m = fmaxf(x[0].x, x[1].x);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            float all = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k) all += x[k].y * (x[k].x == m ? 1.f : exp2_fast(x[k].x - m));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
            const float f = top[n][e] == m ? 1.f : exp2_fast(top[n][e] - m);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
              o[t][n][e] *= f;
              o[t][n][2 + e] *= f;
            }
            top[n][e] = m;
            l[n][e] = all;
          }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int t0 = 0; t0 < kTiles; t0 += kPart) {
            float *mine = parts + (local_head * (slices - 1) + slice - 1) * (kPart * 128) + lane;
            if (slice > 0) {
#pragma unroll
              for (int t = 0; t < kPart; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[(t * 4 + i) * 32] = o[t0 + t][n][i];
            }
            meet();
            if (slice == 0) {
#pragma unroll 4
              for (int k = 1; k < slices; ++k) {
                const float *other = parts + (local_head * (slices - 1) + k - 1) * (kPart * 128) + lane;
#pragma unroll
                for (int t = 0; t < kPart; ++t)
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[t0 + t][n][i] += other[(t * 4 + i) * 32];
              }
            }
            meet();
          }
      }
      if (slice == 0 && live) {
        const bool whole = piece.begin == 0 && piece.end == len.units;
        const long long slot = ((long long)blockIdx.x * 2 + (piece.unit == first ? 0 : 1)) * a.group_heads + local_head;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int row = n * 8 + tig * 2 + e;
            if (row >= rows) continue;
            const int t_row = (int)a.group.div(piece.row0 + row);
            const int q_head = head * (int)a.group.d + (piece.row0 + row - t_row * (int)a.group.d);
            const float inv = !whole ? 1.f : l[n][e] > 0.f ? 1.f / l[n][e] : l[n][e] == 0.f ? 0.f : NAN;
            char *dst = a.out.data + (long long)(len.first + t_row) * a.out.token_stride + (long long)q_head * a.out.head_stride;
            float *part = a.part_o + (slot * a.row_tile + row) * a.c.head_dim;
            // a lane's channels lie side by side, 8 at a time
#pragma unroll
            for (int t = 0; t < kTiles; t += 4) {
              const int d = gid * (DP / 8) + t * 2;
              if (d >= a.c.head_dim) continue;
              const float y[8] = {o[t][n][e] * inv, o[t][n][2 + e] * inv, o[t + 1][n][e] * inv, o[t + 1][n][2 + e] * inv,
                                  o[t + 2][n][e] * inv, o[t + 2][n][2 + e] * inv, o[t + 3][n][e] * inv, o[t + 3][n][2 + e] * inv};
              if (!whole) store8<KVR_F32>(reinterpret_cast<char *>(part + d), y);
              else if (a.out.type == KVR_BF16) store8<KVR_BF16>(dst + d * 2, y);
              else store8<KVR_F16>(dst + d * 2, y);
            }
            if (gid == 0) {
              if (!whole) a.part_ml[slot * a.row_tile + row] = make_float2(top[n][e], l[n][e]);
              else if (a.lse) a.lse[(long long)(len.first + t_row) * a.q_heads + q_head] = l[n][e] == 0.f ? -INFINITY : top[n][e] * 0.69314718f + logf(l[n][e]);
            }
          }
      }
      if (piece.begin != 0 || piece.end != len.units) {
        const int heads = min(a.group_heads, a.c.kv_heads - piece.head_group * a.group_heads);
        hand_in(a, piece, shares, meet, &last_in, warp, lane, [&](const Cut &cut, int c, int step, int n, bool fold) {
          join4(a, piece, cut, c, step, n, fold, rows, heads, warps * 32);
          if (!fold) return;
          meet();
          fold4(a, cut, c, step, n, rows, heads, warps * 32);
        });
      }
      __syncwarp();
      if (lane == 0) {
        Piece next = piece;
        again = next_piece(a, next, last);
        pieces[warp] = next;
      }
      __syncwarp();                    // nor does a shuffle: the piece goes before what the other lanes read of it
      again = __shfl_sync(0xffffffffu, again, 0);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && gave_up_word) report(a.b.status, KVR_DEV_GAVE_UP);
}

template <int DP, int NT, bool EXACT>
cudaError_t launch_rows4(const AttendArgs &a, const Rows4 &r4, const CUtensorMap &map, cudaStream_t s) {
  const int bytes = r4.stages * 32 * rows4_chunks(DP, NT) * r4.slices * r4.stride + rows4_beside(DP, NT, a.group_heads, r4.slices);
  static OncePerDevice once;
  if (const cudaError_t e = allow_shared(once, attend_rows4_kernel<DP, NT, EXACT>, kRows4Shared)) return e;
  attend_rows4_kernel<DP, NT, EXACT><<<a.ctas, (a.group_heads * r4.slices + 1) * 32, bytes, s>>>(a, r4, map);
  return cudaGetLastError();
}
template <int DP>
cudaError_t launch_rows4(const AttendArgs &a, int tiles, const Rows4 &r4, const CUtensorMap &map, cudaStream_t s) {
  if (a.c.head_dim == DP) return tiles == 1 ? launch_rows4<DP, 1, true>(a, r4, map, s) : launch_rows4<DP, 2, true>(a, r4, map, s);
  return tiles == 1 ? launch_rows4<DP, 1, false>(a, r4, map, s) : launch_rows4<DP, 2, false>(a, r4, map, s);
}

}  // namespace
}  // namespace kvr
