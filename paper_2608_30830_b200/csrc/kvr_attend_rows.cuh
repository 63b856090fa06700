// Attention for few query rows a KV head (one token, small trees): bound by reading the cache.
//
// A warp owns one KV head and every `slices`-th chunk of 16 keys of its CTA's run; the CTA's warps take all heads of a
// group at the same keys, so a token's row is read by neighbours at the same time and scales (which lie behind the
// codes of all heads) come from L2 once.  Chunks go to shared memory by 16-byte asynchronous copies, STAGES deep and
// private to the warp: the main loop has no barrier between warps.
//
// Both products keep the cache as the left operand, m = 16: S^T[keys x rows] = K Q^T and O^T[channels x rows] = V^T P^T,
// so the query rows are n and come in steps of 8: one token of four query heads costs half of what rows as m = 16 would.
// S^T's fragment, packed and transposed 8 x 8 in registers (movmatrix), is the right operand of the second product.
//
// 8-bit codes become f16 in registers, exactly; k and m indices of the products are assigned to channels so that a
// lane's fragments are contiguous bytes (16 channels of a key).  A query row is scaled by a power of two into [1, 2)
// first (exact) and rounded to f16: elements down to 2^-14 of the row's largest keep 11 bits, which is all of a bf16 element, smaller
// ones an error of 2^-25 of the largest.  (f16 and not bf16, which codes would fit as well: e4m3 is widened to f16 by one instruction,
// and probabilities keep 11 bits.  tf32 would halve the rate.)  K's scale multiplies the score, V's scale the probability.
//
// Probabilities are rounded to the type of V's operand, bf16 or f16, for a product has both of one type.  Against 64 bits outputs of a bf16 cache are then
// off by 0.0022 (relative, root of the mean square; 32 requests of 8k) where rounding the output alone gives 0.0017; p in two parts would
// mean the second product twice.
//
// Measured, 8 KV heads of 128.  32 requests, median 8k tokens, one token of 4 query heads, bf16: 1.27 GB in 198 us, 6.4 TB/s (DRAM
// traffic is the algorithm's to 0.1 %): bound by memory.  8 requests of 128k, e4m3: 2.21 GB in 439 to 450 us, 5.0 TB/s: half the
// bytes a key, but each element is widened by the ALU, and two warps a scheduler issue in 46 % of the cycles (ALU 47 %): neither is
// full, each warp waits on its own chain.  One request of 333 tokens: 13.5 us, the chain of table, K, softmax, V and join.
#pragma once
#include "kvr_attend_common.cuh"

namespace kvr {
namespace {

template <bool TRANS>
__device__ __forceinline__ void load_matrix4(unsigned (&r)[4], unsigned addr) {
  if constexpr (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ unsigned transpose8(unsigned v) {
  unsigned r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
template <bool BF16>
__device__ __forceinline__ void product(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int FMT, int DP>
struct Shape {
  static constexpr bool kQuant = quantised(FMT);
  static constexpr int kWarps = rows_warps(DP);                          // heads and slices of a CTA
  static constexpr int kRow = DP * (kQuant ? 1 : 2);                     // bytes of a key's head
  static constexpr int kStageBytes = 2 * 16 * kRow + (kQuant ? 128 : 0); // K, V, scales
  static constexpr int kFit = 196608 / kWarps / kStageBytes;
  static constexpr int kStages = kFit > 6 ? 6 : kFit;                    // 3 to 6
};

// where 16-byte column `chunk` of key `key` of a chunk lies: spreads a lane pattern's reads over the banks
template <bool QUANT, int DP>
__device__ __forceinline__ int spread(int key, int chunk) {
  if constexpr (!QUANT) return key * (DP * 2) + ((chunk ^ (key & 7)) << 4);
  else if constexpr (DP == 64) return key * DP + ((chunk ^ (key >> 2)) << 4);
  else return key * DP + ((chunk ^ (((key >> 2) << 1) ^ ((key & 1) << 2))) << 4);
}

template <int FMT, int DP, int NT>
__global__ void __launch_bounds__(Shape<FMT, DP>::kWarps * 32, 1) attend_rows_kernel(const __grid_constant__ AttendArgs a, int slices) {
  using S = Shape<FMT, DP>;
  constexpr bool kQuant = S::kQuant, kBf16 = FMT == KVR_CACHE_BF16;
  constexpr int kStages = S::kStages, kRow = S::kRow, kChunks = kRow / 16, kTiles = DP / 16;
  // Chunks of 16 keys that a turn takes: two where registers allow it, so that one's chain of dependent steps runs beside the other's
  // and the maximum is looked for once.
  constexpr int kAtOnce = chunks_at_once(FMT, NT);
  static_assert(kStages >= 2 * kAtOnce, "");
  constexpr float kLazy = 4.f;         // a row's maximum moves only when a score passes it by 2^4: fewer rescales,
                                       // probabilities up to 16 (room in f16, see the scale of V below)
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ unsigned scratch[39];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const int local_head = warp / slices, slice = warp - local_head * slices;
  __shared__ int last_in;

  Shares shares;
  Piece piece;
  if (!find_share(a, scratch, shares, piece.r, piece.base, piece.len)) return;
  const unsigned first = shares.first(blockIdx.x), last = shares.first(blockIdx.x + 1);
  piece.unit = first;
  if (!open_piece(a, piece, last)) return;     // an opening alone

  const int unit_chunks = (int)a.unit.d / (16 * slices);     // of one warp
  unsigned char *ring = smem + warp * (kStages * S::kStageBytes);
  float *merge = reinterpret_cast<float *>(smem + (blockDim.x >> 5) * (kStages * S::kStageBytes));

  // chunks of a piece that hold keys: c = begin * unit_chunks ..., of which this warp's keys start at (c * slices + slice) * 16
  auto chunk_end = [&](const Piece &p) {
    const int have = (p.len.keys - slice * 16 + 16 * slices - 1) / (16 * slices);
    return min(p.end * unit_chunks, (max(have, 0) + kAtOnce - 1) / kAtOnce * kAtOnce);
  };

  // ---- loads: a second walk that runs ahead
  Piece ahead = piece;
  int load_c = ahead.begin * unit_chunks, load_end = chunk_end(ahead);
  bool more = true;
  auto settle = [&]() {                // to a piece with a chunk left
    while (more && load_c >= load_end) {
      more = next_piece(a, ahead, last);
      if (more) { load_c = ahead.begin * unit_chunks; load_end = chunk_end(ahead); }
    }
  };
  settle();
  // the table entry of the lane's key is fetched one chunk before it is needed
  int next_id = 0, next_j = 0;
  bool next_in = false;
  auto fetch_id = [&]() {
    if (!more) return;
    next_j = (load_c * slices + slice) * 16 + (lane & 15);
    next_in = next_j < ahead.len.keys;
    next_id = next_in ? __ldg(a.b.tables + (long long)ahead.r * a.b.table_stride + a.bs.div(next_j)) : 0;
  };
  fetch_id();
  auto load_chunk = [&](int stage) {
    if (more) {
      const bool known = (unsigned)next_id < (unsigned)a.c.num_blocks;
      if (!known) report(a.b.status, KVR_DEV_BAD_BLOCK);
      const int head = ahead.head_group * a.group_heads + local_head;
      const bool in = next_in && known && head < a.c.kv_heads;
      const int within = next_j - (int)a.bs.div(next_j) * (int)a.bs.d;
      const long long offset = in ? (long long)next_id * a.c.block_stride + (long long)within * a.c.row_bytes : 0;
      const unsigned valid = __ballot_sync(0xffffffffu, in);
      unsigned char *st = ring + stage * S::kStageBytes;
      const unsigned k_at = shared_at(st);
      const int column = head < a.c.kv_heads ? head * a.c.head_dim * (kQuant ? 1 : 2) : 0;
      const int used = a.c.head_dim * (kQuant ? 1 : 2) / 16;             // 16-byte columns of a head
      const char *base = a.c.base + column;
      constexpr int kKeysAtOnce = 32 / kChunks > 0 ? 32 / kChunks : 1;    // kChunks: 4, 8, 16 or 32
      const int chunk = lane % kChunks, sub = lane / kChunks;
#pragma unroll
      for (int i = 0; i < 16 / kKeysAtOnce; ++i) {
        const int key = i * kKeysAtOnce + sub;
        const long long off = __shfl_sync(0xffffffffu, offset, key);
        const bool v = (valid >> key & 1) && chunk < used;
        const char *src = base + off + (v ? chunk * 16 : 0);
        const unsigned dst = k_at + spread<kQuant, DP>(key, chunk);
        copy16(dst, src, v);
        copy16(dst + 16 * kRow, src + a.c.v_offset, v);
      }
      if constexpr (kQuant) {
        const char *src = a.c.base + offset + (in ? a.c.scale_offset + 4 * head : 0) + (lane >= 16 ? a.c.v_offset : 0);
        copy4(k_at + 32 * kRow + 4 * lane, src, in);
      }
      ++load_c;
      settle();
      fetch_id();
    }
    copy_commit();
  };
#pragma unroll
  for (int s = 0; s < kStages - kAtOnce; ++s) load_chunk(s);
  int stage = 0, load_stage = kStages - kAtOnce;

  // ---- pieces
  bool again = true;
  while (again) {
    const Lengths len = piece.len;
    const int head = piece.head_group * a.group_heads + local_head;
    const int rows = min(a.row_tile, len.fresh * (int)a.group.d - piece.row0);     // of this tile
    const bool live = head < a.c.kv_heads;
    // Q^T fragments: lane holds channels of row gid of every n-tile
    unsigned q[NT][kTiles][2];
    float q_scale[NT][2];              // of the rows whose scores this lane holds (tig * 2, + 1)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = piece.row0 + n * 8 + gid;
      const bool have = live && n * 8 + gid < rows;
      const int t = have ? (int)a.group.div(row) : 0, g = have ? row - t * (int)a.group.d : 0;
      const char *src = a.q.data + (long long)(len.first + t) * a.q.token_stride + (long long)((live ? head : 0) * (int)a.group.d + g) * a.q.head_stride;
      if constexpr (!kQuant) {
#pragma unroll
        for (int k = 0; k < kTiles; ++k) {
          const bool in = have && k * 16 < a.c.head_dim;
          q[n][k][0] = in ? *reinterpret_cast<const unsigned *>(src + (k * 16 + tig * 2) * 2) : 0u;
          q[n][k][1] = in ? *reinterpret_cast<const unsigned *>(src + (k * 16 + tig * 2 + 8) * 2) : 0u;
        }
        q_scale[n][0] = q_scale[n][1] = a.scale_log2;
      } else {
        // k-step (group of 64 channels, s): channels 64 * group + 16 * tig + 4 * s + 0..3
        float top = 0.f;
        float x[DP / 64][16];
#pragma unroll
        for (int w = 0; w < DP / 64; ++w) {
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
        // 2^-e with 2^e <= top < 2^(e+1), by the exponent's bits; rows of zeros, subnormals and infinities stay as they are
        const unsigned e = __float_as_uint(top) >> 23;
        const bool plain = e >= 1 && e <= 253;
        const float down = plain ? __uint_as_float((254u - e) << 23) : 1.f, up = plain ? __uint_as_float(e << 23) : 1.f;
#pragma unroll
        for (int w = 0; w < DP / 64; ++w)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            q[n][w * 4 + s][0] = pack_f16(x[w][4 * s] * down, x[w][4 * s + 1] * down);
            q[n][w * 4 + s][1] = pack_f16(x[w][4 * s + 2] * down, x[w][4 * s + 3] * down);
          }
#pragma unroll
        for (int i = 0; i < 2; ++i) q_scale[n][i] = a.scale_log2 * __shfl_sync(0xffffffffu, up, (tig * 2 + i) * 4);
      }
    }
    float o[kTiles][NT][4] = {};
    float top[NT][2], sum[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) top[n][0] = top[n][1] = -INFINITY, sum[n][0] = sum[n][1] = 0.f;
    float unit[NT][2];                 // of V's scales, by row
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) unit[n][e] = unit_first(n * 8 + tig * 2 + e < rows);
    bool odd = false;                  // this lane has found a code of V that is NaN
    // from this turn on chunks reach past the context, where some rows may not see all keys
    const int look_from = len.fresh > 1 || a.mask ? (len.context - slice * 16 + 16 * slices - 1) / (16 * slices) - kAtOnce : 1 << 30;

    const int c_end = chunk_end(piece);
    for (int c = piece.begin * unit_chunks; c < c_end; c += kAtOnce) {
      copy_wait<kStages - 2 * kAtOnce>();
      __syncwarp();
      unsigned char *st_of[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        load_chunk(load_stage);
        load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
        st_of[u] = ring + stage * S::kStageBytes;
        stage = stage + 1 == kStages ? 0 : stage + 1;
      }
      if constexpr (FMT == KVR_CACHE_E4M3) {
        // Codes of V that are NaN must not meet the zero probabilities of rows that do not see their key: set to zero here, and
        // to NaN the sums of the rows that do see it, at the piece's end (append stores no such code).  Done as for 16 bits below, in
        // the loop and channel by channel, the registers it takes cost long caches 6 % (435 against 463 us); so 1 %.
        if (c >= look_from) {
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u)
            for (int i = max(len.context - ((c + u) * slices + slice) * 16, 0) * kChunks + lane; i < 16 * kChunks; i += 32) {
              unsigned *w = reinterpret_cast<unsigned *>(st_of[u] + 16 * kRow + i * 16);        // a key's columns lie side by side
              const uint4 x = *reinterpret_cast<const uint4 *>(w);
              if (!(nan_codes(x.x) | nan_codes(x.y) | nan_codes(x.z) | nan_codes(x.w))) continue;
              odd = true;
#pragma unroll 1
              for (int k = 0; k < 4; ++k) w[k] &= ~(nan_codes(w[k]) / 0x80u * 0xffu);
            }
          __syncwarp();
        }
      }
      // the lane's keys (rows gid and gid + 8 of S^T)
      const int key_a = kQuant ? (gid >> 1) * 4 + (gid & 1) : gid, key_b = kQuant ? key_a + 2 : gid + 8;

      // S^T = K Q^T; the chunks' products in turn, for a product waits for the one before it
      float s[kAtOnce][NT][4] = {}, v_scale[kAtOnce][2];
      if constexpr (!kQuant) {
#pragma unroll
        for (int k = 0; k < kTiles; ++k)
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            unsigned f[4];
            load_matrix4<false>(f, shared_at(st_of[u]) + spread<false, DP>((lane & 7) + ((lane >> 3) & 1) * 8, k * 2 + (lane >> 4)));
#pragma unroll
            for (int n = 0; n < NT; ++n) product<kBf16>(s[u][n], f, q[n][k][0], q[n][k][1]);
          }
      } else {
#pragma unroll
        for (int w = 0; w < DP / 64; ++w) {
          uint4 x[kAtOnce], y[kAtOnce];
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            x[u] = *reinterpret_cast<const uint4 *>(st_of[u] + spread<true, DP>(key_a, w * 4 + tig));
            y[u] = *reinterpret_cast<const uint4 *>(st_of[u] + spread<true, DP>(key_b, w * 4 + tig));
          }
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
              const unsigned xa = k == 0 ? x[u].x : k == 1 ? x[u].y : k == 2 ? x[u].z : x[u].w, yb = k == 0 ? y[u].x : k == 1 ? y[u].y : k == 2 ? y[u].z : y[u].w;
              const unsigned f[4] = {widen<FMT, false>(xa), widen<FMT, false>(yb), widen<FMT, true>(xa), widen<FMT, true>(yb)};
#pragma unroll
              for (int n = 0; n < NT; ++n) product<false>(s[u][n], f, q[n][w * 4 + k][0], q[n][w * 4 + k][1]);
            }
        }
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        unsigned char *st = st_of[u];
        const int key0 = ((c + u) * slices + slice) * 16;
        float k_scale[2] = {1.f, 1.f};
        v_scale[u][0] = v_scale[u][1] = 1.f;
        if constexpr (kQuant) {
          const float *sc = reinterpret_cast<const float *>(st + 32 * kRow);
          k_scale[0] = sc[key_a]; k_scale[1] = sc[key_b];
          v_scale[u][0] = sc[16 + key_a]; v_scale[u][1] = sc[16 + key_b];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[u][n][i] *= kQuant ? q_scale[n][i & 1] * k_scale[i >> 1] : q_scale[n][i & 1];

        // what a row does not see
        if (key0 + 16 > len.context) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int j = key0 + (i ? key_b : key_a) - len.context;      // among the new tokens
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
      }

      // running maximum of each row, over the 8 lanes that share it
      float best[NT][2];
      bool moved = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float m = fmaxf(s[0][n][e], s[0][n][2 + e]);
          if constexpr (kAtOnce == 2) m = fmaxf(m, fmaxf(s[kAtOnce - 1][n][e], s[kAtOnce - 1][n][2 + e]));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
          best[n][e] = m;
          moved = moved || m > top[n][e] + kLazy;                        // from -infinity: any score moves it
        }
      if constexpr (kQuant) {
        float big = fmaxf(v_scale[0][0], v_scale[0][1]);
        if constexpr (kAtOnce == 2) big = fmaxf(big, fmaxf(v_scale[kAtOnce - 1][0], v_scale[kAtOnce - 1][1]));
        bool far = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) far = far || big * unit[n][e] >= kUnitLimit;
        if (__any_sync(0xffffffffu, far)) {
          // the largest that each row sees
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float own = 0.f;
#pragma unroll
              for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  if (s[u][n][i * 2 + e] != -INFINITY) own = fmaxf(own, v_scale[u][i]);
              own = fmaxf(own, __shfl_xor_sync(0xffffffffu, own, 4));
              own = fmaxf(own, __shfl_xor_sync(0xffffffffu, own, 8));
              own = fmaxf(own, __shfl_xor_sync(0xffffffffu, own, 16));
              if (own * unit[n][e] >= kUnitLimit) {
                const float less = unit_of(own) * unit_back(unit[n][e]);
                unit[n][e] = unit_of(own);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                  o[t][n][e] *= less;
                  o[t][n][2 + e] *= less;
                }
              }
            }
        }
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float was = top[n][e];
            if (best[n][e] > was + kLazy) top[n][e] = best[n][e];
            const float f = was == top[n][e] ? 1.f : exp2_fast(was - top[n][e]);   // was = -infinity: 0
            sum[n][e] *= f;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
              o[t][n][e] *= f;
              o[t][n][2 + e] *= f;
            }
          }
      }
      // P^T, as the right operand of the second product
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        unsigned char *st = st_of[u];
        const unsigned v_at = shared_at(st) + 16 * kRow;
        const int key0 = ((c + u) * slices + slice) * 16;
        unsigned p[NT][2];
        // channels of 16-bit V that are not finite must not reach rows that do not see them (0 * infinity): see below
        float pf[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float m = top[n][i & 1];
            const float x = s[u][n][i] == -INFINITY ? 0.f : exp2_fast(s[u][n][i] - m);
            sum[n][i & 1] += x;
            pf[n][i] = x;
          }
        if constexpr (kQuant) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) pf[n][i] = s[u][n][i] == -INFINITY ? 0.f : pf[n][i] * (v_scale[u][i >> 1] * unit[n][i & 1]);
        } else if (key0 + 16 > len.context && (len.fresh > 1 || a.mask)) {
          // lanes 2k and 2k + 1 look through key k's row of V
          bool odd = false;
#pragma unroll
          for (int i = 0; i < kChunks / 2; ++i) {
            const uint4 x = *reinterpret_cast<const uint4 *>(st + 16 * kRow + spread<false, DP>(lane >> 1, (lane & 1) * (kChunks / 2) + i));
            const unsigned w[4] = {x.x, x.y, x.z, x.w};
            constexpr unsigned kExp = kBf16 ? 0x7f80u : 0x7c00u;
#pragma unroll
            for (int j = 0; j < 4; ++j) odd = odd || (w[j] & kExp) == kExp || (w[j] >> 16 & kExp) == kExp;
          }
          unsigned keys = __ballot_sync(0xffffffffu, odd);
          keys |= keys >> 1;
          keys &= 0x55555555u;           // bit 2k: key k
          while (keys) {
            const int key = (__ffs(keys) - 1) >> 1;
            keys &= keys - 1;
            // added row by row, only where the row sees the key; then the key leaves the product
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float w[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                w[e] = __shfl_sync(0xffffffffu, key < 8 ? pf[n][e] : pf[n][2 + e], (key & 7) * 4 + tig);
                if (gid == (key & 7)) { if (key < 8) pf[n][e] = 0.f; else pf[n][2 + e] = 0.f; }
              }
#pragma unroll
              for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const int d = t * 16 + h * 8 + gid;
                  const unsigned char *at = st + 16 * kRow + spread<false, DP>(key, d >> 3) + (d & 7) * 2;
                  const float v = load1<kBf16 ? KVR_BF16 : KVR_F16>(reinterpret_cast<const char *>(at));
#pragma unroll
                  for (int e = 0; e < 2; ++e)
                    if (w[e] > 0.f) o[t][n][h * 2 + e] += w[e] * v;
                }
            }
            __syncwarp();
            for (int i = lane; i < kChunks; i += 32) *reinterpret_cast<uint4 *>(st + 16 * kRow + spread<false, DP>(key, i)) = make_uint4(0, 0, 0, 0);
          }
          __syncwarp();
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          p[n][0] = transpose8(kBf16 ? pack_bf16(pf[n][0], pf[n][1]) : pack_f16(pf[n][0], pf[n][1]));
          p[n][1] = transpose8(kBf16 ? pack_bf16(pf[n][2], pf[n][3]) : pack_f16(pf[n][2], pf[n][3]));
        }
        // O^T += V^T P^T
        if constexpr (!kQuant) {
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            unsigned f[4];
            load_matrix4<true>(f, v_at + spread<false, DP>((lane & 7) + (lane >> 4) * 8, t * 2 + ((lane >> 3) & 1)));
#pragma unroll
            for (int n = 0; n < NT; ++n) product<kBf16>(o[t][n], f, p[n][0], p[n][1]);
          }
        } else {
          // the lane's keys are 4 * tig + 0..3, its channels gid * DP / 8 + 0 .. DP / 8 - 1
          const unsigned char *v_tile = st + 16 * kRow;
          constexpr int kWords = DP / 32;                                  // 4 channels each
          unsigned w[4][kWords];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (DP == 64) {
              const uint2 x = *reinterpret_cast<const uint2 *>(v_tile + spread<true, DP>(tig * 4 + j, gid >> 1) + (gid & 1) * 8);
              w[j][0] = x.x; w[j][1] = x.y;
            } else {
#pragma unroll
              for (int h = 0; h < DP / 128; ++h) {
                const uint4 x = *reinterpret_cast<const uint4 *>(v_tile + spread<true, DP>(tig * 4 + j, gid * (DP / 128) + h));
                w[j][h * 4] = x.x; w[j][h * 4 + 1] = x.y; w[j][h * 4 + 2] = x.z; w[j][h * 4 + 3] = x.w;
              }
            }
          }
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            const int x = t >> 1;
            const unsigned k01 = __byte_perm(w[0][x], w[1][x], t & 1 ? 0x7362 : 0x5140), k23 = __byte_perm(w[2][x], w[3][x], t & 1 ? 0x7362 : 0x5140);
            const unsigned f[4] = {widen<FMT, false>(k01), widen<FMT, true>(k01), widen<FMT, false>(k23), widen<FMT, true>(k23)};
#pragma unroll
            for (int n = 0; n < NT; ++n) product<false>(o[t][n], f, p[n][0], p[n][1]);
          }
        }
      }
    }

    // ---- the piece's result
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], 4);
        sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], 8);
        sum[n][e] += __shfl_xor_sync(0xffffffffu, sum[n][e], 16);
      }
    if constexpr (kQuant) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][n][i] *= unit_back(unit[n][i & 1]);
    }
    if (FMT == KVR_CACHE_E4M3 && __any_sync(0xffffffffu, odd)) {
      // the new tokens among this warp's keys again, as they lie in the cache: a bit for each of the lane's channels
      unsigned nan[NT][2] = {};
#pragma unroll 1
      for (int c = piece.begin * unit_chunks; c < c_end; ++c)
#pragma unroll 1
        for (int j = max((c * slices + slice) * 16, len.context); j < min((c * slices + slice) * 16 + 16, len.keys); ++j) {
          const long long off = token_offset(a.b, a.c, a.bs, piece.r, j);
          const char *v = a.c.base + a.c.v_offset + (long long)head * a.c.head_dim + off;
          unsigned bits = 0;
#pragma unroll 1
          for (int d = gid * (DP / 8); d < min((gid + 1) * (DP / 8), a.c.head_dim) && off >= 0 && live; ++d)
            bits |= (unsigned)((v[d] & 0x7f) == 0x7f) << (d - gid * (DP / 8));
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int row = n * 8 + tig * 2 + e;
              if (row < rows && sees(a, len.first, (int)a.group.div(piece.row0 + row), j - len.context)) nan[n][e] |= bits;
            }
        }
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (nan[n][i & 1] >> (t * 2 + (i >> 1)) & 1) o[t][n][i] = NAN;
    }
    if (slices > 1) {
      // slices of a head are joined through shared memory, one n-tile at a time, in slice order
      constexpr int kPer = DP * 8 + 16;                                  // accumulators, then (maximum, sum) of 8 rows
      const int heads = blockDim.x / 32 / slices;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float *mine = merge + ((slice - 1) * heads + local_head) * kPer;
        if (slice > 0) {
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(t * 4 + i) * 32 + lane] = o[t][n][i];
          if (gid == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              mine[DP * 8 + (tig * 2 + e) * 2] = top[n][e];
              mine[DP * 8 + (tig * 2 + e) * 2 + 1] = sum[n][e];
            }
          }
        }
        __syncthreads();
        if (slice == 0) {
          for (int s = 1; s < slices; ++s) {
            const float *other = merge + ((s - 1) * heads + local_head) * kPer;
            float f[2], g[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float m2 = other[DP * 8 + (tig * 2 + e) * 2], l2 = other[DP * 8 + (tig * 2 + e) * 2 + 1];
              const float m = fmaxf(top[n][e], m2);
              f[e] = top[n][e] == m ? 1.f : exp2_fast(top[n][e] - m);
              g[e] = m2 == m ? 1.f : exp2_fast(m2 - m);
              if (m == -INFINITY) g[e] = 0.f;
              sum[n][e] = sum[n][e] * f[e] + l2 * g[e];
              top[n][e] = m;
            }
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[t][n][i] = o[t][n][i] * f[i & 1] + other[(t * 4 + i) * 32 + lane] * g[i & 1];
          }
        }
        __syncthreads();
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
          if (whole) {
            const float inv = sum[n][e] > 0.f ? 1.f / sum[n][e] : sum[n][e] == 0.f ? 0.f : NAN;
            char *dst = a.out.data + (long long)(len.first + t_row) * a.out.token_stride + (long long)q_head * a.out.head_stride;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int d = kQuant ? gid * (DP / 8) + t * 2 + h : t * 16 + h * 8 + gid;
                if (d >= a.c.head_dim) continue;
                const float x = o[t][n][h * 2 + e] * inv;
                if (a.out.type == KVR_BF16) reinterpret_cast<__nv_bfloat16 *>(dst)[d] = __float2bfloat16_rn(x);
                else reinterpret_cast<__half *>(dst)[d] = __float2half_rn(x);
              }
            if (a.lse && gid == 0)
              a.lse[(long long)(len.first + t_row) * a.q_heads + q_head] = sum[n][e] == 0.f ? -INFINITY : top[n][e] * 0.69314718f + logf(sum[n][e]);
          } else {
            float *dst = a.part_o + (slot * a.row_tile + row) * a.c.head_dim;
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int d = kQuant ? gid * (DP / 8) + t * 2 + h : t * 16 + h * 8 + gid;
                if (d < a.c.head_dim) dst[d] = o[t][n][h * 2 + e];
              }
            if (gid == 0) a.part_ml[slot * a.row_tile + row] = make_float2(top[n][e], sum[n][e]);
          }
        }
    }
    if (piece.begin != 0 || piece.end != len.units) {
      const int heads = min(a.group_heads, a.c.kv_heads - piece.head_group * a.group_heads);
      hand_in(a, piece, shares, [] { __syncthreads(); return true; }, &last_in, warp, lane, [&](const Cut &cut, int c, int step, int n, bool fold) {
        const Piece copy = piece;        // what the call is shown lies in memory
        join_pieces<DP / 128 + DP % 128 / 64>(a, copy, cut, c, step, n, fold, rows, heads, (int)blockDim.x / 32, warp, lane);
      });
    }
    again = next_piece(a, piece, last);
  }
  copy_wait<0>();
}

template <int FMT, int DP, int NT>
cudaError_t launch_rows(const AttendArgs &a, int slices, cudaStream_t s) {
  using S = Shape<FMT, DP>;
  const int warps = a.group_heads * slices;
  const int merge = slices > 1 ? (slices - 1) * a.group_heads * (DP * 8 + 16) * 4 : 0;
  const int bytes = warps * S::kStages * S::kStageBytes + merge;
  static OncePerDevice once;
  if (const cudaError_t e = allow_shared(once, attend_rows_kernel<FMT, DP, NT>, 227 * 1024 - 512)) return e;
  attend_rows_kernel<FMT, DP, NT><<<a.ctas, warps * 32, bytes, s>>>(a, slices);
  return cudaGetLastError();
}

template <int FMT>
cudaError_t launch_rows(const AttendArgs &a, int tiles, int slices, cudaStream_t s) {
  if (a.c.head_dim <= 64) return tiles == 1 ? launch_rows<FMT, 64, 1>(a, slices, s) : launch_rows<FMT, 64, 2>(a, slices, s);
  if (a.c.head_dim <= 128) return tiles == 1 ? launch_rows<FMT, 128, 1>(a, slices, s) : launch_rows<FMT, 128, 2>(a, slices, s);
  return tiles == 1 ? launch_rows<FMT, 256, 1>(a, slices, s) : launch_rows<FMT, 256, 2>(a, slices, s);
}

}  // namespace
}  // namespace kvr
