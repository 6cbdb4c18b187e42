// Attention of few rows over a cache in 8 bits: a decode step, or a few tokens
// of each sequence. What is computed is chunk_attn.cuh's, with the plan, the
// cut by cost and the merge of parts that it explains.
//
// With 16 query rows per kv head or fewer, every byte of the cache meets little
// arithmetic, and what counts is that enough loads are in flight. The
// tensor-memory kernel cannot keep them so here: of its 128 rows 4 or 8 are
// used, and a tile's chain (S, scores to registers, P, PV) is as long as the
// bytes of a tile in 8 bits take. So: several CTAs per SM of four independent
// warps, each with a ring of 16-key pieces of K and V in shared memory filled
// by asynchronous 16-byte copies, and warp-wide MMAs on registers.
//
// A warp takes 16 keys at a time. S^T = K Q^T (m16n8k16, f16: the codes are
// exact in f16, the queries, after a power of two of their row, too) leaves row
// pair 2q, 2q + 1 of keys r and r + 8 in lane 4 r + q; two 8 x 8 transposes
// (movmatrix) turn P into the second operand of O^T += V^T P^T. Which element of
// a head takes which place in the contraction is free as long as both operands
// agree, so a lane's share of a key is 16 (K: 2 x 16) whole bytes, and pairs of
// keys of V become pairs of f16 by a byte permute and the conversion. The
// scales of the 16 keys enter the softmax: s = f 2^ek (K8 . Q), P' = 2^(s + ev -
// m), l += P' 2^-ev, O += P' V8; m, l and O stay in registers, and the reference
// m is raised only when a term passes 2^15 (f16 ends at 2^16; it is set so that
// the largest is 2^7). At the end of an item the warps' (m, l, O) are joined
// through shared memory.
#include "chunk_attn.cuh"

namespace libraspec {

constexpr int kFewWarps = 4, kFewThreads = 32 * kFewWarps;
constexpr int kFewStages = 3;            // of a warp's ring
constexpr int kFewCtas = 3, kFewCtas16 = 2;  // per SM, of 8 rows and of 16
constexpr int kGroup = 8;                // parts merged at a time
constexpr int kTopCounts = kCMaxCtas * kFewCtas;  // counters of a block's groups, behind those of the groups' parts
static_assert(2 * kTopCounts <= kCMaxCounts && 2 * kFewCtas * 8 <= kCBlockRows && 2 * kFewCtas16 * 16 <= kCBlockRows,
              "counters and parts fit the workspace");

struct FewArgs {
  const uint16_t* Q;
  const uint8_t *K8, *V8, *Ks, *Vs;
  __nv_bfloat16* O;
  float* lse;
  const int32_t *cu_new, *kv_len, *block_table;
  const float* slopes;
  MaskArgs mask;
  PlanArgs plan;
  const PlanBlock* blocks;  // NULL: each CTA plans for itself
  const PlanHead* head;
  const uint32_t* seen;
  float *part_o, *part_ml;
  uint32_t* count;
  int* status;
  float scale;
  CapArgs cap;
  int capped, Hq, Hkv, max_pages, page_size, n_pages, block_log2, rows;
  int fixed;  // what a block weighs beside its tiles, in tiles
};

struct FewItem {
  int b, kvh, tok0, pos0, n_tok, n_tiles, tile0, sink, klo, khi, gaps;
  int partial, slot, c0, np, none;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// D += A B, A 16 x 16 and B 16 x 8 of f16, D of binary32
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

template <int D, int NT, bool OPTS>
__global__ void __launch_bounds__(kFewThreads, NT == 1 ? kFewCtas : kFewCtas16) few_q8_kernel(const __grid_constant__ FewArgs A) {
  constexpr int kHalf = 16 * D;              // bytes of 16 keys
  constexpr int kStage = 2 * kHalf;          // K, then V
  constexpr int kSteps = D / 16;             // contraction steps of S
  constexpr int kTiles = D / 16;             // 16-row tiles of O^T
  constexpr int kRows = 8 * NT;
  extern __shared__ __align__(1024) uint8_t smem[];  // the warps' rings, then their O
  __shared__ PlanBlock s_blocks[kWarpBlocks];
  __shared__ FewItem s_item[2];
  __shared__ Place s_at;
  __shared__ long long s_left, s_W;
  __shared__ int s_fixed, s_G, s_last;
  __shared__ float2 s_ml[kFewWarps][kRows];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, q = lane & 3;
  const int g = A.Hq / A.Hkv;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  const PlanBlock* plan = A.blocks ? A.blocks : s_blocks;
  auto next_item = [&](FewItem& out) {  // by one thread
    FewItem it{};
    it.none = s_left <= 0;
    if (!it.none) {
      const Place pl = s_at;
      const PlanBlock p = plan[pl.e];
      const int c = blockIdx.x;
      it.b = p.b;
      it.kvh = pl.kvh;
      it.tok0 = p.tok0;
      it.pos0 = p.pos0;
      it.n_tok = p.n_tok;
      it.n_tiles = (int)min((long long)(p.n_tiles - pl.tile), s_left);
      it.tile0 = p.tile0 + pl.tile;
      it.sink = p.sink << 16 | max(p.sink - pl.tile, 0);
      it.klo = p.klo;
      it.khi = p.khi;
      it.gaps = p.gaps ? pl.e : -1;
      it.partial = it.n_tiles != p.n_tiles;
      it.slot = pl.tile == 0 ? 2 * c + 1 : 2 * c;
      it.c0 = c;
      it.np = 1;
      if (it.partial) {  // the CTAs of the block's first and last tile
        const long long y = (long long)A.Hkv * (p.tiles_before + (long long)s_fixed * pl.e) +
                            (long long)pl.kvh * (p.n_tiles + s_fixed) + s_fixed;
        it.c0 = share_of(y, s_W, s_G);
        it.np = share_of(y + p.n_tiles - 1, s_W, s_G) - it.c0 + 1;
      }
      s_left -= it.n_tiles;
      s_at.tile = 0;
      if (++s_at.kvh == A.Hkv) {
        s_at.kvh = 0;
        ++s_at.e;
      }
    }
    out = it;
  };
  if (warp == 0) {  // the CTA's share, as the other kernel's producer finds it
    PlanHead head;
    if (A.blocks) {
      head = *A.head;
    } else {
      PlanBlock mine[2];
      head = warp_plan(A.plan, mine);
      s_blocks[lane] = mine[0];
      s_blocks[lane + 32] = mine[1];
      __syncwarp();
    }
    const PlanBlock none[2] = {};
    const Blocks blocks{plan, none, head.blocks};
    const long long all = (long long)A.Hkv * head.tiles;
    const int G = (int)min((long long)gridDim.x, all), c = blockIdx.x;
    const FixedCost f{all > 0 ? min(A.fixed, (int)min(1ll << 20, quotient(all, 4ll * G))) : 0, 0};
    const long long W = (long long)A.Hkv * (head.tiles + (long long)f.one * head.blocks);
    Place at{};
    long long left = 0;
    if (c < G) {
      long long end = all;
#pragma unroll 1
      for (int k = 1; k >= 0; --k) {
        const long long x = quotient((c + k) * W, G);
        if (x < W) at = find_place(x, blocks, A.Hkv, g, f);
        if (k && x < W) end = at.before;
      }
      left = end - at.before;
    }
    if (lane == 0) {
      s_at = at;
      s_left = left;
      s_W = W;
      s_fixed = f.one;
      s_G = G;
      next_item(s_item[0]);
    }
  }
  __syncthreads();

  uint8_t* ring = smem + warp * (kFewStages * kStage);
  float2* s_o = reinterpret_cast<float2*>(smem + kFewWarps * kFewStages * kStage);
  const uint32_t s_ring = smem_u32(ring);
  const float scale_log2 = A.scale * kLog2e;
  // Of the item at hand (`it`): 16 keys at a time, the warp's i-th piece is 16-key piece warp + 4 (i & 1) of the item's tile
  // i / 2. Lane i has the page (or sequence) and row of the i-th of 32 pieces, and their exponents. Those of the next 32
  // come in two steps while these are worked on, first the pages, then the exponents, which nobody waits for.
  FewItem it = s_item[0];
  ChunkItem tiles;  // (for the sequence's tiles of the item's)
  const uint32_t* seen = nullptr;
  int n_pieces = 0, sinks_all = 0, row0 = 0, row1 = 0, plane0 = -1, plane1 = -1, page = kNoPage;
  uint32_t exps0 = 0, exps1 = 0;
  auto key_of = [&](int i) { return item_tile<true>(tiles, i >> 1) * kCKeys + 16 * (warp + 4 * (i & 1)); };
  auto page_of = [&](int i) {  // kNoPage: no row of the block sees a key of it
    if (i >= n_pieces) return kNoPage;
    const int key = key_of(i);
    if (key >= it.khi || (key + 16 <= it.klo && key >= sinks_all)) return kNoPage;
    if (it.gaps >= 0 && !some_row_sees(seen, it.pos0, it.n_tok, max(key, it.klo), min(key + 16, it.khi)))
      return kNoPage;
    if (!A.block_table) return it.b;
    return max(-1, __ldg(A.block_table + (size_t)it.b * A.max_pages + key / A.page_size));
  };
  auto plane_of = [&](int i, int page, int& row) {  // -1: none
    row = 0;
    if (page == kNoPage) return -1;
    row = key_of(i);
    if (A.block_table) {
      row %= A.page_size;
      if (page < 0 || page >= A.n_pages) {
        raise_status(A.status, LIBRASPEC_ST_BAD_PAGE);
        page = 0;  // a valid page; the sequence's output is then meaningless
      }
    }
    return page * A.Hkv + it.kvh;
  };
  auto exps_of = [&](int plane, int row) {  // of K, and 2^8 times that of V
    if (plane < 0) return 0u;
    const size_t at = (size_t)plane * (A.rows >> A.block_log2) + (row >> A.block_log2);
    return (uint32_t)__ldg(A.Ks + at) | (uint32_t)__ldg(A.Vs + at) << 8;
  };
  // Where 16-byte chunk c of row x lies within 16 keys, so that the reads below (K: chunks q or 4 + q of rows r; V: chunk
  // r of rows 2 q + ..) meet no bank twice (at a head dim of 64, those of V meet each twice).
  auto k_at = [&](int x, int c) { return x * D + (D == 128 ? c ^ (x & 1) << 2 : c) * 16; };
  auto v_at = [&](int x, int c) { return x * D + (D == 128 ? c ^ (x >> 1 & 3) << 1 : c ^ (x >> 1 & 3)) * 16; };
  auto issue = [&](int i, int base) {  // piece i (of the 32 from base on, or the next) into its stage, if it is seen
    const bool next = i >= base + 32;
    const int row = __shfl_sync(0xffffffffu, next ? row1 : row0, i & 31);
    const int plane = __shfl_sync(0xffffffffu, next ? plane1 : plane0, i & 31);
    if (plane >= 0) {
      const size_t at = ((size_t)plane * A.rows + row) * D;
      const uint32_t to = s_ring + (i % kFewStages) * kStage;
      constexpr int kChunks = D / 16;  // of a row
#pragma unroll
      for (int k = 0; k < kChunks / 2; ++k) {
        const int c = lane + 32 * k, x = c / kChunks, cc = c % kChunks;
        copy16(to + k_at(x, cc), A.K8 + at + c * 16);
        copy16(to + kHalf + v_at(x, cc), A.V8 + at + c * 16);
      }
    }
    copy_commit();
  };
  auto start = [&]() {  // the item's first pieces go out
    tiles.tile0 = it.tile0;
    tiles.sink = it.sink;
    seen = A.seen + (size_t)max(it.gaps, 0) * kSeenWords;
    n_pieces = it.none ? 0 : 2 * it.n_tiles;
    sinks_all = min(A.mask.sinks, it.khi);
    plane0 = plane_of(lane, page_of(lane), row0);
    plane1 = -1;
    row1 = 0;
    page = page_of(lane + 32);
    exps0 = exps_of(plane0, row0);
    exps1 = 0;
#pragma unroll
    for (int i = 0; i < kFewStages - 1; ++i) issue(i, 0);
  };
  start();
  for (int nth = 0; !it.none; ++nth) {
    if (tid == 0) next_item(s_item[(nth + 1) & 1]);
    __syncthreads();
    const int rows = it.n_tok * g;
    // rows: 8 nt + 2 q + j of the block
    float m[NT][2], l[NT][2], unscale[NT][2], slope[NT][2];
    int lo[NT][2], hi[NT][2], pos[NT][2];
    uint32_t qf[NT][kSteps][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // Q: lane 4 r + q has elements [16 q, 16 q + 16) (and 64 more) of row 8 nt + r
      const int rr = 8 * nt + r;
      uint4 v[kSteps / 4][2];
      uint32_t top = 0;
#pragma unroll
      for (int h = 0; h < kSteps / 4; ++h) {
        v[h][0] = v[h][1] = make_uint4(0, 0, 0, 0);
        if (rr < rows) {
          const uint4* src = reinterpret_cast<const uint4*>(
              A.Q + ((size_t)(it.tok0 + rr / g) * A.Hq + it.kvh * g + rr % g) * D + 64 * h + 16 * q);
          v[h][0] = __ldg(src);
          v[h][1] = __ldg(src + 1);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 u = v[h][k];
          const uint32_t a = __vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), b = __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu);
          top = __vmaxu2(top, __vmaxu2(a, b));
        }
      }
      top = max(top & 0xffffu, top >> 16);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // times the power of two that brings the row's largest into [2^14, 2^15): f16 then holds all eight bits of what
      // lies above 2^-31 of it (rows below 2^-112 are not brought up that far: factor and inverse are normal numbers)
      const int fe = min(268 - (int)(top >> 7), 253);
      const float f = power_of_two_biased(fe);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const uint4 u = v[s / 4][s % 4 / 2];
        const uint32_t a = s % 2 ? u.z : u.x, b = s % 2 ? u.w : u.y;
        qf[nt][s][0] = pack_f16(bf16_lo(a) * f, bf16_hi(a) * f);
        qf[nt][s][1] = pack_f16(bf16_lo(b) * f, bf16_hi(b) * f);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = 8 * nt + 2 * q + j;
        unscale[nt][j] = power_of_two_biased(254u - __shfl_sync(0xffffffffu, fe, 4 * (2 * q + j)));
        m[nt][j] = -INFINITY;
        l[nt][j] = 0.f;
        lo[nt][j] = pos[nt][j] = 0;
        hi[nt][j] = 0x7fffffff;  // (a row past the block's scores 0 with every key: it asks for no masks)
        slope[nt][j] = 0.f;
        if (row < rows) {
          const int tok = it.tok0 + row / g;
          pos[nt][j] = it.pos0 + row / g;
          const int n_keys = A.kv_len[it.b] + A.cu_new[it.b + 1] - A.cu_new[it.b];
          row_range(pos[nt][j], n_keys, A.mask.prefix_len ? A.mask.prefix_len[it.b] : 0,
                    A.mask.first_key ? A.mask.first_key[tok] : 0, A.mask.window, lo[nt][j], hi[nt][j]);
          if (OPTS && A.slopes) slope[nt][j] = A.slopes[it.kvh * g + row % g] * kLog2e;
        }
      }
    }
    float o[NT][kTiles][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[nt][i][k] = 0.f;

    int base = 0;
#pragma unroll 1
    for (int i = 0; i < n_pieces; ++i) {
      if ((i & 31) == 8) {
        plane1 = plane_of(base + 32 + lane, page, row1);
        exps1 = exps_of(plane1, row1);
      }
      if (i == base + 32) {  // the next 32 pieces become the current ones
        base += 32;
        plane0 = plane1;
        row0 = row1;
        exps0 = exps1;
        page = page_of(base + 32 + lane);
      }
      __syncwarp();  // (the stage has been read by all lanes)
      issue(i + kFewStages - 1, base);
      copy_wait<kFewStages - 1>();
      __syncwarp();
      if (__shfl_sync(0xffffffffu, plane0, i & 31) < 0) continue;
      const uint32_t e = __shfl_sync(0xffffffffu, exps0, i & 31);
      const int ek = min(max((int)(e & 0xffu), 67), 187), ev = min(max((int)(e >> 8), 67), 187);
      const float ks = power_of_two_biased(ek), il = power_of_two_biased(254u - ev);
      const float lv = (float)(ev - 127);
      const uint8_t* st = ring + (i % kFewStages) * kStage;
      const int key0 = key_of(i);

      float s[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[nt][k] = 0.f;
#pragma unroll
      for (int h = 0; h < kSteps / 4; ++h) {
        const uint4 ka = *reinterpret_cast<const uint4*>(st + k_at(r, 4 * h + q));
        const uint4 kb = *reinterpret_cast<const uint4*>(st + k_at(r + 8, 4 * h + q));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t a = word(ka, j), b = word(kb, j);
          const uint32_t a0 = f16_of_e4m3((uint16_t)a), a2 = f16_of_e4m3((uint16_t)(a >> 16));
          const uint32_t a1 = f16_of_e4m3((uint16_t)b), a3 = f16_of_e4m3((uint16_t)(b >> 16));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma16816(s[nt], a0, a1, a2, a3, qf[nt][4 * h + j][0], qf[nt][4 * h + j][1]);
        }
      }
      // scores in units of log 2: s[nt][2 k + j] of key key0 + r + 8 k and row 8 nt + 2 q + j
      bool edge = false, high = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) edge |= key0 < lo[nt][j] || key0 + 16 > hi[nt][j];
      edge = __any_sync(0xffffffffu, edge);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float f = fmaxf(scale_log2 * unscale[nt][j] * ks, kFloatMin);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float x = s[nt][2 * k + j];
            const int key = key0 + r + 8 * k;
            if constexpr (OPTS) {
              x *= unscale[nt][j] * ks;
              x = A.capped ? wide_cap(x, rcp_approx(ex2_approx(x * A.cap.twice_inverse) + 1.f), scale_log2, A.cap)
                           : x * scale_log2;
              x -= slope[nt][j] * fabsf((float)(pos[nt][j] - key));
            } else {
              x *= f;
            }
            if (edge && !(key < hi[nt][j] && (key >= lo[nt][j] || key < A.mask.sinks))) x = -INFINITY;
            x += lv;
            high |= x - m[nt][j] > kCRescaleLog2 + kHeadroomLog2;
            s[nt][2 * k + j] = x;
          }
        }
      if (__any_sync(0xffffffffu, high)) {  // a new reference for some row
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float mx = fmaxf(s[nt][j], s[nt][2 + j]);
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            if (mx - m[nt][j] > kCRescaleLog2 + kHeadroomLog2) {
              const float to = mx - kHeadroomLog2, f = m[nt][j] == -INFINITY ? 0.f : ex2_approx(m[nt][j] - to);
              m[nt][j] = to;
              l[nt][j] *= f;
#pragma unroll
              for (int t = 0; t < kTiles; ++t) {
                o[nt][t][j] *= f;
                o[nt][t][2 + j] *= f;
              }
            }
          }
      }
      uint32_t pb[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float neg = m[nt][j] == -INFINITY ? 0.f : m[nt][j];
          s[nt][j] = ex2_approx(s[nt][j] - neg);
          s[nt][2 + j] = ex2_approx(s[nt][2 + j] - neg);
          l[nt][j] = fmaf(s[nt][j] + s[nt][2 + j], il, l[nt][j]);
        }
        pb[nt][0] = transpose8x8(pack_f16(s[nt][0], s[nt][1]));
        pb[nt][1] = transpose8x8(pack_f16(s[nt][2], s[nt][3]));
      }
      // V: keys 2 q, 2 q + 1, 2 q + 8, 2 q + 9; D / 8 elements from D / 8 r on
      constexpr int kWords = D / 32;
      uint32_t v[4][kWords];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int x = 2 * q + (k & 1) + 8 * (k >> 1);
        if constexpr (D == 128) {
          const uint4 u = *reinterpret_cast<const uint4*>(st + kHalf + v_at(x, r));
          v[k][0] = u.x, v[k][1] = u.y, v[k][2] = u.z, v[k][3] = u.w;
        } else {
          const uint2 u = *reinterpret_cast<const uint2*>(st + kHalf + v_at(x, r >> 1) + 8 * (r & 1));
          v[k][0] = u.x, v[k][1] = u.y;
        }
        if (edge) {  // what a key that no row sees holds (NaN, say) does not meet the zeros of P
          const int key = key0 + x;
          bool some = key < it.khi && (key >= it.klo || key < sinks_all);
          if (some && it.gaps >= 0) some = some_row_sees(seen, it.pos0, it.n_tok, key, key + 1);
          if (!some)
#pragma unroll
            for (int w = 0; w < kWords; ++w) v[k][w] = 0;
        }
      }
#pragma unroll
      for (int w = 0; w < kWords; ++w)
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // elements 4 w + 2 half and the next, of two keys side by side
          const uint32_t a = __byte_perm(v[0][w], v[1][w], half ? 0x7362 : 0x5140);
          const uint32_t b = __byte_perm(v[2][w], v[3][w], half ? 0x7362 : 0x5140);
          const uint32_t a0 = f16_of_e4m3((uint16_t)a), a1 = f16_of_e4m3((uint16_t)(a >> 16));
          const uint32_t a2 = f16_of_e4m3((uint16_t)b), a3 = f16_of_e4m3((uint16_t)(b >> 16));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma16816(o[nt][2 * w + half], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
        }
    }
    __syncwarp();
    // the next item's first pieces are on their way while this one's parts are joined
    const FewItem done = it;
    it = s_item[(nth + 1) & 1];
    start();

    // ---- the warps' parts, joined ----
    // o[nt][t]: elements D / 8 r + 2 t (and the next) of rows 8 nt + 2 q + j; in shared memory [t][r][row] pairs of them
    float2* mine = s_o + warp * (kRows * D / 2);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float sum = l[nt][j];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (r == 0) s_ml[warp][8 * nt + 2 * q + j] = make_float2(m[nt][j], sum);
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
          mine[(t * 8 + r) * kRows + 8 * nt + 2 * q + j] = make_float2(o[nt][t][j], o[nt][t][2 + j]);
      }
    __syncthreads();
    for (int u = tid; u < rows * (D / 2); u += kFewThreads) {
      const int row = u / (D / 2), d = 2 * (u % (D / 2)), at = (d % (D / 8) / 2 * 8 + d / (D / 8)) * kRows + row;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) M = fmaxf(M, s_ml[w][row].x);
      float2 acc = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) {
        const float2 ml = s_ml[w][row];
        const float f = M == -INFINITY ? 1.f : ex2_approx(ml.x - M);  // (no reference: nothing seen, or NaN alone)
        const float2 x = s_o[w * (kRows * D / 2) + at];
        L += f * ml.y;
        acc.x += f * x.x;
        acc.y += f * x.y;
      }
      if (done.partial) {
        const size_t prow = (size_t)done.slot * kRows + row;
        *reinterpret_cast<float2*>(A.part_o + prow * D + d) = acc;
        if (d == 0) *reinterpret_cast<float2*>(A.part_ml + prow * 2) = make_float2(M, L);
      } else {
        const size_t out = (size_t)(done.tok0 + row / g) * A.Hq + done.kvh * g + row % g;
        const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;  // (NaN stays)
        *reinterpret_cast<uint32_t*>(A.O + out * D + d) = c_pack(acc.x * inv, acc.y * inv);
        if (A.lse && d == 0) A.lse[out] = (M + __log2f(L)) * kLn2;
      }
    }
    // The CTA that delivers the last part of kGroup merges them, and the one that merges the last group merges the groups,
    // each in CTA order: a block's parts then take two rounds of loads and not np / 8 (one sequence over 8000 keys and 32
    // heads, 57 parts of a head: 14.6 us, with eight parts of the row at a
    // time in one round after the other 22.4; of four tokens 24 and 41).
    if (done.partial) {
      auto arrive = [&](int at, int of) {
        __syncthreads();
        if (tid == 0) {
          uint32_t old;
          asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(old) : "l"(A.count + at) : "memory");
          s_last = old == (uint32_t)of - 1;
          if (s_last) A.count[at] = 0u;
        }
        __syncthreads();
        return s_last != 0;
      };
      const int slots = 2 * gridDim.x;  // (those of the groups lie behind the parts')
      auto slot_of = [&](int p) { return p == 0 ? 2 * done.c0 + 1 : 2 * (done.c0 + p); };
      auto merge = [&](int from, int to, int step, int first_slot, int into) {  // into < 0: the results
        for (int u = tid; u < rows * (D / 4); u += kFewThreads) {
          const int row = u / (D / 4), d = 4 * (u % (D / 4));
          float M = -INFINITY, L = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int p0 = from; p0 < to; p0 += kGroup * step) {
            float2 ml[kGroup];
            float4 x[kGroup];
            float top = M;
#pragma unroll
            for (int k = 0; k < kGroup; ++k) {
              ml[k] = make_float2(-INFINITY, 0.f);
              x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (p0 + k * step < to) {
                const size_t at = (size_t)(first_slot + slot_of(p0 + k * step)) * kRows + row;
                ml[k] = __ldcg(reinterpret_cast<const float2*>(A.part_ml) + at);
                x[k] = __ldcg(reinterpret_cast<const float4*>(A.part_o + at * D + d));
              }
            }
#pragma unroll
            for (int k = 0; k < kGroup; ++k) top = fmaxf(top, ml[k].x);
            const float old = top == -INFINITY ? 1.f : ex2_approx(M - top);
            M = top;
            L *= old;
            acc.x *= old, acc.y *= old, acc.z *= old, acc.w *= old;
#pragma unroll
            for (int k = 0; k < kGroup; ++k) {
              const float f = top == -INFINITY ? 1.f : ex2_approx(ml[k].x - top);
              L += f * ml[k].y;
              acc.x += f * x[k].x, acc.y += f * x[k].y, acc.z += f * x[k].z, acc.w += f * x[k].w;
            }
          }
          if (into >= 0) {
            const size_t at = (size_t)into * kRows + row;
            *reinterpret_cast<float4*>(A.part_o + at * D + d) = acc;
            if (d == 0) *reinterpret_cast<float2*>(A.part_ml + at * 2) = make_float2(M, L);
          } else {
            const size_t out = (size_t)(done.tok0 + row / g) * A.Hq + done.kvh * g + row % g;
            const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;
            *reinterpret_cast<uint2*>(A.O + out * D + d) =
                make_uint2(c_pack(acc.x * inv, acc.y * inv), c_pack(acc.z * inv, acc.w * inv));
            if (A.lse && d == 0) A.lse[out] = (M + __log2f(L)) * kLn2;
          }
        }
      };
      // (no other block's parts begin in a CTA before its last, so a counter at a group's first CTA is its own)
      const int first = ((int)blockIdx.x - done.c0) / kGroup * kGroup, n = min(kGroup, done.np - first);
      if (n == 1) __syncthreads();  // (a group of this CTA's part alone: it is written by all threads)
      if (done.np <= kGroup) {
        if (arrive(done.c0, done.np)) merge(0, done.np, 1, 0, -1);
      } else if (n == 1 || arrive(done.c0 + first, n)) {
        merge(first, first + n, 1, 0, slots + slot_of(first));
        if (arrive(kTopCounts + done.c0, (done.np + kGroup - 1) / kGroup)) merge(0, done.np, kGroup, slots, -1);
      }
    }
    __syncthreads();
  }
}

template <int D, int NT, bool OPTS>
static cudaError_t launch_few_t(const FewArgs& a, int grid, cudaStream_t stream) {
  constexpr int kBytes = kFewWarps * (kFewStages * 32 * D + 8 * NT * D * 4);
  static std::atomic<uint64_t> devices{0};
  const cudaError_t e = allow_shared(few_q8_kernel<D, NT, OPTS>, kBytes, devices);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = kBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, few_q8_kernel<D, NT, OPTS>, a);
}

cudaError_t launch_few_attn_q8(const ChunkCall& c) {
  if (c.T == 0 || c.B == 0) return cudaSuccess;
  const ChunkWs lay = chunk_ws(c.T, c.B, c.Hq, c.Hkv, c.D);
  const int g = c.Hq / c.Hkv;
  const bool eight = few_rows(c.T, c.B, g) == 8;
  const int tokens = (eight ? 8 : 16) / g;
  char* ws = c.ws;
  FewArgs a{};
  a.Q = c.Q;
  a.K8 = static_cast<const uint8_t*>(c.K);
  a.V8 = static_cast<const uint8_t*>(c.V);
  a.Ks = c.Ks;
  a.Vs = c.Vs;
  a.O = reinterpret_cast<__nv_bfloat16*>(c.O);
  a.lse = c.lse;
  a.cu_new = c.cu_new;
  a.kv_len = c.kv_len;
  a.block_table = c.block_table;
  a.slopes = c.slopes;
  a.mask = MaskArgs{c.first_key, c.prefix_len, c.window, c.window > 0 ? c.sinks : 0};
  a.blocks = reinterpret_cast<const PlanBlock*>(ws + lay.blocks);
  a.head = reinterpret_cast<const PlanHead*>(ws + lay.head);
  a.seen = reinterpret_cast<const uint32_t*>(ws + lay.seen);
  a.part_o = reinterpret_cast<float*>(ws + lay.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + lay.part_ml);
  a.count = reinterpret_cast<uint32_t*>(ws + lay.count);
  a.status = reinterpret_cast<int*>(ws + lay.status);
  a.scale = c.scale;
  a.capped = c.softcap > 0.f;
  if (a.capped) a.cap = cap_args(c.scale, c.softcap);
  a.Hq = c.Hq;
  a.Hkv = c.Hkv;
  a.max_pages = c.max_pages;
  a.page_size = c.page_size;
  a.n_pages = c.n_pages;
  a.rows = c.block_table ? c.page_size : c.S_cap;
  while ((1 << a.block_log2) < c.block) ++a.block_log2;
  a.fixed = 6;  // (a decoding batch of 64 sequences: 189 us at 2, 186 at 4, 183 at 6)
  const int grid = std::min(num_sms_current(), kCMaxCtas) * (eight ? kFewCtas : kFewCtas16);
  a.plan = PlanArgs{c.cu_new, c.kv_len, a.mask, c.T, c.B, tokens, std::min(c.S_cap, kCMaxKeys), c.Hkv, grid, 0x7fffffff,
                    0, few_alone(c.T, g) ? 0x7fffffff : tokens, a.status};
  if (few_blocks(c.T, c.B, tokens) <= kWarpBlocks && c.B <= kWarpSeqs && !c.first_key) {
    a.blocks = nullptr;
  } else {
    chunk_plan_kernel<<<1, kPlanThreads, 0, c.stream>>>(a.plan, reinterpret_cast<PlanBlock*>(ws + lay.blocks),
                                                        reinterpret_cast<PlanHead*>(ws + lay.head),
                                                        reinterpret_cast<uint32_t*>(ws + lay.seen));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const bool opts = a.capped || c.slopes;
  if (c.D == 128) {
    if (eight) return opts ? launch_few_t<128, 1, true>(a, grid, c.stream) : launch_few_t<128, 1, false>(a, grid, c.stream);
    return opts ? launch_few_t<128, 2, true>(a, grid, c.stream) : launch_few_t<128, 2, false>(a, grid, c.stream);
  }
  if (eight) return opts ? launch_few_t<64, 1, true>(a, grid, c.stream) : launch_few_t<64, 1, false>(a, grid, c.stream);
  return opts ? launch_few_t<64, 2, true>(a, grid, c.stream) : launch_few_t<64, 2, false>(a, grid, c.stream);
}

}  // namespace libraspec
