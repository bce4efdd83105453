// Included by hisparse.cu: attention of chunks with many query rows a request, on pairs of SMs.  The same problem and the
// same rounding as record_attention_kernel.cuh; this kernel is for 128 rows a block of work and bf16 records that lie in
// boxes of 64 rows.
//
// What bounds attention over these records is the accumulator and shared memory: 128 rows of O with 512 numbers fill the
// tensor memory of one SM, and 64 rows a tile read every operand from shared memory so often that the tensor cores reach
// half of their rate.  A pair of SMs (cta_group::2, M = 128) works on 64 rows each and N columns together, at the full
// rate (measured: 32.4 cycles for M 128 x N 128 x K 16, 64.4 for N 256, where one SM alone takes 32.4 for M 64 x N 64):
//   S = Q K^T   128 rows x 128 keys: either SM holds its 64 rows of Q and 64 of the tile's keys
//   O = P V     128 rows x Dv: either SM holds its 64 rows of P, all 128 keys, and half of the numbers of every block of 256
// so a tile costs an SM 64 (D) + 128 (Dv / 2) numbers of loads.  In tensor memory lanes 0-63 are the SM's rows over the first
// half of the columns, lanes 64-127 the same rows over the second half.
// 2048 tokens x 16 heads over 32768 keys: 1.88 ms, 1200 TFLOP/s (72 % of the measured burst rate, 87 % of the sustained
// one); the tensor pipe is active 76 % of a block's life, a tile takes 2650 cycles of which 2200 are its MMAs.
//   shared memory (D 576, Dv 512): Q 72 KB, K 72 KB, V 64 KB, P 16 KB: one buffer each.  K is refilled in groups of two
//   64-number chunks while V is multiplied, V in blocks while K is.
//   warps   0-7 softmax (a thread has 32 keys of a row; with four warps and 64 it took 2900 cycles a tile, longer than the
//   products), 8 issues S (first SM), 9 issues O (first SM), 10-13 bring chunks of K by TMA, 14 and 15 blocks of V.

namespace {

constexpr int kCaTile = 128;                     // keys a tile
constexpr int kCaRows = 64;                      // rows an SM
constexpr int kCaKeyWarps = 4, kCaValueWarps = 2;
constexpr int kCaSoftWarps = 8, kCaSoft = kCaSoftWarps * 32;
constexpr int kCaThreads = (kCaSoftWarps + 2 + kCaKeyWarps + kCaValueWarps) * 32;
constexpr int kCaMasks = 4;
constexpr int kCaChunk = kCaRows * 128;          // bytes of a 64 x 64 chunk (Q, K, P); of V twice that

struct CaSmem {
  static constexpr int kKGroups = kRaMaxGroups, kVBlocks = 2;
  static constexpr int kBars = 2 * kKGroups + 2 * kVBlocks + 2 + 2 + 1 + kCaMasks + 2;
  __host__ __device__ static constexpr uint32_t k(const int chunks) { return (uint32_t)(chunks * kCaChunk); }
  __host__ __device__ static constexpr uint32_t v(const int chunks) { return 2 * k(chunks); }
  __host__ __device__ static constexpr uint32_t p(const int chunks, const int vchunks) { return v(chunks) + (uint32_t)(vchunks * 2 * kCaChunk); }
  __host__ __device__ static constexpr uint32_t bars(const int chunks, const int vchunks) { return p(chunks, vchunks) + 2 * kCaChunk; }
  __host__ __device__ static constexpr uint32_t masks(const int chunks, const int vchunks) { return bars(chunks, vchunks) + 8 * kBars + 8; }
  __host__ __device__ static constexpr uint32_t tmem(const int chunks, const int vchunks) { return masks(chunks, vchunks) + kCaMasks * 16; }
  __host__ __device__ static constexpr uint32_t red(const int chunks, const int vchunks) { return tmem(chunks, vchunks) + 16; }
  __host__ __device__ static constexpr uint32_t odd(const int chunks, const int vchunks) { return red(chunks, vchunks) + 4 * kCaRows * 4; }
  __host__ __device__ static constexpr uint32_t total(const int chunks, const int vchunks) { return odd(chunks, vchunks) + kCaRows; }
};

__device__ __forceinline__ uint32_t in_first(const uint32_t addr) {   // this shared-memory address in the pair's first SM
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
// Arrival at a barrier of the other SM.  What it announces is read by the tensor cores of the SM that wrote it, behind the
// writer's proxy fence, so it need not be a release for the whole pair (which took 2100 cycles).
__device__ __forceinline__ void mbar_arrive_pair(const uint32_t addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ void umma2_bf16(const uint32_t d, const uint32_t a_lo, const uint32_t b_lo, const uint32_t idesc, const bool add) {
  asm volatile("{ .reg .pred p; .reg .b64 a, b; setp.ne.u32 p, %5, 0; mov.b64 a, {%1, %4}; mov.b64 b, {%2, %4};"
               " tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p; }"
               ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(kUmmaDescHi), "r"((uint32_t)add) : "memory");
}
// arrives on the barrier at this offset in both SMs when everything issued so far is done
__device__ __forceinline__ void umma2_commit(const uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// loads into this SM, counted by a barrier of the pair's first SM
__device__ __forceinline__ void tma2_rows(const uint32_t dst, const CUtensorMap *map, const int x, const int y, const uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma2_gather4(const uint32_t dst, const CUtensorMap *map, const int x, const int4 y, const uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w), "r"(bar) : "memory");
}
// 32 lanes x 32 columns
__device__ __forceinline__ void tmem_ld32(const uint32_t addr, float *v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
               "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                 "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                 "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
                 "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
               : "r"(addr));
}

// `dense` > 0: the records of request n are rows n * dense + j of the maps, whatever the table says about where they were
// (expand_records_kernel laid them out); the table still says which of them there are.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kCaThreads, 1)
chunk_attention_kernel(const RecAtt a, const int dense, const __grid_constant__ CUtensorMap rows_map,
                       const __grid_constant__ CUtensorMap eight_map, const __grid_constant__ CUtensorMap gather_map) {
  extern __shared__ __align__(1024) unsigned char ra_smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = blockIdx.x & 1u;
  const int chunks = (a.f.D + 63) / 64, groups = (chunks + 1) / 2;
  const int vblocks = a.Dv > 256 ? 2 : 1, vper = a.Dv == 128 ? 1 : 2, vchunks = vblocks * vper;   // chunks of V this SM holds
  const uint32_t sbase = smem_u32(ra_smem);
  const uint32_t s_q = sbase, s_k = sbase + CaSmem::k(chunks), s_v = sbase + CaSmem::v(chunks), s_p = sbase + CaSmem::p(chunks, vchunks);
  const uint32_t bars = sbase + CaSmem::bars(chunks, vchunks);
  // in the first SM: K groups and V blocks filled, P of either buffer, Q; in both: K, V free again, S of either buffer, masks
  const uint32_t b_kfull = bars, b_vfull = b_kfull + 8 * CaSmem::kKGroups, b_p = b_vfull + 8 * CaSmem::kVBlocks, b_q = b_p + 16;
  const uint32_t b_kfree = b_q + 8, b_vfree = b_kfree + 8 * CaSmem::kKGroups, b_s = b_vfree + 8 * CaSmem::kVBlocks, b_m = b_s + 16;
  const uint32_t b_end = b_m + 8 * kCaMasks;
  unsigned long long *s_mask = reinterpret_cast<unsigned long long *>(ra_smem + CaSmem::masks(chunks, vchunks));   // [buffer][half]
  float *s_red = reinterpret_cast<float *>(ra_smem + CaSmem::red(chunks, vchunks));                                // [quarter][row]
  uint8_t *s_odd = ra_smem + CaSmem::odd(chunks, vchunks);

  const uint32_t item = (blockIdx.x >> 1) / (uint32_t)a.splits, split = (blockIdx.x >> 1) - item * a.splits;
  const int n = (int)(item / (uint32_t)a.row_tiles);
  const int rt = a.row_tiles - 1 - (int)(item - (uint32_t)n * a.row_tiles);
  bool bad_req;
  const RaRequest rq = ra_request(a, n, bad_req);
  if (bad_req && tid == 0 && a.status) atomicOr(a.status, HISPARSE_STATUS_OUT_OF_RANGE);
  const int pair0 = rt * 2 * kCaRows, pair_rows = min(2 * kCaRows, rq.qlen * a.H - pair0);
  if (pair_rows <= 0) return;                    // (both SMs of the pair)
  const int row0 = pair0 + (int)rank * kCaRows, rows = min(kCaRows, rq.qlen * a.H - row0);   // of this SM, may be none
  const int hi_all = min(rq.kv, ra_limit(a, rq, (pair0 + pair_rows - 1) / a.H));
  const int tiles_all = (hi_all + kCaTile - 1) / kCaTile, per = (tiles_all + a.splits - 1) / a.splits;
  // (bounds in tiles first: a split's end in keys may lie beyond 2^31)
  const int lo = min((int)split * per, tiles_all) * kCaTile, hi = min(hi_all, min(((int)split + 1) * per, tiles_all) * kCaTile);
  const int nt = hi > lo ? (hi - lo + kCaTile - 1) / kCaTile : 0;

  bool dead = false;
  auto wait = [&](const uint32_t bar, const uint32_t parity) { if (!dead && !mbar_wait_quick(bar, parity)) dead = true; };

  if (tid < CaSmem::kBars) {
    const uint32_t b = bars + 8 * tid;
    uint32_t count = 1;
    if (b < b_vfull) count = (uint32_t)min(2, max(1, chunks - 2 * tid));    // one arrival a chunk
    else if (b < b_p) count = (uint32_t)vper;
    else if (b < b_kfree) count = 2 * kCaSoftWarps;                         // softmax warps of both SMs
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(count) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kCaSoftWarps) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(sbase + CaSmem::tmem(chunks, vchunks)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
  for (int i = tid; i < kCaRows; i += kCaThreads) s_odd[i] = 0;
  // what global memory is asked for first is on its way while the pair meets: the query's rows, and the table entries of a
  // tile's 128 keys (lane + 32 i), which are asked for a tile ahead all along
  uint4 qv[kCaRows / kCaSoftWarps][kRaQParts];
  int32_t e[4];
  auto ask = [&](const int t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = lo + t * kCaTile + 32 * i + lane;
      e[i] = j < hi ? ra_entry(a, n, j) : -1;
    }
  };
  if (warp < kCaSoftWarps) ra_fetch_q<kCaSoftWarps>(a, rq, row0, rows, warp, lane, qv);
  if (warp >= kCaSoftWarps + 2) ask(0);
  tmem_fence_before();
  __syncthreads();
  // (the barriers' initialisation is released by its own fence; a release here would wait for the loads above)
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  tmem_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(ra_smem + CaSmem::tmem(chunks, vchunks));
  const uint32_t ocols = (uint32_t)(a.Dv / 2), t_s = tmem + ocols;   // O, then two buffers of S with 64 columns each
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (warp >= kCaSoftWarps + 2) {
    // ------------------------------------------------------------------ loaders
    // warp w < 4 brings chunks w, w + 4, .. of K (this SM's 64 keys), warp 4 + b block b of V (its half, all 128 keys)
    const int w = warp - kCaSoftWarps - 2;
    const bool issuer = elect_one();
    bool bad_page = false;
    const int none = dense ? a.N * dense : ra_none(a);   // a row that does not exist
    // one chunk of 64 keys from j0: as a box where all of it may be read (what lies behind the context in a page may not),
    // eight keys at a time otherwise
    auto bring = [&](const uint32_t dst, const int c, const int j0, const int first, const int r0, const int r1, const uint32_t bar) {
      if (dense || j0 + 64 <= hi || first == none) {
        if (issuer) tma2_rows(dst, &rows_map, c * 64, first, bar);
        return;
      }
#pragma unroll 1
      for (int k = 0; k < 64; k += 8) {
        const int src = k < 32 ? r0 : r1;
        int4 x, y;
        x.x = __shfl_sync(0xffffffffu, src, (k + 0) & 31); x.y = __shfl_sync(0xffffffffu, src, (k + 1) & 31);
        x.z = __shfl_sync(0xffffffffu, src, (k + 2) & 31); x.w = __shfl_sync(0xffffffffu, src, (k + 3) & 31);
        y.x = __shfl_sync(0xffffffffu, src, (k + 4) & 31); y.y = __shfl_sync(0xffffffffu, src, (k + 5) & 31);
        y.z = __shfl_sync(0xffffffffu, src, (k + 6) & 31); y.w = __shfl_sync(0xffffffffu, src, (k + 7) & 31);
        if (issuer) {
          if (j0 + k + 8 <= hi || j0 + k >= hi) tma2_rows(dst + k * 128, &eight_map, c * 64, x.x, bar);
          else {
            tma2_gather4(dst + k * 128, &gather_map, c * 64, x, bar);
            tma2_gather4(dst + k * 128 + 512, &gather_map, c * 64, y, bar);
          }
        }
      }
    };
    const uint32_t kfull = in_first(b_kfull), vfull = in_first(b_vfull);
    for (int t = 0; t < nt; ++t) {
      const int j0 = lo + t * kCaTile;
      int r[4];
      uint32_t there[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = j0 + 32 * i + lane;
        const int32_t idx = ra_resolve(a, e[i], j, bad_page);
        r[i] = dense ? (j < hi ? n * dense + j : none) : idx < 0 ? none : idx;
        there[i] = __ballot_sync(0xffffffffu, idx >= 0);
      }
      ask(t + 1);
      const int f0 = __shfl_sync(0xffffffffu, r[0], 0), f1 = __shfl_sync(0xffffffffu, r[2], 0);
      if (w == 0 && lane == 0) {
        // (the masks of tile t - 4 are read: K of tile t - 1 came after S of t - 2, which came after the weights of t - 4)
        s_mask[(t % kCaMasks) * 2] = (unsigned long long)there[1] << 32 | there[0];
        s_mask[(t % kCaMasks) * 2 + 1] = (unsigned long long)there[3] << 32 | there[2];
        mbar_arrive(b_m + 8 * (t % kCaMasks));
      }
      __syncwarp();
      if (w < kCaKeyWarps) {
        for (int c = w; c < chunks; c += kCaKeyWarps) {
          if (t > 0) wait(b_kfree + 8 * (c >> 1), (uint32_t)((t - 1) & 1));
          dead = __any_sync(0xffffffffu, dead);   // (the warp goes on as one)
          if (rank == 0 && issuer) mbar_arrive_tx(b_kfull + 8 * (c >> 1), dead ? 0u : 2u * kCaChunk);
          if (!dead) bring(s_k + (uint32_t)c * kCaChunk, c, j0 + (int)rank * 64, rank ? f1 : f0, rank ? r[2] : r[0], rank ? r[3] : r[1], kfull + 8 * (c >> 1));
          __syncwarp();
        }
      } else if (w - kCaKeyWarps < vblocks) {
        const int b = w - kCaKeyWarps;
        if (t > 0) wait(b_vfree + 8 * b, (uint32_t)((t - 1) & 1));
        dead = __any_sync(0xffffffffu, dead);
        for (int x = 0; x < vper; ++x) {          // numbers 256 b + 128 rank + 64 x (64 rank where there are 128 in all)
          const int c = b * 4 + (int)rank * vper + x;
          const uint32_t dst = s_v + (uint32_t)((b * vper + x) * 2 * kCaChunk), bar = vfull + 8 * b;
          if (rank == 0 && issuer) mbar_arrive_tx(b_vfull + 8 * b, dead ? 0u : 4u * kCaChunk);
          if (!dead) {
            bring(dst, c, j0, f0, r[0], r[1], bar);
            bring(dst + kCaChunk, c, j0 + 64, f1, r[2], r[3], bar);
          }
          __syncwarp();
        }
      }
    }
    if (bad_page && a.status) atomicOr(a.status, HISPARSE_STATUS_OUT_OF_RANGE);
  } else if (warp == kCaSoftWarps) {
    // ------------------------------------------------------------------ S = Q K^T
    if (rank == 0) {
      const int ksteps = a.f.D / 16;
      constexpr uint32_t kIdS = umma_idesc(128, 128, false, false);
      const uint32_t q_lo = umma_desc_lo(s_q, 16), k_lo = umma_desc_lo(s_k, 16);
      const bool issuer = elect_one();
      wait(b_q, 0);
      for (int t = 0; t < nt; ++t) {
        const uint32_t d = t_s + (uint32_t)((t & 1) * 64);
        if (t >= 2) wait(b_p + 8 * (t & 1), (uint32_t)((t / 2 - 1) & 1));
#pragma unroll
        for (int g = 0; g < CaSmem::kKGroups; ++g) {
          if (g < groups) {
            wait(b_kfull + 8 * g, (uint32_t)(t & 1));
            tmem_fence_after();
            if (issuer && !dead) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (g * 8 + k < ksteps)
                  umma2_bf16(d, q_lo + (2 * g + k / 4) * (kCaChunk >> 4) + k % 4 * 2, k_lo + (2 * g + k / 4) * (kCaChunk >> 4) + k % 4 * 2, kIdS, g > 0 || k > 0);
              umma2_commit(b_kfree + 8 * g);
            }
            __syncwarp();
          }
        }
        if (issuer && !dead) umma2_commit(b_s + 8 * (t & 1));
        __syncwarp();
      }
      if (issuer) umma2_commit(b_end);
    }
    __syncwarp();
  } else if (warp == kCaSoftWarps + 1) {
    // ------------------------------------------------------------------ O += P V
    if (rank == 0) {
      const uint32_t id_o = umma_idesc(128, a.Dv < 256 ? a.Dv : 256, false, true);
      const uint32_t p_lo = umma_desc_lo(s_p, 16), v_lo = umma_desc_lo(s_v, 2 * kCaChunk);
      const bool issuer = elect_one();
      for (int t = 0; t < nt; ++t) {
        wait(b_p + 8 * (t & 1), (uint32_t)((t / 2) & 1));
#pragma unroll
        for (int b = 0; b < CaSmem::kVBlocks; ++b) {
          if (b < vblocks) {
            wait(b_vfull + 8 * b, (uint32_t)(t & 1));
            tmem_fence_after();
            if (issuer && !dead) {
              const uint32_t vb = v_lo + (uint32_t)(b * vper) * (2 * kCaChunk >> 4);
#pragma unroll
              for (int k = 0; k < kCaTile / 16; ++k)
                umma2_bf16(tmem + (uint32_t)(b * 128), p_lo + k / 4 * (kCaChunk >> 4) + k % 4 * 2, vb + k * (2048 >> 4), id_o, t > 0 || k > 0);
              umma2_commit(b_vfree + 8 * b);
            }
            __syncwarp();
          }
        }
      }
      if (issuer) umma2_commit(b_end + 8);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax
    const int row = tid & 63, half = tid >> 6 & 1, part = tid >> 7;   // keys 64 half + 32 part .. of the row
    {
      ra_put_q<kCaRows, kCaSoftWarps>(a, ra_smem, warp, lane, qv);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive_pair(in_first(b_q));
    }
    const int limit = row < rows ? min(rq.kv, ra_limit(a, rq, (row0 + row) / a.H)) : rq.kv;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t b_vdone = b_vfree + 8 * (vblocks - 1), p_first = in_first(b_p);
    const uint32_t o0 = (uint32_t)part * (ocols / 2), o1 = o0 + ocols / 2;   // columns of O that this thread scales and writes
    unsigned char *prow = ra_smem + CaSmem::p(chunks, vchunks) + half * kCaChunk + row * 128;
    float m = kRaLowest, l = 0.f;
    for (int t = 0; t < nt; ++t) {
      const int j0 = lo + t * kCaTile + half * 64 + part * 32;
      wait(b_m + 8 * (t % kCaMasks), (uint32_t)((t / kCaMasks) & 1));
      const uint32_t there = (uint32_t)(s_mask[(t % kCaMasks) * 2 + half] >> (32 * part));
      wait(b_s + 8 * (t & 1), (uint32_t)((t / 2) & 1));
      tmem_fence_after();
      float s[32];
      tmem_ld32(t_s + lanes + (uint32_t)((t & 1) * 64 + part * 32), s);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 32; ++i) s[i] *= a.scale_log2e;
      if (j0 + 32 > limit) {                      // the row does not see all of these keys
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (j0 + i >= limit) {
            odd |= !(fabsf(s[i]) <= 3.402823466e38f);
            s[i] = -INFINITY;
          }
        if (odd) s_odd[row] = 1;
      }
      if (there != ~0u) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (!(there >> i & 1)) s[i] = -INFINITY;
      }
      float x0 = s[0], x1 = s[1], x2 = s[2], x3 = s[3];
#pragma unroll
      for (int i = 4; i < 32; i += 4) { x0 = fmaxf(x0, s[i]); x1 = fmaxf(x1, s[i + 1]); x2 = fmaxf(x2, s[i + 2]); x3 = fmaxf(x3, s[i + 3]); }
      const float top = fmaxf(fmaxf(x0, x1), fmaxf(x2, x3));
      if (softmax_any<kCaSoft>(top - m > 8.f)) {
        s_red[(2 * half + part) * kCaRows + row] = top;
        softmax_sync<kCaSoft>();
        const float mn = fmaxf(m, fmaxf(fmaxf(s_red[row], s_red[kCaRows + row]), fmaxf(s_red[2 * kCaRows + row], s_red[3 * kCaRows + row])));
        const float al = exp2f(m - mn);
        softmax_sync<kCaSoft>();
        l *= al;
        m = mn;
        if (t > 0) {
          wait(b_vdone, (uint32_t)((t - 1) & 1));
          tmem_fence_after();
          for (uint32_t c = o0; c < o1; c += 16) {
            float o[16];
            tmem_ld_o(tmem + lanes + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= al;
            tmem_st_o(tmem + lanes + c, o);
          }
          tmem_wait_st();
        }
      }
      float l0 = 0.f, l1 = 0.f;
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        s[i] = ex2(s[i] - m);
        s[i + 1] = ex2(s[i + 1] - m);
        l0 += s[i];
        l1 += s[i + 1];
      }
      l += l0 + l1;
      if (t > 0) wait(b_vdone, (uint32_t)((t - 1) & 1));    // P of the last tile is used up
#pragma unroll
      for (int u = 0; u < 4; ++u)
        *reinterpret_cast<uint4 *>(prow + (((4 * part + u) ^ (row & 7)) << 4)) =
            make_uint4(pack_bf16(s[8 * u], s[8 * u + 1]), pack_bf16(s[8 * u + 2], s[8 * u + 3]), pack_bf16(s[8 * u + 4], s[8 * u + 5]),
                       pack_bf16(s[8 * u + 6], s[8 * u + 7]));
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tmem_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_pair(p_first + 8 * (t & 1));
    }
    // ---------------------------------------------------------------- epilogue
    softmax_sync<kCaSoft>();                       // (the last maxima are read)
    s_red[(2 * half + part) * kCaRows + row] = l;
    if (nt > 0) {
      wait(b_vdone, (uint32_t)((nt - 1) & 1));
      tmem_fence_after();
    }
    softmax_sync<kCaSoft>();
    const float sum = (s_red[row] + s_red[kCaRows + row]) + (s_red[2 * kCaRows + row] + s_red[3 * kCaRows + row]);
    const bool whole = a.splits == 1, live = row < rows && !s_odd[row];
    const int64_t grow = rq.q0 * a.H + row0;
    float *part_out = whole ? nullptr : a.partial + ((grow + row) * a.splits + split) * (a.Dv + 4);
    if (live && half == 0 && part == 0) {
      if (whole) a.lse[grow + row] = sum == 0.f ? -INFINITY : 0.6931471805599453f * (m + log2f(sum));
      else *reinterpret_cast<float2 *>(part_out + a.Dv) = make_float2(m, sum);
    }
    // rows go through shared memory (K, V and P are used up), so that they are written as whole lines
    const float fac = sum == 0.f ? 0.f : whole ? 1.f / sum : 1.f;
    const int width = a.Dv < 256 ? 64 : 128;      // columns of a block in this half's lanes
    const uint32_t pitch = (uint32_t)(a.Dv * (whole ? 2 : 4) + 16);   // (an odd number of 16-byte units: no bank conflicts)
    unsigned char *stage = ra_smem + CaSmem::k(chunks);
    for (uint32_t c = o0; c < o1; c += 32) {      // (32 columns at least: Dv = 128 has 64 in all)
      float o[32];
      if (nt > 0) {
        tmem_ld32(tmem + lanes + c, o);
        tmem_wait_ld();
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = nt > 0 && fac != 0.f ? o[i] * fac : 0.f;
      const int d = (int)(c / width) * 2 * width + half * width + (int)(c % width);
      if (whole) {
        uint4 *dst = reinterpret_cast<uint4 *>(stage + row * pitch + d * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          dst[i] = make_uint4(pack_bf16(o[8 * i], o[8 * i + 1]), pack_bf16(o[8 * i + 2], o[8 * i + 3]), pack_bf16(o[8 * i + 4], o[8 * i + 5]),
                              pack_bf16(o[8 * i + 6], o[8 * i + 7]));
      } else {
        float4 *dst = reinterpret_cast<float4 *>(stage + row * pitch + d * 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
      }
    }
    softmax_sync<kCaSoft>();
    // (eight rows a warp, their pieces taken out together: one after the other they took 3500 cycles)
    constexpr int kRowsWarp = kCaRows / kCaSoftWarps;
    const int units = a.Dv * (whole ? 2 : 4) / 16;
    const int64_t out_pitch = whole ? (int64_t)a.Dv * 2 : (int64_t)a.splits * (a.Dv + 4) * 4;
    char *to = whole ? reinterpret_cast<char *>(a.out + grow * a.Dv) : reinterpret_cast<char *>(a.partial + (grow * a.splits + split) * (a.Dv + 4));
    uint32_t live_rows = 0;
#pragma unroll
    for (int k = 0; k < kRowsWarp; ++k) {
      const int r = warp + k * kCaSoftWarps;
      live_rows |= (r < rows && !s_odd[r] ? 1u : 0u) << k;
    }
    for (int u = lane; u < units; u += 32) {
      uint4 v[kRowsWarp];
#pragma unroll
      for (int k = 0; k < kRowsWarp; ++k) v[k] = *reinterpret_cast<const uint4 *>(stage + (warp + k * kCaSoftWarps) * pitch + u * 16);
#pragma unroll
      for (int k = 0; k < kRowsWarp; ++k)
        if (live_rows >> k & 1) *reinterpret_cast<uint4 *>(to + (warp + k * kCaSoftWarps) * out_pitch + u * 16) = v[k];
    }
    tmem_fence_before();
    for (int r = warp; r < rows; r += kCaSoftWarps) {
      if (!s_odd[r]) continue;
      float o[kRaMaxDims / 32], pm, pl;
      const int g = row0 + r, tok = g / a.H;
      const int lim = min(rq.kv, ra_limit(a, rq, tok));
      ra_plain_row(a, n, a.q + (rq.q0 + tok) * a.q_token + (int64_t)(g - tok * a.H) * a.q_head, lo, min(hi, lim), o, pm, pl);
      const float inv = whole ? (pl == 0.f ? 0.f : 1.f / pl) : 1.f;
      float *to = whole ? nullptr : a.partial + ((grow + r) * a.splits + split) * (a.Dv + 4);
#pragma unroll
      for (int i = 0; i < kRaMaxDims / 32; ++i) {
        const int d = lane + 32 * i;
        if (d < a.Dv) {
          if (whole) a.out[(grow + r) * a.Dv + d] = __float2bfloat16(o[i] * inv);
          else to[d] = o[i];
        }
      }
      if (lane == 0) {
        if (whole) a.lse[grow + r] = pl == 0.f ? -INFINITY : 0.6931471805599453f * (pm + log2f(pl));
        else { to[a.Dv] = pm; to[a.Dv + 1] = pl; }
      }
    }
  }
  // both products over (the first SM's commits arrive here as well) before the tensor memory goes and the pair parts
  if (warp == kCaSoftWarps) { wait(b_end, 0); wait(b_end + 8, 0); }
  if (__syncthreads_or(dead)) ra_gave_up(a.status);
  // (relaxed: nothing is handed over, and a release would wait for the output to reach memory)
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
  if (warp == kCaSoftWarps) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Lays the records that a chunk's keys are out side by side as bf16 rows, dense rows a request, zeros where a key is absent
// or behind the context up to the end of its tile.  One pass over the records, for pages or formats that the pair kernel's
// boxes cannot take: many blocks then read what is expanded once.  One warp two keys.
__global__ void __launch_bounds__(256)
expand_records_kernel(const RecAtt a, const int dense, __nv_bfloat16 *__restrict__ out) {
  const int lane = threadIdx.x & 31;
  bool bad;
  const int per = (dense + 15) / 16;
  const int n = blockIdx.x / per, j0 = (blockIdx.x - n * per) * 16 + (threadIdx.x >> 5) * 2;
  const RaRequest rq = ra_request(a, n, bad);
  const int end = min(dense, (rq.kv + kCaTile - 1) / kCaTile * kCaTile);
  if (rq.qlen == 0 || j0 >= end) return;
  const uint8_t *rec[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int32_t idx = j0 + r < rq.kv ? ra_index(a, n, j0 + r, bad) : -1;
    rec[r] = idx < 0 ? nullptr : a.records + (int64_t)idx * a.f.E;
  }
  __nv_bfloat16 *o = out + ((int64_t)n * dense + j0) * a.f.D;
  for (int p = lane * 8; p < a.f.D; p += 256) {
    uint4 v[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      v[r] = make_uint4(0, 0, 0, 0);
      if (rec[r]) {
        if (p < a.f.Dq) {
          const uint2 c = *reinterpret_cast<const uint2 *>(rec[r] + p);
          const float s = *reinterpret_cast<const float *>(rec[r] + a.f.scales + p / kRecGroup * 4);
          const uint2 x = e4m3x4_to_bf16(c.x, s), y = e4m3x4_to_bf16(c.y, s);
          v[r] = make_uint4(x.x, x.y, y.x, y.y);
        } else {
          v[r] = *reinterpret_cast<const uint4 *>(rec[r] + a.f.Dq + 2 * (p - a.f.Dq));
        }
      }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
      if (j0 + r < end) *reinterpret_cast<uint4 *>(o + (int64_t)r * a.f.D + p) = v[r];
  }
}

}  // namespace
