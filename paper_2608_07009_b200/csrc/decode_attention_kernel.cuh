// Included by hisparse.cu: attention of single tokens over quantised records, without expanding them.  The same problem as
// record_attention_kernel.cuh for one token a request, where a record is read once and what counts is bytes: expanding a
// record to bf16 costs more shared-memory traffic (written, read as K, read as V: 3.3 KB) than its 656 bytes may take at the
// memory's rate.  Here the codes are the tensor cores' operand as they come (kind::f8f6f4), and the other operand is split
// into e4m3 terms, each 1/32 of the one before it (a term of at most 2^8 leaves at most 8, which is 2^8 / 32):
//   query    q / 2^a = t1 + t2 / 32, 2^a by row so that the largest is in [128, 256): two terms hold a bf16 number's 8 bits
//            exactly down to 2^-13 of the largest; below that they are off by at most 2^-22 of it.  S_g = codes_g t1^T,
//            codes_g t2^T by group of 128 numbers, because the scales are by record and group:
//            s = 2^a sum_g scale_g (S_g1 + S_g2 / 32) + tail, the bf16 tail in a product of its own.
//   weights  p scale_g / 2^k = w1 + w2 / 32 + w3 / 1024, k by row and group: p is rounded to f16 (11 bits; bf16 weights are 8),
//            which three terms hold, and what is too small for them is off by 2^-20.  What k follows is the largest p scale_g
//            so far, the weight and the size of one and the same record, which comes to lie above 2^lift and at most at 2^8, with
//            lift such that all keys together are off by at most 2^-8 of the largest p max |value| of the group, no more than
//            bf16's rounding: 0 for 2048 keys, 6 for 131072, the most that this kernel is given.  A small lift leaves the
//            maximum room, so that it moves for a fraction of the tiles (13 of 64; 32 x 32768 keys take 152 us with a lift of 4,
//            141 if it never moves).  A group of zeros has scale 1 and no size: it does not count, for which the codes of
//            groups with that scale are looked at.  (With the largest scale in place of the largest p scale, 142 us, a record of
//            zeros, or a large one that is not attended, took the weights of all others below the terms' reach.)  The running
//            maximum of a row is a whole number, so that k moves with it exactly.
//            O_g += codes_g w^T, out = 2^k (O_g1 + O_g2 / 32 + O_g3 / 1024).
// Splits of a context meet in a cluster where there are 2, 4 or 8: every block leaves its O, m and l in shared memory and merges
// a share of the numbers out of all of them, which saves the second kernel and its 2 x 33 KB a block through memory.
// Both products are transposed as there: 128 keys or 128 numbers are M, R query rows times their terms are N.
// 32 requests x 32768 keys of 656 bytes, 16 heads: 152 us, 4.5 TB/s, bound by the TMA's rows (each 128 bytes of such a record
// lie in two lines; loads alone take 129 us) and by the softmax warps (3000 cycles a tile, 2600 more where maxima move); with
// stages released as a whole instead of by group 14 us more.  32 x 2048 keys through a slot table: 22.1 us, where four-row
// gathers (25 cycles each) and a block's start and end count as much as its four tiles.
//   tile     128 keys: [group][key][128 bytes] of codes (K-major for S^T, MN-major for O^T) and [key][128 bytes] of tail, by TMA
//            boxes or four-row gathers; two stages
//   warps    0-7 softmax, two threads a key with half of the rows each (the key's scales come by plain loads a tile ahead;
//            with four warps the weights' terms took 2500 to 3100 cycles a tile, as long as its loads), 8 issues S^T, 9 O^T,
//            10-13 load

namespace {

constexpr int kDaTile = 128;
constexpr int kDaLoadWarps = 4;
constexpr int kDaSoftWarps = 8, kDaSoft = kDaSoftWarps * 32;
constexpr int kDaThreads = (kDaSoftWarps + 2 + kDaLoadWarps) * 32;
constexpr int kDaChunk = kDaTile * 128;          // bytes of a group of a tile
constexpr int kDaTermsQ = 2, kDaTermsP = 3;

template <int R>
struct DaSmem {
  static constexpr int kVG = R == 16 ? 4 : R == 32 ? 2 : 1;   // groups of values that tensor memory has room for beside R rows
  static constexpr int kRed = R / 2 * (1 + kVG);              // numbers that a softmax warp reduces: its rows, then [row][group]
  // stages, query codes [group][2 R][128], query tail [R][128], weights [group][term][R / 16][key][16]
  __host__ __device__ static constexpr uint32_t stage(const int cg, const int tail) { return (uint32_t)((cg + tail) * kDaChunk); }
  __host__ __device__ static constexpr uint32_t q(const int cg, const int tail) { return 2 * stage(cg, tail); }
  __host__ __device__ static constexpr uint32_t qt(const int cg, const int tail) { return q(cg, tail) + (uint32_t)(cg * kDaTermsQ * R * 128); }
  __host__ __device__ static constexpr uint32_t p(const int cg, const int tail) { return qt(cg, tail) + (uint32_t)(tail * R * 128); }
  __host__ __device__ static constexpr uint32_t bars(const int cg, const int tail, const int vg) { return p(cg, tail) + (uint32_t)(vg * kDaTermsP * R * kDaTile); }
  static constexpr int kBars = 2 + 2 * 4 + 2 + 2 + 1 + 2;
  __host__ __device__ static constexpr uint32_t tmem(const int cg, const int tail, const int vg) { return bars(cg, tail, vg) + 8 * (kBars + 1); }
  __host__ __device__ static constexpr uint32_t red(const int cg, const int tail, const int vg) { return (tmem(cg, tail, vg) + 31) / 16 * 16; }
  __host__ __device__ static constexpr uint32_t fac(const int cg, const int tail, const int vg) { return red(cg, tail, vg) + kDaSoftWarps * kRed * 4; }   // (a multiple of 16)
  __host__ __device__ static constexpr uint32_t qs(const int cg, const int tail, const int vg) { return fac(cg, tail, vg) + R * kVG * 4; }
  __host__ __device__ static constexpr uint32_t max(const int cg, const int tail, const int vg) { return qs(cg, tail, vg) + R * 4; }
  __host__ __device__ static constexpr uint32_t inv(const int cg, const int tail, const int vg) { return max(cg, tail, vg) + R * 4; }
  __host__ __device__ static constexpr uint32_t total(const int cg, const int tail, const int vg) { return inv(cg, tail, vg) + R * kVG * 4; }
};

__host__ __device__ constexpr int da_cols(const int R, const int cg, const int tail, const int vg) {   // tensor-memory columns
  return 2 * (cg * kDaTermsQ + tail) * R + vg * kDaTermsP * R;
}
// kind::f8f6f4, e4m3 operands, fp32 accumulators
__host__ __device__ constexpr uint32_t umma_idesc_e4m3(const int M, const int N, const bool a_mn, const bool b_mn) {
  return 1u << 4 | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;
}
__device__ __forceinline__ void umma_e4m3(const uint32_t d, const uint32_t a_lo, const uint32_t a_hi, const uint32_t b_lo, const uint32_t b_hi,
                                          const uint32_t idesc, const bool add) {
  asm volatile("{ .reg .pred p; .reg .b64 a, b; setp.ne.u32 p, %6, 0; mov.b64 a, {%1, %2}; mov.b64 b, {%3, %4};"
               " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %5, p; }"
               ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// MN-major without swizzle: blocks of 16 numbers x 8 keys, 128 bytes each; keys go on at `lbo` (low word), numbers at 2048
constexpr uint32_t kDaPDescHi = 2048u >> 4 | 1u << 14;

constexpr float kDaStep = 32.f;                  // from one term to the next
constexpr int kDaMaxKeys = 1 << 17;
constexpr int kDaLeast = -120;                   // smallest k: 2^-k times a scale and a weight stays a number

// The codes of a pair of f16 numbers, and kDaStep times what they leave (exact: both are multiples of the number's last bit)
__device__ __forceinline__ uint32_t e4m3_term(__half2 &x) {
  const __half2_raw in = x;
  const uint32_t c = (uint32_t)__nv_cvt_halfraw2_to_fp8x2(in, __NV_SATFINITE, __NV_E4M3);
  const __half2 back = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3));
  x = __hmul2(__hsub2(x, back), __float2half2_rn(kDaStep));
  return c;
}

// 2^e of a whole number, 0 below 2^-126
__device__ __forceinline__ float pow2_whole(const float e) {
  return __int_as_float((min(max(__float2int_rn(e), -127), 127) + 127) << 23);
}
__device__ __forceinline__ float warp_max(const float v) {   // (a NaN is ignored)
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// Lane i's v[0] becomes the largest v[i] of the warp's lanes: every step hands over half of the numbers that are left.
__device__ __forceinline__ void warp_max_each(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = 16; n; n >>= 1) {
    const bool up = lane & n;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float away = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + n], n);
      v[i] = fmaxf(up ? v[i + n] : v[i], away);
    }
  }
}
// 32 lanes x 8 columns
__device__ __forceinline__ void tmem_ld8(const uint32_t addr, float *v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(addr));
}
__device__ __forceinline__ void tmem_st8(const uint32_t addr, const float *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
               ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "r"(addr) : "memory");
}

__device__ __forceinline__ float peer_f32(const uint32_t addr, const uint32_t rank) {
  float v;
  asm volatile("{ .reg .b32 r; mapa.shared::cluster.u32 r, %1, %2; ld.shared::cluster.f32 %0, [r]; }" : "=f"(v) : "r"(addr), "r"(rank) : "memory");
  return v;
}
__device__ __forceinline__ float4 peer_f32x4(const uint32_t addr, const uint32_t rank) {
  float4 v;
  asm volatile("{ .reg .b32 r; mapa.shared::cluster.u32 r, %4, %5; ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [r]; }"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr), "r"(rank) : "memory");
  return v;
}

// Merges the blocks of a cluster, one split each: o [row][Dv], m [row] and l [row] at these shared-memory addresses in all of
// them; `w` is R * splits + R floats of the block's own.  All threads of the cluster.
template <int R>
__device__ __forceinline__ void da_merge(const RecAtt &a, const int64_t grow, const int rows, const uint32_t rank, const uint32_t o,
                                         const uint32_t m, const uint32_t l, float *w) {
  __syncwarp();                                   // (lanes whose waits ran out one by one)
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  const int tid = threadIdx.x;
  if (tid < rows) {
    float ms[8], ls[8], M = kRaLowest, sum = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < a.splits) { ms[s] = peer_f32(m + tid * 4, s); ls[s] = peer_f32(l + tid * 4, s); }
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < a.splits && ls[s] != 0.f) M = fmaxf(M, ms[s]);
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < a.splits) {
        const float x = ls[s] != 0.f ? exp2f(ms[s] - M) : 0.f;
        w[s * R + tid] = x;
        if (ls[s] != 0.f) sum += x * ls[s];
      }
    w[a.splits * R + tid] = sum != 0.f ? 1.f / sum : 0.f;
    if (rank == 0) a.lse[grow + tid] = sum == 0.f ? -INFINITY : 0.6931471805599453f * (M + log2f(sum));
  }
  __syncthreads();
  const int quads = a.Dv / 4, total = rows * quads, share = (total + a.splits - 1) / a.splits;
  const int end = min(total, ((int)rank + 1) * share);
  for (int i = (int)rank * share + tid; i < end; i += kDaThreads) {
    const int r = i / quads;
    float4 v[8], x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < a.splits) v[s] = peer_f32x4(o + (uint32_t)i * 16, s);
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < a.splits) {
        const float ws = w[s * R + r];
        if (ws != 0.f) { x.x += ws * v[s].x; x.y += ws * v[s].y; x.z += ws * v[s].z; x.w += ws * v[s].w; }
      }
    const float inv = w[a.splits * R + r];
    *reinterpret_cast<uint2 *>(a.out + grow * a.Dv + (int64_t)i * 4) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
  }
  // (relaxed: only that no block goes while another reads from it)
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}

template <int R>
__global__ void __launch_bounds__(kDaThreads, 1)
decode_attention_kernel(const RecAtt a, const float lift, const int cluster, const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap gather_map) {
  extern __shared__ __align__(1024) unsigned char ra_smem[];
  using L = DaSmem<R>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cg = a.f.Dq / 128, tail = a.f.D > a.f.Dq ? 1 : 0, vg = a.Dv / 128;
  const uint32_t sbase = smem_u32(ra_smem), s_q = sbase + L::q(cg, tail), s_qt = sbase + L::qt(cg, tail), s_p = sbase + L::p(cg, tail);
  const uint32_t stage_bytes = L::stage(cg, tail);
  const uint32_t b_full = sbase + L::bars(cg, tail, vg), b_empty = b_full + 16, b_s = b_empty + 64, b_p = b_s + 16, b_q = b_p + 16, b_end = b_q + 8;
  float *s_red = reinterpret_cast<float *>(ra_smem + L::red(cg, tail, vg));   // [warp][kRed]
  float *s_fac = reinterpret_cast<float *>(ra_smem + L::fac(cg, tail, vg));   // [row][group], at the end [row]
  float *s_qs = reinterpret_cast<float *>(ra_smem + L::qs(cg, tail, vg));     // [row] 2^a times the scale, in the base-2 domain

  float *s_max = reinterpret_cast<float *>(ra_smem + L::max(cg, tail, vg));   // [row] running maximum of the scores, base 2, a whole number
  float *s_inv = reinterpret_cast<float *>(ra_smem + L::inv(cg, tail, vg));   // [row][group] 2^-k

  const uint32_t item = blockIdx.x / (uint32_t)a.splits, split = blockIdx.x - item * a.splits;
  const int n = (int)(item / (uint32_t)a.row_tiles), rt = (int)(item - (uint32_t)n * a.row_tiles);
  bool bad_req;
  const RaRequest rq = ra_request(a, n, bad_req);
  if (bad_req && tid == 0 && a.status) atomicOr(a.status, HISPARSE_STATUS_OUT_OF_RANGE);
  const int row0 = rt * R, rows = min(R, rq.qlen * a.H - row0);
  if (rows <= 0) return;
  // (one token a request: every row sees the whole context)
  const int tiles_all = (rq.kv + kDaTile - 1) / kDaTile, per = (tiles_all + a.splits - 1) / a.splits;
  const int lo = (int)split * per * kDaTile, hi = min(rq.kv, lo + per * kDaTile);
  const int nt = hi > lo ? (hi - lo + kDaTile - 1) / kDaTile : 0;

  bool dead = false;
  auto wait = [&](const uint32_t bar, const uint32_t parity) { if (!dead && !mbar_wait_quick(bar, parity)) dead = true; };

  // the first tiles' table entries are on their way while barriers and tensor memory are set up
  const int mykey = warp >= kDaSoftWarps + 2 ? (warp - kDaSoftWarps - 2) * 32 + lane : tid & 127;
  auto entry = [&](const int t) { const int j = lo + t * kDaTile + mykey; return j < hi ? ra_entry(a, n, j) : -1; };
  int32_t e = -1, e1 = -1;
  if (warp < kDaSoftWarps || warp >= kDaSoftWarps + 2) { e = entry(0); e1 = entry(1); }
  const uint32_t scols = (uint32_t)((cg * kDaTermsQ + tail) * R), need = (uint32_t)da_cols(R, cg, tail, vg);
  const uint32_t cols = need <= 128 ? 128 : need <= 256 ? 256 : 512;
  if (tid < L::kBars) {
    // full, empty by stage and group of values, S, P, Q, ends
    const uint32_t count = tid < 2 ? kDaLoadWarps : tid == 12 || tid == 13 ? kDaSoft : tid == 14 ? kDaSoftWarps : 1;
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b_full + 8 * tid), "r"(count) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kDaSoftWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + L::tmem(cg, tail, vg)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(ra_smem + L::tmem(cg, tail, vg));
  const uint32_t t_o = tmem + 2 * scols;          // two buffers of S^T, then O^T
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (warp >= kDaSoftWarps + 2) {
    // ------------------------------------------------------------------ loaders: 32 keys a warp
    const int w = warp - kDaSoftWarps - 2;
    const bool issuer = elect_one();
    const int none = ra_none(a);
    bool bad_page = false;
    for (int t = 0; t < nt; ++t) {
      const int st = t & 1, j0 = lo + t * kDaTile;
      const int32_t idx = ra_resolve(a, e, j0 + mykey, bad_page), y = idx < 0 ? none : idx;
      e = e1;
      e1 = entry(t + 2);
      // A chunk may be overwritten when the products that read it are done: S^T, and for a group of values its O^T.
      const uint32_t bar = b_full + 8 * st, dst = sbase + (uint32_t)st * stage_bytes + (uint32_t)(w * 32 * 128);
      const bool boxes = a.box && j0 + kDaTile <= hi;   // 32 keys of a page
      const int first = __shfl_sync(0xffffffffu, y, 0);
      // otherwise lane i takes keys 4 i .. 4 i + 3 (against one lane for all: 36.6 us instead of 38.4 on 77 x 1333 short records)
      int4 r;
      r.x = __shfl_sync(0xffffffffu, y, 4 * lane & 31); r.y = __shfl_sync(0xffffffffu, y, (4 * lane + 1) & 31);
      r.z = __shfl_sync(0xffffffffu, y, (4 * lane + 2) & 31); r.w = __shfl_sync(0xffffffffu, y, (4 * lane + 3) & 31);
      if (t < 2 && !boxes) {                      // (nothing to wait for: all of a lane's copies at once)
        if (issuer) mbar_arrive_tx(bar, (uint32_t)((cg + tail) * 32 * 128));
        __syncwarp();
        if (lane < 8)
          for (int c = 0; c < cg + tail; ++c) tma_gather4(dst + (uint32_t)(c * kDaChunk + lane * 4 * 128), &gather_map, c * 128, r, bar);
        __syncwarp();
        continue;
      }
      for (int i = 0; i < cg + tail; ++i) {
        const int c = i + vg < cg + tail ? i + vg : i + vg - cg - tail;   // (chunks that are no values are free first)
        if (t >= 2) {
          wait(c < vg ? b_empty + 8 * (4 * st + c) : b_s + 8 * st, (uint32_t)((t / 2 - 1) & 1));
          dead = __any_sync(0xffffffffu, dead);
        }
        if (i == 0) {
          if (issuer) mbar_arrive_tx(bar, dead ? 0u : (uint32_t)((cg + tail) * 32 * 128));
          __syncwarp();
        }
        if (dead) continue;
        if (boxes) {
          if (issuer) tma_rows(dst + (uint32_t)c * kDaChunk, &rows_map, c * 128, first, bar);
        } else if (lane < 8) {
          tma_gather4(dst + (uint32_t)(c * kDaChunk + lane * 4 * 128), &gather_map, c * 128, r, bar);
        }
      }
      if (boxes && !dead) {
        // the tile after the next into L2: a load from there takes a third of the time
        const int ahead = ra_resolve(a, __shfl_sync(0xffffffffu, e1, 0), j0 + 2 * kDaTile + w * 32, bad_page);
        if (issuer && ahead >= 0 && j0 + 3 * kDaTile <= hi)
          for (int c = 0; c < cg + tail; ++c)
            asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(&rows_map), "r"(c * 128), "r"(ahead) : "memory");
      }
      __syncwarp();
    }
    if (bad_page && a.status) atomicOr(a.status, HISPARSE_STATUS_OUT_OF_RANGE);
  } else if (warp == kDaSoftWarps) {
    // ------------------------------------------------------------------ S^T = K Q^T, by group and term
    constexpr uint32_t kIdS = umma_idesc_e4m3(128, kDaTermsQ * R, false, false), kIdT = umma_idesc(128, R, false, false);
    const int tsteps = (a.f.D - a.f.Dq) / 16;
    const uint32_t k_lo = umma_desc_lo(sbase, 16), q_lo = umma_desc_lo(s_q, 16), qt_lo = umma_desc_lo(s_qt, 16);
    const bool issuer = elect_one();
    wait(b_q, 0);
    for (int t = 0; t < nt; ++t) {
      const int st = t & 1;
      const uint32_t d = tmem + (uint32_t)st * scols, ka = k_lo + ((uint32_t)st * stage_bytes >> 4);
      if (t >= 2) wait(b_p + 8 * st, (uint32_t)((t / 2 - 1) & 1));   // S^T of the last tile but one is read
      wait(b_full + 8 * st, (uint32_t)((t / 2) & 1));
      tmem_fence_after();
      if (issuer && !dead) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if (g < cg)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              umma_e4m3(d + (uint32_t)(g * kDaTermsQ * R), ka + g * (kDaChunk >> 4) + 2 * k, kUmmaDescHi,
                        q_lo + g * (kDaTermsQ * R * 128 >> 4) + 2 * k, kUmmaDescHi, kIdS, k > 0);
        const uint32_t kt = ka + (uint32_t)cg * (kDaChunk >> 4), dt = d + (uint32_t)(cg * kDaTermsQ * R);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < tsteps) umma_bf16(dt, kt + 2 * k, qt_lo + 2 * k, kIdT, k > 0);
        umma_commit(b_s + 8 * st);
      }
      __syncwarp();
    }
    if (issuer) umma_commit(b_end);
    wait(b_end, 0);
    __syncwarp();
  } else if (warp == kDaSoftWarps + 1) {
    // ------------------------------------------------------------------ O^T += V^T W^T, by group
    constexpr uint32_t kIdO = umma_idesc_e4m3(128, kDaTermsP * R, true, true);
    const uint32_t v_lo = umma_desc_lo(sbase, 16), p_lo = umma_desc_lo(s_p, 128);
    const bool issuer = elect_one();
    for (int t = 0; t < nt; ++t) {
      const int st = t & 1;
      const uint32_t va = v_lo + ((uint32_t)st * stage_bytes >> 4);
      wait(b_p + 8 * st, (uint32_t)((t / 2) & 1));
      tmem_fence_after();
      if (issuer && !dead) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          if (g >= vg) break;
#pragma unroll
          for (int k = 0; k < kDaTile / 32; ++k)
            umma_e4m3(t_o + (uint32_t)(g * kDaTermsP * R), va + g * (kDaChunk >> 4) + k * (4096 >> 4), kUmmaDescHi,
                        p_lo + g * (kDaTermsP * R * kDaTile >> 4) + k * (512 >> 4), kDaPDescHi, kIdO, t > 0 || k > 0);
          umma_commit(b_empty + 8 * (4 * st + g));
        }
      }
      __syncwarp();
    }
    if (issuer) umma_commit(b_end + 8);
    wait(b_end + 8, 0);
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax
    constexpr int RH = R / 2, VG = L::kVG, W = L::kRed;
    const int key = tid & 127, part = tid >> 7, r0 = part * RH;   // this thread's key and rows
    // the records' scales, a tile ahead
    bool ignore = false;
    auto resolve = [&](const int t, const int32_t e) { return ra_resolve(a, e, lo + t * kDaTile + key, ignore); };
    auto scales = [&](const int32_t idx) {
      return idx < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4 *>(a.records + (int64_t)idx * a.f.E + a.f.scales);
    };
    // query rows: a lane has 16 numbers of the codes' part, which become 16 codes of either term, and 8 of the tail
    // (two rows in flight a warp)
    constexpr int kRowsWarp = 2;
#pragma unroll 1
    for (int base = 0; base < R; base += kRowsWarp * kDaSoftWarps) {
    uint4 raw[kRowsWarp][2], rawt[kRowsWarp];
#pragma unroll
    for (int i = 0; i < kRowsWarp; ++i) {
      const int r = base + warp + i * kDaSoftWarps, g = row0 + r, tok = g / a.H;
      const __nv_bfloat16 *src = a.q + (rq.q0 + tok) * a.q_token + (int64_t)(g - tok * a.H) * a.q_head;
      raw[i][0] = raw[i][1] = rawt[i] = make_uint4(0, 0, 0, 0);
      if (r < rows && lane * 16 < a.f.Dq) {
        raw[i][0] = reinterpret_cast<const uint4 *>(src + lane * 16)[0];
        raw[i][1] = reinterpret_cast<const uint4 *>(src + lane * 16)[1];
      }
      const int d = a.f.Dq + lane * 8;
      if (r < rows && lane < 8 && d < a.f.D) rawt[i] = *reinterpret_cast<const uint4 *>(src + d);
    }
#pragma unroll
    for (int i = 0; i < kRowsWarp; ++i) {
      const int r = base + warp + i * kDaSoftWarps;
      const uint32_t x[8] = {raw[i][0].x, raw[i][0].y, raw[i][0].z, raw[i][0].w, raw[i][1].x, raw[i][1].y, raw[i][1].z, raw[i][1].w};
      uint32_t top = 0;                           // pattern of the largest magnitude (bf16 patterns are ordered as the numbers)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, max(x[j] & 0x7fffu, x[j] >> 16 & 0x7fffu));
#pragma unroll
      for (int o = 16; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      // 2^a: the largest magnitude comes to lie in [128, 256) (a row below 2^-112 stays smaller: its scores are zeros)
      int ex = (int)(top >> 7) - 127 - 7;
      ex = ex > 120 ? 120 : ex < -119 ? -119 : ex;
      const float down = __uint_as_float((uint32_t)(127 - ex) << 23), up = __uint_as_float((uint32_t)(127 + ex) << 23);
      uint32_t c1[4], c2[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c1[j] = c2[j] = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t v = x[2 * j + h];
          float f0 = __uint_as_float(v << 16), f1 = __uint_as_float(v & 0xffff0000u);
          // (an infinity must not saturate to the largest code)
          f0 = fabsf(f0) <= 3.402823466e38f ? f0 * down : __uint_as_float(0x7fc00000u);
          f1 = fabsf(f1) <= 3.402823466e38f ? f1 * down : __uint_as_float(0x7fc00000u);
          __half2 f = __floats2half2_rn(f0, f1);
          c1[j] |= e4m3_term(f) << (16 * h);
          c2[j] |= e4m3_term(f) << (16 * h);
        }
      }
      if (lane * 16 < a.f.Dq) {
        unsigned char *to = ra_smem + L::q(cg, tail) + (lane >> 3) * (kDaTermsQ * R * 128);
        const int u = lane & 7;
        *reinterpret_cast<uint4 *>(to + r * 128 + ((u ^ (r & 7)) << 4)) = make_uint4(c1[0], c1[1], c1[2], c1[3]);
        *reinterpret_cast<uint4 *>(to + (R + r) * 128 + ((u ^ (r & 7)) << 4)) = make_uint4(c2[0], c2[1], c2[2], c2[3]);
      }
      if (tail && lane < 8) *reinterpret_cast<uint4 *>(ra_smem + L::qt(cg, tail) + r * 128 + ((lane ^ (r & 7)) << 4)) = rawt[i];
      if (lane == 0) s_qs[r] = up * a.scale_log2e;
    }
    }
    if (tid < R) s_max[tid] = kRaLowest;
    if (tid < R * VG) s_inv[tid] = pow2_whole((float)-kDaLeast);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(b_q);
    softmax_sync<kDaSoft>();                      // s_qs of every warp's rows
    int32_t mine = resolve(0, e);
    float4 sc = scales(mine);
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float *red = s_red + part * 4 * W;      // of this part's four warps
    float l[RH];
#pragma unroll
    for (int r = 0; r < RH; ++r) l[r] = 0.f;
    for (int t = 0; t < nt; ++t) {
      const int st = t & 1;
      const float sg[4] = {sc.x, sc.y, sc.z, sc.w};
      const bool here = mine >= 0;
      mine = resolve(t + 1, e1);
      e1 = entry(t + 2);
      sc = scales(mine);
      wait(b_s + 8 * st, (uint32_t)((t / 2) & 1));
      tmem_fence_after();
      // scores of this thread's key
      float x[RH];
      const uint32_t ts = tmem + lanes + (uint32_t)st * scols + (uint32_t)r0;
#pragma unroll
      for (int h = 0; h < RH; h += 8) {
        float acc[8], s3[8];
        if (tail) tmem_ld8(ts + (uint32_t)(cg * kDaTermsQ * R + h), s3);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          if (g < cg) {
            float s1[8], s2[8];
            tmem_ld8(ts + (uint32_t)(g * kDaTermsQ * R + h), s1);
            tmem_ld8(ts + (uint32_t)(g * kDaTermsQ * R + R + h), s2);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += sg[g] * (s1[i] + (1.f / kDaStep) * s2[i]);
          }
        }
        float qs[8];
        *reinterpret_cast<float4 *>(qs) = *reinterpret_cast<const float4 *>(s_qs + r0 + h);
        *reinterpret_cast<float4 *>(qs + 4) = *reinterpret_cast<const float4 *>(s_qs + r0 + h + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[h + i] = here ? acc[i] * qs[i] + (tail ? s3[i] * a.scale_log2e : 0.f) : -INFINITY;
      }
      // the scales that the weights are measured with: none where the group is zeros
      // (one branch for all groups: one each took 250 cycles a tile)
      float se[VG];
      bool ones = false;
#pragma unroll
      for (int g = 0; g < VG; ++g) {
        se[g] = here && g < vg ? sg[g] : 0.f;
        ones |= se[g] == 1.f;
      }
      if (ones) {
        wait(b_full + 8 * st, (uint32_t)((t / 2) & 1));   // (it has come; the wait makes the codes visible to this thread)
#pragma unroll
        for (int g = 0; g < VG; ++g) {
          if (se[g] != 1.f) continue;
          const unsigned char *row = ra_smem + (uint32_t)st * stage_bytes + g * kDaChunk + key * 128;
          uint32_t some = 0;
#pragma unroll 1
          for (int u = 0; u < 8 && !some; ++u) {
            const uint4 v = *reinterpret_cast<const uint4 *>(row + ((u ^ (key & 7)) << 4));
            some = (v.x | v.y | v.z | v.w) & 0x7f7f7f7fu;
          }
          if (!some) se[g] = 0.f;
        }
      }
      // weights against the running maxima, and whether one is above 2^8
      float p[RH], w[RH * VG];
      auto weigh = [&] {
        bool over = false;
#pragma unroll
        for (int r = 0; r < RH; r += 4) {
          const float4 m = *reinterpret_cast<const float4 *>(s_max + r0 + r);
          p[r] = ex2(x[r] - m.x); p[r + 1] = ex2(x[r + 1] - m.y); p[r + 2] = ex2(x[r + 2] - m.z); p[r + 3] = ex2(x[r + 3] - m.w);
          over |= fmaxf(fmaxf(p[r], p[r + 1]), fmaxf(p[r + 2], p[r + 3])) > 256.f;
        }
#pragma unroll
        for (int i = 0; i < RH * VG; i += 4) {
          const float4 inv = *reinterpret_cast<const float4 *>(s_inv + r0 * VG + i);
          // (in this order no product is out of range before it is known to be above 2^8)
          w[i] = p[i / VG] * se[i % VG] * inv.x;
          w[i + 1] = p[(i + 1) / VG] * se[(i + 1) % VG] * inv.y;
          w[i + 2] = p[(i + 2) / VG] * se[(i + 2) % VG] * inv.z;
          w[i + 3] = p[(i + 3) / VG] * se[(i + 3) % VG] * inv.w;
          over |= fmaxf(fmaxf(w[i], w[i + 1]), fmaxf(w[i + 2], w[i + 3])) > 256.f;
        }
        return over;
      };
      if (softmax_any<kDaSoft>(weigh())) {
#pragma unroll
        for (int r = 0; r < RH; ++r) {
          const float v = warp_max(x[r]);
          if (lane == 0) s_red[warp * W + r] = v;
        }
        float y[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const float sc2 = i < RH * VG ? se[i % VG] : 0.f;
          // (the exponent of the power of two at or above the scale)
          y[i] = sc2 > 0.f ? x[i / VG < RH ? i / VG : 0] + (float)((int)((__float_as_uint(sc2) + 0x7fffffu) >> 23) - 127) : -INFINITY;
        }
        warp_max_each(y);
        if (lane < RH * VG) s_red[warp * W + RH + lane] = y[0];
        float before[RH];
#pragma unroll
        for (int r = 0; r < RH; r += 4) *reinterpret_cast<float4 *>(before + r) = *reinterpret_cast<const float4 *>(s_max + r0 + r);
        softmax_sync<kDaSoft>();
        const int mr = key / VG;                   // a thread a row and group
        float mn = 0.f, inv = 0.f;
        if (key < RH * VG) {
          const float *v4 = red + mr, *y4 = red + RH + key;
          const float v = fmaxf(fmaxf(v4[0], v4[W]), fmaxf(v4[2 * W], v4[3 * W])), top = fmaxf(fmaxf(y4[0], y4[W]), fmaxf(y4[2 * W], y4[3 * W]));
          mn = fmaxf(s_max[r0 + mr], ceilf(v));
          // k such that the largest weight so far lies between 2^lift and 2^(lift + 1)
          const float drop = s_max[r0 + mr] - mn, k0 = (float)(127 - (int)(__float_as_uint(s_inv[r0 * VG + key]) >> 23));
          const float k = fminf(fmaxf(ceilf(fmaxf(top - mn, k0 + lift + 1.f + drop)) - (lift + 1.f), (float)kDaLeast), 126.f);
          inv = pow2_whole(-k);
          s_fac[r0 * VG + key] = pow2_whole(drop + k0 - k);
        }
        softmax_sync<kDaSoft>();
        if (key < RH * VG) {
          s_inv[r0 * VG + key] = inv;
          if (key % VG == 0) s_max[r0 + mr] = mn;
        }
        if (t > 0) {
          wait(b_empty + 8 * (4 * ((t - 1) & 1) + vg - 1), (uint32_t)(((t - 1) / 2) & 1));
          tmem_fence_after();
#pragma unroll
          for (int g = 0; g < VG; ++g) {
            if (g >= vg) break;
#pragma unroll 1
            for (int h = 0; h < RH; h += 8) {
              float o[kDaTermsP][8];
              const uint32_t at = t_o + lanes + (uint32_t)(g * kDaTermsP * R + r0 + h);
#pragma unroll
              for (int k = 0; k < kDaTermsP; ++k) tmem_ld8(at + (uint32_t)(k * R), o[k]);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float f = s_fac[(r0 + h + i) * VG + g];
#pragma unroll
                for (int k = 0; k < kDaTermsP; ++k) o[k][i] *= f;
              }
#pragma unroll
              for (int k = 0; k < kDaTermsP; ++k) tmem_st8(at + (uint32_t)(k * R), o[k]);
            }
          }
          tmem_wait_st();
        }
        softmax_sync<kDaSoft>();                   // (s_max and s_inv are written, s_fac and s_red may be again)
        weigh();
#pragma unroll
        for (int r = 0; r < RH; r += 4) {
          const float4 m = *reinterpret_cast<const float4 *>(s_max + r0 + r);
          l[r] *= pow2_whole(before[r] - m.x); l[r + 1] *= pow2_whole(before[r + 1] - m.y);
          l[r + 2] *= pow2_whole(before[r + 2] - m.z); l[r + 3] *= pow2_whole(before[r + 3] - m.w);
        }
      }
#pragma unroll
      for (int r = 0; r < RH; ++r) l[r] += p[r];
      if (t > 0) wait(b_empty + 8 * (4 * ((t - 1) & 1) + vg - 1), (uint32_t)(((t - 1) / 2) & 1));   // the weights of the last tile are used up
#pragma unroll
      for (int g = 0; g < VG; ++g) {
        if (g < vg) {
#pragma unroll
          for (int h = 0; h < RH; h += 8) {
            uint32_t c[kDaTermsP][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float *v = w + (h + 4 * i) * VG + g;
              __half2 y0 = __floats2half2_rn(v[0], v[VG]);
              __half2 y1 = __floats2half2_rn(v[2 * VG], v[3 * VG]);
#pragma unroll
              for (int k = 0; k < kDaTermsP; ++k) { const uint32_t lo2 = e4m3_term(y0); c[k][i] = lo2 | e4m3_term(y1) << 16; }
            }
            const int unit = (r0 + h) / 8;         // eight rows: half of a block of 16
            unsigned char *to = ra_smem + L::p(cg, tail) + (unit >> 1) * (kDaTile * 16) + key * 16 + (unit & 1) * 8;
#pragma unroll
            for (int k = 0; k < kDaTermsP; ++k)
              *reinterpret_cast<uint2 *>(to + (g * kDaTermsP + k) * (R / 16) * (kDaTile * 16)) = make_uint2(c[k][0], c[k][1]);
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tmem_fence_before();
      mbar_arrive(b_p + 8 * st);
    }
    // ---------------------------------------------------------------- epilogue
    softmax_sync<kDaSoft>();
#pragma unroll
    for (int r = 0; r < RH; ++r) {
      float v = l[r];
#pragma unroll
      for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane == 0) s_red[warp * W + r] = v;
    }
    if (nt > 0) {
      wait(b_empty + 8 * (4 * ((nt - 1) & 1) + vg - 1), (uint32_t)(((nt - 1) / 2) & 1));
      tmem_fence_after();
    }
    softmax_sync<kDaSoft>();
    const bool whole = a.splits == 1;
    const int64_t grow = rq.q0 * a.H + row0;
    const int64_t pstride = cluster ? a.Dv : (int64_t)a.splits * (a.Dv + 4);
    // (in a cluster O goes to shared memory, where the stages are used up)
    float *part_out = whole ? nullptr : cluster ? reinterpret_cast<float *>(ra_smem) : a.partial + (grow * a.splits + split) * (a.Dv + 4);
    if (key < RH) {
      const int r = r0 + key;
      const float sum = (red[key] + red[W + key]) + (red[2 * W + key] + red[3 * W + key]);
      s_fac[r] = sum == 0.f ? 0.f : whole ? 1.f / sum : 1.f;
      s_qs[r] = sum;                               // (the query's factors are no longer needed)
      if (r < rows && !cluster) {
        if (whole) a.lse[grow + r] = sum == 0.f ? -INFINITY : 0.6931471805599453f * (s_max[r] + log2f(sum));
        else *reinterpret_cast<float2 *>(part_out + r * pstride + a.Dv) = make_float2(s_max[r], sum);
      }
    }
    softmax_sync<kDaSoft>();
#pragma unroll 1
    for (int g = 0; g < vg; ++g) {
      const int d = g * 128 + key;                 // (a lane is a number of the group now)
#pragma unroll
      for (int h = 0; h < RH; h += 8) {
        if (r0 + h >= rows) break;
        float o[8], o2[8], o3[8];
        if (nt > 0) {
          const uint32_t at = t_o + lanes + (uint32_t)(g * kDaTermsP * R + r0 + h);
          tmem_ld8(at, o);
          tmem_ld8(at + R, o2);
          tmem_ld8(at + 2 * R, o3);
          tmem_wait_ld();
        }
        float fac[8];
        *reinterpret_cast<float4 *>(fac) = *reinterpret_cast<const float4 *>(s_fac + r0 + h);
        *reinterpret_cast<float4 *>(fac + 4) = *reinterpret_cast<const float4 *>(s_fac + r0 + h + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = r0 + h + i;
          const float up = __uint_as_float(0x7f000000u - __float_as_uint(s_inv[r * VG + g])) * fac[i];   // 2^k, and the normaliser
          const float v = nt > 0 && fac[i] != 0.f ? (o[i] + (1.f / kDaStep) * (o2[i] + (1.f / kDaStep) * o3[i])) * up : 0.f;
          if (r < rows) {
            if (whole) a.out[(grow + r) * a.Dv + d] = __float2bfloat16(v);
            else part_out[r * pstride + d] = v;
          }
        }
      }
    }
    tmem_fence_before();
  }
  if (cluster) da_merge<R>(a, rq.q0 * a.H + row0, rows, split, sbase, sbase + L::max(cg, tail, vg), sbase + L::qs(cg, tail, vg),
                           reinterpret_cast<float *>(ra_smem + L::p(cg, tail)));
  if (__syncthreads_or(dead)) ra_gave_up(a.status);
  if (warp == kDaSoftWarps) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
}

}  // namespace
