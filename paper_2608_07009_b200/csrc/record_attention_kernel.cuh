// Included by hisparse.cu: attention over records of a caller's pool, in either record format, for one new token a
// request (a slot table) or a chunk of them (a paged cache).
//
//   s[r, j] = scale * q[r] . key(j),   out[r] = sum_j softmax_j(s[r, :]) value(j),   lse[r] = log sum_j exp s[r, j]
//
// Rows r = (token, head) of one request share every key: record j's key is all D numbers, its value the first Dv.
//
// Both products run on the tensor cores transposed, S^T = K Q^T and O^T = V^T P^T, so that the long axis of a tile is
// the M of the instruction and the query rows are its N: 16, 32 or 64 rows a block without padding to 128.
// O^T (Dv x N fp32) then takes Dv / 128 * N tensor-memory columns, at most 256 of 512, next to two buffers of S^T,
// where 128 rows of O with Dv = 512 would fill the tensor memory alone.
//   tile     64 keys, staged in shared memory once as [64-number chunk][key][128 bytes], 128-byte swizzle.  The same bytes
//            are the K-major operand of S^T (M = 64 keys) and the MN-major operand of O^T (M = 128 numbers).
//   stages   two, filled and released in groups of 128 numbers: a group is free again when the block of O^T that reads it
//            is done, so the next but one tile arrives behind the products instead of after them (with whole tiles
//            the load of a tile and the products of another took turns).
//            Quantised tiles are filled as a whole: their loads wait in registers, not in the stage.
//   warps    0-3 softmax and epilogue, 4 issues S^T, 5 issues O^T (two, so that the waits of one are covered by the
//            products of the other), 6-13 bring tiles: bf16 records as TMA boxes of a page's rows or, where pages do not
//            line up with a tile, as four-row gathers; quantised records to registers, from where they are expanded to
//            bf16 and stored.  S^T of tile t + 1 is computed while the softmax of tile t runs.
//   softmax  S^T is read in 16x256b pieces: a thread holds 2 keys x N / 4 rows.  The running maximum of a row is only
//            raised when a score passes it by 2^8 (one barrier vote a tile): weights are at most 2^8, sums and O are fp32,
//            so nothing overflows, and a maximum that moves little costs neither shuffles nor a pass over O.
//   weights  are rounded to bf16, as the operand type demands (2^-9 relative each); the normaliser sums them in fp32
//            before that rounding.
// A row of keys is split over blocks when there are few rows; the partial (O, m, l) are merged by a second kernel.
// With 16 rows it is bound by loads (32 x 32768 bf16 records of 1152 bytes: 230 us, 5.2 TB/s; 32 x 2048: 27.5 us), with 64 by
// the MMAs' operand reads (36 of M 64 x N 64 at 32 cycles and 16 of M 128 x N 64 at 48 a tile, of which half would be the
// full rate) and by two stages being all that fits: 2048 tokens x 16 heads over 32768 keys 3.66 ms, 619 TFLOP/s, which is
// why chunk_attention_kernel.cuh exists.

namespace {

constexpr int kRaTile = 64;                     // keys a tile
constexpr int kRaStages = 2;
constexpr int kRaSoftmaxWarps = 4, kRaLoadWarps = 8;
constexpr int kRaThreads = (kRaSoftmaxWarps + 2 + kRaLoadWarps) * 32;
constexpr int kRaMaxDims = 576;
constexpr int kRaChunkBytes = kRaTile * 128;    // one 64-number chunk of a tile
constexpr int kRaMaxGroups = (kRaMaxDims / 64 + 1) / 2;   // groups of 128 numbers
constexpr float kRaLowest = -3.402823466e38f;   // running maximum of a row that has seen no key

struct RecAtt {
  RecFmt f;
  const uint8_t *records;
  int64_t num_records;
  const int32_t *table;        // [n][table_stride]: first record / page_size of each page, negative = absent
  int64_t table_stride;
  int32_t page, page_shift;    // page_shift >= 0: page == 1 << page_shift
  int32_t room;                // keys a request may have: the table's, at most the caller's bound
  const int32_t *kv_len;       // [n], null: room
  const int32_t *q_start;      // [n + 1], null: one token a request
  int32_t N, H, Dv, causal;
  const __nv_bfloat16 *q;
  int64_t q_token, q_head;     // strides in numbers
  int64_t total_q;
  int32_t max_q, row_tiles, splits;
  int32_t box;                 // rows of a TMA box of a page (8, 16, 32, 64); 0: gathers only
  float scale_log2e;
  __nv_bfloat16 *out;
  float *lse;
  float *partial;              // [row][split][Dv + 4]: O, m, l
  uint32_t *status;
};

// ---- tcgen05 ----

// Shared-memory operand descriptors, 128-byte swizzle.  K-major: 8-row groups `sbo` bytes apart.  MN-major: 8-k groups
// `sbo` bytes apart, blocks of 64 numbers of the MN axis `lbo` bytes apart.  The low word is address and lbo in 16-byte
// units, so a step along the operand is an addition to it.
__device__ __forceinline__ uint32_t umma_desc_lo(const uint32_t addr, const uint32_t lbo) { return (addr & 0x3ffffu) >> 4 | (lbo >> 4) << 16; }
constexpr uint32_t kUmmaDescHi = 1024u >> 4 | 1u << 14 | 2u << 29;   // sbo = 1024 bytes, version 1, 128-byte swizzle
// kind::f16, bf16 operands, fp32 accumulators
__host__ __device__ constexpr uint32_t umma_idesc(const int M, const int N, const bool a_mn, const bool b_mn) {
  return 1u << 4 | 1u << 7 | 1u << 10 | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;
}
__device__ __forceinline__ void umma_bf16(const uint32_t d, const uint32_t a_lo, const uint32_t b_lo, const uint32_t idesc, const bool add) {
  asm volatile("{ .reg .pred p; .reg .b64 a, b; setp.ne.u32 p, %5, 0; mov.b64 a, {%1, %4}; mov.b64 b, {%2, %4};"
               " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p; }"
               ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(kUmmaDescHi), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void umma_commit(const uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(const uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Bounded wait whose first look costs little: most waits of the pipeline find their phase complete (60 cycles instead
// of 120 to 160 for the loop of the general one).
__device__ __forceinline__ bool mbar_wait_quick(const uint32_t bar, const uint32_t parity) {
  uint32_t done;
  asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done ? true : mbar_wait_bounded(bar, parity);
}
// The end of a block in which a bounded wait ran out (all its threads): the status, and a bounded time in which copies that are
// still in flight land, before its shared memory goes to another block.
__device__ __noinline__ void ra_gave_up(uint32_t *status) {
  if (threadIdx.x == 0 && status) atomicOr(status, HISPARSE_STATUS_TIMEOUT);
  const uint64_t t0 = global_ns();
  for (int i = 0; i < 10000 && global_ns() - t0 < 1000000; ++i) __nanosleep(1000);
}
__device__ __forceinline__ void mbar_arrive_tx(const uint32_t bar, const uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// box of rows y .. of the record matrix, 64 numbers from x
__device__ __forceinline__ void tma_rows(const uint32_t dst, const CUtensorMap *map, const int x, const int y, const uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
// four rows anywhere; a row that does not exist is filled with zeros
__device__ __forceinline__ void tma_gather4(const uint32_t dst, const CUtensorMap *map, const int x, const int4 y, const uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w), "r"(bar) : "memory");
}
__device__ __forceinline__ float ex2(const float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// 16 lanes x 16 columns: registers (4 i + 0, 1) are row lane / 4, columns 8 i + 2 (lane % 4) + 0, 1; (4 i + 2, 3) row + 8
__device__ __forceinline__ void tmem_ld_s(const uint32_t addr, float *v) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(addr));
}
// 32 lanes x 16 columns: register i is column i of the thread's lane
__device__ __forceinline__ void tmem_ld_o(const uint32_t addr, float (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                 "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_st_o(const uint32_t addr, const float (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
               ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
                 "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "r"(addr)
               : "memory");
}

template <int THREADS = kRaSoftmaxWarps * 32>
__device__ __forceinline__ void softmax_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(THREADS) : "memory"); }
template <int THREADS = kRaSoftmaxWarps * 32>
__device__ __forceinline__ bool softmax_any(const bool p) {
  uint32_t r;
  asm volatile("{ .reg .pred a, b; setp.ne.u32 a, %1, 0; barrier.cta.red.or.pred b, 1, %2, a; selp.u32 %0, 1, 0, b; }"
               : "=r"(r) : "r"((uint32_t)p), "n"(THREADS) : "memory");
  return r != 0;
}

// ---- one request's rows and keys, the same in both kernels ----

struct RaRequest { int64_t q0; int qlen, kv; };

__device__ __forceinline__ RaRequest ra_request(const RecAtt &a, const int n, bool &bad) {
  RaRequest r;
  r.q0 = a.q_start ? a.q_start[n] : n;
  const int64_t q1 = a.q_start ? a.q_start[n + 1] : n + 1;
  const int64_t kv = a.kv_len ? a.kv_len[n] : a.room;
  bad = r.q0 < 0 || q1 > a.total_q || q1 < r.q0 || q1 - r.q0 > a.max_q || kv < 0 || kv > a.room;
  // (a request whose rows are not in the tensor is skipped, a longer chunk or context than announced is cut)
  r.qlen = r.q0 < 0 || q1 > a.total_q || q1 <= r.q0 ? 0 : (int)(q1 - r.q0 < a.max_q ? q1 - r.q0 : a.max_q);
  r.kv = (int)(kv < 0 ? 0 : kv < a.room ? kv : a.room);
  return r;
}

// Keys that query token t of the request sees: [0, limit)
__device__ __forceinline__ int ra_limit(const RecAtt &a, const RaRequest &r, const int t) {
  if (!a.causal) return r.kv;
  const int v = r.kv - r.qlen + t + 1;
  return v < 0 ? 0 : v;
}

// Record of key j, -1 where its page is absent.  In two steps, so that a loader can ask for a table entry a tile before it
// looks at it.
__device__ __forceinline__ int32_t ra_entry(const RecAtt &a, const int n, const int j) {
  return a.table[(int64_t)n * a.table_stride + (a.page_shift >= 0 ? j >> a.page_shift : j / a.page)];
}
__device__ __forceinline__ int32_t ra_resolve(const RecAtt &a, const int32_t e, const int j, bool &bad) {
  const int64_t idx = (int64_t)e * a.page + (a.page_shift >= 0 ? j & (a.page - 1) : j % a.page);
  bad |= e >= 0 && idx >= a.num_records;
  return e < 0 || idx >= a.num_records ? -1 : (int32_t)idx;
}
// A row that the pool's tensor maps do not have: filled with zeros.  (The map of an empty pool has one row.)
__device__ __forceinline__ int32_t ra_none(const RecAtt &a) { return a.num_records > 0 ? (int32_t)a.num_records : 1; }
__device__ __forceinline__ int32_t ra_index(const RecAtt &a, const int n, const int j, bool &bad) {
  return ra_resolve(a, ra_entry(a, n, j), j, bad);
}

__device__ __forceinline__ float ra_number(const RecFmt &f, const uint8_t *rec, const int d) {
  if (d >= f.Dq) return __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(rec + f.Dq + 2 * (d - f.Dq)));
  const float s = *reinterpret_cast<const float *>(rec + f.scales + d / kRecGroup * 4);
  return __bfloat162float(__float2bfloat16(e4m3x4_to_float(rec[d]).x * s));
}

// Query rows of a block into shared memory, K-major [chunk][row][128 bytes], rows behind the last one as zeros, by WARPS warps.
// In two steps, K rows a warp (base + WARPS k), so that their loads are in flight together: written one after the other, 64
// rows of 576 numbers took 22000 cycles, because the compiler may not move a load over a store to shared memory.
constexpr int kRaQParts = (kRaMaxDims / 8 + 31) / 32;
template <int WARPS, int K>
__device__ __forceinline__ void ra_fetch_q(const RecAtt &a, const RaRequest &rq, const int row0, const int rows, const int base,
                                           const int lane, uint4 (&v)[K][kRaQParts]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int r = base + k * WARPS, g = row0 + r, tok = g / a.H;
    const __nv_bfloat16 *src = a.q + (rq.q0 + tok) * a.q_token + (int64_t)(g - tok * a.H) * a.q_head;
#pragma unroll
    for (int i = 0; i < kRaQParts; ++i) {
      v[k][i] = make_uint4(0, 0, 0, 0);
      if (r < rows && i * 32 + lane < a.f.D / 8) v[k][i] = *reinterpret_cast<const uint4 *>(src + (i * 32 + lane) * 8);
    }
  }
}
template <int ROWS, int WARPS, int K>
__device__ __forceinline__ void ra_put_q(const RecAtt &a, unsigned char *to, const int base, const int lane, const uint4 (&v)[K][kRaQParts]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int r = base + k * WARPS;
#pragma unroll
    for (int i = 0; i < kRaQParts; ++i) {
      const int u = i * 32 + lane;
      if (u < a.f.D / 8) *reinterpret_cast<uint4 *>(to + (u >> 3) * (ROWS * 128) + r * 128 + (((u & 7) ^ (r & 7)) << 4)) = v[k][i];
    }
  }
}

// One row in plain arithmetic by one warp, for rows whose masked keys hold NaN or infinities: a weight of zero does not
// remove those from a matrix product.
__device__ __noinline__ void ra_plain_row(const RecAtt &a, const int n, const __nv_bfloat16 *q, const int lo, const int hi,
                                          float (&o)[kRaMaxDims / 32], float &m, float &l) {
  const int lane = threadIdx.x & 31;
  m = kRaLowest; l = 0.f;
#pragma unroll
  for (int i = 0; i < kRaMaxDims / 32; ++i) o[i] = 0.f;
  for (int j = lo; j < hi; ++j) {
    bool bad = false;
    const int32_t idx = ra_index(a, n, j, bad);
    if (idx < 0) continue;
    const uint8_t *rec = a.records + (int64_t)idx * a.f.E;
    float s = 0.f;
    for (int d = lane; d < a.f.D; d += 32) s += __bfloat162float(q[d]) * ra_number(a.f, rec, d);
#pragma unroll
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= a.scale_log2e;
    const float m2 = fmaxf(m, s), al = exp2f(m - m2), p = exp2f(s - m2);
    l = l * al + p;
#pragma unroll
    for (int i = 0; i < kRaMaxDims / 32; ++i)
      if (lane + 32 * i < a.Dv) o[i] = o[i] * al + p * ra_number(a.f, rec, lane + 32 * i);
    m = m2;
  }
}

template <int N>
struct RaSmem {
  static constexpr int kColsPerThread = N / 4;
  static constexpr uint32_t q = 0;
  __host__ __device__ static constexpr uint32_t kv(const int chunks) { return (uint32_t)(chunks * N * 128); }
  __host__ __device__ static constexpr uint32_t p(const int chunks) { return kv(chunks) + (uint32_t)(kRaStages * chunks * kRaChunkBytes); }
  __host__ __device__ static constexpr uint32_t bars(const int chunks) { return p(chunks) + N * 128; }
  // mbarriers (full, empty per stage and group; S, P per stage; Q; end of either product), tensor-memory address, per-key and per-row arrays
  static constexpr int kBars = 2 * kRaStages * kRaMaxGroups + 2 * kRaStages + 3;
  __host__ __device__ static constexpr uint32_t tmem(const int chunks) { return bars(chunks) + 16 * ((kBars + 1) / 2); }
  __host__ __device__ static constexpr uint32_t valid(const int chunks) { return tmem(chunks) + 16; }
  __host__ __device__ static constexpr uint32_t lim(const int chunks) { return valid(chunks) + kRaStages * kRaTile; }
  __host__ __device__ static constexpr uint32_t red(const int chunks) { return lim(chunks) + N * 4; }
  __host__ __device__ static constexpr uint32_t fac(const int chunks) { return red(chunks) + 4 * N * 4; }
  __host__ __device__ static constexpr uint32_t max(const int chunks) { return fac(chunks) + N * 4; }
  __host__ __device__ static constexpr uint32_t odd(const int chunks) { return max(chunks) + N * 4; }
  __host__ __device__ static constexpr uint32_t total(const int chunks) { return odd(chunks) + N; }
};

template <int N, bool QUANT>
__global__ void __launch_bounds__(kRaThreads, 1) record_attention_kernel(const RecAtt a, const __grid_constant__ CUtensorMap rows_map,
                                                                        const __grid_constant__ CUtensorMap gather_map) {
  extern __shared__ __align__(1024) unsigned char ra_smem[];
  using L = RaSmem<N>;
  constexpr int NC = N / 4;                       // rows (columns of S^T) a softmax thread holds
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int chunks = (a.f.D + 63) / 64;
  const uint32_t sbase = smem_u32(ra_smem);
  const uint32_t s_q = sbase + L::q, s_kv = sbase + L::kv(chunks), s_p = sbase + L::p(chunks), s_bar = sbase + L::bars(chunks);
  const uint32_t stage_bytes = (uint32_t)chunks * kRaChunkBytes;
  uint8_t *s_valid = ra_smem + L::valid(chunks);                            // [stage][key]
  int32_t *s_lim = reinterpret_cast<int32_t *>(ra_smem + L::lim(chunks));   // [row] keys seen
  float *s_red = reinterpret_cast<float *>(ra_smem + L::red(chunks));       // [warp][row]
  float *s_fac = reinterpret_cast<float *>(ra_smem + L::fac(chunks));       // [row]
  float *s_max = reinterpret_cast<float *>(ra_smem + L::max(chunks));       // [row]
  uint8_t *s_odd = ra_smem + L::odd(chunks);                                // [row] a masked key is not finite
  const uint32_t b_full = s_bar, b_empty = b_full + 8 * kRaStages * kRaMaxGroups, b_s = b_empty + 8 * kRaStages * kRaMaxGroups;
  const uint32_t b_p = b_s + 8 * kRaStages, b_q = b_p + 8 * kRaStages, b_end = b_q + 8;
  auto at = [](const int st, const int g) { return (uint32_t)(8 * (st * kRaMaxGroups + g)); };   // of a group's barrier
  const int groups = (chunks + 1) / 2, vgroups = a.Dv / 128;   // groups below vgroups are values, too
  const int vlast = QUANT ? 0 : vgroups - 1;      // the barrier that says that O^T has a whole tile behind it

  const uint32_t item = blockIdx.x / (uint32_t)a.splits, split = blockIdx.x - item * a.splits;
  const int n = (int)(item / (uint32_t)a.row_tiles);
  const int rt = a.row_tiles - 1 - (int)(item - (uint32_t)n * a.row_tiles);   // (from the last: with a causal mask it is the longest)
  bool bad_req;
  const RaRequest rq = ra_request(a, n, bad_req);
  if (bad_req && tid == 0 && a.status) atomicOr(a.status, HISPARSE_STATUS_OUT_OF_RANGE);
  const int row0 = rt * N;                        // first row in the request (the host keeps rows below 2^31)
  const int rows = min(N, rq.qlen * a.H - row0);  // of this tile
  if (rows <= 0) return;
  const int hi_all = min(rq.kv, ra_limit(a, rq, (row0 + rows - 1) / a.H));
  const int lo_full = min(rq.kv, ra_limit(a, rq, row0 / a.H));             // keys below are seen by every row
  const int tiles_all = (hi_all + kRaTile - 1) / kRaTile, per = (tiles_all + a.splits - 1) / a.splits;
  // (bounds in tiles first: a split's end in keys may lie beyond 2^31)
  const int lo = min((int)split * per, tiles_all) * kRaTile, hi = min(hi_all, min(((int)split + 1) * per, tiles_all) * kRaTile);
  const int nt = hi > lo ? (hi - lo + kRaTile - 1) / kRaTile : 0;

  bool dead = false;                              // a bounded wait ran out: finish without waiting
  auto wait = [&](const uint32_t bar, const uint32_t parity) {
    if (!dead && !mbar_wait_quick(bar, parity)) dead = true;
  };

  const uint32_t kCols = (uint32_t)(a.Dv / 128 * N + 2 * N);
  const uint32_t cols = kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
  if (tid < L::kBars) {
    const uint32_t count = tid < kRaStages * kRaMaxGroups ? kRaLoadWarps
                           : tid >= L::kBars - 3 - kRaStages && tid < L::kBars - 3 ? kRaSoftmaxWarps * 32
                           : tid == L::kBars - 3                                        ? kRaSoftmaxWarps
                                                                                        : 1;
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(s_bar + 8 * tid), "r"(count) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kRaSoftmaxWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + L::tmem(chunks)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  for (int i = tid; i < N; i += kRaThreads) {
    s_lim[i] = i < rows ? min(rq.kv, ra_limit(a, rq, (row0 + i) / a.H)) : 0;
    s_odd[i] = 0;
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(ra_smem + L::tmem(chunks));
  const uint32_t t_s = tmem + (uint32_t)(a.Dv / 128 * N);   // two buffers of S^T behind O^T
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (warp > kRaSoftmaxWarps + 1) {
    // ------------------------------------------------------------------ loaders
    const int w = warp - kRaSoftmaxWarps - 2;
    const int units = a.f.D / 8;                  // 16-byte units of a bf16 row
    bool bad_page = false;
    const int mykey = w * 8 + (lane & 7);         // lanes hold the record of one of the warp's 8 keys each
    auto entry = [&](const int t) { const int j = lo + t * kRaTile + mykey; return j < hi ? ra_entry(a, n, j) : -1; };
    auto resolve = [&](const int t, const int32_t e) { return ra_resolve(a, e, lo + t * kRaTile + mykey, bad_page); };
    // A group may be overwritten when the block of O^T that reads it is done, or S^T where it is no value.  The groups
    // that are no values come first: they are free first.
    auto wait_free = [&](const int t, const int g) {
      if (t >= kRaStages)
        wait(g < vgroups ? b_empty + at(t & 1, g) : b_s + 8 * (t & 1), (uint32_t)((t / kRaStages - 1) & 1));
    };
    if constexpr (!QUANT) {
      const bool issuer = elect_one();
      int32_t ahead = entry(0);
      for (int t = 0; t < nt; ++t) {
        const int st = t & 1, j0 = lo + t * kRaTile;
        const int32_t idx = resolve(t, ahead);
        ahead = entry(t + 1);
        // whole pages, or rows of one, as boxes; a tile that is not full row by row, so that what lies behind the context
        // is never read
        const bool boxes = a.box && j0 + kRaTile <= hi;
        const int rows_here = boxes ? (w * 8 % a.box == 0 ? a.box : 0) : 8;
        const int y_box = __shfl_sync(0xffffffffu, idx, 0);
        const int none = ra_none(a);
        const int yi = idx < 0 ? none : idx;
        int4 y0, y1;
        y0.x = __shfl_sync(0xffffffffu, yi, 0); y0.y = __shfl_sync(0xffffffffu, yi, 1);
        y0.z = __shfl_sync(0xffffffffu, yi, 2); y0.w = __shfl_sync(0xffffffffu, yi, 3);
        y1.x = __shfl_sync(0xffffffffu, yi, 4); y1.y = __shfl_sync(0xffffffffu, yi, 5);
        y1.z = __shfl_sync(0xffffffffu, yi, 6); y1.w = __shfl_sync(0xffffffffu, yi, 7);
        const uint32_t base = s_kv + (uint32_t)st * stage_bytes + (uint32_t)(w * 8 * 128);
        for (int i = 0; i < groups; ++i) {
          const int g = i + vgroups < groups ? i + vgroups : i + vgroups - groups;
          wait_free(t, g);
          if (g == 0 && lane < 8) s_valid[st * kRaTile + mykey] = idx >= 0;
          __syncwarp();
          if (issuer) {
            const int c1 = 2 * g + 2 < chunks ? 2 * g + 2 : chunks;
            const uint32_t bar = b_full + at(st, g);
            if (dead || rows_here == 0) mbar_arrive(bar);
            else {
              mbar_arrive_tx(bar, (uint32_t)((c1 - 2 * g) * rows_here * 128));
              for (int c = 2 * g; c < c1; ++c) {
                const uint32_t dst = base + (uint32_t)c * kRaChunkBytes;
                if (boxes) tma_rows(dst, &rows_map, c * 64, y_box < 0 ? none : y_box, bar);
                else {
                  tma_gather4(dst, &gather_map, c * 64, y0, bar);
                  tma_gather4(dst + 512, &gather_map, c * 64, y1, bar);
                }
              }
            }
          }
          __syncwarp();
        }
      }
    } else {
      // Eight lanes a record and 128 numbers, so a lane has 16 codes of two of the warp's keys in each group.
      const int u = lane & 7, k0 = lane >> 3;
      const int cgroups = a.f.Dq / 128;           // groups of codes; the numbers behind them are bf16
      uint4 code[4][2], tail[2];
      float4 scale[2];
      auto pointer = [&](const int32_t idx, const int k) -> const uint8_t * {
        const int32_t x = __shfl_sync(0xffffffffu, idx, k);
        return x < 0 ? nullptr : a.records + (int64_t)x * a.f.E;
      };
      auto load16 = [](const uint8_t *p) { return p ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0, 0, 0, 0); };
      const int last = chunks - 1;                // the last chunk is prefetched where it is bf16
      const bool tail_lane = 64 * last >= a.f.Dq && last * 8 + u < units;
      auto load_tail = [&](const uint8_t *r) { return load16(r && tail_lane ? r + a.f.Dq + (last * 64 - a.f.Dq + u * 8) * 2 : nullptr); };
      // Records two tiles ahead of the registers are asked into L2, sector by sector: the registers alone hold too little
      // in flight for the memory's latency.
      auto prefetch = [&](const int32_t idx) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t *p = pointer(idx, k0 + 4 * h);
          if (p)
            for (int o = u * 32; o < a.f.E; o += 256) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + o));
        }
      };
      int32_t mine = resolve(0, entry(0)), next = resolve(1, entry(1)), then = resolve(2, entry(2)), ahead = entry(3);
      const uint8_t *r[2] = {pointer(mine, k0), pointer(mine, k0 + 4)};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int g = 0; g < 4; ++g) code[g][h] = load16(r[h] && g < cgroups ? r[h] + g * 128 + u * 16 : nullptr);
        tail[h] = load_tail(r[h]);
        scale[h] = r[h] ? *reinterpret_cast<const float4 *>(r[h] + a.f.scales) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      prefetch(next);
      prefetch(then);
      for (int t = 0; t < nt; ++t) {
        const int st = t & 1;
        const uint8_t *nx[2] = {pointer(next, k0), pointer(next, k0 + 4)};
        unsigned char *base = ra_smem + L::kv(chunks) + (uint32_t)st * stage_bytes;
        if (t >= kRaStages) wait(b_empty + at(st, 0), (uint32_t)((t / kRaStages - 1) & 1));
        if (lane < 8) s_valid[st * kRaTile + mykey] = mine >= 0;
        mine = next; next = then; then = resolve(t + 3, ahead);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          if (g < cgroups) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int key = w * 8 + k0 + 4 * h;
              const float s = g == 0 ? scale[h].x : g == 1 ? scale[h].y : g == 2 ? scale[h].z : scale[h].w;
              const uint4 cd = code[g][h];
              const uint2 v0 = e4m3x4_to_bf16(cd.x, s), v1 = e4m3x4_to_bf16(cd.y, s), v2 = e4m3x4_to_bf16(cd.z, s), v3 = e4m3x4_to_bf16(cd.w, s);
              const uint4 e0 = make_uint4(v0.x, v0.y, v1.x, v1.y), e1 = make_uint4(v2.x, v2.y, v3.x, v3.y);
              // the two 16-byte units of the chunk's row; the lanes of the second chunk take them the other way round, so
              // that eight lanes store to eight different bank groups
              const bool up = u >= 4;
              unsigned char *row = base + (2 * g + (u >> 2)) * kRaChunkBytes + key * 128;
              const int d = 2 * (u & 3);
              *reinterpret_cast<uint4 *>(row + (((d + (up ? 1 : 0)) ^ (key & 7)) << 4)) = up ? e1 : e0;
              *reinterpret_cast<uint4 *>(row + (((d + (up ? 0 : 1)) ^ (key & 7)) << 4)) = up ? e0 : e1;
            }
          }
        }
        for (int c = 2 * cgroups; c < chunks; ++c) {
          if (c * 8 + u < units) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int key = w * 8 + k0 + 4 * h;
              const uint4 v = c == last ? tail[h] : load16(r[h] ? r[h] + a.f.Dq + (c * 64 - a.f.Dq + u * 8) * 2 : nullptr);
              *reinterpret_cast<uint4 *>(base + c * kRaChunkBytes + key * 128 + ((u ^ (key & 7)) << 4)) = v;
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(b_full + at(st, 0));
        // (behind the arrival: it is a release, which waits for the loads before it)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          r[h] = nx[h];
#pragma unroll
          for (int g = 0; g < 4; ++g) code[g][h] = load16(r[h] && g < cgroups ? r[h] + g * 128 + u * 16 : nullptr);
          tail[h] = load_tail(r[h]);
          scale[h] = r[h] ? *reinterpret_cast<const float4 *>(r[h] + a.f.scales) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        ahead = entry(t + 4);
        prefetch(then);
      }
    }
    if (bad_page && a.status) atomicOr(a.status, HISPARSE_STATUS_OUT_OF_RANGE);
  } else if (warp == kRaSoftmaxWarps) {
    // ------------------------------------------------------------------ S^T = K Q^T
    // (the warp runs as one, one lane issues: operands then stay in uniform registers)
    const int ksteps = a.f.D / 16;
    constexpr uint32_t kIdS = umma_idesc(64, N, false, false);
    const uint32_t q_lo = umma_desc_lo(s_q, 16), k_lo = umma_desc_lo(s_kv, 16);
    const bool issuer = elect_one();
    wait(b_q, 0);
    for (int t = 0; t < nt; ++t) {
      const int st = t & 1;
      const uint32_t d = t_s + (uint32_t)(st * N), kst = k_lo + ((uint32_t)st * stage_bytes >> 4);
      if (t >= kRaStages) wait(b_p + 8 * st, (uint32_t)((t / kRaStages - 1) & 1));   // S^T of the last tile but one is read
#pragma unroll
      for (int g = 0; g < kRaMaxGroups; ++g) {
        if (g < groups) {
          if (!QUANT || g == 0) {
            wait(b_full + at(st, g), (uint32_t)((t / kRaStages) & 1));
            tmem_fence_after();
          }
          if (issuer && !dead) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              if (g * 8 + k < ksteps)
                umma_bf16(d, kst + (2 * g + k / 4) * (kRaChunkBytes >> 4) + k % 4 * 2, q_lo + (2 * g + k / 4) * (N * 128 >> 4) + k % 4 * 2, kIdS, g > 0 || k > 0);
          }
          __syncwarp();
        }
      }
      if (issuer && !dead) umma_commit(b_s + 8 * st);
      __syncwarp();
    }
    if (issuer) umma_commit(b_end);               // everything issued has finished before the tensor memory is freed
    if (!mbar_wait_bounded(b_end, 0)) dead = true;
    __syncwarp();
  } else if (warp == kRaSoftmaxWarps + 1) {
    // ------------------------------------------------------------------ O^T += V^T P^T
    constexpr uint32_t kIdO = umma_idesc(128, N, true, false);
    const uint32_t p_lo = umma_desc_lo(s_p, 16), v_lo = umma_desc_lo(s_kv, kRaChunkBytes);
    const bool issuer = elect_one();
    for (int t = 0; t < nt; ++t) {
      const int st = t & 1;
      const uint32_t vst = v_lo + ((uint32_t)st * stage_bytes >> 4);
      wait(b_p + 8 * st, (uint32_t)((t / kRaStages) & 1));
      tmem_fence_after();
      if (issuer && !dead) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if (b >= vgroups) break;
#pragma unroll
          for (int k = 0; k < kRaTile / 16; ++k)
            umma_bf16(tmem + (uint32_t)(b * N), vst + (uint32_t)b * (2 * kRaChunkBytes >> 4) + k * (2048 >> 4), p_lo + 2 * k, kIdO, t > 0 || k > 0);
          if (!QUANT || b == vgroups - 1) umma_commit(b_empty + at(st, QUANT ? 0 : b));
        }
      }
      __syncwarp();
    }
    if (issuer) umma_commit(b_end + 8);
    if (!mbar_wait_bounded(b_end + 8, 0)) dead = true;
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ softmax
    float m[NC], l[NC];                           // column 8 i + 2 (lane % 4) + c is entry 2 i + c
#pragma unroll
    for (int i = 0; i < NC; ++i) { m[i] = kRaLowest; l[i] = 0.f; }
    {
#pragma unroll 1
      for (int base = warp; base < N; base += 4 * kRaSoftmaxWarps) {
        uint4 v[4][kRaQParts];
        ra_fetch_q<kRaSoftmaxWarps>(a, rq, row0, rows, base, lane, v);
        ra_put_q<N, kRaSoftmaxWarps>(a, ra_smem + L::q, base, lane, v);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(b_q);
    }
    const int c0 = 2 * (lane & 3), key0 = warp * 16 + (lane >> 2);
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    for (int t = 0; t < nt; ++t) {
      const int st = t & 1, j0 = lo + t * kRaTile;
      wait(b_full + at(st, 0), (uint32_t)((t / kRaStages) & 1));   // (for s_valid)
      wait(b_s + 8 * st, (uint32_t)((t / kRaStages) & 1));
      tmem_fence_after();
      float s[2 * NC];
#pragma unroll
      for (int i = 0; i < N / 16; ++i) tmem_ld_s(t_s + lanes + (uint32_t)(st * N + 16 * i), s + 8 * i);
      const bool v0 = s_valid[st * kRaTile + key0] != 0, v1 = s_valid[st * kRaTile + key0 + 8] != 0;
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 2 * NC; ++i) s[i] *= a.scale_log2e;
      if (j0 + kRaTile > lo_full) {               // some row does not see all of this tile
#pragma unroll
        for (int i = 0; i < 2 * NC; ++i) {
          const int col = (i >> 2) * 8 + c0 + (i & 1);
          if (j0 + key0 + ((i & 2) << 2) >= s_lim[col]) {
            if (!(fabsf(s[i]) <= 3.402823466e38f)) s_odd[col] = 1;
            s[i] = -INFINITY;
          }
        }
      }
      if (!(v0 && v1)) {
#pragma unroll
        for (int i = 0; i < 2 * NC; ++i)
          if (!((i & 2) ? v1 : v0)) s[i] = -INFINITY;
      }
      float over = kRaLowest;                     // (max ignores a NaN)
#pragma unroll
      for (int i = 0; i < NC; ++i) over = fmaxf(over, fmaxf(s[(i >> 1) * 4 + (i & 1)], s[(i >> 1) * 4 + 2 + (i & 1)]) - m[i]);
      const bool raise = over > 8.f;
      if (softmax_any(raise)) {
        // new maxima of every row: over the thread's two keys, the warp's 16, the four warps
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          float x = fmaxf(s[(i >> 1) * 4 + (i & 1)], s[(i >> 1) * 4 + 2 + (i & 1)]);
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
          if (lane < 4) s_red[warp * N + (i >> 1) * 8 + c0 + (i & 1)] = x;
        }
        softmax_sync();
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          const int col = (i >> 1) * 8 + c0 + (i & 1);
          const float x = fmaxf(fmaxf(s_red[col], s_red[N + col]), fmaxf(s_red[2 * N + col], s_red[3 * N + col]));
          const float mn = fmaxf(m[i], x), al = exp2f(m[i] - mn);
          l[i] *= al;
          m[i] = mn;
          if (warp == 0 && lane < 4) s_fac[col] = al;
        }
        softmax_sync();
        if (t > 0) {
          wait(b_empty + at((t - 1) & 1, vlast), (uint32_t)(((t - 1) / kRaStages) & 1));
          tmem_fence_after();
          for (int b = 0; b < a.Dv / 128 * (N / 16); ++b) {
            float o[16];
            tmem_ld_o(tmem + lanes + (uint32_t)(b * 16), o);
            tmem_wait_ld();
            const float *fc = s_fac + (b * 16) % N;
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] *= fc[i];
            tmem_st_o(tmem + lanes + (uint32_t)(b * 16), o);
          }
          tmem_wait_st();
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * NC; ++i) {
        s[i] = ex2(s[i] - m[(i >> 2) * 2 + (i & 1)]);
        l[(i >> 2) * 2 + (i & 1)] += s[i];
      }
      if (t > 0) wait(b_empty + at((t - 1) & 1, vlast), (uint32_t)(((t - 1) / kRaStages) & 1));   // P of the last tile is used up
      // P^T, K-major [row][64 keys]: 8 x 8 blocks of (keys, rows) stored transposed
#pragma unroll
      for (int i = 0; i < N / 16; ++i) {
        const int mat = lane >> 3, row = 16 * i + 8 * (mat >> 1) + (lane & 7), kc = 2 * warp + (mat & 1);
        const float *v = s + 8 * i;
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};"
                     ::"r"(s_p + (uint32_t)(row * 128 + ((kc ^ (row & 7)) << 4))), "r"(pack_bf16(v[0], v[1])), "r"(pack_bf16(v[2], v[3])),
                       "r"(pack_bf16(v[4], v[5])), "r"(pack_bf16(v[6], v[7])) : "memory");
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tmem_fence_before();
      mbar_arrive(b_p + 8 * st);
    }
    // ---------------------------------------------------------------- epilogue
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 4);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 8);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 16);
      if (lane < 4) s_red[warp * N + (i >> 1) * 8 + c0 + (i & 1)] = l[i];
      if (warp == 0 && lane < 4) s_max[(i >> 1) * 8 + c0 + (i & 1)] = m[i];
    }
    if (nt > 0) {
      wait(b_empty + at((nt - 1) & 1, vlast), (uint32_t)(((nt - 1) / kRaStages) & 1));
      tmem_fence_after();
    }
    softmax_sync();
    const bool whole = a.splits == 1;
    const int64_t grow = rq.q0 * a.H + row0;      // row in out and lse
    const int64_t pstride = (int64_t)a.splits * (a.Dv + 4);
    float *part = whole ? nullptr : a.partial + (grow * a.splits + split) * (a.Dv + 4);
    for (int r = tid; r < N; r += kRaSoftmaxWarps * 32) {
      const float sum = (s_red[r] + s_red[N + r]) + (s_red[2 * N + r] + s_red[3 * N + r]);
      const float mr = s_max[r];
      s_fac[r] = whole ? (sum == 0.f ? 0.f : 1.f / sum) : (sum == 0.f ? 0.f : 1.f);
      if (r < rows && !s_odd[r]) {
        if (whole) a.lse[grow + r] = sum == 0.f ? -INFINITY : 0.6931471805599453f * (mr + log2f(sum));
        else *reinterpret_cast<float2 *>(part + r * pstride + a.Dv) = make_float2(mr, sum);
      }
    }
    softmax_sync();
    // rows to write, as bits
    uint32_t live[(N + 31) / 32];
#pragma unroll
    for (int i = 0; i < (N + 31) / 32; ++i) live[i] = __ballot_sync(0xffffffffu, 32 * i + lane < rows && !s_odd[(32 * i + lane) & (N - 1)]);
#pragma unroll
    for (int g = 0; g < N / 16; ++g) {
      if (g * 16 >= rows) break;
      float fac[16];
#pragma unroll
      for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4 *>(fac + i) = *reinterpret_cast<const float4 *>(s_fac + g * 16 + i);
      const uint32_t lv = live[g / 2] >> (g % 2 * 16);
      for (int b = 0; b < vgroups; ++b) {
        const int d = b * 128 + warp * 32 + lane;
        float o[16];
        if (nt > 0) {
          tmem_ld_o(tmem + lanes + (uint32_t)(b * N + g * 16), o);
          tmem_wait_ld();
        }
        if (whole) {
          __nv_bfloat16 *dst = a.out + (grow + g * 16) * a.Dv + d;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (lv >> i & 1) dst[i * a.Dv] = __float2bfloat16(fac[i] != 0.f ? o[i] * fac[i] : 0.f);
        } else {
          float *dst = part + g * 16 * pstride + d;
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (lv >> i & 1) dst[i * pstride] = fac[i] != 0.f ? o[i] : 0.f;
        }
      }
    }
    tmem_fence_before();
    for (int r = warp; r < rows; r += kRaSoftmaxWarps) {
      if (!s_odd[r]) continue;
      float o[kRaMaxDims / 32], pm, pl;
      const int g = row0 + r, tok = g / a.H;
      ra_plain_row(a, n, a.q + (rq.q0 + tok) * a.q_token + (int64_t)(g - tok * a.H) * a.q_head, lo, min(hi, s_lim[r]), o, pm, pl);
      const float inv = whole ? (pl == 0.f ? 0.f : 1.f / pl) : 1.f;
#pragma unroll
      for (int i = 0; i < kRaMaxDims / 32; ++i) {
        const int d = lane + 32 * i;
        if (d < a.Dv) {
          if (whole) a.out[(grow + r) * a.Dv + d] = __float2bfloat16(o[i] * inv);
          else part[r * pstride + d] = o[i];
        }
      }
      if (lane == 0) {
        if (whole) a.lse[grow + r] = pl == 0.f ? -INFINITY : 0.6931471805599453f * (pm + log2f(pl));
        else { part[r * pstride + a.Dv] = pm; part[r * pstride + a.Dv + 1] = pl; }
      }
    }
  }
  if (__syncthreads_or(dead)) ra_gave_up(a.status);
  if (warp == kRaSoftmaxWarps)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
}

// Merges the splits of a row: out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s, lse = ln 2 (M + log2 L).  One block of
// 128 threads a row (n, r); rows beyond a request's own are left alone.
__global__ void __launch_bounds__(128) record_attention_combine_kernel(const RecAtt a) {
  __shared__ float s_w[128];
  __shared__ float s_red[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t per = (uint32_t)(a.max_q * a.H);
  const int n = (int)(blockIdx.x / per), r = (int)(blockIdx.x - n * per);
  bool bad;
  const RaRequest rq = ra_request(a, n, bad);
  asm volatile("griddepcontrol.wait;" ::: "memory");   // (every block, or the pair of kernels could end before the first)
  if (r >= rq.qlen * a.H) return;
  const int64_t grow = rq.q0 * a.H + r;
  const int stride = a.Dv + 4;
  const float *p = a.partial + grow * a.splits * stride;
  const float l = tid < a.splits ? p[(int64_t)tid * stride + a.Dv + 1] : 0.f;
  const float m = tid < a.splits && l != 0.f ? p[(int64_t)tid * stride + a.Dv] : kRaLowest;   // (l is NaN where a score is)
  float M = m;
#pragma unroll
  for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (lane == 0) s_red[warp] = M;
  __syncthreads();
  M = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
  const float w = l != 0.f ? exp2f(m - M) : 0.f;
  s_w[tid] = w;
  float L = l != 0.f ? w * l : 0.f;
#pragma unroll
  for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  if (lane == 0) s_red[4 + warp] = L;
  __syncthreads();
  L = (s_red[4] + s_red[5]) + (s_red[6] + s_red[7]);
  const float inv = L != 0.f ? 1.f / L : 0.f;
  for (int c = tid * 4; c < a.Dv; c += 128 * 4) {
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    // (eight splits' numbers in flight; a split without keys has left what was there before, which is not used)
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) {
      const float ws = s_w[s];
      const float4 v = *reinterpret_cast<const float4 *>(p + (int64_t)s * stride + c);
      o.x += ws != 0.f ? ws * v.x : 0.f; o.y += ws != 0.f ? ws * v.y : 0.f;
      o.z += ws != 0.f ? ws * v.z : 0.f; o.w += ws != 0.f ? ws * v.w : 0.f;
    }
    *reinterpret_cast<uint2 *>(a.out + grow * a.Dv + c) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  }
  if (tid == 0) a.lse[grow] = L == 0.f ? -INFINITY : 0.6931471805599453f * (M + log2f(L));
}

}  // namespace
