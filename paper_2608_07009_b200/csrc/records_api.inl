// Included by hisparse.cu: the C-ABI of the record operators (formats, write, read, attention over a caller's pool).

namespace {

// Makes `device` current for one call and restores the caller's.
struct RecDevice {
  int restore = -1;
  int rc = HISPARSE_OK;
  explicit RecDevice(int device) {
    int cur = -1;
    cudaError_t e = cudaGetDevice(&cur);
    if (e == cudaSuccess && cur != device) {
      e = cudaSetDevice(device);
      if (e == cudaSuccess) restore = cur;
    }
    if (e != cudaSuccess) { g_last_cuda_error = (int)e; rc = HISPARSE_ECUDA; }
  }
  ~RecDevice() { if (restore >= 0) cudaSetDevice(restore); }
};

int rec_format(const hisparse_record_format_t *f, RecFmt *out) {
  if (!f || f->dims < 16 || f->dims % 16 || f->dims > HISPARSE_MAX_RECORD_DIMS) return HISPARSE_EINVAL;
  if (f->quant_dims < 0 || f->quant_dims % kRecGroup || f->quant_dims > f->dims) return HISPARSE_EINVAL;
  out->D = f->dims;
  out->Dq = f->quant_dims;
  out->scales = f->quant_dims + 2 * (f->dims - f->quant_dims);
  out->E = (out->scales + f->quant_dims / kRecGroup * 4 + 15) / 16 * 16;
  return HISPARSE_OK;
}

int rec_blocks(int64_t count, int warps) { return (int)std::min<int64_t>((count + warps - 1) / warps, 148 * 64); }

template <typename Src>
int launch_write(const RecFmt &f, const void *src, int64_t stride, int64_t count, const int64_t *slots, void *records,
                 int64_t num_records, uint32_t *status, cudaStream_t st) {
  write_records_kernel<Src><<<rec_blocks(count, kWriteWarps), kWriteWarps * 32, 0, st>>>(
      f, static_cast<const Src *>(src), stride, count, slots, static_cast<uint8_t *>(records), num_records, status);
  HS_CUDA(cudaGetLastError());
  return HISPARSE_OK;
}

constexpr uint32_t kRaSmemLimit = 227 * 1024;   // shared memory a block may have
constexpr int kRaMaxSplits = 128;   // threads of a combine block

// cuTensorMapEncodeTiled through the runtime, so that the library does not link against the driver.
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_tiled(EncodeTiled *out) {
  static EncodeTiled encode = nullptr;            // (two threads that race here store the same pointer)
  if (!encode) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    HS_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q));
    if (!fn || q != cudaDriverEntryPointSuccess) return HISPARSE_ECUDA;
    encode = reinterpret_cast<EncodeTiled>(fn);
  }
  *out = encode;
  return HISPARSE_OK;
}

// Map of a pool of plain records as a matrix [num_records][D] of bf16, boxes of `rows` x 64 numbers.
int record_map(const RecFmt &f, const void *records, int64_t num_records, int rows, CUtensorMap *map) {
  EncodeTiled encode = nullptr;
  int rc = encode_tiled(&encode);
  if (rc) return rc;
  const cuuint64_t dims[2] = {(cuuint64_t)f.D, (cuuint64_t)std::max<int64_t>(1, num_records)}, strides[1] = {(cuuint64_t)f.E};
  const cuuint32_t box[2] = {64, (cuuint32_t)rows}, step[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(records), dims, strides, box, step,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? HISPARSE_OK : HISPARSE_EINVAL;
}

// Map of a pool of quantised records as a matrix [num_records][E] of bytes, boxes of `rows` x 128.
int byte_map(const RecFmt &f, const void *records, int64_t num_records, int rows, CUtensorMap *map) {
  EncodeTiled encode = nullptr;
  int rc = encode_tiled(&encode);
  if (rc) return rc;
  const cuuint64_t dims[2] = {(cuuint64_t)f.E, (cuuint64_t)std::max<int64_t>(1, num_records)}, strides[1] = {(cuuint64_t)f.E};
  const cuuint32_t box[2] = {128, (cuuint32_t)rows}, step[2] = {1, 1};
  const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(records), dims, strides, box, step,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? HISPARSE_OK : HISPARSE_EINVAL;
}

struct RaGeom {
  int rows, chunks, row_tiles, splits, room;
  bool pair;                     // chunk_attention_kernel, 128 rows a pair of SMs
  bool codes;                    // decode_attention_kernel: quantised records as they are
  bool cluster;                  // and its splits merge in a cluster
  int dense;                     // its rows a request in the workspace (expand_records_kernel); 0: the pages are taken as they are
  size_t smem, partial, workspace;
};

size_t ra_smem_bytes(int rows, int chunks) {
  return rows == 16 ? RaSmem<16>::total(chunks) : rows == 32 ? RaSmem<32>::total(chunks) : RaSmem<64>::total(chunks);
}

int ra_geometry(const hisparse_record_attention_t *p, RecFmt *f, RaGeom *g) {
  if (!p) return HISPARSE_EINVAL;
  int rc = rec_format(&p->format, f);
  if (rc) return rc;
  if (f->D > kRaMaxDims || !(p->value_dims == 128 || p->value_dims == 256 || p->value_dims == 512) || p->value_dims > f->D)
    return HISPARSE_EINVAL;
  if (p->num_requests < 1 || p->num_heads < 1 || p->num_heads > HISPARSE_MAX_HEADS || p->page_size < 1 || p->table_width < 1 ||
      (p->table_stride < p->table_width && p->table_stride != 0) || p->num_records < 0 || p->num_records > INT32_MAX || p->total_q < 0 || p->max_q_len < 1)
    return HISPARSE_EINVAL;
  // (the kernels count keys and rows in 32 bits and look a few tiles ahead)
  if ((int64_t)p->table_width * p->page_size > INT32_MAX - 1023 || (int64_t)p->max_q_len * p->num_heads > INT32_MAX - 1023) return HISPARSE_EINVAL;
  if (!p->q_start_dev && (p->max_q_len != 1 || p->total_q != p->num_requests)) return HISPARSE_EINVAL;
  const int64_t rows = (int64_t)p->max_q_len * p->num_heads;
  const int64_t width = (int64_t)p->table_width * p->page_size;
  const int64_t kv = p->max_kv_len > 0 ? std::min<int64_t>(p->max_kv_len, width) : width;
  g->room = (int)kv;
  g->chunks = (f->D + 63) / 64;
  // More than 64 rows go to pairs of SMs if their boxes can take the pages, or if there are so many rows that laying the
  // records out once is cheaper than reading (and expanding) them again for every 64 rows: with 128 rows it is not yet, with
  // 256 it is.  Up to 2 GB of workspace.
  const int64_t dense = (kv + kCaTile - 1) / kCaTile * kCaTile, dense_bytes = (int64_t)p->num_requests * dense * f->D * 2;
  const bool direct = f->Dq == 0 && p->page_size % 64 == 0;
  g->pair = rows > 64 && (direct || (rows > 192 && dense_bytes <= (int64_t)1 << 31 && p->num_requests * dense <= INT32_MAX));
  g->dense = g->pair && !direct ? (int)dense : 0;
  // Single tokens over quantised records whose values are all codes: 16, 32 or 48 rows, as tensor memory has room for.
  const int cg = f->Dq / 128, tail = f->D > f->Dq ? 1 : 0, vg = p->value_dims / 128;
  g->codes = f->Dq > 0 && p->max_q_len == 1 && p->value_dims <= f->Dq && f->D - f->Dq <= 64 && kv <= kDaMaxKeys;
  g->rows = g->pair ? 128 : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  if (g->codes) {
    g->pair = false;
    g->dense = 0;
    g->rows = rows > 32 && da_cols(48, cg, tail, vg) <= 512 && DaSmem<48>::total(cg, tail, vg) <= kRaSmemLimit   ? 48
              : rows > 16 && da_cols(32, cg, tail, vg) <= 512 && DaSmem<32>::total(cg, tail, vg) <= kRaSmemLimit ? 32
                                                                                                                 : 16;
  }
  const int vchunks = p->value_dims == 512 ? 4 : p->value_dims == 256 ? 2 : 1;
  g->smem = g->codes ? (g->rows == 16   ? DaSmem<16>::total(cg, tail, vg)
                          : g->rows == 32 ? DaSmem<32>::total(cg, tail, vg) : DaSmem<48>::total(cg, tail, vg))
            : g->pair ? CaSmem::total(g->chunks, vchunks) : ra_smem_bytes(g->rows, g->chunks);
  const int64_t row_tiles = (rows + g->rows - 1) / g->rows, tile = g->codes ? kDaTile : g->pair ? kCaTile : kRaTile;
  const int64_t tiles = std::max<int64_t>(1, (kv + tile - 1) / tile);
  // row tiles that there can be: every request's own, the last one of each partly filled
  const int64_t items = std::min<int64_t>((int64_t)p->num_requests * row_tiles,
                                          p->num_requests + (int64_t)p->total_q * p->num_heads / g->rows);
  if ((int64_t)p->num_requests * row_tiles > INT32_MAX / kRaMaxSplits / 2 || (int64_t)p->num_requests * rows > INT32_MAX) return HISPARSE_EINVAL;
  g->row_tiles = (int)row_tiles;
  // Blocks run one to an SM (or pair) in waves; a block costs its key tiles and what it takes to start and end (about three
  // tiles; eight of a pair's, whose start and end are 17,000 cycles and whose tile is 2650), a further split of a context the merge.
  // The cheapest number of splits of the longest context, counted in key tiles.
  const int64_t slots = g->pair ? 74 : 148, ends = g->pair ? 8 : 3;
  int64_t splits = 1, best = INT64_MAX;
  for (int64_t s = 1; s <= std::min<int64_t>(tiles, kRaMaxSplits); ++s) {
    const int64_t cost = (items * s + slots - 1) / slots * ((tiles + s - 1) / s + ends) + (s > 1 ? 2 : 0);
    if (cost < best) { best = cost; splits = s; }
    if (items * s > 8 * slots) break;
  }
  const int64_t per = (tiles + splits - 1) / splits;
  g->splits = (int)((tiles + per - 1) / per);
  g->cluster = g->codes && (g->splits == 2 || g->splits == 4 || g->splits == 8);
  g->partial = g->splits > 1 && !g->cluster ? (size_t)p->total_q * p->num_heads * g->splits * (p->value_dims + 4) * sizeof(float) : 0;
  g->workspace = g->dense ? (g->partial + 127) / 128 * 128 + (size_t)dense_bytes : g->partial;
  return HISPARSE_OK;
}

int launch_chunk_attention(const RecAtt &a, const RaGeom &g, cudaStream_t st) {
  HS_CUDA(cudaFuncSetAttribute(chunk_attention_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)CaSmem::total(kRaMaxDims / 64, 4)));
  RecFmt f = a.f;
  const void *rows = a.records;
  int64_t count = a.num_records;
  if (g.dense) {
    __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(reinterpret_cast<char *>(a.partial) + (g.partial + 127) / 128 * 128);
    expand_records_kernel<<<(unsigned)((int64_t)a.N * ((g.dense + 15) / 16)), 256, 0, st>>>(a, g.dense, out);
    HS_CUDA(cudaGetLastError());
    rows = out;
    count = (int64_t)a.N * g.dense;
    f.Dq = 0; f.E = 2 * f.D;
  }
  CUtensorMap rows_map, eight_map, gather_map;
  int rc = record_map(f, rows, count, 64, &rows_map);
  if (!rc) rc = record_map(f, rows, count, 8, &eight_map);
  if (!rc) rc = record_map(f, rows, count, 1, &gather_map);
  if (rc) return rc;
  chunk_attention_kernel<<<(unsigned)(2 * a.N * a.row_tiles * a.splits), kCaThreads, g.smem, st>>>(a, g.dense, rows_map, eight_map, gather_map);
  HS_CUDA(cudaGetLastError());
  return HISPARSE_OK;
}

template <int R>
int launch_decode_attention(const RecAtt &args, const RaGeom &g, cudaStream_t st) {
  HS_CUDA(cudaFuncSetAttribute(decode_attention_kernel<R>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRaSmemLimit));
  RecAtt a = args;
  a.box = a.page % 32 == 0 ? 32 : 0;
  CUtensorMap rows_map, gather_map;
  int rc = byte_map(a.f, a.records, a.num_records, 32, &rows_map);
  if (!rc) rc = byte_map(a.f, a.records, a.num_records, 1, &gather_map);
  if (rc) return rc;
  int lift = 0;
  while (lift < 6 && (int64_t)a.room > (int64_t)2048 << lift) ++lift;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.N * a.row_tiles * a.splits));
  cfg.blockDim = dim3(kDaThreads);
  cfg.dynamicSmemBytes = g.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = g.cluster ? (unsigned)a.splits : 1u; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  HS_CUDA(cudaLaunchKernelEx(&cfg, decode_attention_kernel<R>, a, (float)lift, g.cluster ? 1 : 0, rows_map, gather_map));
  return HISPARSE_OK;
}

template <int N, bool QUANT>
int launch_record_attention(const RecAtt &a, const RaGeom &g, cudaStream_t st) {
  // (always the most that any record takes: another thread's launch must not find a smaller limit)
  HS_CUDA(cudaFuncSetAttribute(record_attention_kernel<N, QUANT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               (int)RaSmem<N>::total(kRaMaxDims / 64)));
  CUtensorMap rows_map{}, gather_map{};
  if (!QUANT) {
    int rc = record_map(a.f, a.records, a.num_records, a.box ? a.box : 1, &rows_map);
    if (!rc) rc = record_map(a.f, a.records, a.num_records, 1, &gather_map);
    if (rc) return rc;
  }
  record_attention_kernel<N, QUANT><<<(unsigned)(a.N * a.row_tiles * a.splits), kRaThreads, g.smem, st>>>(a, rows_map, gather_map);
  HS_CUDA(cudaGetLastError());
  return HISPARSE_OK;
}

}  // namespace

extern "C" {

int hisparse_record_bytes(const hisparse_record_format_t *format, int64_t *bytes) {
  RecFmt f;
  const int rc = rec_format(format, &f);
  if (rc || !bytes) return HISPARSE_EINVAL;
  *bytes = f.E;
  return HISPARSE_OK;
}

int hisparse_write_records(const hisparse_record_format_t *format, int device, const void *src_dev, int src_type, int64_t src_stride,
                           int64_t count, const int64_t *slots_dev, void *records_dev, int64_t num_records,
                           uint32_t *status_dev, void *stream) {
  RecFmt f;
  const int rc = rec_format(format, &f);
  if (rc) return rc;
  if (device < 0 || count < 0 || num_records < 0 || (src_stride < f.D && src_stride != 0) || (!slots_dev && count > num_records)) return HISPARSE_EINVAL;
  if (src_type != HISPARSE_BF16 && src_type != HISPARSE_FP16 && src_type != HISPARSE_FP32) return HISPARSE_EINVAL;
  if (count == 0) return HISPARSE_OK;
  if (!src_dev || (!records_dev && num_records)) return HISPARSE_EINVAL;
  if (((uintptr_t)src_dev | (uintptr_t)records_dev) & 15 || src_stride * (src_type == HISPARSE_FP32 ? 4 : 2) % 16) return HISPARSE_EINVAL;
  RecDevice guard(device);
  if (guard.rc) return guard.rc;
  cudaStream_t st = as_stream(stream);
  switch (src_type) {
    case HISPARSE_BF16: return launch_write<__nv_bfloat16>(f, src_dev, src_stride, count, slots_dev, records_dev, num_records, status_dev, st);
    case HISPARSE_FP16: return launch_write<__half>(f, src_dev, src_stride, count, slots_dev, records_dev, num_records, status_dev, st);
    default: return launch_write<float>(f, src_dev, src_stride, count, slots_dev, records_dev, num_records, status_dev, st);
  }
}

int hisparse_read_records(const hisparse_record_format_t *format, int device, const void *records_dev, int64_t num_records,
                          const int32_t *table_dev, int64_t count, void *out_dev, uint32_t *status_dev, void *stream) {
  RecFmt f;
  const int rc = rec_format(format, &f);
  if (rc) return rc;
  if (device < 0 || count < 0 || num_records < 0) return HISPARSE_EINVAL;
  if (count == 0) return HISPARSE_OK;
  if ((!records_dev && num_records) || !table_dev || !out_dev || ((uintptr_t)records_dev | (uintptr_t)out_dev) & 15) return HISPARSE_EINVAL;
  RecDevice guard(device);
  if (guard.rc) return guard.rc;
  const bool few = count <= 148 * 4 * kReadWarps;   // a warp for each entry, and all of them resident
  auto *kernel = few ? read_records_kernel<1> : read_records_kernel<kReadRows>;
  kernel<<<rec_blocks(count, kReadWarps * (few ? 1 : kReadRows)), kReadWarps * 32, 0, as_stream(stream)>>>(
      f, static_cast<const uint8_t *>(records_dev), num_records, table_dev, count, static_cast<__nv_bfloat16 *>(out_dev), status_dev);
  HS_CUDA(cudaGetLastError());
  return HISPARSE_OK;
}

int hisparse_record_attention_workspace_bytes(const hisparse_record_attention_t *p, size_t *bytes) {
  RecFmt f;
  RaGeom g;
  const int rc = ra_geometry(p, &f, &g);
  if (rc || !bytes) return HISPARSE_EINVAL;
  *bytes = g.workspace;
  return HISPARSE_OK;
}

int hisparse_record_attention(const hisparse_record_attention_t *p, void *workspace_dev, size_t workspace_bytes, void *stream) {
  RecFmt f;
  RaGeom g;
  int rc = ra_geometry(p, &f, &g);
  if (rc) return rc;
  if (p->total_q == 0) return HISPARSE_OK;
  if (p->device < 0 || (!p->records_dev && p->num_records) || !p->table_dev || !p->q_dev || !p->out_dev || !p->lse_dev) return HISPARSE_EINVAL;
  if (((uintptr_t)p->records_dev | (uintptr_t)p->q_dev | (uintptr_t)p->out_dev | (uintptr_t)workspace_dev) & 15) return HISPARSE_EINVAL;
  if (p->q_token_stride % 8 || p->q_head_stride % 8 || p->q_token_stride < 0 || p->q_head_stride < 0) return HISPARSE_EINVAL;
  if (workspace_bytes < g.workspace || (g.workspace && !workspace_dev)) return HISPARSE_EINVAL;
  RecDevice guard(p->device);
  if (guard.rc) return guard.rc;
  RecAtt a{};
  a.f = f;
  // (an empty pool may have no address; the tensor maps want one, of which nothing is read)
  a.records = static_cast<const uint8_t *>(p->num_records ? p->records_dev : p->q_dev);
  a.num_records = p->num_records;
  a.table = p->table_dev; a.table_stride = p->table_stride; a.room = g.room; a.page = p->page_size;
  a.page_shift = -1;
  for (int s = 0; s < 31; ++s)
    if (p->page_size == 1 << s) a.page_shift = s;
  a.box = p->page_size % kRaTile == 0 ? kRaTile : p->page_size == 32 || p->page_size == 16 || p->page_size == 8 ? p->page_size : 0;
  a.kv_len = p->kv_len_dev; a.q_start = p->q_start_dev;
  a.N = p->num_requests; a.H = p->num_heads; a.Dv = p->value_dims; a.causal = p->causal != 0;
  a.q = static_cast<const __nv_bfloat16 *>(p->q_dev);
  a.q_token = p->q_token_stride; a.q_head = p->q_head_stride; a.total_q = p->total_q;
  a.max_q = p->max_q_len; a.row_tiles = g.row_tiles; a.splits = g.splits;
  a.scale_log2e = p->scale * 1.4426950408889634f;
  a.out = static_cast<__nv_bfloat16 *>(p->out_dev); a.lse = p->lse_dev;
  a.partial = static_cast<float *>(workspace_dev);
  a.status = p->status_dev;
  cudaStream_t st = as_stream(stream);
  const bool quant = f.Dq > 0;
  if (g.codes) rc = g.rows == 16   ? launch_decode_attention<16>(a, g, st)
                       : g.rows == 32 ? launch_decode_attention<32>(a, g, st) : launch_decode_attention<48>(a, g, st);
  else switch (g.rows) {
    case 128: rc = launch_chunk_attention(a, g, st); break;
    case 16: rc = quant ? launch_record_attention<16, true>(a, g, st) : launch_record_attention<16, false>(a, g, st); break;
    case 32: rc = quant ? launch_record_attention<32, true>(a, g, st) : launch_record_attention<32, false>(a, g, st); break;
    default: rc = quant ? launch_record_attention<64, true>(a, g, st) : launch_record_attention<64, false>(a, g, st); break;
  }
  if (rc || g.splits == 1 || g.cluster) return rc;
  // programmatic dependent launch: the merge is scheduled while the attention kernel drains
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)a.N * a.max_q * a.H));
  cfg.blockDim = dim3(128);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  HS_CUDA(cudaLaunchKernelEx(&cfg, record_attention_combine_kernel, a));
  return HISPARSE_OK;
}

}  // extern "C"
