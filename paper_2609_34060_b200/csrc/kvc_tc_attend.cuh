// What the tensor-core kernels of kvc_attend share: the tensor maps of one layer of a cache as tiles of 128 tokens, the
// operand descriptors of such tiles, and a few instructions.
//
// A tile is 128 token rows of one KV head, each row one part of 64 or 128 bytes (two for bf16 at d = 128), parts swizzled
// over their own width.  Rows come in groups of 8; a group's parts are `ps` bytes apart, groups `gs` bytes:
// (rows of one part: the group is only a matter of counting)
//   contiguous caches  one box of 128 rows: [part][128 rows], gs = 8 rows, ps = 128 rows
//   paged caches       one box a page: (channel, row in group, part, group, page x head): [group][part][8 rows], so the
//                      boxes of a tile follow each other and gs is the same inside a page and from page to page
// Both are canonical operand layouts of the tensor cores: the keys as a K-major matrix (channels are contracted), the
// values as an MN-major one (tokens are contracted).  Page and head share a tensor-map dimension, X = page * ratio + head,
// which needs s_page to be a multiple of s_head (head-major and token-major pools both are).
#pragma once
#include "kvc_attend.h"
#include "kvc_tc_maps.h"
#include "kvc_tc_ptx.cuh"

namespace kvc {
namespace tc {

struct TileGeo {
  int32_t gs, ps;            // bytes from group to group, from part to part
  int32_t box_rows;          // token rows a box holds (paged; a power of two), 128 (contiguous)
  int32_t box_shift;         // its logarithm
  int32_t box_bytes;
  int32_t ratio;             // X = page * ratio + head
  int32_t paged;
  int32_t flat;              // rows have one part: tensors and boxes of three dimensions (channel, row, head or X)
};

template <typename T>
inline bool encode_attend_tile(CUtensorMap* m, TileGeo* geo, const DevCache& c, const T* base, int layer, int H, int d) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  constexpr int E = (int)sizeof(T);
  const int pe = E == 2 ? 64 : d;                          // channels of a part
  const int np = d / pe;
  void* at = const_cast<T*>(base + (int64_t)layer * c.s_layer);
  const CUtensorMapDataType type = E == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
  const CUtensorMapSwizzle sw = pe * E == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
  const cuuint32_t es[5] = {1, 1, 1, 1, 1};
  geo->paged = is_paged(c);
  geo->flat = np == 1;
  auto encode3 = [&](int64_t rows, int64_t units, int64_t unit_stride, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)pe, (cuuint64_t)rows, (cuuint64_t)units};
    const cuuint64_t st[2] = {(cuuint64_t)c.s_tok * E, (cuuint64_t)unit_stride * E};
    const cuuint32_t box[3] = {(cuuint32_t)pe, (cuuint32_t)box_rows, 1};
    return fn(m, type, 3, at, dims, st, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (!geo->paged) {
    geo->gs = 8 * pe * E;
    geo->ps = 128 * pe * E;
    geo->box_rows = 128;
    geo->box_shift = 7;
    geo->box_bytes = 128 * d * E;
    geo->ratio = 0;
    if (c.T < 1) return false;
    if (geo->flat) return encode3(c.T, H, c.s_head, 128);
    const cuuint64_t dims[5] = {(cuuint64_t)pe, (cuuint64_t)c.T, (cuuint64_t)np, (cuuint64_t)H, 1};
    const cuuint64_t st[4] = {(cuuint64_t)c.s_tok * E, (cuuint64_t)pe * E, (cuuint64_t)c.s_head * E, (cuuint64_t)pe * E};
    const cuuint32_t box[5] = {(cuuint32_t)pe, 128, (cuuint32_t)np, 1, 1};
    return fn(m, type, 5, at, dims, st, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  }
  const int page = c.page_mask + 1, rows = page < 128 ? page : 128;
  const int64_t hs = H == 1 ? c.s_page : c.s_head;         // one head: X is the page
  if (hs <= 0 || c.s_page % hs) return false;
  const int64_t ratio = c.s_page / hs, x = (int64_t)(c.n_phys - 1) * ratio + H;
  if (x >= (int64_t)1 << 31) return false;
  geo->gs = np * 8 * pe * E;
  geo->ps = 8 * pe * E;
  geo->box_rows = rows;
  geo->box_shift = 0;
  while ((1 << geo->box_shift) < rows) ++geo->box_shift;
  geo->box_bytes = rows * d * E;
  geo->ratio = (int32_t)ratio;
  if (geo->flat) return encode3(page, x, hs, rows);
  const cuuint64_t dims[5] = {(cuuint64_t)pe, 8, (cuuint64_t)np, (cuuint64_t)(page / 8), (cuuint64_t)x};
  const cuuint64_t st[4] = {(cuuint64_t)c.s_tok * E, (cuuint64_t)pe * E, (cuuint64_t)c.s_tok * 8 * E, (cuuint64_t)hs * E};
  const cuuint32_t box[5] = {(cuuint32_t)pe, 8, (cuuint32_t)np, (cuuint32_t)(rows / 8), 1};
  return fn(m, type, 5, at, dims, st, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); }

// One lane of the warp, always the same.  The control flow around copies and products stays the whole warp's, with
// operands that are the same in all lanes, and only the instruction itself is the elected lane's: operands then live in
// uniform registers.  (Inside a branch taken by one lane they are moved there for every instruction: about 110 cycles a
// product and 100 a copy, which bounded both kernels.)
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
// a whole warp's wait: one answer for all lanes, so that the warp stays together
__device__ __forceinline__ bool wait_all(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}

// Loads of a tile (whole warp).  `rows` are the tile's valid rows; pages behind them are not looked up.  tile_entry reads
// the table (a tile ahead, so that nobody waits for it), tile_load checks the ids and issues the copies; a page the table
// does not name is read from outside the tensor, where the copy fills in zeros.
__device__ __forceinline__ int tile_boxes(const TileGeo& g, int rows) { return g.paged ? (rows + g.box_rows - 1) >> g.box_shift : 1; }
__device__ __forceinline__ int tile_entry(const AttendLaunch& a, const TileGeo& g, int b, int t0, int rows, int lane) {
  if (!g.paged || lane >= tile_boxes(g, rows)) return 0;
  const int32_t* tab = a.req.table ? a.req.table + (int64_t)b * a.req.table_stride : a.c.page_table;
  return tab[(t0 + lane * g.box_rows) >> a.c.page_shift];
}
// kFlat: rows of one part, as g.flat says (known where the kernel is compiled: half the code)
template <bool kFlat>
__device__ __forceinline__ void tile_load(const CUtensorMap* map, const AttendLaunch& a, const TileGeo& g, uint32_t dst, uint32_t bar,
                                          int t0, int rows, int h, int entry, int lane) {
  const int nb = tile_boxes(g, rows);
  if (g.paged) {
    const bool bad = lane < nb && (unsigned)entry >= (unsigned)a.c.n_phys;
    if (bad) atomicOr(a.status, KVC_FLAG_BAD_PAGE);
    const int x = bad ? -1 : entry * g.ratio + h;
    const int row = t0 & a.c.page_mask & ~(g.box_rows - 1);         // inside a page longer than a tile
    if (elect_one()) mbar_expect_tx(bar, (uint32_t)(nb * g.box_bytes));
    // eight boxes at a time (a tile of 16-token pages), their coordinates fetched first
    for (int j0 = 0; j0 < nb; j0 += 8) {
      int xs[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) xs[j] = __shfl_sync(0xffffffffu, x, j0 + j);
      if (elect_one()) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j0 + j < nb) {
            if (kFlat)
              tma_load_3d(dst + (uint32_t)((j0 + j) * g.box_bytes), map, bar, 0, row, xs[j]);
            else
              tma_load_5d(dst + (uint32_t)((j0 + j) * g.box_bytes), map, bar, 0, 0, 0, row >> 3, xs[j]);
          }
      }
    }
  } else if (elect_one()) {
    mbar_expect_tx(bar, (uint32_t)g.box_bytes);
    if (kFlat)
      tma_load_3d(dst, map, bar, 0, t0, h);
    else
      tma_load_5d(dst, map, bar, 0, t0, 0, h, 0);
  }
}

// Shared-memory operand descriptor: `swizzle` 2 = 128 B, 4 = 64 B, 6 = 32 B.  K-major: sbo = bytes from one group of 8
// rows to the next.  MN-major: lbo = from one swizzle-wide block of the M / N axis to the next, sbo = from one group of 8
// contracted rows to the next.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lbo, uint32_t sbo, uint32_t swizzle) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | ((uint64_t)((sbo >> 4) & 0x3FFFu) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)swizzle << 61);
}
// kind::f16, A = B = bf16, D = f32
__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, int a_mn, int b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// A in tensor memory (bf16 pairs, one 32-bit column a pair), B in shared memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// A kernel launched with launch_after() may start while the one before it in the stream ends (once all of that one's
// blocks have called grid_dependents_launch, or have ended); every block of it calls grid_dependency_wait(), which lasts
// until the one before is done and its memory is visible, before it touches global memory or ends.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dependents_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... P>
inline cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, const P&... p) {
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p...);
}

template <int R>
__device__ __forceinline__ void regs_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R));
}
template <int R>
__device__ __forceinline__ void regs_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R));
}

}  // namespace tc
}  // namespace kvc
