// Gated feed-forward product and its gradient on the fifth-generation tensor cores.
//
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u;   dg = dh u act'(g),  du = dh act(g),
//   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x.
//
// Every product runs on one main loop.  A pair of CTAs (a cluster of two, cta_group::2) owns a tile of 256 rows and up to
// 256 columns: each CTA brings 128 rows of A and half of B's columns into its shared memory by TMA, 64 deep at a time in
// 128-byte-swizzled tiles, seven stages in flight; one thread of the pair issues the 256 x N x 16 products; each CTA's tensor
// memory holds the 128 x N binary32 sums of its rows, twice, so that the epilogue of one tile runs beside the products of the next.
//   forward   A = x, B = 128 rows of Wg (first CTA) and the same rows of Wu (second): columns 0.. of the sums are g and
//             columns ftile.. are u of the same places, so a thread holds both and forms act(g) u in registers
//   dx        A = dg then du, B = Wg then Wu read across their rows (N-major): one sum over 2 * inner
//   dW        A = dg (du) read across its rows (M-major), B = x N-major: the sum runs over the tokens
//
// Bound by the tensor cores, and over longer stretches by the power limit: 8192 x 1600 x 6400 fp16 forward with g and u kept
// 221 us (1520 TFLOP/s) after a pause and 286 to 302 us (1110 to 1170) back to back, where the library's one product of the same
// size takes 270; backward 603 and 698 to 736 us, of them about 80 for dg and du (memory), where the library's two products take 305 and 316 back to back.
// A stage of a full tile brings a multiprocessor 32 KB for 512 cycles of products, about what L2 delivers, so that smaller
// tiles are bound by that.  Waits that poll instead of sleeping cost the backward pass 11 % (695 against 622 us).

#include <cuda.h>

#include <atomic>

#include "aq_stage.h"
#include "aq_stage_device.cuh"

namespace aq {
namespace {

template <typename T> struct Operand;        // how the tensor cores and TMA name a type
template <> struct Operand<__half> {
  static constexpr CUtensorMapDataType kMap = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  static constexpr uint32_t kFormat = 0;
};
template <> struct Operand<__nv_bfloat16> {
  static constexpr CUtensorMapDataType kMap = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  static constexpr uint32_t kFormat = 1;
};

// Phi(-|g|), the normal distribution's tail: e^(-g^2/2) times a polynomial in t = 1 / (1 + 0.375 |g| / sqrt(2)), fitted to
// erfc(x) e^(x^2) / 2 over x = 0..12 by reweighted least squares.  The fit is good to 4.5e-8; as evaluated here, in binary32, what
// counts is the rounding of the exponent: relative error 4.8e-7 up to |g| = 2, 1.5e-6 up to 5, 2.8e-6 up to 8, 7.6e-6 up
// to 13, far below one rounding of the 16-bit outputs (4.9e-4 or 3.9e-3) everywhere.
// Against erfcf: the forward kernel's epilogue at 256 x 128 outputs a tile 15000 cycles with erfcf.
__device__ float normal_tail(float g) {
  const float x = fabsf(g), t = __fdividef(1.0f, fmaf(x, 0.2651650429f, 1.0f));
  float p = 0.029775582253932953f;
  p = fmaf(p, t, -0.13898201286792755f);
  p = fmaf(p, t, 0.2068338394165039f);
  p = fmaf(p, t, -0.10435142368078232f);
  p = fmaf(p, t, 0.12995630502700806f);
  p = fmaf(p, t, 0.06359007209539413f);
  p = fmaf(p, t, 0.10195682942867279f);
  p = fmaf(p, t, 0.10541940480470657f);
  p = fmaf(p, t, 0.10580138117074966f);
  return p * t * __expf(-0.5f * g * g);
}

// act(g) and act'(g)
template <int ACT> __device__ void activation(float g, float* a, float* da) {
  if (ACT == AQ_ACT_GELU) {
    const float tail = normal_tail(g), cdf = g < 0.0f ? tail : 1.0f - tail;
    *a = g * cdf;
    *da = fmaf(g * 0.3989422804f, __expf(-0.5f * g * g), cdf);
    return;
  }
  // g sigmoid(y): y = g, or the cubic whose sigmoid is (1 + tanh(y / 2)) / 2
  const float y = ACT == AQ_ACT_SILU ? g : 1.5957691216f * g * fmaf(0.044715f * g, g, 1.0f);
  const float dy = ACT == AQ_ACT_SILU ? 1.0f : 1.5957691216f * fmaf(3.0f * 0.044715f * g, g, 1.0f);
  const float sig = __fdividef(1.0f, 1.0f + __expf(-y));
  *a = g * sig;
  const float bend = g * (sig * (1.0f - sig));                  // 0 long before the cubic's derivative overflows
  *da = bend == 0.0f ? sig : fmaf(bend, dy, sig);
}

// ---- instructions ------------------------------------------------------------------------------------------------

// four bytes into the shared memory of either CTA, counted by that CTA's barrier
__device__ void send(uint32_t to, uint32_t value, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];" ::"r"(to), "r"(value), "r"(bar) : "memory");
}
__device__ uint32_t in_cta(uint32_t addr, uint32_t rank) { uint32_t r; asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank)); return r; }
__device__ void barrier_arrive_remote(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// a box of this GPU's memory into this CTA's shared memory, counted by the first CTA's barrier
__device__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ void multiply(uint32_t sums, uint64_t a, uint64_t b, uint32_t what, uint32_t add) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(sums), "l"(a), "l"(b), "r"(what),
               "r"(add)
               : "memory");
}
// arrives on both CTAs' copies of a barrier when the products issued so far are done
__device__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ void read_sums(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
      "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
        "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
// The values are there after this; named as operands so that nothing that uses them moves ahead of it.
__device__ void sums_read(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                 "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
// 32 aligned bytes
__device__ void write_sector(void* to, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h) : "memory");
}
__device__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- the kernel --------------------------------------------------------------------------------------------------

constexpr int kDeep = 64;                     // depth of a stage: 128 bytes, one swizzled row
constexpr int kStages = 7;
constexpr int kHalfTile = 128 * kDeep * 2;    // bytes of one CTA's share of A (or B) of a stage
constexpr int kEpilogueWarps = 8;
constexpr int kFfnThreads = 128 + 32 * kEpilogueWarps;
constexpr int kChunk = 32;                    // columns an epilogue warp takes at a time
constexpr int kColumns = 512;                 // tensor memory: two tiles' sums of up to 256 columns
constexpr int kSharedBytes = 1024 + kStages * 2 * kHalfTile;
constexpr int kMaxPairs = 128;

constexpr int kClasses = 2;                   // kinds of tiles of one launch: dx and dW

// `count` tiles, `columns` wide but for the last, in each of m_tiles rows of tiles, `parts` times over (dx: parts of the
// depth; dW: dWg and dWu).  The tiles of a row follow one another, so that the pairs at work on them share its operand in L2.
struct TileClass {
  int problem, m_tiles, count, columns, last, parts, k_blocks;
};

struct Products {
  CUtensorMap a[2], b[2];                     // forward and dx
  CUtensorMap a2[2], b2;                      // dW: dg and du across their rows, x
  void* out[3];                               // forward: h, g, u; backward: dx, dWg, dWu
  long long ld[3];
  int sectors[3];                             // its rows begin on 32-byte boundaries
  int k_total;                                // stages of the whole depth of forward and dx
  int rows[2], cols[2];                       // of the outputs
  int save;                                   // forward: write g and u
  float* partial;                             // dx in parts: float[parts][rows][cols], else null
  TileClass cls[kClasses];                    // the longest tiles first
  int tiles;                                  // of all classes
  uint32_t* next;                             // tiles taken beyond each pair's first, pairs that take no more; both 0 between launches
  uint32_t format;
  uint32_t* status;
};

struct Tile {
  int problem, part, m0, n0, columns, k0, k_blocks;
};

__device__ void place(const Products& p, const TileClass& c, unsigned at, Tile* t) {
  const unsigned n = at % (unsigned)c.count, rest = at / (unsigned)c.count;
  t->problem = c.problem;
  t->part = (int)(rest / (unsigned)c.m_tiles);
  t->m0 = (int)(rest % (unsigned)c.m_tiles) * 256;
  t->n0 = (int)n * c.columns;
  t->columns = (int)n == c.count - 1 ? c.last : c.columns;
  t->k0 = c.problem == 0 ? t->part * c.k_blocks : 0;
  t->k_blocks = c.problem == 0 ? min(c.k_blocks, p.k_total - t->k0) : c.k_blocks;
}

// Tile `at` of the launch; false past the last one.
template <bool BACKWARD>
__device__ bool tile_at(const Products& p, unsigned at, Tile* t) {
  if (at >= (unsigned)p.tiles) return false;
  if constexpr (!BACKWARD) {
    // rows of tiles fastest: the pairs at work share their columns' weights
    const TileClass& c = p.cls[0];
    *t = {0, 0, (int)(at % (unsigned)c.m_tiles) * 256, (int)(at / (unsigned)c.m_tiles) * (c.columns / 2), c.columns, 0, c.k_blocks};
  } else {
    for (int k = 0; k < kClasses; ++k) {
      const TileClass& c = p.cls[k];
      const unsigned n = (unsigned)c.m_tiles * (unsigned)c.count * (unsigned)c.parts;
      if (at < n) {
        place(p, c, at, t);
        break;
      }
      at -= n;
    }
  }
  return true;
}

// what the tensor cores are told of a stage's tile in shared memory: rows of 128 bytes swizzled in groups of eight (1024
// bytes); across (M- or N-major) the next 64 rows of the operand follow after a whole 64 x 64 box
__device__ uint64_t describe(uint32_t addr, bool across) {
  return (2ull << 61) | (1ull << 46) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)(across ? 8192 >> 4 : 1) << 16) | ((addr & 0x3ffffu) >> 4);
}

template <typename T, int ACT, bool BACKWARD>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFfnThreads, 1) products_kernel(const __grid_constant__ Products p) {
  extern __shared__ uint8_t shared_raw[];
  __shared__ __align__(8) uint64_t barriers[2 * kStages + 9];
  __shared__ uint32_t tensor_base, tile_ids[2];
  const uint32_t base = (shared_address(shared_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const uint32_t rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const uint32_t bars = shared_address(barriers);
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (kStages + s); };
  auto sums_full = [&](int s) { return bars + 8u * (2 * kStages + s); };
  auto sums_empty = [&](int s) { return bars + 8u * (2 * kStages + 2 + s); };
  auto tile_sent = [&](int s) { return bars + 8u * (2 * kStages + 4 + s); };
  auto tile_read = [&](int s) { return bars + 8u * (2 * kStages + 6 + s); };   // the first CTA's counts both CTAs' readers

  const uint32_t tile_wanted = bars + 8u * (2 * kStages + 8);

  if (warp == 3 && lane == 0) {               // fetch the maps that every tile begins with
    prefetch_map(&p.a[0]); prefetch_map(&p.b[0]); prefetch_map(&p.b[1]);
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { barrier_init(full(s), 1); barrier_init(empty(s), 1); }
    barrier_init(tile_wanted, 1);
    for (int s = 0; s < 2; ++s) {
      barrier_init(sums_full(s), 1);
      barrier_init(sums_empty(s), 2 * kEpilogueWarps);
      barrier_init(tile_sent(s), 1);
      barrier_init(tile_read(s), 2 * kEpilogueWarps + 4);      // epilogue warps and loaders of both CTAs, the issuing thread, the second CTA's warp 3
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(&tensor_base)), "r"(kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  pair_sync();                                // the barriers of both CTAs exist before either signals the other's
  fence_after();
  const uint32_t tensor = tensor_base;
  next_may_launch();
  wait_for_previous();

  // A pair's first tile is its own number; the next ones are whatever tile nobody has taken yet (the longest come first), so
  // that pairs end together whatever their speed.  Which pair computes a tile does not touch its result.
  // `turn` numbers the tiles that this thread or warp has asked for.
  auto next_tile = [&](int turn, Tile* t) {
    if (turn == 0) return tile_at<BACKWARD>(p, pair, t);
    const int slot = (turn - 1) & 1;
    const bool sent = warp < 4 ? barrier_wait(tile_sent(slot), ((turn - 1) >> 1) & 1, p.status)
                               : warp_wait(lane, tile_sent(slot), ((turn - 1) >> 1) & 1, p.status);
    if (!sent) return false;
    uint32_t at;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(at) : "r"(shared_address(&tile_ids[slot])) : "memory");
    if (warp >= 4) __syncwarp();
    if (warp < 4 || lane == 0) barrier_arrive_remote(in_cta(tile_read(slot), 0));
    return tile_at<BACKWARD>(p, at, t);
  };

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool going = true;
      Tile t;
      for (int i = 0; going && next_tile(i, &t); ++i) {
        if (rank == 0) barrier_arrive(tile_wanted);
        const int half_n = t.columns / 2;
        const int b_boxes = BACKWARD ? (half_n + 63) / 64 : 0;
        const uint32_t bytes = kHalfTile + (BACKWARD ? (uint32_t)b_boxes * 8192u : (uint32_t)half_n * 128u);
        for (int i_k = 0; i_k < t.k_blocks; ++i_k) {
          const int k = t.k0 + i_k;
          if (!barrier_wait(empty(stage), phase ^ 1, p.status)) { going = false; break; }
          const uint32_t bar = in_cta(full(stage), 0);
          if (rank == 0) barrier_expect(full(stage), 2 * bytes);
          const uint32_t to_a = base + (uint32_t)stage * 2 * kHalfTile, to_b = to_a + kHalfTile;
          if constexpr (!BACKWARD) {
            load_box(to_a, &p.a[0], k * kDeep, t.m0 + (int)rank * 128, bar);
            load_box(to_b, &p.b[rank], k * kDeep, t.n0, bar);
          } else if (t.problem == 0) {
            const int z = 2 * k >= p.k_total, k0 = (z ? k - p.k_total / 2 : k) * kDeep;
            load_box(to_a, &p.a[z], k0, t.m0 + (int)rank * 128, bar);
            load_box(to_a + 8192, &p.a[z], k0, t.m0 + (int)rank * 128 + 64, bar);
            for (int j = 0; j < b_boxes; ++j) load_box(to_b + j * 8192, &p.b[z], t.n0 + (int)rank * half_n + j * 64, k0, bar);
          } else {
            load_box(to_a, &p.a2[t.part], t.m0 + (int)rank * 128, k * kDeep, bar);
            load_box(to_a + 8192, &p.a2[t.part], t.m0 + (int)rank * 128 + 64, k * kDeep, bar);
            for (int j = 0; j < b_boxes; ++j) load_box(to_b + j * 8192, &p.b2, t.n0 + (int)rank * half_n + j * 64, k * kDeep, bar);
          }
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
      }
      // the products that release the last stages signal both CTAs: none may leave before
      for (int s = 0; going && s < kStages; ++s) {
        going = barrier_wait(empty(stage), phase ^ 1, p.status);
        if (++stage == kStages) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1 && rank == 0) {
    if (lane == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool going = true;
      Tile t;
      for (int i = 0; going && next_tile(i, &t); ++i) {
        const bool a_across = BACKWARD && t.problem == 1, b_across = BACKWARD;
        // binary32 sums (bit 4), operand types, which operands run across, N / 8, M / 16
        const uint32_t what = (1u << 4) | (p.format << 7) | (p.format << 10) | ((uint32_t)a_across << 15) | ((uint32_t)b_across << 16) |
                              ((uint32_t)(t.columns >> 3) << 17) | (16u << 24);
        // 16 deep: 32 bytes along a row, or sixteen rows
        const uint32_t step_a = a_across ? 2048 >> 4 : 32 >> 4, step_b = b_across ? 2048 >> 4 : 32 >> 4;
        if (!barrier_wait(sums_empty(acc), acc_phase ^ 1, p.status)) break;
        fence_after();
        const uint32_t sums = tensor + (uint32_t)acc * 256u;
        for (int k = 0; k < t.k_blocks; ++k) {
          if (!barrier_wait(full(stage), phase, p.status)) { going = false; break; }
          fence_after();
          const uint32_t at = base + (uint32_t)stage * 2 * kHalfTile;
          const uint64_t da = describe(at, a_across), db = describe(at + kHalfTile, b_across);
#pragma unroll
          for (int j = 0; j < kDeep / 16; ++j) multiply(sums, da + j * step_a, db + j * step_b, what, (k | j) != 0);
          commit(empty(stage));
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
        commit(sums_full(acc));
        acc ^= 1;
        if (!acc) acc_phase ^= 1;
      }
    }
  } else if (warp == 3) {
    if (lane == 0) {
      // Each CTA says what its barrier is to receive; the first CTA takes a tile when the loader has begun with the one before
      // (no earlier, so that none waits at a busy pair) and sends it to both.
      for (int i = 0;; ++i) {
        const int slot = i & 1;
        uint32_t at = 0;
        if (rank == 0) {
          if (!barrier_wait(tile_wanted, i & 1, p.status) || !barrier_wait(tile_read(slot), ((i >> 1) & 1) ^ 1, p.status)) break;
          barrier_expect(tile_sent(slot), 4);
          at = pairs + atomicAdd(p.next, 1u);
          for (uint32_t r = 0; r < 2; ++r) send(in_cta(shared_address(&tile_ids[slot]), r), at, in_cta(tile_sent(slot), r));
        } else {
          barrier_expect(tile_sent(slot), 4);
          if (!barrier_wait(tile_sent(slot), (i >> 1) & 1, p.status)) break;
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(at) : "r"(shared_address(&tile_ids[slot])) : "memory");
          barrier_arrive_remote(in_cta(tile_read(slot), 0));
        }
        if (at >= (unsigned)p.tiles) break;
      }
      // The last pair that has done with taking, however it came to that, leaves the counters as the next launch expects them.
      __threadfence();                         // its takes come first
      if (rank == 0 && atomicAdd(p.next + 1, 1u) == pairs - 1) { p.next[0] = 0; p.next[1] = 0; }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, turn = (warp - 4) / 4;
    int acc = 0;
    uint32_t acc_phase = 0;
    // 32 rows x 32 columns, each lane a row, to (y, x) of an output: 32 bytes (one sector) a store where the output is aligned
    // for that.  Turning the tile round in shared memory first, for stores along rows or by TMA, took longer beside the products,
    // whose operands fill that memory's bandwidth (1200 to 1700 cycles for 32 x 32 values of a warp, 800 to 1200 as here), and
    // took a stage's room.
    auto put16 = [&](const uint32_t (&v)[32], int out, int problem, int x, int y) {
      const int row = y + lane;
      if (row >= p.rows[problem]) return;
      T* const to = static_cast<T*>(p.out[out]) + (long long)row * p.ld[out] + x;
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = Num<T>::close(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
      if (p.sectors[out] && x + kChunk <= p.cols[problem]) {
        write_sector(to, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
        write_sector(to + 16, w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (x + j * 8 < p.cols[problem]) *reinterpret_cast<uint4*>(to + j * 8) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
      }
    };
    auto put32 = [&](const uint32_t (&v)[32], float* out, int x, int y) {
      const int row = y + lane;
      if (row >= p.rows[0]) return;
      float* const to = out + (long long)row * p.cols[0] + x;
#pragma unroll
      for (int j = 0; j < 4; ++j)                         // cols is a multiple of 8
        if (x + j * 8 < p.cols[0]) write_sector(to + j * 8, v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3], v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]);
    };
    Tile t;
    for (int i = 0; next_tile(i, &t); ++i) {
      if (!warp_wait(lane, sums_full(acc), acc_phase, p.status)) break;
      fence_after();
      const uint32_t sums = tensor + (uint32_t)acc * 256u + ((uint32_t)quarter << 21);
      const int width = BACKWARD ? t.columns : t.columns / 2;
      const int y = t.m0 + (int)rank * 128 + quarter * 32;
      const bool rows_there = y < p.rows[t.problem];
      for (int c = turn * kChunk; c < width; c += 2 * kChunk) {
        uint32_t r[32], q[32];
        read_sums(sums + (uint32_t)c, r);
        if constexpr (!BACKWARD) read_sums(sums + (uint32_t)(width + c), q);
        sums_read(r);
        if constexpr (!BACKWARD) sums_read(q);
        if (c + 2 * kChunk >= width) {                    // this warp's last columns are in registers
          fence_before();
          __syncwarp();
          if (lane == 0) barrier_arrive_remote(in_cta(sums_empty(acc), 0));
        }
        if (!rows_there || t.n0 + c >= p.cols[t.problem]) continue;
        if constexpr (BACKWARD) {
          if (t.problem == 0 && p.partial) put32(r, p.partial + (long long)t.part * p.rows[0] * p.cols[0], t.n0 + c, y);
          else put16(r, t.problem ? 1 + t.part : 0, t.problem, t.n0 + c, y);
        } else {
          if (p.save) {
            put16(r, 1, 0, t.n0 + c, y);
            put16(q, 2, 0, t.n0 + c, y);
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float act, dact;
            activation<ACT>(__uint_as_float(r[j]), &act, &dact);
            r[j] = __float_as_uint(act * __uint_as_float(q[j]));
          }
          put16(r, 0, 0, t.n0 + c, y);
        }
      }
      if (turn * kChunk >= width) {                       // a narrow tile: nothing here for this warp
        if (lane == 0) barrier_arrive_remote(in_cta(sums_empty(acc), 0));
      }
      acc ^= 1;
      if (!acc) acc_phase ^= 1;
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  pair_sync();                                // no CTA leaves while the other may still signal it or use its memory
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tensor), "r"(kColumns) : "memory");
}

// dg and du to the workspace, eight elements per thread.  Rounded to T, what the tensor cores take: two 16-bit parts of each would be
// twice the products.  The one rounding more takes the relative error of dx and dW from 2.1e-4 to 2.9e-4 (fp16) and from 1.7e-3
// to 2.4e-3 (bf16).
template <typename T, int ACT>
__global__ void __launch_bounds__(256) ffn_dgu_kernel(const FfnGradArgs a) {
  next_may_launch();
  wait_for_previous();
  const unsigned per_row = (unsigned)a.inner / 8;
  const unsigned long long n = (unsigned long long)a.rows * per_row;
  for (unsigned long long i = (unsigned long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (unsigned long long)gridDim.x * 256) {
    const unsigned long long r = i / per_row;
    const unsigned c = (unsigned)(i - r * per_row) * 8;
    const uint4 vd = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(a.dh) + r * a.lddh + c));
    const uint4 vg = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(a.g) + r * a.ldgu + c));
    const uint4 vu = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(a.u) + r * a.ldgu + c));
    const uint32_t d[4] = {vd.x, vd.y, vd.z, vd.w}, g[4] = {vg.x, vg.y, vg.z, vg.w}, u[4] = {vu.x, vu.y, vu.z, vu.w};
    uint32_t og[4], ou[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 df = Num<T>::open(d[j]), gf = Num<T>::open(g[j]), uf = Num<T>::open(u[j]);
      float a0, a1, d0, d1;
      activation<ACT>(gf.x, &a0, &d0);
      activation<ACT>(gf.y, &a1, &d1);
      og[j] = Num<T>::close(df.x * uf.x * d0, df.y * uf.y * d1);
      ou[j] = Num<T>::close(df.x * a0, df.y * a1);
    }
    reinterpret_cast<uint4*>(a.dg)[i] = make_uint4(og[0], og[1], og[2], og[3]);
    reinterpret_cast<uint4*>(a.du)[i] = make_uint4(ou[0], ou[1], ou[2], ou[3]);
  }
}

// dx = the sum of its parts, in their order
template <typename T>
__global__ void __launch_bounds__(256) ffn_join_kernel(const float* part, int parts, long long rows, int cols, T* out, long long ld) {
  next_may_launch();
  wait_for_previous();
  const unsigned per_row = (unsigned)cols / 8;
  const unsigned long long n = (unsigned long long)rows * per_row, i = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const unsigned long long r = i / per_row;
  const unsigned c = (unsigned)(i - r * per_row) * 8;
  const float4* from = reinterpret_cast<const float4*>(part + r * (unsigned)cols + c);
  const unsigned long long next = (unsigned long long)rows * (unsigned)cols / 4;
  float4 a = __ldcs(from), b = __ldcs(from + 1);
#pragma unroll 4
  for (int p = 1; p < parts; ++p) {
    from += next;
    const float4 c4 = __ldcs(from), d4 = __ldcs(from + 1);
    a.x += c4.x; a.y += c4.y; a.z += c4.z; a.w += c4.w;
    b.x += d4.x; b.y += d4.y; b.z += d4.z; b.w += d4.w;
  }
  *reinterpret_cast<uint4*>(out + r * ld + c) = make_uint4(Num<T>::close(a.x, a.y), Num<T>::close(a.z, a.w), Num<T>::close(b.x, b.y), Num<T>::close(b.z, b.w));
}

// ---- forward for few rows ---------------------------------------------------------------------------------------
//
// Bound by the weights, 4 * inner * hidden bytes, which every token shares: a CTA takes sixteen rows of Wg and Wu, its eight
// warps share their depth, and all of the loads are in flight at once (no staging).  The products are warp-level 16 x 8 x 16
// ones: rows 0..7 of the sixteen are Wg's, rows 8..15 Wu's of the same outputs, columns are tokens.  Which place of the depth a
// lane's element takes does not matter as long as weights and tokens agree, so each lane loads 16 contiguous bytes of a row
// and uses them for two products of depth 16.

constexpr int kRowsThreads = 256, kRowsWarps = 8, kRowsAhead = 4;
// At 32 rows 14.5 us (1600 x 6400) and 6.3 us (2048 x 520), where the CTA pairs take 15.4 and 12.8 us; one row 7.1 us, 5.8 TB/s.
constexpr int kFewRows = 32;

__device__ void multiply_warp(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __half) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ void multiply_warp(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __nv_bfloat16) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T, int ACT, int TOKENS8>
__global__ void __launch_bounds__(kRowsThreads, TOKENS8 == 2 ? 3 : 1) ffn_rows_kernel(const FfnArgs a) {
  __shared__ float4 sums[kRowsWarps][2 * TOKENS8][32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int f0 = blockIdx.x * 16;
  const int rows = (int)a.rows;
  const bool there[2] = {true, f0 + 8 < a.inner};            // inner is a multiple of 8
  const T* const wg = static_cast<const T*>(a.wg) + (long long)(f0 + g) * a.ldw;
  const T* const wu = static_cast<const T*>(a.wu) + (long long)(f0 + g) * a.ldw;
  const T* const x = static_cast<const T*>(a.x);
  float c[2][TOKENS8][4] = {};
  next_may_launch();
  // a hint while the stream's previous kernel drains: the weights into L2, a row of each matrix a lane of the first warp
  if (warp == 0 && f0 + (lane & 15) < a.inner) {
    const T* const row = static_cast<const T*>(lane < 16 ? a.wg : a.wu) + (long long)(f0 + (lane & 15)) * a.ldw;
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row), "r"(a.hidden * 2) : "memory");
  }
  wait_for_previous();
  const int steps = (a.hidden + 31) / 32;
  for (int s0 = warp; s0 < steps; s0 += kRowsWarps * kRowsAhead) {
    uint4 vg[kRowsAhead][2], vu[kRowsAhead][2];
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int k = (s0 + i * kRowsWarps) * 32 + q * 8;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bool in = k < a.hidden && there[t];
        vg[i][t] = in ? __ldcs(reinterpret_cast<const uint4*>(wg + t * 8 * a.ldw + k)) : make_uint4(0, 0, 0, 0);
        vu[i][t] = in ? __ldcs(reinterpret_cast<const uint4*>(wu + t * 8 * a.ldw + k)) : make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < kRowsAhead; ++i) {
      const int k = (s0 + i * kRowsWarps) * 32 + q * 8;
#pragma unroll
      for (int n = 0; n < TOKENS8; ++n) {
        const int token = n * 8 + g;
        const uint4 v = k < a.hidden && token < rows ? __ldg(reinterpret_cast<const uint4*>(x + token * a.ldx + k)) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          multiply_warp(c[t][n], vg[i][t].x, vu[i][t].x, vg[i][t].y, vu[i][t].y, v.x, v.y, T());
          multiply_warp(c[t][n], vg[i][t].z, vu[i][t].z, vg[i][t].w, vu[i][t].w, v.z, v.w, T());
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int n = 0; n < TOKENS8; ++n) sums[warp][t * TOKENS8 + n][lane] = make_float4(c[t][n][0], c[t][n][1], c[t][n][2], c[t][n][3]);
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * TOKENS8 * 32; i += kRowsThreads) {
    const int l = i & 31, t = (i >> 5) / TOKENS8, n = (i >> 5) % TOKENS8;
    float4 v = sums[0][i >> 5][l];
#pragma unroll
    for (int w = 1; w < kRowsWarps; ++w) {
      const float4 o = sums[w][i >> 5][l];
      v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
    }
    const int f = f0 + t * 8 + (l >> 2), token = n * 8 + (l & 3) * 2;
    if (f >= a.inner) continue;
    const float gate[2] = {v.x, v.y}, up[2] = {v.z, v.w};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (token + j >= rows) break;
      float act, dact;
      activation<ACT>(gate[j], &act, &dact);
      static_cast<T*>(a.h)[(token + j) * a.ldh + f] = Num<T>::one(act * up[j]);
      if (a.g) {
        static_cast<T*>(a.g)[(token + j) * a.ldgu + f] = Num<T>::one(gate[j]);
        static_cast<T*>(a.u)[(token + j) * a.ldgu + f] = Num<T>::one(up[j]);
      }
    }
  }
}

// ---- host --------------------------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

cudaError_t encoder(EncodeTiled* out) {
  static std::atomic<EncodeTiled> known{nullptr};          // the same address for every thread that finds it
  EncodeTiled fn = known.load(std::memory_order_relaxed);
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !p) return cudaErrorNotSupported;
    fn = reinterpret_cast<EncodeTiled>(p);
    known.store(fn, std::memory_order_relaxed);
  }
  *out = fn;
  return cudaSuccess;
}

struct Maps {
  EncodeTiled fn = nullptr;
  cudaError_t error = cudaSuccess;
  Maps() { error = encoder(&fn); }
  // T[rows][ld], `cols` of a row, in boxes of 64 columns (128 bytes, swizzled) x box_rows
  template <typename T>
  void set(CUtensorMap* m, const void* p, long long rows, long long cols, long long ld, int box_rows) {
    if (error != cudaSuccess) return;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {kDeep, (cuuint32_t)box_rows}, one[2] = {1, 1};
    const CUresult r = fn(m, Operand<T>::kMap, 2, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) error = cudaErrorInvalidValue;
  }
};

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// The cost of tiles, in cycles.  A stage's products take 2 n for n columns; its operands, 16384 + 64 n bytes to each
// multiprocessor, take about 480 + n / 4.  Starting a tile costs about 1500, its epilogue 11 n, which hides behind the next
// tile's stages.  The constants are those that order the times of 16 widths and depths of five backward calls best (509 to 3000
// rows; what they choose is within 1.18 of the fastest, four times the fastest itself).
long long stage_cycles(int n) { return 2 * n > 480 + n / 4 ? 2 * n : 480 + n / 4; }
long long epilogue_cycles(int n) { return 11 * n; }
long long tile_cycles(int stages, int n) {
  const long long work = (long long)stages * stage_cycles(n), before = epilogue_cycles(n);
  return (work > before ? work : before) + 1500;
}

// Pairs that are on the GPU at the same time: the parts of the chip with an odd number of multiprocessors hold one CTA less.
// A grid with more would run its last pairs after all others had finished their share.
cudaError_t resident_pairs(int* pairs) {
  auto kernel = products_kernel<__half, AQ_ACT_SILU, true>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(2 * kMaxPairs);
  cfg.blockDim = dim3(kFfnThreads);
  cfg.dynamicSmemBytes = kSharedBytes;
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 2;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(pairs, kernel, &cfg);
  if (e == cudaSuccess && *pairs < 1) e = cudaErrorInvalidConfiguration;
  if (*pairs > kMaxPairs) *pairs = kMaxPairs;
  return e;
}

template <typename T, int ACT, bool BACKWARD>
cudaError_t launch_products(Products& p, int pairs, cudaStream_t s) {
  for (int i = 0; i < 3; ++i) p.sectors[i] = (reinterpret_cast<uintptr_t>(p.out[i]) & 31) == 0 && p.ld[i] % 16 == 0;
  auto kernel = products_kernel<T, ACT, BACKWARD>;
  static std::atomic<uint64_t> allowed{0};    // devices on which this kernel may have that much shared memory
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (!(allowed.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
    if (e != cudaSuccess) return e;
    allowed.fetch_or(bit, std::memory_order_relaxed);
  }
  return launch(kernel, 2u * pairs, kFfnThreads, kSharedBytes, s, p);
}

template <typename T, int ACT>
cudaError_t run_rows(const FfnArgs& a, cudaStream_t s) {
  const unsigned ctas = (unsigned)ceil_div(a.inner, 16);
  if (a.rows <= 8) return launch(ffn_rows_kernel<T, ACT, 1>, ctas, kRowsThreads, 0, s, a);
  if (a.rows <= 16) return launch(ffn_rows_kernel<T, ACT, 2>, ctas, kRowsThreads, 0, s, a);
  return launch(ffn_rows_kernel<T, ACT, 4>, ctas, kRowsThreads, 0, s, a);
}

template <typename T, int ACT>
cudaError_t run(const FfnArgs& a, cudaStream_t s) {
  if (a.rows <= kFewRows) return run_rows<T, ACT>(a, s);
  Products p{};
  const int m_tiles = ceil_div(a.rows, 256), kb = ceil_div(a.hidden, kDeep);
  int best = 0;
  long long least = 0;
  for (int f = 128; f >= 32; f -= 32) {
    // rounds of the grid, and the last one's epilogue
    const long long tiles = (long long)m_tiles * ceil_div(a.inner, f), c = ((tiles + a.pairs - 1) / a.pairs) * tile_cycles(kb, 2 * f) + epilogue_cycles(2 * f);
    if (!best || c < least) { best = f; least = c; }
  }
  p.cls[0] = {0, m_tiles, ceil_div(a.inner, best), 2 * best, 2 * best, 1, kb};
  p.k_total = kb;
  p.rows[0] = (int)a.rows;
  p.cols[0] = a.inner;
  p.save = a.g != nullptr;
  p.format = Operand<T>::kFormat;
  p.status = a.status;
  Maps maps;
  maps.set<T>(&p.a[0], a.x, a.rows, a.hidden, a.ldx, 128);
  maps.set<T>(&p.b[0], a.wg, a.inner, a.hidden, a.ldw, best);
  maps.set<T>(&p.b[1], a.wu, a.inner, a.hidden, a.ldw, best);
  p.out[0] = a.h;
  p.out[1] = a.g;
  p.out[2] = a.u;
  p.ld[0] = a.ldh;
  p.ld[1] = p.ld[2] = a.ldgu;
  if (maps.error != cudaSuccess) return maps.error;
  const long long tiles = (long long)m_tiles * p.cls[0].count;
  if (tiles > 0x7fffffff - kMaxPairs) return cudaErrorInvalidValue;
  p.tiles = (int)tiles;
  p.next = a.next;
  return launch_products<T, ACT, false>(p, tiles < a.pairs ? (int)tiles : a.pairs, s);
}

// ---- the gradient's plan

constexpr long long kMostPartialBytes = 256ll << 20;

struct Plan {
  int n = 256, parts = 1;
  long long cycles = -1;
};

// The classes of tiles of a plan, the longest first; their number.  Columns that a row of full tiles leaves over widen its
// last tile where they fit, and are a narrow tile of their own otherwise.
int classes_of(const Plan& plan, long long rows, int hidden, int inner, bool dx, bool dw, TileClass* out) {
  int count = hidden / plan.n, last = plan.n;
  const int rest = (hidden - count * plan.n + 31) / 32 * 32;
  if (rest && count && plan.n + rest <= 256) last = plan.n + rest;
  else if (rest) { ++count; last = rest; }
  const int kb0 = 2 * ceil_div(inner, kDeep), part = ceil_div(kb0, plan.parts);
  int c = 0;
  if (dx) out[c++] = {0, ceil_div(rows, 256), count, plan.n, last, ceil_div(kb0, part), part};
  if (dw) out[c++] = {1, ceil_div(inner, 256), count, plan.n, last, 2, ceil_div(rows, kDeep)};
  if (c == 2 && out[1].k_blocks > out[0].k_blocks) {
    const TileClass t = out[0];
    out[0] = out[1];
    out[1] = t;
  }
  return c;
}

long long tiles_of(const TileClass& c) { return (long long)c.m_tiles * c.count * c.parts; }
// Widths and parts by an estimate of the longest load.  Parts of dx's depth, 2 * inner, serve few rows, whose dx is a
// handful of very long tiles; joining them is another kernel of about 2200 cycles more that moves 8 bytes a value and part, some
// 2800 a cycle.
Plan plan_of(const FfnGradArgs& a) {
  Plan best;
  const int kb0 = 2 * ceil_div(a.inner, kDeep);
  for (int parts = 1; parts <= 32 && parts <= kb0; parts *= 2) {
    if (parts > 1 && (!a.dx || (long long)parts * a.rows * a.hidden * 4 > kMostPartialBytes)) break;
    for (int n = 256; n >= 64; n -= 32) {
      Plan plan;
      plan.n = n;
      plan.parts = parts;
      TileClass cls[kClasses];
      const int count = classes_of(plan, a.rows, a.hidden, a.inner, a.dx != nullptr, a.dwg != nullptr, cls);
      long long work = 0, tiles = 0;
      for (int c = 0; c < count; ++c) {
        work += (long long)cls[c].m_tiles * cls[c].parts * ((cls[c].count - 1) * tile_cycles(cls[c].k_blocks, n) + tile_cycles(cls[c].k_blocks, cls[c].last));
        tiles += tiles_of(cls[c]);
      }
      // taken longest first, the pairs end within about half of a short tile of one another
      const long long longest = tile_cycles(cls[0].k_blocks, cls[0].count > 1 && n > cls[0].last ? n : cls[0].last);
      plan.cycles = tiles <= a.pairs ? 0 : work / a.pairs + tile_cycles(cls[count - 1].k_blocks, n) / 2;
      if (plan.cycles < longest) plan.cycles = longest;
      plan.cycles += epilogue_cycles(n) + (parts > 1 ? 2200 + (long long)parts * a.rows * a.hidden * 8 / 2800 : 0);
      if (best.cycles < 0 || plan.cycles < best.cycles) best = plan;
    }
  }
  return best;
}

template <typename T>
cudaError_t run_grad(const FfnGradArgs& a, cudaStream_t s) {
  const long long vectors = a.rows * (a.inner / 8), want = (vectors + 255) / 256, most = 16ll * a.sms;
  const unsigned ctas = (unsigned)(want < most ? want : most);
  cudaError_t e = a.act == AQ_ACT_SILU   ? launch(ffn_dgu_kernel<T, AQ_ACT_SILU>, ctas, 256, 0, s, a)
                  : a.act == AQ_ACT_GELU ? launch(ffn_dgu_kernel<T, AQ_ACT_GELU>, ctas, 256, 0, s, a)
                                         : launch(ffn_dgu_kernel<T, AQ_ACT_GELU_TANH>, ctas, 256, 0, s, a);
  if (e != cudaSuccess) return e;
  const Plan plan = plan_of(a);
  Products p{};
  Maps maps;
  p.format = Operand<T>::kFormat;
  p.status = a.status;
  p.k_total = 2 * ceil_div(a.inner, kDeep);
  p.rows[0] = (int)a.rows;
  p.rows[1] = a.inner;
  p.cols[0] = p.cols[1] = a.hidden;
  p.partial = plan.parts > 1 ? a.partial : nullptr;
  const int count = classes_of(plan, a.rows, a.hidden, a.inner, a.dx != nullptr, a.dwg != nullptr, p.cls);
  long long tiles = 0;
  for (int c = 0; c < count; ++c) tiles += tiles_of(p.cls[c]);
  if (tiles > 0x7fffffff - kMaxPairs) return cudaErrorInvalidValue;
  p.tiles = (int)tiles;
  p.next = a.next;
  const int pairs = tiles < a.pairs ? (int)tiles : a.pairs;
  maps.set<T>(&p.a[0], a.dg, a.rows, a.inner, a.inner, 64);
  maps.set<T>(&p.a[1], a.du, a.rows, a.inner, a.inner, 64);
  p.a2[0] = p.a[0];
  p.a2[1] = p.a[1];
  maps.set<T>(&p.b[0], a.wg, a.inner, a.hidden, a.ldw, 64);
  maps.set<T>(&p.b[1], a.wu, a.inner, a.hidden, a.ldw, 64);
  maps.set<T>(&p.b2, a.x, a.rows, a.hidden, a.ldx, 64);
  p.out[0] = a.dx;
  p.out[1] = a.dwg;
  p.out[2] = a.dwu;
  p.ld[0] = a.lddx;
  p.ld[1] = p.ld[2] = a.lddw;
  if (maps.error != cudaSuccess) return maps.error;
  e = launch_products<T, AQ_ACT_SILU, true>(p, pairs, s);
  if (e != cudaSuccess || !p.partial) return e;
  int parts = 1;
  for (int c = 0; c < count; ++c) if (p.cls[c].problem == 0) parts = p.cls[c].parts;
  return launch(ffn_join_kernel<T>, (unsigned)((a.rows * (a.hidden / 8) + 255) / 256), 256, 0, s, (const float*)a.partial, parts, a.rows, a.hidden,
                static_cast<T*>(a.dx), a.lddx);
}

template <typename T>
cudaError_t run_act(const FfnArgs& a, cudaStream_t s) {
  return a.act == AQ_ACT_SILU ? run<T, AQ_ACT_SILU>(a, s) : a.act == AQ_ACT_GELU ? run<T, AQ_ACT_GELU>(a, s) : run<T, AQ_ACT_GELU_TANH>(a, s);
}

}  // namespace

long long ffn_grad_partial_bytes(const FfnGradArgs& a) {
  const Plan plan = plan_of(a);
  return plan.parts > 1 ? (long long)plan.parts * a.rows * a.hidden * 4 : 0;
}
cudaError_t ffn_resident_pairs(int* pairs) { return resident_pairs(pairs); }
cudaError_t launch_ffn(int dtype, const FfnArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run_act<__half>(a, s) : run_act<__nv_bfloat16>(a, s);
}
cudaError_t launch_ffn_grad(int dtype, const FfnGradArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run_grad<__half>(a, s) : run_grad<__nv_bfloat16>(a, s);
}

}  // namespace aq
