// Gated feed-forward product and its gradient on the fifth-generation tensor cores.
//
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u;   dg = dh u act'(g),  du = dh act(g),
//   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x.
//
// Every product runs on one main loop.  A pair of CTAs (a cluster of two, cta_group::2) owns a tile of 256 rows and up to
// 256 columns: each CTA brings 128 rows of A and half of B's columns into its shared memory by TMA, 64 deep at a time in
// 128-byte-swizzled tiles, six stages in flight; one thread of the pair issues the 256 x N x 16 products; each CTA's tensor
// memory holds the 128 x N binary32 sums of its rows, twice, so that the epilogue of one tile runs beside the products of the next.
//   forward   A = x, B = 128 rows of Wg (first CTA) and the same rows of Wu (second): columns 0.. of the sums are g and
//             columns ftile.. are u of the same places, so a thread holds both and forms act(g) u in registers
//   dx        A = dg then du, B = Wg then Wu read across their rows (N-major): one sum over 2 * inner
//   dW        A = dg (du) read across its rows (M-major), B = x N-major: the sum runs over the tokens

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/aq_b200.h"
#include "aq_stage.h"

namespace aq {
namespace {

template <typename T> struct Num;
template <> struct Num<__half> {
  static constexpr CUtensorMapDataType kMap = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  static constexpr uint32_t kFormat = 0;
  static __device__ float2 open(uint32_t u) { return __half22float2(*reinterpret_cast<__half2*>(&u)); }
  static __device__ uint32_t close(float a, float b) { const __half2 p = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&p); }
};
template <> struct Num<__nv_bfloat16> {
  static constexpr CUtensorMapDataType kMap = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  static constexpr uint32_t kFormat = 1;
  static __device__ float2 open(uint32_t u) { return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
  static __device__ uint32_t close(float a, float b) { const __nv_bfloat162 p = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&p); }
};

// act(g) and act'(g)
template <int ACT> __device__ void activation(float g, float* a, float* da) {
  if (ACT == AQ_ACT_GELU) {
    const float cdf = 0.5f * erfcf(-0.70710678f * g);
    *a = g * cdf;
    *da = fmaf(g * 0.3989422804f, __expf(-0.5f * g * g), cdf);
    return;
  }
  // g sigmoid(y): y = g, or the cubic whose sigmoid is (1 + tanh(y / 2)) / 2
  const float y = ACT == AQ_ACT_SILU ? g : 1.5957691216f * g * fmaf(0.044715f * g, g, 1.0f);
  const float dy = ACT == AQ_ACT_SILU ? 1.0f : 1.5957691216f * fmaf(3.0f * 0.044715f * g, g, 1.0f);
  const float sig = __fdividef(1.0f, 1.0f + __expf(-y));
  *a = g * sig;
  // sig (1 - sig) is 0 long before the cubic's derivative could overflow
  *da = fmaf(g * (sig * (1.0f - sig)), dy, sig);
}

// ---- instructions ------------------------------------------------------------------------------------------------

__device__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// the address of the pair's first CTA's copy of a shared variable
__device__ uint32_t in_first_cta(uint32_t addr) { uint32_t r; asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr)); return r; }
__device__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ void barrier_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ void barrier_arrive_remote(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ bool barrier_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
__device__ unsigned long long now_ns() { unsigned long long t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }
// Waits for a phase; false (and the status bit) when it has not come within four seconds: the caller leaves its loop.
__device__ __noinline__ bool barrier_wait_long(uint32_t bar, uint32_t parity, uint32_t* status) {
  const unsigned long long until = now_ns() + 4000000000ull;
  do {
    for (int i = 0; i < 256; ++i)
      if (barrier_try(bar, parity)) return true;
  } while (now_ns() < until);
  atomicOr(status, (uint32_t)AQ_ST_STALLED);
  return false;
}
__device__ bool barrier_wait(uint32_t bar, uint32_t parity, uint32_t* status) {
#pragma unroll 1
  for (int i = 0; i < 64; ++i)
    if (barrier_try(bar, parity)) return true;
  return barrier_wait_long(bar, parity, status);
}
// a box of this GPU's memory into this CTA's shared memory, counted by the first CTA's barrier
__device__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ void store_box(const CUtensorMap* map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
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
__device__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- the kernel --------------------------------------------------------------------------------------------------

constexpr int kDeep = 64;                     // depth of a stage: 128 bytes, one swizzled row
constexpr int kStages = 6;
constexpr int kHalfTile = 128 * kDeep * 2;    // bytes of one CTA's share of A (or B) of a stage
constexpr int kEpilogueWarps = 8;
constexpr int kFfnThreads = 128 + 32 * kEpilogueWarps;
constexpr int kChunk = 32;                    // columns an epilogue warp takes at a time
constexpr int kOutBytes = 32 * kChunk * 2;    // ... of 32 rows: one TMA store
constexpr int kOutBuffers = 2;
constexpr int kColumns = 512;                 // tensor memory: two tiles' sums of up to 256 columns
constexpr int kSharedBytes = 1024 + kStages * 2 * kHalfTile + kEpilogueWarps * kOutBuffers * kOutBytes;
constexpr int kMaxPairs = 128;

struct Products {
  CUtensorMap a[2], b[2];                     // first problem
  CUtensorMap a2[2], b2;                      // dW: dg and du across their rows, x
  CUtensorMap out[3];                         // forward: h, g, u; backward: dx, dWg, dWu
  int m_tiles[2], n_tiles[2];                 // of the first problem and of dW
  int k_blocks[2];                            // stages per tile
  int n[2];                                   // columns of a tile (both halves of the pair)
  int rows[2], cols[2];                       // of the outputs
  int save;                                   // forward: write g and u
  uint32_t first[2][kMaxPairs + 1];           // backward: the tiles of each problem that a pair works on
  uint32_t format;
  uint32_t* status;
};

struct Tile {
  int problem, z, m0, n0;
};

template <bool BACKWARD>
__device__ bool tile_at(const Products& p, unsigned pair, unsigned pairs, unsigned i, Tile* t) {
  if constexpr (!BACKWARD) {
    const unsigned at = pair + i * pairs;
    if (at >= (unsigned)p.m_tiles[0] * (unsigned)p.n_tiles[0]) return false;
    *t = {0, 0, (int)(at % (unsigned)p.m_tiles[0]) * 256, (int)(at / (unsigned)p.m_tiles[0]) * (p.n[0] / 2)};
    return true;
  } else {
    unsigned at = p.first[0][pair] + i;
    if (at < p.first[0][pair + 1]) {
      *t = {0, 0, (int)(at / (unsigned)p.n_tiles[0]) * 256, (int)(at % (unsigned)p.n_tiles[0]) * p.n[0]};
      return true;
    }
    at = p.first[1][pair] + (at - p.first[0][pair + 1]);
    if (at >= p.first[1][pair + 1]) return false;
    const unsigned per = (unsigned)p.m_tiles[1] * (unsigned)p.n_tiles[1], in = at % per;
    *t = {1, (int)(at / per), (int)(in / (unsigned)p.n_tiles[1]) * 256, (int)(in % (unsigned)p.n_tiles[1]) * p.n[1]};
    return true;
  }
}

// what the tensor cores are told of a stage's tile in shared memory: rows of 128 bytes swizzled in groups of eight (1024
// bytes); across (M- or N-major) the next 64 rows of the operand follow after a whole 64 x 64 box
__device__ uint64_t describe(uint32_t addr, bool across) {
  return (2ull << 61) | (1ull << 46) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)(across ? 8192 >> 4 : 1) << 16) | ((addr & 0x3ffffu) >> 4);
}

template <typename T, int ACT, bool BACKWARD>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFfnThreads, 1) products_kernel(const __grid_constant__ Products p) {
  extern __shared__ uint8_t shared_raw[];
  __shared__ __align__(8) uint64_t barriers[2 * kStages + 4];
  __shared__ uint32_t tensor_base;
  const uint32_t base = (shared_address(shared_raw) + 1023u) & ~1023u;
  const uint32_t out_base = base + kStages * 2 * kHalfTile;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const unsigned rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const uint32_t bars = shared_address(barriers);
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (kStages + s); };
  auto sums_full = [&](int s) { return bars + 8u * (2 * kStages + s); };
  auto sums_empty = [&](int s) { return bars + 8u * (2 * kStages + 2 + s); };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { barrier_init(full(s), 1); barrier_init(empty(s), 1); }
    for (int s = 0; s < 2; ++s) { barrier_init(sums_full(s), 1); barrier_init(sums_empty(s), 2 * kEpilogueWarps); }
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

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool going = true;
      Tile t;
      for (unsigned i = 0; going && tile_at<BACKWARD>(p, pair, pairs, i, &t); ++i) {
        const int half_n = p.n[t.problem] / 2, kb = p.k_blocks[t.problem];
        const int b_boxes = BACKWARD ? (half_n + 63) / 64 : 0;
        const uint32_t bytes = kHalfTile + (BACKWARD ? (uint32_t)b_boxes * 8192u : (uint32_t)half_n * 128u);
        for (int k = 0; k < kb; ++k) {
          if (!barrier_wait(empty(stage), phase ^ 1, p.status)) { going = false; break; }
          const uint32_t bar = in_first_cta(full(stage));
          if (rank == 0) barrier_expect(full(stage), 2 * bytes);
          const uint32_t to_a = base + (uint32_t)stage * 2 * kHalfTile, to_b = to_a + kHalfTile;
          if constexpr (!BACKWARD) {
            load_box(to_a, &p.a[0], k * kDeep, t.m0 + (int)rank * 128, bar);
            load_box(to_b, &p.b[rank], k * kDeep, t.n0, bar);
          } else if (t.problem == 0) {
            const int z = 2 * k >= kb, k0 = (z ? k - kb / 2 : k) * kDeep;
            load_box(to_a, &p.a[z], k0, t.m0 + (int)rank * 128, bar);
            load_box(to_a + 8192, &p.a[z], k0, t.m0 + (int)rank * 128 + 64, bar);
            for (int j = 0; j < b_boxes; ++j) load_box(to_b + j * 8192, &p.b[z], t.n0 + (int)rank * half_n + j * 64, k0, bar);
          } else {
            load_box(to_a, &p.a2[t.z], t.m0 + (int)rank * 128, k * kDeep, bar);
            load_box(to_a + 8192, &p.a2[t.z], t.m0 + (int)rank * 128 + 64, k * kDeep, bar);
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
      for (unsigned i = 0; going && tile_at<BACKWARD>(p, pair, pairs, i, &t); ++i) {
        const bool a_across = BACKWARD && t.problem == 1, b_across = BACKWARD;
        // binary32 sums (bit 4), operand types, which operands run across, N / 8, M / 16
        const uint32_t what = (1u << 4) | (p.format << 7) | (p.format << 10) | ((uint32_t)a_across << 15) | ((uint32_t)b_across << 16) |
                              ((uint32_t)(p.n[t.problem] >> 3) << 17) | (16u << 24);
        // 16 deep: 32 bytes along a row, or sixteen rows
        const uint32_t step_a = a_across ? 2048 >> 4 : 32 >> 4, step_b = b_across ? 2048 >> 4 : 32 >> 4;
        if (!barrier_wait(sums_empty(acc), acc_phase ^ 1, p.status)) break;
        fence_after();
        const uint32_t sums = tensor + (uint32_t)acc * 256u;
        const int kb = p.k_blocks[t.problem];
        for (int k = 0; k < kb; ++k) {
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
  } else if (warp >= 4) {
    const int quarter = warp & 3, turn = (warp - 4) / 4;
    const uint32_t out_buf = out_base + (uint32_t)(warp - 4) * kOutBuffers * kOutBytes;
    int acc = 0, buffer = 0;
    uint32_t acc_phase = 0;
    // 32 rows x 32 columns of binary32, rounded, to the output at (x, y); each lane holds a row
    auto store = [&](const CUtensorMap* map, const float (&v)[32], int x, int y) {
      if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kOutBuffers - 1) : "memory");
      __syncwarp();
      const uint32_t to = out_buf + (uint32_t)buffer * kOutBytes;
#pragma unroll
      for (int j = 0; j < 4; ++j) {                       // 64-byte rows, their 16-byte pieces swizzled over four rows' worth
        const uint32_t at = to + (uint32_t)lane * 64u + (uint32_t)((j ^ ((lane >> 1) & 3)) * 16);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(Num<T>::close(v[8 * j], v[8 * j + 1])),
                     "r"(Num<T>::close(v[8 * j + 2], v[8 * j + 3])), "r"(Num<T>::close(v[8 * j + 4], v[8 * j + 5])),
                     "r"(Num<T>::close(v[8 * j + 6], v[8 * j + 7]))
                     : "memory");
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) store_box(map, x, y, to);
      buffer ^= 1;
    };
    Tile t;
    for (unsigned i = 0; tile_at<BACKWARD>(p, pair, pairs, i, &t); ++i) {
      if (!barrier_wait(sums_full(acc), acc_phase, p.status)) break;
      fence_after();
      const uint32_t sums = tensor + (uint32_t)acc * 256u + ((uint32_t)quarter << 21);
      const int width = BACKWARD ? p.n[t.problem] : p.n[0] / 2;
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
          if (lane == 0) barrier_arrive_remote(in_first_cta(sums_empty(acc)));
        }
        if (!rows_there || t.n0 + c >= p.cols[t.problem]) continue;
        float v[32];
        if constexpr (BACKWARD) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
          store(&p.out[t.problem + t.z], v, t.n0 + c, y);
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float act, dact;
            activation<ACT>(__uint_as_float(r[j]), &act, &dact);
            v[j] = act * __uint_as_float(q[j]);
          }
          store(&p.out[0], v, t.n0 + c, y);
          if (p.save) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
            store(&p.out[1], v, t.n0 + c, y);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(q[j]);
            store(&p.out[2], v, t.n0 + c, y);
          }
        }
      }
      if (turn * kChunk >= width) {                       // a narrow tile: nothing here for this warp
        if (lane == 0) barrier_arrive_remote(in_first_cta(sums_empty(acc)));
      }
      acc ^= 1;
      if (!acc) acc_phase ^= 1;
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  pair_sync();                                // no CTA leaves while the other may still signal it or use its memory
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tensor), "r"(kColumns) : "memory");
}

// dg and du to the workspace, eight elements per thread
template <typename T, int ACT>
__global__ void __launch_bounds__(256) ffn_dgu_kernel(const FfnGradArgs a) {
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

// ---- host --------------------------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

cudaError_t encoder(EncodeTiled* out) {
  static EncodeTiled fn = nullptr;            // the same address for every thread that finds it
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !p) return cudaErrorNotSupported;
    fn = reinterpret_cast<EncodeTiled>(p);
  }
  *out = fn;
  return cudaSuccess;
}

struct Maps {
  EncodeTiled fn = nullptr;
  cudaError_t error = cudaSuccess;
  Maps() { error = encoder(&fn); }
  // T[rows][ld], `cols` of a row, in boxes of box_cols x box_rows
  template <typename T>
  void set(CUtensorMap* m, const void* p, long long rows, long long cols, long long ld, int box_cols, int box_rows) {
    if (error != cudaSuccess) return;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, one[2] = {1, 1};
    const CUresult r = fn(m, Num<T>::kMap, 2, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          box_cols * 2 == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) error = cudaErrorInvalidValue;
  }
};

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// The rounds of a grid of `tiles` on `pairs`, each of `kb` stages of n columns: a stage's products take 2 n cycles, an
// epilogue that nothing hides (the last one) about 16 n, filling and draining the pipeline about 1500.
long long cost(long long tiles, int pairs, int kb, int n) { return ((tiles + pairs - 1) / pairs) * (long long)kb * 2 * n + 16 * n + 1500; }

template <typename Kernel>
cudaError_t launch(Kernel kernel, const Products& p, int pairs, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes);
  if (e != cudaSuccess) return e;
  kernel<<<2 * pairs, kFfnThreads, kSharedBytes, s>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t run(const FfnArgs& a, cudaStream_t s) {
  const int pairs = a.sms / 2 < kMaxPairs ? a.sms / 2 : kMaxPairs;
  Products p{};
  p.m_tiles[0] = ceil_div(a.rows, 256);
  p.k_blocks[0] = ceil_div(a.hidden, kDeep);
  int best = 0;
  for (int f = 128; f >= 32; f -= 32) {
    const long long c = cost((long long)p.m_tiles[0] * ceil_div(a.inner, f), pairs, p.k_blocks[0], 2 * f);
    if (!best || c < cost((long long)p.m_tiles[0] * ceil_div(a.inner, best), pairs, p.k_blocks[0], 2 * best)) best = f;
  }
  p.n[0] = 2 * best;
  p.n_tiles[0] = ceil_div(a.inner, best);
  p.rows[0] = (int)a.rows;
  p.cols[0] = a.inner;
  p.save = a.g != nullptr;
  p.format = Num<T>::kFormat;
  p.status = a.status;
  Maps maps;
  maps.set<T>(&p.a[0], a.x, a.rows, a.hidden, a.ldx, kDeep, 128);
  maps.set<T>(&p.b[0], a.wg, a.inner, a.hidden, a.ldw, kDeep, best);
  maps.set<T>(&p.b[1], a.wu, a.inner, a.hidden, a.ldw, kDeep, best);
  maps.set<T>(&p.out[0], a.h, a.rows, a.inner, a.ldh, kChunk, 32);
  if (p.save) {
    maps.set<T>(&p.out[1], a.g, a.rows, a.inner, a.ldgu, kChunk, 32);
    maps.set<T>(&p.out[2], a.u, a.rows, a.inner, a.ldgu, kChunk, 32);
  }
  if (maps.error != cudaSuccess) return maps.error;
  const long long tiles = (long long)p.m_tiles[0] * p.n_tiles[0];
  const int used = tiles < pairs ? (int)tiles : pairs;
  if (a.act == AQ_ACT_SILU) return launch(products_kernel<T, AQ_ACT_SILU, false>, p, used, s);
  if (a.act == AQ_ACT_GELU) return launch(products_kernel<T, AQ_ACT_GELU, false>, p, used, s);
  return launch(products_kernel<T, AQ_ACT_GELU_TANH, false>, p, used, s);
}

// Tiles of two problems, of different lengths, over the pairs: the first problem's evenly, then the second's one round at
// a time to whichever pairs (those with a tile more of the first, or those with one less) are less loaded.
void share(Products* p, long long tiles0, long long tiles1, int pairs) {
  const long long c0 = (long long)p->k_blocks[0] * p->n[0], c1 = (long long)p->k_blocks[1] * p->n[1];
  const int more = (int)(tiles0 % pairs);                        // pairs 0..more-1 have one more
  const long long base = tiles0 / pairs;
  long long load[2] = {(base + 1) * c0, base * c0}, count[2] = {more, pairs - more}, got[2] = {0, 0}, rest[2] = {0, 0}, left = tiles1;
  while (left > 0) {
    const int to = count[0] && (!count[1] || load[0] + c1 <= load[1] + c1) && load[0] <= load[1] ? 0 : count[1] ? 1 : 0;
    if (left >= count[to]) {
      ++got[to];
      left -= count[to];
      load[to] += c1;
    } else {
      rest[to] = left;
      left = 0;
    }
  }
  uint32_t at0 = 0, at1 = 0;
  for (int i = 0; i < pairs; ++i) {
    const int cls = i < more ? 0 : 1, in = i < more ? i : i - more;
    p->first[0][i] = at0;
    p->first[1][i] = at1;
    at0 += (uint32_t)(base + (cls == 0));
    at1 += (uint32_t)(got[cls] + (in < rest[cls]));
  }
  p->first[0][pairs] = at0;
  p->first[1][pairs] = at1;
}

template <typename T>
cudaError_t run_grad(const FfnGradArgs& a, cudaStream_t s) {
  const long long vectors = a.rows * (a.inner / 8), want = (vectors + 255) / 256, most = 16ll * a.sms;
  const unsigned ctas = (unsigned)(want < most ? want : most);
  if (a.act == AQ_ACT_SILU) ffn_dgu_kernel<T, AQ_ACT_SILU><<<ctas, 256, 0, s>>>(a);
  else if (a.act == AQ_ACT_GELU) ffn_dgu_kernel<T, AQ_ACT_GELU><<<ctas, 256, 0, s>>>(a);
  else ffn_dgu_kernel<T, AQ_ACT_GELU_TANH><<<ctas, 256, 0, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int pairs = a.sms / 2 < kMaxPairs ? a.sms / 2 : kMaxPairs;
  Products p{};
  Maps maps;
  p.format = Num<T>::kFormat;
  p.status = a.status;
  p.m_tiles[0] = ceil_div(a.rows, 256);
  p.k_blocks[0] = 2 * ceil_div(a.inner, kDeep);
  p.m_tiles[1] = ceil_div(a.inner, 256);
  p.k_blocks[1] = ceil_div(a.rows, kDeep);
  const long long m0 = a.dx ? p.m_tiles[0] : 0, m1 = a.dwg ? 2 * p.m_tiles[1] : 0;
  long long best = -1;
  for (int n = 256; n >= 64; n -= 32) {
    const int nt = ceil_div(a.hidden, n);
    // the work of all tiles over the pairs, and one shorter tile that the last round leaves uneven
    const long long c0 = (long long)p.k_blocks[0] * 2 * n, c1 = (long long)p.k_blocks[1] * 2 * n;
    const long long whole = (m0 * nt * c0 + m1 * nt * c1) / pairs, uneven = m0 && m1 ? (c0 < c1 ? c0 : c1) / 2 : 0;
    const long long alone = m0 && !m1 ? cost(m0 * nt, pairs, p.k_blocks[0], n) : m1 && !m0 ? cost(m1 * nt, pairs, p.k_blocks[1], n) : 0;
    const long long least = m0 ? c0 : c1;
    long long c = alone ? alone : whole + uneven + 16 * n;
    if (c < least) c = least;
    if (best < 0 || c < best) { best = c; p.n[0] = p.n[1] = n; }
  }
  p.n_tiles[0] = p.n_tiles[1] = ceil_div(a.hidden, p.n[0]);
  p.rows[0] = (int)a.rows;
  p.rows[1] = a.inner;
  p.cols[0] = p.cols[1] = a.hidden;
  maps.set<T>(&p.a[0], a.dg, a.rows, a.inner, a.inner, 64, 64);
  maps.set<T>(&p.a[1], a.du, a.rows, a.inner, a.inner, 64, 64);
  p.a2[0] = p.a[0];
  p.a2[1] = p.a[1];
  maps.set<T>(&p.b[0], a.wg, a.inner, a.hidden, a.ldw, 64, 64);
  maps.set<T>(&p.b[1], a.wu, a.inner, a.hidden, a.ldw, 64, 64);
  maps.set<T>(&p.b2, a.x, a.rows, a.hidden, a.ldx, 64, 64);
  if (a.dx) maps.set<T>(&p.out[0], a.dx, a.rows, a.hidden, a.lddx, kChunk, 32);
  if (a.dwg) {
    maps.set<T>(&p.out[1], a.dwg, a.inner, a.hidden, a.lddw, kChunk, 32);
    maps.set<T>(&p.out[2], a.dwu, a.inner, a.hidden, a.lddw, kChunk, 32);
  }
  if (maps.error != cudaSuccess) return maps.error;
  const long long tiles0 = m0 * p.n_tiles[0], tiles1 = m1 * p.n_tiles[1];
  const int used = tiles0 + tiles1 < pairs ? (int)(tiles0 + tiles1) : pairs;
  share(&p, tiles0, tiles1, used);
  return launch(products_kernel<T, AQ_ACT_SILU, true>, p, used, s);
}

}  // namespace

cudaError_t launch_ffn(int dtype, const FfnArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run<__half>(a, s) : run<__nv_bfloat16>(a, s);
}
cudaError_t launch_ffn_grad(int dtype, const FfnGradArgs& a, cudaStream_t s) {
  return dtype == AQ_FP16 ? run_grad<__half>(a, s) : run_grad<__nv_bfloat16>(a, s);
}

}  // namespace aq
