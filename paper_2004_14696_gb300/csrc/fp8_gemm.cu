// Products of 8-bit operands with a scale for each block of 128, on the tensor cores.
//
//   out[g][m, n] = sum_kb sa[m, kb] sb[n, kb] sum_{k in block kb} a[m, k] b[n, k]
//
// a and b are e4m3, K-major.  The inner sum of 128 products is tcgen05.mma's, in fp32 in tensor
// memory; its two scales are no powers of two, so the outer sum cannot stay there: epilogue
// warps read every 128-deep partial tile back, scale it and add it into fp32 registers, while
// the next one runs into a second buffer.
//
// Two kernels: tiles of one CTA for few rows or few tiles, pairs of CTAs for large products.
//
// Measured: 8192 x 4096 x 4096 107 us (2,570 TFLOP/s; bound by the scaled sums, MMAs and loads alone take 84), with b's
// scales per row 154; 128 weight gradients of 1024 x 1024 x 128 to fp32 91.5 (6.2 TB/s of writes); a single row by
// 4096 x 4096 6.5 and 1003 x 1000 x 1622 8.7, the chain of a launch, loads, products and their join.
//
// Every wait on an mbarrier is bounded (2 s).  One that runs out sets bit 0 of *status and ends its warp's loop; the
// others' waits run out in turn.  Then the MMAs issued are waited for, and the loads, each of these waits
// bounded again, tensor memory is freed and the CTA returns.
#include "elements.cuh"
#include "gemm_tc.cuh"
#include "tc_ptx.cuh"

namespace dbw {

namespace {

using namespace tcx;

constexpr int BM = 128, BK = 128;    // a K block is a block of scales and a 128-byte row

// acc[j] += r[j] * (f * scales[j])  (F: with the factor f, else without), j < N; scales in shared memory, 16-byte aligned.
template <bool F, int N>
__device__ __forceinline__ void add_scaled(float* acc, const uint32_t* r, float f, const float* scales) {
    const uint64_t f2 = pack_f32x2(f, f);
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        float s[4];
        if constexpr (F) {
            const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(scales + j);
            unpack_f32x2(mul_f32x2(f2, v.x), s[0], s[1]);
            unpack_f32x2(mul_f32x2(f2, v.y), s[2], s[3]);
        } else {
            const float4 v = *reinterpret_cast<const float4*>(scales + j);
            s[0] = v.x, s[1] = v.y, s[2] = v.z, s[3] = v.w;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[j + u] = fmaf(u2f(r[j + u]), s[u], acc[j + u]);
    }
}
// A wait of a whole warp: every lane's, or none's.  CLUSTER: on what the pair's other CTA does as well.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint64_t limit_ns) {
    return __all_sync(0xffffffffu, mbar_sleep<CLUSTER>(bar, parity, limit_ns)) != 0;
}

struct Fp8Args {
    CUtensorMap tmA, tmB, tmOut;
    int tma_out;                     // out leaves through tmOut
    const float *sa, *sb;
    void* out;
    int64_t ldsa, ldsb, ldo, out_stride;
    int M, N, K, groups, blocks;     // K of one group
    int mt, nt, nk;                  // tiles, K blocks of a group
    int tile_bytes;                  // one CTA per tile: of a stage's loads
    int* status;
    uint64_t wait_ns;                // bound of every wait
    int64_t skip;                    // the first tile's stage that stays without its loads (tests of the waits); -1: none
};

// Keeps what reads r behind the tcgen05.wait that stands before.
template <int N>
__device__ __forceinline__ void tie(uint32_t (&r)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+r"(r[j]));
}

// ------------------------------------------------------------------ one CTA per tile
// Few rows of a (single tokens, ragged batches) or few tiles: a CTA takes 128 rows of b and BT rows of a,
// with b as the MMA's M, so that a single token costs one read of b's rows and 16 columns of
// the MMA; a cluster of up to 8 CTAs splits the K blocks of a tile, and each adds and writes its
// share of the tile's rows of a, in the order of the ranks.  A lane of the epilogue is a row of
// b, a column of out: a warp writes neighbouring entries.
//
// Warps: 0 TMA producer, 1 MMA issuer and TMEM owner, from 2 on epilogue: warp w reads lane quarter w % 4, and
// rows of a 64 ((w - 2) / 4) .. + 63.  Tensor memory holds four partial tiles.  The scales of 8 K blocks
// are brought at a time, the next ones while these are worked on.
template <int BT, bool BLOCKS>
struct TileCfg {
    static constexpr int EPI_WARPS = BT > 64 ? 8 : 4;
    static constexpr int THREADS = 64 + 32 * EPI_WARPS;
    static constexpr int COLS = BT > 64 ? 64 : BT;      // rows of a per epilogue thread
    static constexpr int NB = 4;
    // two CTAs share an SM up to BT = 64; the loads of three stages are enough (two: the same times)
    static constexpr int STAGES = BT == 16 ? 5 : BT == 32 ? 4 : BT == 64 && !BLOCKS ? 2 : 3;
    static constexpr int B_BYTES = BM * BK, A_BYTES = BT * BK;
    static constexpr int KC = 8;                        // K blocks of scales
    // of a K block: the rows of a (times b's scale where it is one for all 128), then of b (where each has its own)
    static constexpr int ROW = BT + (BLOCKS ? 0 : BM);
    static constexpr int SCALES = KC * ROW;             // per chunk, two chunks
    static constexpr int PER_THREAD = SCALES / (32 * EPI_WARPS);
    static constexpr int BASE = STAGES * (A_BYTES + B_BYTES) + 256 + 1024;   // and 2 * SCALES floats that are static
    static constexpr int JOIN = BT * BM * 4;            // the cluster's partial sums of this CTA's rows
    static_assert(SCALES % (32 * EPI_WARPS) == 0 && NB * BT >= 32, "tile shape");
};

template <int COLS>
__device__ __forceinline__ void load_cols(uint32_t t, uint32_t (&r)[COLS]) {
    if constexpr (COLS == 16) {
        tc_ld_16cols(t, r);
    } else {
#pragma unroll
        for (int c = 0; c < COLS / 32; ++c) tc_ld_32cols(t + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(r + 32 * c));
    }
}

template <class T, int BT, bool BLOCKS>
__global__ void __launch_bounds__(TileCfg<BT, BLOCKS>::THREADS, BT > 64 ? 1 : 2)
    fp8_tile_kernel(const __grid_constant__ Fp8Args a) {
    grid_begin();
    using Cfg = TileCfg<BT, BLOCKS>;
    constexpr int STAGES = Cfg::STAGES, NB = Cfg::NB, COLS = Cfg::COLS, KC = Cfg::KC;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sB = smem;
    uint8_t* sA = smem + STAGES * Cfg::B_BYTES;
    __shared__ __align__(16) float scales[2 * Cfg::SCALES];   // [2][KC][ROW]
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + STAGES * (Cfg::A_BYTES + Cfg::B_BYTES));
    uint64_t* empty_bar = full_bar + STAGES;
    uint64_t* tfull_bar = empty_bar + STAGES;     // [NB] partial tile ready
    uint64_t* tempty_bar = tfull_bar + NB;        // [NB] read back by the epilogue warps
    uint64_t* done_bar = tempty_bar + NB;         // every MMA issued has completed
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done_bar + 1);
    int* abort_flag = reinterpret_cast<int*>(tmem_slot + 1);
    float* join = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(full_bar) + 256);   // [rank][row of a][128]
    volatile int* vabort = abort_flag;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int split = static_cast<int>(cluster_size()), rank = split > 1 ? static_cast<int>(cluster_rank()) : 0;
    const int tile = blockIdx.x / split, g = tile / (a.mt * a.nt), rem = tile % (a.mt * a.nt);
    const int m0 = rem / a.nt * BT, n0 = rem % a.nt * BM;
    const int kb0 = static_cast<int>(static_cast<int64_t>(a.nk) * rank / split);
    const int nk = static_cast<int>(static_cast<int64_t>(a.nk) * (rank + 1) / split) - kb0;

    // stage s of K block i: the caller has found it empty
    auto load_stage = [&](int i) {
        const int s = i % STAGES, k = (g * a.nk + kb0 + i) * BK;
        if (i == a.skip && blockIdx.x == 0) return;
        mbar_expect_tx(smem_u32(full_bar + s), a.tile_bytes);
        tma_load_2d(smem_u32(sB + s * Cfg::B_BYTES), &a.tmB, k, n0, smem_u32(full_bar + s));
        tma_load_2d(smem_u32(sA + s * Cfg::A_BYTES), &a.tmA, k, m0, smem_u32(full_bar + s));
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(full_bar + s), 1);
            mbar_init(smem_u32(empty_bar + s), 1);
        }
        for (int b = 0; b < NB; ++b) {
            mbar_init(smem_u32(tfull_bar + b), 1);
            mbar_init(smem_u32(tempty_bar + b), Cfg::EPI_WARPS);
        }
        mbar_init(smem_u32(done_bar), 1);
        *abort_flag = 0;
        fence_mbar_init();
        // the first loads do not wait for the others
        for (int i = 0; i < STAGES && i < nk; ++i) load_stage(i);
    }
    if (warp == 1) {
        tc_alloc(smem_u32(tmem_slot), NB * BT);
        tc_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    if (split > 1) cluster_arrive();   // this CTA runs: its join buffer may be written

    int issued = nk < STAGES ? nk : STAGES;    // warp 0: stages loaded so far
    if (warp == 0) {
        for (int i = STAGES; i < nk && !*vabort; ++i) {
            if (!warp_wait(smem_u32(empty_bar + i % STAGES), (i / STAGES & 1) ^ 1, a.wait_ns)) {
                atomicOr(a.status, 1);
                *vabort = 1;
                break;
            }
            if (elect_one()) load_stage(i);
            __syncwarp();
            issued = i + 1;
        }
    } else if (warp == 1) {
        constexpr uint32_t idesc = instr_desc_e4m3(BM, BT);
        const uint64_t da = smem_desc(smem_u32(sB), 128), db = smem_desc(smem_u32(sA), 128);   // + 16 bytes per 1
        for (int i = 0; i < nk; ++i) {
            const int s = i % STAGES, b = i % NB;
            if (!warp_wait(smem_u32(full_bar + s), i / STAGES & 1, a.wait_ns) ||
                !warp_wait(smem_u32(tempty_bar + b), (i / NB & 1) ^ 1, a.wait_ns)) {
                atomicOr(a.status, 1);
                *vabort = 1;
                break;
            }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t d0 = da + s * (Cfg::B_BYTES / 16), d1 = db + s * (Cfg::A_BYTES / 16);
#pragma unroll
                for (int kk = 0; kk < BK / 32; ++kk)   // columns past K are zero
                    tc_mma_f8(tmem + b * BT, d0 + 2 * kk, d1 + 2 * kk, idesc, kk > 0);
                tc_commit(smem_u32(tfull_bar + b));
                tc_commit(smem_u32(empty_bar + s));
            }
            __syncwarp();
        }
        if (elect_one()) tc_commit(smem_u32(done_bar));   // after an abort: nothing may read the stages or tensor memory any more
        __syncwarp();
        if (!warp_wait(smem_u32(done_bar), 0, a.wait_ns)) atomicOr(a.status, 1);
    } else if (warp >= 2) {
        const int q = warp & 3, h = (warp - 2) >> 2, tid = threadIdx.x - 64;
        const int n = n0 + 32 * q + lane;
        const int64_t kg = static_cast<int64_t>(g) * a.nk + kb0;
        // entry e of a chunk: K block e / ROW, row e % ROW.  Two factors, multiplied when they are needed, so that
        // nothing waits for the loads
        float next[Cfg::PER_THREAD], times[Cfg::PER_THREAD];
        auto load_scales = [&](int first) {
#pragma unroll
            for (int u = 0; u < Cfg::PER_THREAD; ++u) {
                const int e = tid + u * 32 * Cfg::EPI_WARPS, kb = first + e / Cfg::ROW, c = e % Cfg::ROW;
                next[u] = 0.f;
                if (BLOCKS) times[u] = 0.f;
                if (kb >= nk) continue;
                if (c < BT) {
                    if (m0 + c < a.M) next[u] = __ldg(a.sa + (kg + kb) * a.ldsa + m0 + c);
                    if (BLOCKS) times[u] = __ldg(a.sb + (n0 >> 7) * a.ldsb + kg + kb);
                } else if (n0 + c - BT < a.N) {
                    next[u] = __ldg(a.sb + (kg + kb) * a.ldsb + n0 + c - BT);
                }
            }
        };
        load_scales(0);
        float x[COLS];
#pragma unroll
        for (int j = 0; j < COLS; ++j) x[j] = 0.f;
        bool ok = true;
        for (int i = 0; i < nk; ++i) {
            float* chunk = scales + (i / KC & 1) * Cfg::SCALES;
            if (i % KC == 0) {
#pragma unroll
                for (int u = 0; u < Cfg::PER_THREAD; ++u) 
                    chunk[tid + u * 32 * Cfg::EPI_WARPS] = BLOCKS ? next[u] * times[u] : next[u];
                asm volatile("bar.sync 1, %0;" ::"n"(32 * Cfg::EPI_WARPS) : "memory");
                load_scales(i + KC);
            }
            const float* sk = chunk + i % KC * Cfg::ROW;
            const float sb = BLOCKS ? 1.f : sk[BT + 32 * q + lane];
            const int b = i % NB;
            if (ok && !warp_wait(smem_u32(tfull_bar + b), i / NB & 1, a.wait_ns)) {
                ok = false;   // as a warp; its part in the barriers goes on
                atomicOr(a.status, 1);
                *vabort = 1;
            }
            tc_fence_after();
            uint32_t r[COLS];
            load_cols(tmem + b * BT + h * COLS + (static_cast<uint32_t>(32 * q) << 16), r);
            tc_wait_ld();
            tie(r);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(tempty_bar + b));
            add_scaled<!BLOCKS, COLS>(x, r, sb, sk + h * COLS);
        }
        T* out = static_cast<T*>(a.out) + g * a.out_stride + static_cast<int64_t>(m0) * a.ldo + n;
        if (split == 1) {
            if (n < a.N) {
#pragma unroll
                for (int j = 0; j < COLS; ++j)
                    if (m0 + h * COLS + j < a.M) put(out + (h * COLS + j) * a.ldo, x[j]);
            }
        } else {
            // row j of a goes to rank j / share, as its piece of this rank
            const int share = BT / split, log_share = 31 - __clz(share);
            cluster_wait();
#pragma unroll
            for (int j = 0; j < COLS; ++j) {
                const int row = h * COLS + j;
                const uint32_t at = smem_u32(join + (rank * share + (row & (share - 1))) * BM + 32 * q + lane);
                store_remote(map_to_rank(at, row >> log_share), x[j]);
            }
            cluster_arrive();
            cluster_wait();
            // eight rows at a time, so that a rank's pieces are on their way together
            const uint32_t mine = smem_u32(join + 32 * q + lane);
            for (int row = 8 * h; row < share; row += 8 * (Cfg::EPI_WARPS / 4)) {
                float s[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) s[u] = 0.f;
                for (int r = 0; r < split; ++r)
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (row + u < share) s[u] += lds(mine + ((r * share + row + u) * BM) * 4);
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int m = rank * share + row + u;
                    if (row + u < share && m0 + m < a.M && n < a.N) put(out + m * a.ldo, s[u]);
                }
            }
        }
    }
    if (split > 1 && warp < 2) {
        cluster_wait();
        cluster_arrive();
        cluster_wait();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0 && *vabort)     // loads that no MMA has waited for
        for (int i = issued < STAGES ? 0 : issued - STAGES; i < issued; ++i)
            warp_wait(smem_u32(full_bar + i % STAGES), i / STAGES & 1, a.wait_ns);
    if (warp == 1) {
        tc_fence_after();
        tc_dealloc(tmem, NB * BT);
    }
}

template <class T, int BT, bool BLOCKS>
cudaError_t launch_fp8_tile(Fp8Args& p, int split, const uint8_t* a, int64_t lda, const uint8_t* b, int64_t ldb,
                            cudaStream_t st) {
    using Cfg = TileCfg<BT, BLOCKS>;
    const int64_t cols = static_cast<int64_t>(p.groups) * p.K;
    // Boxes of no more rows than there are: rows outside cost more than rows inside (7790 x 33 x 1222 14.0 us against 7.8).
    // The stage's other rows stay as they are; what the MMA makes of them is not written.
    const int rows_a = p.M < BT ? p.M : BT, rows_b = p.N < BM ? p.N : BM;
    if (!tc_make_map_u8(&p.tmA, a, p.M, cols, lda, rows_a) || !tc_make_map_u8(&p.tmB, b, p.N, cols, ldb, rows_b))
        return cudaErrorInvalidValue;
    p.tile_bytes = (rows_a + rows_b) * BK;
    p.mt = (p.M + BT - 1) / BT;
    p.nt = (p.N + BM - 1) / BM;
    const int64_t ctas = static_cast<int64_t>(p.mt) * p.nt * p.groups * split;
    auto kern = fp8_tile_kernel<T, BT, BLOCKS>;
    const cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::BASE + Cfg::JOIN);
    if (err != cudaSuccess) return err;
    launch_clusters(split, kern, static_cast<unsigned>(ctas), Cfg::THREADS, Cfg::BASE + (split > 1 ? Cfg::JOIN : 0), st, p);
    return cudaGetLastError();
}

// ------------------------------------------------------------------ CTA pairs
// Large products: two-CTA clusters that take 256 x 256 output tiles one after another, of a grid of as many as run at a
// time or, ASK, of clusters that have not been launched yet.  CTA r stages rows 128 r .. + 127 of the tile's a and b;
// the even CTA's MMA warp reads both CTAs' stages and leaves output rows 128 r .. in CTA r's tensor memory, 256
// columns, two buffers.  A K block is 512 cycles of MMA; in that time 8 epilogue warps read 128 x 256 partial sums back
// and add them, 128 a thread: thread = one row, 128 columns, so that a's scale is the thread's and b's, where it is one
// per block, the warp's.
//
// Twelve warps: 0 TMA producer and TMEM owner, 1 MMA issuer, 2 and 3 bring a's and b's scales of eight K blocks at a time
// to shared memory, 4-11 epilogue: warp w reads lane quarter w % 4, column half (w - 4) / 4.  (An epilogue warp's wait
// for its reads of tensor memory is a wait for its loads from global memory too: with the scales loaded by these warps,
// even four K blocks ahead, 8192 x 4096 x 4096 took 15 us longer.)  The first four give registers to the others
// (40 x 128 + 232 x 256 = 168 x 384).
constexpr int kPairThreads = 384;
constexpr int PN = 256;
constexpr int kPairStages = 4;
constexpr int HALF_BYTES = BM * BK;         // a CTA's rows of a, and of b, in a stage
// Answers to ask_cluster that there is room for.  A cluster asks for the tile after the one whose loads it begins; its other
// warps are then at most the stages and the two accumulators behind, 7 tiles of one K block, so that an answer's place
// has been read by all of them before the next one comes to it.
constexpr int kAsked = 16;
constexpr int kChunk = 8, kChunks = 2;      // K blocks of scales at a time, and how many such chunks there is room for
// Floats of a K block's scales: a's 128 rows, and b's 256 rows or two blocks.
__host__ __device__ constexpr int pair_scales(bool blocks) { return BM + (blocks ? 4 : PN); }
// an epilogue warp's outputs on their way: two boxes of 32 rows x 128 bytes, or 32 rows of 17 pieces of 16 bytes
constexpr int kPiecePitch = 17 * 16;
constexpr int kWarpBoxes = 2 * 32 * 128, kWarpOut = 32 * kPiecePitch;
constexpr int kPairSmem = kPairStages * 2 * HALF_BYTES + 8 * kWarpOut + 256 + 1024;   // and the scales, which are static
static_assert(kPairSmem + kChunks * kChunk * pair_scales(false) * 4 + 24 * kAsked <= 227 * 1024, "shared memory");

__device__ __forceinline__ void fp8_pair_tile(const Fp8Args& a, int t, int& g, int& m, int& n) {
    g = t / (a.mt * a.nt);
    const int rem = t % (a.mt * a.nt);
    m = rem / a.nt;
    n = rem % a.nt;
}

// A warp's 32 rows x 128 columns (one row per lane) to out by way of its shared memory, in boxes of 128 bytes a row;
// 16-byte pieces lie where the 128-byte swizzle puts them, so that a quarter warp's are in different banks.  The
// copies go on while the next tile is computed: with the stores issued by the warps themselves, all SMs at the
// same time, a tile of 32 K blocks took 5,000 cycles longer.
template <class T>
__device__ __forceinline__ void fill_box(uint32_t box, int lane, const float* x) {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        uint4 w;
        if constexpr (sizeof(T) == 2) {
            const float* v = x + 8 * p;
            w = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        } else {
            const float* v = x + 4 * p;
            w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
        sts4(box + lane * 128 + ((p ^ (lane & 7)) << 4), w);
    }
}
// Where out's rows do not lie on 16 bytes: word i of a row (its lane's) that begins ``shift`` bytes behind a multiple of
// 16, counted from that multiple.  x: 256 bytes of a row's entries.
template <class T>
__device__ __forceinline__ uint32_t word_of(const float* x, int i) {
    if (i < 0 || i >= 64) return 0u;
    if constexpr (sizeof(T) == 2) return bf16_pair(x[2 * i], x[2 * i + 1]);
    else return __float_as_uint(x[i]);
}
template <class T>
__device__ __forceinline__ uint32_t shifted_word(const float* x, int i, uint32_t shift) {
    uint32_t v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        v[u] = word_of<T>(x, i - u);
        if constexpr (sizeof(T) == 2) v[u] = __funnelshift_l(word_of<T>(x, i - u - 1), v[u], (shift & 2) * 8);
    }
    const uint32_t even = shift & 4 ? v[1] : v[0], odd = shift & 4 ? v[3] : v[2];
    return shift & 8 ? odd : even;
}
// ``rows`` rows of ``bytes`` <= 256 bytes from ``to`` on, by way of shared memory in 16-byte pieces as memory has them:
// the whole ones two rows at a time, then every lane the ends of its row.  (Entries a lane each, 64 or 128 bytes of a row an
// instruction, leave every other sector in parts: 23 x 2710 x 653 x 128 to fp32 84 us against 53, 8000 x 1001 x 1024 to bf16
// 23.6 against 17.2.)
template <class T>
__device__ __forceinline__ void write_rows(T* to, int64_t ldo, uint32_t buf, int rows, int bytes, int lane, const float* x) {
    auto phase = [](const T* p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15; };
    __syncwarp();
    T* mine = to + lane * ldo;
    const uint32_t shift = phase(mine);
#pragma unroll
    for (int u = 0; u < 17; ++u)
        sts4(buf + lane * kPiecePitch + 16 * u,
             make_uint4(shifted_word<T>(x, 4 * u, shift), shifted_word<T>(x, 4 * u + 1, shift),
                        shifted_word<T>(x, 4 * u + 2, shift), shifted_word<T>(x, 4 * u + 3, shift)));
    __syncwarp();
    T* row = to + (lane >> 4) * ldo;
    const int u = lane & 15;
#pragma unroll 4
    for (int r = lane >> 4; r < rows; r += 2, row += 2 * ldo) {
        const int first = 16 * u - static_cast<int>(phase(row));
        if (first >= 0 && first + 16 <= bytes)
            *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(row) + first) = lds4(buf + r * kPiecePitch + 16 * u);
    }
    if (lane >= rows) return;
    const int end = static_cast<int>(shift) + bytes;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        if (!(side ? end & 15 : shift)) continue;
        const int piece = side ? end >> 4 : 0, first = 16 * piece - static_cast<int>(shift);
        const uint4 v = lds4(buf + lane * kPiecePitch + 16 * piece);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint8_t* p = reinterpret_cast<uint8_t*>(mine) + first + 4 * i;
            const int o = first + 4 * i;
            if constexpr (sizeof(T) == 2) {
                const bool lo = o >= 0 && o < bytes, hi = o >= -2 && o + 2 < bytes;
                if (lo && hi) *reinterpret_cast<uint32_t*>(p) = w[i];
                else if (lo) *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[i]);
                else if (hi) *reinterpret_cast<uint16_t*>(p + 2) = static_cast<uint16_t>(w[i] >> 16);
            } else if (o >= 0 && o < bytes) {
                *reinterpret_cast<uint32_t*>(p) = w[i];
            }
        }
    }
}
template <class T>
__device__ __forceinline__ void store_boxes(const Fp8Args& a, uint8_t* buf, int n0, int row0, int g, int lane,
                                            const float (&x)[128]) {
    constexpr int W = 128 / sizeof(T);   // columns of a box
    if (a.tma_out) {
#pragma unroll
        for (int c = 0; c < 128 / W; ++c) {
            if (lane == 0) bulk_wait_read<1>();   // the box that was here, before the last one
            __syncwarp();
            const uint32_t box = smem_u32(buf) + (c & 1) * (32 * 128);
            fill_box<T>(box, lane, x + W * c);
            fence_async_shared();
            __syncwarp();
            if (lane == 0) {
                if (row0 < a.M && n0 + W * c < a.N) tma_store_3d(&a.tmOut, box, n0 + W * c, row0, g);
                bulk_commit();
            }
        }
    } else {
        const int rows = a.M - row0 < 32 ? a.M - row0 : 32;
#pragma unroll
        for (int c = 0; c < 128; c += 2 * W) {
            const int n = n0 + c, cols = a.N - n < 2 * W ? a.N - n : 2 * W;
            if (cols > 0)
                write_rows(static_cast<T*>(a.out) + g * a.out_stride + row0 * a.ldo + n, a.ldo, smem_u32(buf), rows,
                           cols * static_cast<int>(sizeof(T)), lane, x + c);
        }
    }
}

// The scales of ``left`` K blocks, entries first .. + 32 J - 1 of each (zero from ``end`` on), to rows of ``row`` floats.
template <int J>
__device__ __forceinline__ void bring_scales(float* to, int row, const float* from, int64_t ld, int first, int end, int left,
                                             int lane) {
    constexpr int kTogether = 16 / J;
    for (int k = 0; k < left; k += kTogether) {
        float v[kTogether][J];
#pragma unroll
        for (int u = 0; u < kTogether; ++u)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int i = first + lane + 32 * j;
                v[u][j] = k + u < left && i < end ? __ldg(from + (k + u) * ld + i) : 0.f;
            }
#pragma unroll
        for (int u = 0; u < kTogether; ++u)
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (k + u < left) to[(k + u) * row + lane + 32 * j] = v[u][j];
    }
}

// a.mt, a.nt: tiles of 256 x 256
template <class T, bool BLOCKS, bool ASK>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
    fp8_pair_kernel(const __grid_constant__ Fp8Args a) {
    grid_begin();
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sA = smem;
    uint8_t* sB = smem + kPairStages * HALF_BYTES;
    uint8_t* sOut = smem + kPairStages * 2 * HALF_BYTES;
    constexpr int kScales = pair_scales(BLOCKS);
    __shared__ __align__(16) float scales[kChunks * kChunk * kScales];
    uint64_t* full_bar = reinterpret_cast<uint64_t*>(sOut + 8 * kWarpOut);
    uint64_t* empty_bar = full_bar + kPairStages;    // full: in the even CTA, of both CTAs' loads
    uint64_t* tfull_bar = empty_bar + kPairStages;   // [2] partial tile ready
    uint64_t* tempty_bar = tfull_bar + 2;            // [2] even CTA: read back by both CTAs' epilogue warps
    uint64_t* sfull_bar = tempty_bar + 2;            // [kChunks] a chunk of scales is there
    uint64_t* sempty_bar = sfull_bar + kChunks;      // [kChunks] the epilogue warps are through with it
    uint64_t* done_bar = sempty_bar + kChunks;       // every MMA issued has completed
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done_bar + 1);
    int* abort_flag = reinterpret_cast<int*>(tmem_slot + 1);
    volatile int* vabort = abort_flag;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_rank());
    __shared__ __align__(16) uint4 answers[ASK ? kAsked : 1];
    __shared__ uint64_t asked_bar[ASK ? kAsked : 1];
    const int npairs = gridDim.x >> 1, tiles = a.mt * a.nt * a.groups;
    // The cluster's j-th tile, the one after t, as every warp asks for it in turn; -1: none.
    auto tile_after = [&](int t, uint32_t j) {
        if constexpr (ASK) {
            const uint32_t s = (j - 1) % kAsked;
            if (warp_wait<true>(smem_u32(asked_bar + s), (j - 1) / kAsked & 1, a.wait_ns)) return asked_cluster(smem_u32(answers + s)) >> 1;
            atomicOr(a.status, 1);
            *vabort = 1;
            return -1;
        } else {
            return t + npairs < tiles ? t + npairs : -1;
        }
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(smem_u32(full_bar + s), 1);
            mbar_init(smem_u32(empty_bar + s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(tfull_bar + b), 1);
            mbar_init(smem_u32(tempty_bar + b), 16);
        }
        for (int c = 0; c < kChunks; ++c) {
            mbar_init(smem_u32(sfull_bar + c), 2);
            mbar_init(smem_u32(sempty_bar + c), 8);
        }
        mbar_init(smem_u32(done_bar), 1);
        if constexpr (ASK)
            for (int c = 0; c < kAsked; ++c) mbar_init(smem_u32(asked_bar + c), 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 0) {
        tc2_alloc(smem_u32(tmem_slot), 2 * PN);
        tc2_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    uint32_t loaded = 0;      // warp 0: stages loaded so far
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0) {
            uint32_t& it = loaded;
            const uint32_t full0 = map_to_rank(smem_u32(full_bar), 0);
            uint32_t j = 0;
            for (int t = blockIdx.x >> 1; t >= 0 && !*vabort; t = tile_after(t, ++j)) {
                if constexpr (ASK) {
                    if (elect_one()) {     // for the tile after this one
                        mbar_expect_tx(smem_u32(asked_bar + j % kAsked), 16);
                        if (rank == 0) ask_cluster(smem_u32(answers + j % kAsked), smem_u32(asked_bar + j % kAsked));
                    }
                    __syncwarp();
                }
                int g, m, n;
                fp8_pair_tile(a, t, g, m, n);
                for (int kb = 0; kb < a.nk; ++kb, ++it) {
                    const int s = it % kPairStages;
                    if (!warp_wait<true>(smem_u32(empty_bar + s), (it / kPairStages & 1) ^ 1, a.wait_ns)) {
                        atomicOr(a.status, 1);
                        *vabort = 1;
                        break;
                    }
                    if (!(it == a.skip && blockIdx.x < 2) && elect_one()) {
                        const int k = (g * a.nk + kb) * BK;
                        if (rank == 0) mbar_expect_tx(smem_u32(full_bar + s), 4 * HALF_BYTES);
                        tma_load_2d_pair(smem_u32(sA + s * HALF_BYTES), &a.tmA, k, (2 * m + rank) * BM, full0 + 8 * s);
                        tma_load_2d_pair(smem_u32(sB + s * HALF_BYTES), &a.tmB, k, n * PN + rank * (PN / 2), full0 + 8 * s);
                    }
                    __syncwarp();
                }
            }
            // the last use of every stage has been consumed: no load or commit is on its way any more
            if (!*vabort) {
                for (uint32_t q = it < kPairStages ? 0 : it - kPairStages; q < it; ++q)
                    if (!warp_wait<true>(smem_u32(empty_bar + q % kPairStages), q / kPairStages & 1, a.wait_ns)) {
                        atomicOr(a.status, 1);
                        *vabort = 1;
                        break;
                    }
            }
        } else if (warp == 1 && rank == 0) {
            constexpr uint32_t idesc = instr_desc_e4m3(2 * BM, PN);
            const uint64_t da = smem_desc(smem_u32(sA), 128), db = smem_desc(smem_u32(sB), 128);   // + 16 bytes per 1
            uint32_t it = 0, j = 0;
            for (int t = blockIdx.x >> 1; t >= 0 && !*vabort; t = tile_after(t, ++j)) {
                for (int kb = 0; kb < a.nk; ++kb, ++it) {
                    const int s = it % kPairStages, b = it & 1;
                    if (!warp_wait<true>(smem_u32(full_bar + s), it / kPairStages & 1, a.wait_ns) ||
                        !warp_wait<true>(smem_u32(tempty_bar + b), (it >> 1 & 1) ^ 1, a.wait_ns)) {
                        atomicOr(a.status, 1);
                        *vabort = 1;
                        break;
                    }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t d0 = da + s * (HALF_BYTES / 16), d1 = db + s * (HALF_BYTES / 16);
#pragma unroll
                        for (int kk = 0; kk < BK / 32; ++kk)
                            tc2_mma_f8(tmem + b * PN, d0 + 2 * kk, d1 + 2 * kk, idesc, kk > 0);
                        tc2_commit_multicast(smem_u32(tfull_bar + b), 0x3);
                        tc2_commit_multicast(smem_u32(empty_bar + s), 0x3);
                    }
                    __syncwarp();
                }
            }
            if (elect_one()) tc2_commit_multicast(smem_u32(done_bar), 0x3);
            __syncwarp();
        } else if (warp >= 2) {
            uint32_t ch = 0, j = 0;
            bool ok = true;
            for (int t = blockIdx.x >> 1; t >= 0; t = ok ? tile_after(t, ++j) : -1) {
                int g, m, n;
                fp8_pair_tile(a, t, g, m, n);
                for (int kb = 0; kb < a.nk; kb += kChunk, ++ch) {
                    ok = warp_wait(smem_u32(sempty_bar + ch % kChunks), (ch / kChunks & 1) ^ 1, a.wait_ns);
                    if (!ok) {
                        atomicOr(a.status, 1);
                        *vabort = 1;
                        break;
                    }
                    float* to = scales + ch % kChunks * kChunk * kScales;
                    const int64_t k0 = static_cast<int64_t>(g) * a.nk + kb;
                    const int left = a.nk - kb < kChunk ? a.nk - kb : kChunk;
                    if (warp == 2)
                        bring_scales<4>(to, kScales, a.sa + k0 * a.ldsa, a.ldsa, (2 * m + rank) * BM, a.M, left, lane);
                    else if (!BLOCKS)
                        bring_scales<8>(to + BM, kScales, a.sb + k0 * a.ldsb, a.ldsb, n * PN, a.N, left, lane);
                    else if (lane < 2 * kChunk && lane % kChunk < left)   // of the tile's two blocks
                        to[lane % kChunk * kScales + BM + lane / kChunk] =
                            n * PN + 128 * (lane / kChunk) < a.N
                                ? __ldg(a.sb + (2 * n + lane / kChunk) * a.ldsb + k0 + lane % kChunk)
                                : 0.f;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(sfull_bar + ch % kChunks));
                }
            }
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int q = warp & 3, h = (warp - 4) >> 2;
        const uint32_t tempty0 = map_to_rank(smem_u32(tempty_bar), 0);
        uint32_t ch = 0;
        const uint32_t tcol = tmem + h * 128 + (static_cast<uint32_t>(32 * q) << 16);
        uint32_t it = 0, j = 0;
        for (int t = blockIdx.x >> 1; t >= 0; t = tile_after(t, ++j)) {
            int g, m, n;
            fp8_pair_tile(a, t, g, m, n);
            const int row = (2 * m + rank) * BM + 32 * q + lane, n0 = n * PN + 128 * h;
            float acc[128];
#pragma unroll
            for (int j = 0; j < 128; ++j) acc[j] = 0.f;
            uint32_t r[2][32];
            // The partial tile of K block ``i`` is complete.
            auto ready = [&](uint32_t i) {
                const bool got = warp_wait<true>(smem_u32(tfull_bar + (i & 1)), i >> 1 & 1, a.wait_ns);
                if (!got) {
                    atomicOr(a.status, 1);
                    *vabort = 1;
                }
                tc_fence_after();
                return got;   // a warp leaves as one
            };
            // What the next MMA but one waits for is the reads, so that only the sums that make room for the second
            // half of them stand before the arrival.
            bool ok = true;
            for (int kb = 0; kb < a.nk; ++kb, ++it) {
                if (kb % kChunk == 0) {
                    ok = warp_wait(smem_u32(sfull_bar + ch % kChunks), ch / kChunks & 1, a.wait_ns);
                    if (!ok) {
                        atomicOr(a.status, 1);
                        *vabort = 1;
                        break;
                    }
                }
                const float* sk = scales + (ch % kChunks * kChunk + kb % kChunk) * kScales;
                const float s = BLOCKS ? sk[32 * q + lane] * sk[BM + h] : sk[32 * q + lane];
                const float* sbk = sk + BM + 128 * h;
                const uint32_t ta = tcol + (it & 1) * PN;
                auto add = [&](int c) {
                    if constexpr (BLOCKS) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[32 * c + j] = fmaf(u2f(r[c & 1][j]), s, acc[32 * c + j]);
                    } else {
                        add_scaled<true, 32>(acc + 32 * c, r[c & 1], s, sbk + 32 * c);
                    }
                };
                ok = ready(it);
                if (!ok) break;
                tc_ld_32cols(ta, r[0]);
                tc_ld_32cols(ta + 32, r[1]);
                tc_wait_ld();
                tie(r[0]);
                tie(r[1]);
                add(0);
                tc_ld_32cols(ta + 64, r[0]);
                add(1);
                tc_ld_32cols(ta + 96, r[1]);
                tc_wait_ld();
                tie(r[0]);
                tie(r[1]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote_ld(tempty0 + 8 * (it & 1));
                add(2);
                add(3);
                if (kb % kChunk == kChunk - 1 || kb + 1 == a.nk) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(sempty_bar + ch % kChunks));
                    ++ch;
                }
            }
            if (!ok) break;
            store_boxes<T>(a, sOut + (warp - 4) * (a.tma_out ? kWarpBoxes : kWarpOut), n0, row - lane, g, lane, acc);
        }
        bulk_wait();
    }
    tc_fence_before();
    __syncthreads();
    // Nothing of the pair's may be on its way any more when a CTA leaves: neither MMAs, which read both CTAs' stages and
    // write both's tensor memory, nor, after a wait that ran out, loads that no MMA has waited for (the even CTA's
    // barriers count both CTAs').
    if (warp == 1 && !warp_wait<true>(smem_u32(done_bar), 0, a.wait_ns)) atomicOr(a.status, 1);
    if (warp == 0 && rank == 0 && *vabort)
        for (uint32_t q = loaded < kPairStages ? 0 : loaded - kPairStages; q < loaded; ++q)
            warp_wait<true>(smem_u32(full_bar + q % kPairStages), q / kPairStages & 1, a.wait_ns);
    __syncthreads();
    cluster_sync();
    if (warp == 0) {
        tc_fence_after();
        tc2_dealloc(tmem, 2 * PN);
    }
}

template <class T, bool BLOCKS>
cudaError_t launch_fp8_pair(Fp8Args& p, const uint8_t* a, int64_t lda, const uint8_t* b, int64_t ldb, cudaStream_t st) {
    const int64_t cols = static_cast<int64_t>(p.groups) * p.K;
    if (!tc_make_map_u8(&p.tmA, a, p.M, cols, lda, BM) || !tc_make_map_u8(&p.tmB, b, p.N, cols, ldb, PN / 2))
        return cudaErrorInvalidValue;
    // Tiles with little to compute are bound by their stores, and SMs differ in how fast these go: asked for one by one,
    // 128 x 1024 x 1024 x 128 took 91.5 us, dealt out evenly 103 (16 x 1024 x 1024 x 1024 38.1 and 38.9); with more to
    // compute asking costs more than it evens out, 8192 x 4096 x 4096 107.5 and 104.6, as with b's scales per block and
    // bf16 outputs, 16384 x 4096 x 512 48.5 and 47.8.
    const bool ask = !BLOCKS && p.nk <= 8;
    auto kern = ask ? fp8_pair_kernel<T, BLOCKS, !BLOCKS> : fp8_pair_kernel<T, BLOCKS, false>;
    const cudaError_t err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem);
    if (err != cudaSuccess) return err;
    p.tma_out = tc_make_out_map(&p.tmOut, p.out, sizeof(T) == 2, p.M, p.N, p.groups, p.ldo, p.out_stride);
    p.mt = (p.M + 2 * BM - 1) / (2 * BM);
    p.nt = (p.N + PN - 1) / PN;
    const int tiles = p.mt * p.nt * p.groups, slots = sm_count() / 2;
    launch(kern, 2u * (ask || tiles < slots ? tiles : slots), kPairThreads, kPairSmem, st, p);
    return cudaGetLastError();
}

// How a product is cut: BT rows of a per CTA and K over ``split`` CTAs, or pairs (BT = 256).
struct Fp8Cut {
    int bt, split;
};

// The cheapest by an estimate in us, from the times of single products at K = 4096 (GB300, b's scales per
// block): a launch 1, the first loads and last stores of a round 3; a K block 0.23, 0.25, 0.33 and 0.41 for BT = 16, 32, 64 and
// 128 with an SM to itself, 0.29, 0.33 and 0.46 where two CTAs share one; the join of a split 0.02 BT + 0.2
// split; pairs 0.40 a K block and 2 a round of 76 tiles (0.64 where b's scales are per row).  Measured beside
// the alternatives: 1 x 4096 x 4096 on 16 rows / 4 splits 6.6 us (16 / 8: 7.2, 16 / 1: 11.0, 64 / 4: 8.6); 64 rows 64 / 4 8.6
// (16 / 1 11.4, 128 / 4 10.8); 512 rows 128 / 1 17.5 (64 / 1 18.8, pairs 19.7); 1024 rows pairs 20.7 (128 / 1
// 34.0); 1003 x 1000 x 1622 64 / 1 8.3 (128 / 1 9.5, pairs 11.2); 300 x 300 x 8192 32 / 8 9.6 (128 / 1 38).
Fp8Cut choose_cut(const Fp8Args& p) {
    const int64_t sms = sm_count(), nt = (p.N + BM - 1) / BM, g = p.groups;
    const double one[4] = {0.23, 0.25, 0.33, 0.41}, two[3] = {0.29, 0.33, 0.46};
    Fp8Cut best{16, 1};
    double least = 1e30;
    for (int i = 0; i < 4; ++i) {
        const int bt = 16 << i;
        const int64_t tiles = (p.M + bt - 1) / bt * nt * g;
        for (int split = 1; split <= 8; split *= 2) {
            if (split > 1 && p.nk < 2 * split) break;
            const int64_t ctas = tiles * split;
            const int nk = (p.nk + split - 1) / split;
            double t;
            if (ctas <= sms || bt == 128)
                t = static_cast<double>((ctas + sms - 1) / sms) * nk * one[i];
            else
                t = static_cast<double>((ctas + 2 * sms - 1) / (2 * sms)) * nk * two[i];
            t += 1.0 + 3.0 * static_cast<double>((ctas + sms - 1) / sms) / (bt == 128 || ctas <= sms ? 1 : 2);
            if (split > 1) t += 0.02 * bt + 0.2 * split;
            if (t < least) least = t, best = {bt, split};
        }
    }
    const int64_t pairs = (p.M + 2 * BM - 1) / (2 * BM) * ((p.N + PN - 1) / PN) * g, rounds = (2 * pairs + sms - 1) / sms;
    if (pairs <= 0x7fffffff && 4.0 + static_cast<double>(rounds) * (p.nk * (p.blocks ? 0.40 : 0.64) + 2.0) < least)
        best = {256, 1};
    return best;
}

template <class T, bool BLOCKS>
cudaError_t launch_fp8_cut(Fp8Args& p, const uint8_t* a, int64_t lda, const uint8_t* b, int64_t ldb, cudaStream_t st) {
    const Fp8Cut c = choose_cut(p);
    if (c.bt == 16) return launch_fp8_tile<T, 16, BLOCKS>(p, c.split, a, lda, b, ldb, st);
    if (c.bt == 32) return launch_fp8_tile<T, 32, BLOCKS>(p, c.split, a, lda, b, ldb, st);
    if (c.bt == 64) return launch_fp8_tile<T, 64, BLOCKS>(p, c.split, a, lda, b, ldb, st);
    if (c.bt == 128) return launch_fp8_tile<T, 128, BLOCKS>(p, c.split, a, lda, b, ldb, st);
    return launch_fp8_pair<T, BLOCKS>(p, a, lda, b, ldb, st);
}

template <class T>
cudaError_t launch_fp8(Fp8Args& p, const uint8_t* a, int64_t lda, const uint8_t* b, int64_t ldb, cudaStream_t st) {
    return p.blocks ? launch_fp8_cut<T, true>(p, a, lda, b, ldb, st) : launch_fp8_cut<T, false>(p, a, lda, b, ldb, st);
}

}  // namespace

}  // namespace dbw

using namespace dbw;

extern "C" int dbw_fp8_matmul(int64_t M, int64_t N, int64_t K, int groups, const uint8_t* a, int64_t lda,
                              const float* a_scale, int64_t ldas, const uint8_t* b, int64_t ldb, const float* b_scale,
                              int64_t ldbs, int blocks, void* out, int type, int64_t ldo, int64_t out_stride,
                              int* status, void* stream) {
    clear_error();
    Call call("dbw_fp8_matmul", as_stream(stream));
    const int64_t most = 0x7fffff00;
    if (M < 0 || N < 1 || K < 1 || M > most || N > most || K > most)
        return fail(DBW_EINVAL, "dbw_fp8_matmul: M must be >= 0, N and K >= 1, all below 2^31 - 255");
    if (groups < 1 || groups > DBW_NMAX || K > most / groups)
        return fail(DBW_EINVAL, "dbw_fp8_matmul: groups must be in [1, %d] and groups K below 2^31 - 255", DBW_NMAX);
    if (groups > 1 && K % 128 != 0) return fail(DBW_EINVAL, "dbw_fp8_matmul: K must be a multiple of 128 with groups");
    if (type != DBW_F32 && type != DBW_BF16) return fail(DBW_EINVAL, "dbw_fp8_matmul: unknown type");
    if (blocks != 0 && blocks != 1) return fail(DBW_EINVAL, "dbw_fp8_matmul: blocks must be 0 or 1");
    if (M == 0) return DBW_OK;
    if (!a || !a_scale || !b || !b_scale || !out || !status)
        return fail(DBW_EINVAL, "dbw_fp8_matmul: NULL pointer argument");
    const int64_t nk = (K + 127) / 128;
    if (lda < groups * K || ldb < groups * K || ldas < M || ldbs < (blocks ? groups * nk : N) || ldo < N)
        return fail(DBW_EALIGN, "dbw_fp8_matmul: a leading dimension is shorter than its rows");
    if (!aligned16(a) || !aligned16(b) || lda % 16 != 0 || ldb % 16 != 0)
        return fail(DBW_EALIGN, "dbw_fp8_matmul: a and b must be 16-byte aligned with leading dimensions of multiples of 16");
    if (!aligned_to(a_scale, 4) || !aligned_to(b_scale, 4) || !aligned_to(out, elem_bytes(type)) || !aligned_to(status, 4))
        return fail(DBW_EALIGN, "dbw_fp8_matmul: a pointer is not aligned to its elements");
    if ((M + 15) / 16 > 0x7fffffffll / 8 / ((N + BM - 1) / BM) / groups)   // the finest cut's CTAs
        return fail(DBW_EINVAL, "dbw_fp8_matmul: more than 2^28 output tiles of 16 x 128");
    int rc = check_device();
    if (rc) return rc;
    Fp8Args p{};
    p.sa = a_scale, p.sb = b_scale, p.out = out;
    p.ldsa = ldas, p.ldsb = ldbs, p.ldo = ldo, p.out_stride = out_stride;
    p.M = static_cast<int>(M), p.N = static_cast<int>(N), p.K = static_cast<int>(K);
    p.groups = groups, p.blocks = blocks, p.nk = static_cast<int>(nk);
    p.status = status;
    const TestWaits test = take_test_waits();
    p.wait_ns = test.limit_ns, p.skip = test.skip_stage;
    cudaStream_t st = as_stream(stream);
    const cudaError_t err = type == DBW_BF16 ? launch_fp8<__nv_bfloat16>(p, a, lda, b, ldb, st)
                                             : launch_fp8<float>(p, a, lda, b, ldb, st);
    if (err != cudaSuccess) return fail(DBW_ECUDA, "dbw_fp8_matmul: %s", cudaGetErrorString(err));
    return call.done(DBW_OK);
}
