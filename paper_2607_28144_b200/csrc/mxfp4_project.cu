// Product of two matrices in microscaled 4-bit floating point, y = x w^T + b, on the block-scaled tensor instruction
// (tcgen05.mma kind::mxf4, 64 elements of K per instruction, fp32 accumulators in tensor memory): the 4-bit form of the
// projections beside the attention.  Products of 4-bit values and power-of-two scales are exact; a result is rounded
// once, to y's type.
//
// A work item is a tile of tokens and `NT` output features; the grid is persistent.
//   warp 0      TMA producer: codes of x and w (rows of 128 bytes = 256 elements, 128-byte swizzle) and their scales
//               (tiles of 512 bytes, no swizzle), all counted on the stage's barrier
//   warp 1      copies the scales of a stage to tensor memory (tcgen05.cp, replicated to the four lane groups), issues
//               the MMAs and commits
//   warps 2-9   epilogue: accumulator -> + bias -> 16 bits -> swizzled staging block -> tiled store, in two halves that work
//               on alternate blocks of 64 columns (as one group with one staging tile the epilogue was the longest part of
//               an item at inner extents of 1536: 10920 x 1536 -> 4608 took 49 us instead of 43.5)
// Two accumulators of NT columns, used in turn, the scales behind them.
//
// Bound: the operands' way from L2.  All CTAs together take about 11.7 TB/s (45 bytes per SM and cycle), and a pair's
// 256 x 192 tile needs 31 KB per CTA for 384 cycles of tensor work, a 256 x 256 tile 35 KB for 512: at 31200 x 5120 x
// 15360 the two take 1.02 and 0.93 ms, single CTAs (43 KB for 128 x 192) 1.33 ms.  (Keeping a tile's weights in shared
// memory while the tokens go by, possible up to inner extents of 1536, halves those bytes there but leaves room for three
// stages only: 47.6 us.)
#include "common.cuh"
#include "cta_pair.cuh"
#include "mxfp4.cuh"
#include "ptx.cuh"
#include "umma_desc.cuh"

namespace regenvc {
namespace {

constexpr int kRowBytes = 128;                           // 256 codes: one swizzled row
constexpr uint32_t kCodesA = kTile * kRowBytes;          // 16 KB: this CTA's tokens
constexpr uint32_t kScalesA = 2 * 512;                   // 128 tokens x 256 elements
constexpr uint32_t kScalesB = 2 * kScalesA;              // up to 256 features
constexpr int kEpiThreads = 256;
constexpr int kThreadsMx = 64 + kEpiThreads;
constexpr uint64_t kWaitNs = 500000000ull;
constexpr int kScaleColumns = 24;                        // tensor-memory columns of one stage's scales: 2 x (4 + 8)

template <int CG, int NT>
struct Cfg {
    static constexpr uint32_t kCodesB = NT / CG * kRowBytes;   // this CTA's share of the weight rows
    static constexpr uint32_t kStage = kCodesA + kCodesB + kScalesA + kScalesB;
    static constexpr uint32_t kOutBlock = kTile * 64 * 2;      // [128 tokens][64 features] 16-bit, staged for TMA
    static constexpr uint32_t kOut = (NT > 64 ? 4 : 2) * kOutBlock;   // two slots for each half of the epilogue warps
    static constexpr int kStages = (int)((232448 - 4096 - kOut) / kStage) < 6 ? (int)((232448 - 4096 - kOut) / kStage) : 6;
    // Tensor-memory columns: two accumulators used in turn, then two sets of scales.  Two of 256 columns and the scales do
    // not fit 512 columns: the accumulators then share 48 columns, which an epilogue reads out first.
    static constexpr bool kShare = 2 * NT + 2 * kScaleColumns > 512;
    static constexpr uint32_t kAccStep = kShare ? 512 - 2 * kScaleColumns - NT : NT;
    static constexpr uint32_t kScaleBase = kAccStep + NT;
    static_assert(NT % 64 == 0 && kScaleBase + 2 * kScaleColumns <= 512 && NT - kAccStep <= 64, "tensor memory");
    // instruction descriptor of kind::mxf4: A and B e2m1 (1 at bits 7 and 10), N / 8 at bit 17, scales e8m0 (bit 23),
    // M / 16 at bit 24; the scales' place inside their words (bits 4 and 29) is added per instruction
    static constexpr uint32_t kIdesc = (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | (1u << 23) |
                                       ((uint32_t)(128 * CG >> 4) << 24);
};

struct MxShared {
    uint64_t full[6], empty[6];
    uint64_t acc_full[2], acc_empty[2];
    uint32_t tmem_base;
    int abort_flag;
    alignas(16) float bias[256];
};
template <int CG, int NT>
constexpr uint32_t mx_smem() {
    return Cfg<CG, NT>::kStages * Cfg<CG, NT>::kStage + Cfg<CG, NT>::kOut + 1024 + sizeof(MxShared);
}

// 32 rows x 16 bytes from shared memory (rows packed: eight of them 128 bytes apart) to four tensor-memory columns,
// replicated over the four groups of 32 lanes.
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem) {
    return static_cast<uint64_t>((smem & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128 >> 4) << 32) |
           (static_cast<uint64_t>(1) << 46);
}
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t smem) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(scale_desc(smem)) : "memory");
    else
        asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(scale_desc(smem)) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                       uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
template <int CG>
__device__ __forceinline__ void load_tile(uint32_t dst, const void* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1) tma_load_2d(dst, map, x, y, bar);
    else tma_load_2d_pair(dst, map, x, y, bar);
}
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if constexpr (CG == 1) {
        umma_commit(smem_u32(bar));
    } else {
        umma_commit_pair(smem_u32(bar));
        umma_commit_pair(map_to_rank(smem_u32(bar), 1));
    }
}

// The 128 threads of one half of the epilogue warps.
__device__ __forceinline__ void epi_barrier(int half) { asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory"); }
// All of this thread's stores but the last have read their shared memory.
__device__ __forceinline__ void tma_store_wait_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
// One arrival of a warp that has read an accumulator out (the barrier that counts is the leader's).
template <int CG>
__device__ __forceinline__ void release_accumulator(uint64_t* bar) {
    if constexpr (CG == 2) mbar_arrive_peer(map_to_rank(smem_u32(bar), 0));
    else mbar_arrive(smem_u32(bar));
}

template <int CG, int NT>
__global__ void __launch_bounds__(kThreadsMx, 1)
mxfp4_project_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_xs,
                     const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_ws,
                     const __grid_constant__ CUtensorMap tmap_y, const MxProjectParams p) {
    using C = Cfg<CG, NT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* stage_out = base + C::kStages * C::kStage;
    MxShared* sh = reinterpret_cast<MxShared*>(stage_out + C::kOut);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = CG == 2 ? static_cast<int>(cluster_rank()) : 0;
    const int n_rank = (p.features + NT - 1) / NT;
    const int n_tiles = (p.n_tokens + kTile - 1) / kTile;
    const int n_slices = (n_tiles + CG - 1) / CG * n_rank;
    const int slice0 = CG == 2 ? static_cast<int>(cluster_id_x()) : static_cast<int>(blockIdx.x);
    const int slice_step = CG == 2 ? static_cast<int>(n_clusters_x()) : static_cast<int>(gridDim.x);
    const int n_kb = (p.k_blocks + 1) / 2;                   // stages of 256 elements, the last one maybe half
    const WaitCtl ctl{&sh->abort_flag, p.status, kStatusTimeout, kWaitNs};

    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(smem_u32(&sh->full[s]), 1);
            mbar_init(smem_u32(&sh->empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sh->acc_full[b]), 1);
            mbar_init(smem_u32(&sh->acc_empty[b]), CG * (kEpiThreads / 32));
        }
        sh->abort_flag = (*reinterpret_cast<volatile int*>(p.status) != 0) ? 1 : 0;
        fence_mbar_init();
    }
    __syncwarp();
    if (warp == 1) {
        if constexpr (CG == 1) {
            tmem_alloc(smem_u32(&sh->tmem_base), 512);
            tmem_relinquish();
        } else {
            tmem_alloc_pair(smem_u32(&sh->tmem_base), 512);
            tmem_relinquish_pair();
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = sh->tmem_base;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        if (elect_one()) {
            tma_prefetch_desc(&tmap_x);
            tma_prefetch_desc(&tmap_w);
            // launched early behind the kernel that quantises x (launch_mxfp4_project): all set-up above ran beside its end
            asm volatile("griddepcontrol.wait;" ::: "memory");
            int fill = 0;
            bool ok = true;
            for (int slice = slice0; ok && slice < n_slices; slice += slice_step) {
                const int tile = CG * (slice / n_rank) + rank;       // this CTA's token tile (may lie past the end)
                const int f0 = slice % n_rank * NT;
                for (int kb = 0; kb < n_kb; ++kb, ++fill) {
                    const int s = fill % C::kStages, round = fill / C::kStages;
                    if (round > 0) ok = mbar_wait(smem_u32(&sh->empty[s]), (round - 1) & 1, ctl);
                    if (!ok) break;
                    if (rank == 0) mbar_expect_tx(smem_u32(&sh->full[s]), CG * C::kStage);
                    const uint32_t full = CG == 2 ? map_to_rank(smem_u32(&sh->full[s]), 0) : smem_u32(&sh->full[s]);
                    const uint32_t dst = smem_u32(base + s * C::kStage), sc = dst + kCodesA + C::kCodesB;
                    // rows past the last token or feature and bytes past the last column arrive as zeros; the second
                    // scale tile of a half stage is not read
                    load_tile<CG>(dst, &tmap_x, kb * kRowBytes, tile * kTile, full);
                    load_tile<CG>(dst + kCodesA, &tmap_w, kb * kRowBytes, f0 + rank * (NT / CG), full);
                    load_tile<CG>(sc, &tmap_xs, 0, tile * p.k_blocks + 2 * kb, full);
                    load_tile<CG>(sc + kScalesA, &tmap_ws, 0, f0 / 128 * p.k_blocks + 2 * kb, full);
                    load_tile<CG>(sc + 2 * kScalesA, &tmap_ws, 0, (f0 / 128 + 1) * p.k_blocks + 2 * kb, full);
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ scales to tensor memory, MMAs
        if (rank == 0 && elect_one()) {
            int fill = 0, it = 0;
            bool ok = true;
            for (int slice = slice0; ok && slice < n_slices; slice += slice_step, ++it) {
                const int b = it & 1;
                const uint32_t acc = tmem_base + b * C::kAccStep;
                // a tile that starts in the middle of 128 features takes its scales from the middle of their columns
                const uint32_t sb_off = (uint32_t)(slice % n_rank * NT % 128) / 32;
                // accumulator b was read out two slices ago; where it shares columns with the other one, that one's
                // shared columns have been read too (which comes later)
                if (it >= (C::kShare ? 1 : 2)) {
                    const int before = it - (C::kShare ? 1 : 2);
                    ok = mbar_wait(smem_u32(&sh->acc_empty[before & 1]), (before >> 1) & 1, ctl);
                    if (!ok) break;
                    tc_fence_after();
                }
                for (int kb = 0; kb < n_kb; ++kb, ++fill) {
                    const int s = fill % C::kStages;
                    ok = mbar_wait(smem_u32(&sh->full[s]), (fill / C::kStages) & 1, ctl);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(base + s * C::kStage), sb = sa + kCodesA, sc = sb + C::kCodesB;
                    const uint64_t da = umma_smem_desc_k_sw128(sa), db = umma_smem_desc_k_sw128(sb);
                    const uint32_t t_sc = tmem_base + C::kScaleBase + (fill & 1) * kScaleColumns;
                    const int halves = min(2, p.k_blocks - 2 * kb);
                    // copies and MMAs of one thread run in the order of their issue
                    for (int k2 = 0; k2 < halves; ++k2) {
                        const uint32_t t_a = t_sc + k2 * 12, t_b = t_a + 4;
                        copy_scales<CG>(t_a, sc + k2 * 512);
                        copy_scales<CG>(t_b, sc + kScalesA + k2 * 512);
                        copy_scales<CG>(t_b + 4, sc + 2 * kScalesA + k2 * 512);
                    }
                    for (int k2 = 0; k2 < halves; ++k2) {
                        const uint32_t t_a = t_sc + k2 * 12, t_b = t_a + 4 + sb_off;
#pragma unroll
                        for (uint32_t kk = 0; kk < 2; ++kk) {
                            // an instruction's two scales per row are bytes 0-1 or 2-3 of the row's word
                            const uint32_t idesc = C::kIdesc | (2 * kk) << 4 | (2 * kk) << 29;
                            mma_mx<CG>(acc, da + 2 * (2 * k2 + kk), db + 2 * (2 * k2 + kk), idesc, t_a, t_b,
                                       (kb > 0 || k2 > 0 || kk > 0) ? 1u : 0u);
                        }
                    }
                    commit<CG>(&sh->empty[s]);
                }
                if (ok) commit<CG>(&sh->acc_full[b]);
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue warps
        // Blocks of 64 columns; the four warps of half h (128 threads, one per accumulator row) take blocks h, h + 2, ...
        // on their own, through two staging slots in turn: a slot is written again once the store before last has read it.
        const int half = (warp - 2) >> 2;
        const int row = (warp & 3) * 32 + lane;       // accumulator row = TMEM lane
        const int et = (tid - 64) & 127;
        constexpr int kBlocks = NT / 64;
        const int mine = (kBlocks - half + 1) / 2;    // blocks of this half
        float* bias = sh->bias + half * 128;
        uint8_t* slots = stage_out + half * 2 * C::kOutBlock;
        bool ok = true;
        int it = 0, used = 0;
        for (int slice = slice0; slice < n_slices; slice += slice_step, ++it) {
            const int f0 = slice % n_rank * NT, b = it & 1;
            const int tile = CG * (slice / n_rank) + rank;
            const uint32_t t_acc = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + b * C::kAccStep;
            if (et < mine * 64) {   // (the slice before's readers are past the barrier behind their last block)
                const int f = f0 + (half + et / 64 * 2) * 64 + et % 64;
                bias[et] = p.bias && f < p.features ? __ldg(p.bias + f) : 0.0f;
            }
            if (ok) ok = mbar_wait(smem_u32(&sh->acc_full[b]), (it >> 1) & 1, ctl);
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
            if (mine == 0 && lane == 0) release_accumulator<CG>(&sh->acc_empty[b]);
#pragma unroll 1
            for (int i = 0; i < mine; ++i, ++used) {
                // accumulator 0 shares its last columns with the other one, accumulator 1 its first: those go first
                const int k = C::kShare && b == 0 ? mine - 1 - i : i;
                const int col = (half + 2 * k) * 64;
                uint32_t a[64];
                if (ok) {
                    tmem_ld32(t_acc + col, a);
                    tmem_ld32(t_acc + col + 32, a + 32);
                    tmem_wait_ld();
                }
                if (i == (C::kShare ? 0 : mine - 1)) {
                    // this warp's part of what the next MMAs overwrite is in registers: all of the accumulator, or the
                    // shared columns (and the slice before's accumulator was finished earlier)
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) release_accumulator<CG>(&sh->acc_empty[b]);
                }
                uint8_t* slot = slots + (used & 1) * C::kOutBlock;
                if (et == 0) tma_store_wait_read_but_one();
                epi_barrier(half);
#pragma unroll
                for (int c8 = 0; c8 < 8; ++c8) {
                    const float4* b4 = reinterpret_cast<const float4*>(bias + k * 64 + c8 * 8);
                    const float4 b0 = b4[0], b1 = b4[1];
                    const float v0 = __uint_as_float(a[c8 * 8 + 0]) + b0.x, v1 = __uint_as_float(a[c8 * 8 + 1]) + b0.y;
                    const float v2 = __uint_as_float(a[c8 * 8 + 2]) + b0.z, v3 = __uint_as_float(a[c8 * 8 + 3]) + b0.w;
                    const float v4 = __uint_as_float(a[c8 * 8 + 4]) + b1.x, v5 = __uint_as_float(a[c8 * 8 + 5]) + b1.y;
                    const float v6 = __uint_as_float(a[c8 * 8 + 6]) + b1.z, v7 = __uint_as_float(a[c8 * 8 + 7]) + b1.w;
                    const uint4 w = p.y_f16
                        ? make_uint4(pack_f16x2(v0, v1), pack_f16x2(v2, v3), pack_f16x2(v4, v5), pack_f16x2(v6, v7))
                        : make_uint4(pack_bf16x2(v0, v1), pack_bf16x2(v2, v3), pack_bf16x2(v4, v5), pack_bf16x2(v6, v7));
                    if (ok) *reinterpret_cast<uint4*>(slot + sw128_offset(row, c8)) = w;
                }
                fence_proxy_async_smem();
                epi_barrier(half);
                if (et == 0) {
                    // what lies past the last token or feature is dropped by the store
                    if (ok && tile < n_tiles && f0 + col < p.features) tma_store_2d(&tmap_y, f0 + col, tile * kTile, smem_u32(slot));
                    tma_store_commit();
                }
            }
        }
        if (et == 0) tma_store_wait_read();
        __syncwarp();
    }

    // ---------------------------------------------------------------- tear-down
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    if (warp == 1) {
        __syncwarp();
        if (sh->abort_flag) {   // copies and MMAs in flight end first
            const uint64_t t0 = global_timer_ns();
            while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
        }
        __syncwarp();
        if constexpr (CG == 1) tmem_dealloc(tmem_base, 512);
        else tmem_dealloc_pair(tmem_base, 512);
    }
}

template <int CG, int NT>
cudaError_t launch_cfg(const CUtensorMap& x, const CUtensorMap& xs, const CUtensorMap& w, const CUtensorMap& ws,
                       const CUtensorMap& y, const MxProjectParams& p, bool early, int sm_count, cudaStream_t stream) {
    const int n_tiles = (p.n_tokens + kTile - 1) / kTile;
    const long long n_slices = (long long)((n_tiles + CG - 1) / CG) * ((p.features + NT - 1) / NT);
    const int slots = sm_count / CG;
    const int items = n_slices < slots ? (int)n_slices : slots;
    if (items < 1) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CG * items));
    cfg.blockDim = dim3(kThreadsMx);
    cfg.dynamicSmemBytes = mx_smem<CG, NT>();
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n_attr = 0;
    if (CG == 2) {
        attr[n_attr].id = cudaLaunchAttributeClusterDimension;
        attr[n_attr].val.clusterDim.x = CG;
        attr[n_attr].val.clusterDim.y = 1;
        attr[n_attr++].val.clusterDim.z = 1;
    }
    if (early) {
        attr[n_attr].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n_attr++].val.programmaticStreamSerializationAllowed = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n_attr;
    return cudaLaunchKernelEx(&cfg, mxfp4_project_kernel<CG, NT>, x, xs, w, ws, y, p);
}

}  // namespace

// Which build: the one with the least estimated time.  An item costs its operand bytes at what an SM can take (80 bytes
// per cycle alone, 45 when all SMs load) and about 1500 cycles beside, more for wider epilogues; items run in rounds.
// (With pairs or 192-wide single items wherever there were enough of them and 64-wide ones elsewhere, 512 x 5120 -> 5120
// took 27 us instead of 17 and 128 x 5120 -> 15360 24 instead of 15.)
MxProjectPlan plan_mxfp4_project(int n_tokens, int features, int in_features, int sm_count) {
    struct Build {
        MxProjectPlan plan;
        int kilobytes;   // per CTA and 256 elements of K
    };
    static const Build builds[4] = {{{1, 256, 128}, 35}, {{1, 192, 96}, 31}, {{0, 192, 192}, 43}, {{0, 64, 64}, 27}};
    const long long tiles = (n_tokens + kTile - 1) / kTile;
    const double stages = (in_features + 255) / 256;
    double best = 0.0;
    const Build* pick = nullptr;
    for (const Build& b : builds) {
        const int group = b.plan.pair ? 2 : 1;
        const long long items = (tiles + group - 1) / group * ((features + b.plan.tile_features - 1) / b.plan.tile_features);
        const long long slots = sm_count / group;
        const long long rounds = (items + slots - 1) / slots;
        const double busy = (double)(items < slots ? items : slots) * group;
        double rate = 45.0 * sm_count / busy;
        if (rate > 80.0) rate = 80.0;
        const double cycles = rounds * (stages * b.kilobytes * 1024.0 / rate + 1500.0 + 4.0 * b.plan.tile_features);
        if (!pick || cycles < best) {
            best = cycles;
            pick = &b;
        }
    }
    return pick->plan;
}

cudaError_t configure_mxfp4_project() {
    cudaError_t e = cudaFuncSetAttribute(mxfp4_project_kernel<1, 192>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)mx_smem<1, 192>());
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(mxfp4_project_kernel<1, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)mx_smem<1, 64>());
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(mxfp4_project_kernel<2, 192>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)mx_smem<2, 192>());
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(mxfp4_project_kernel<2, 256>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)mx_smem<2, 256>());
    return e;
}

cudaError_t launch_mxfp4_project(const MxProjectPlan& plan, const CUtensorMap& x, const CUtensorMap& xs, const CUtensorMap& w,
                                 const CUtensorMap& ws, const CUtensorMap& y, const MxProjectParams& p, bool early,
                                 int sm_count, cudaStream_t stream) {
    if (plan.pair && plan.tile_features == 256) return launch_cfg<2, 256>(x, xs, w, ws, y, p, early, sm_count, stream);
    if (plan.pair) return launch_cfg<2, 192>(x, xs, w, ws, y, p, early, sm_count, stream);
    if (plan.tile_features == 64) return launch_cfg<1, 64>(x, xs, w, ws, y, p, early, sm_count, stream);
    return launch_cfg<1, 192>(x, xs, w, ws, y, p, early, sm_count, stream);
}

}  // namespace regenvc
