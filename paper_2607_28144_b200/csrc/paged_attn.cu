// Attention of chunks of new tokens over a paged key/value cache, ragged over sequences.
//
//     out[i] = sum_j softmax_j(q_i k_j scale) v_j       over the cached tokens j that token i's position sees
//
// Rows: the new tokens of a sequence times the query heads that share a head of the cache, (token, head) in order, so that
// a chunk of few tokens still fills a tile.  An item is one sequence, one head of the cache and up to 256 rows; it walks over
// the tiles of 128 keys that any of its rows sees.  One thread block per SM:
//   warps 0-3, 4-7  two streams of softmax, a thread per row (TMEM lane): scores from tensor memory, running reference and
//                   sum in registers, probabilities back to tensor memory
//   warp  8         issues the products (one thread) and owns the tensor memory
//   warp  9         copies: looks the pages up (a lane per box) and fetches K and V tiles into a ring by TMA
// More than 128 rows: each stream has 128 rows of its own and both take every tile of keys.  At most 128 rows (single
// tokens): both streams have the same rows and take every other tile of keys, and their results are joined in tensor memory
// at the end.  Either way one stream's products run under the other's exponentials.
//
// Tensor memory: S0 [0,128) S1 [128,256) O0 [256,..) O1 [384,..); the probabilities (16-bit pairs) lie over the scores.
// K comes as [keys][64 columns] blocks with the 128-byte swizzle, which is a K-major operand of Q K^T, V in the same form,
// which is an MN-major operand of P V: neither is rewritten.
//
// Softmax: a row's reference is its maximum at the time it was last set, and is set again only when a later tile's maximum
// lies more than 8 log2 units above it (probabilities up to 2^8, in range of either type); then the row's O is rescaled.
// Scores, sums, O are fp32; probabilities are rounded to the cache's type, which the product P V takes both operands in
// (half a step of 2^-9 or 2^-12 each, independent from key to key).  Keys that no row of the item sees (behind the length,
// before the window) are zeroed in V's tile, so that what lies there does not reach a sum as 0 * NaN.
//
// Work: the units (item, key tile) form one line, cut into equal parts for the thread blocks; an item that is cut leaves
// unnormalised pieces which a second kernel joins in order.  Where several tiles of rows share a head's keys, whole items
// are dealt out in rounds first (neighbours of a round read the same keys at a time, out of L2), and only the rest is cut.
// Every thread block derives its part from the lengths on the device, so that a captured graph follows them.
#include "attn_core.cuh"
#include "common.cuh"
#include "paged_attn.cuh"

namespace regenvc {
namespace {

constexpr int kPgThreads = 384, kPgSoftmax = 256;
constexpr int kPgLaunchRegs = 168, kPgControlRegs = 64;
constexpr int kPgSoftmaxRegs = ((kPgLaunchRegs * kPgThreads - kPgControlRegs * 128) / kPgSoftmax) / 8 * 8;
static_assert(kPgSoftmaxRegs * kPgSoftmax + kPgControlRegs * 128 <= kPgLaunchRegs * kPgThreads, "register budget");
constexpr int kPgMmaWarp = 8, kPgTmaWarp = 9;
constexpr int kMaxRounds = 64;
constexpr float kRaise = 8.0f;

template <int D>
struct Shape {
    static constexpr int kTileB = 128 * D * 2;               // one tile of Q, K or V
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kRing = kStages * kTileB;
    static constexpr int kBlocks = D / 64;                    // 64-column blocks of a tile, 16 KB each
};

struct Control {
    uint64_t kv_full[10], kv_empty[10], q_full, s_full[2], p_full[2], o_full[2];
    uint32_t tmem_base;
    int abort_flag;
    // this thread block's part of the work
    int rounds, seq, head, tile, off;
    long long left;
    int item_seq[kMaxRounds], item_head[kMaxRounds], item_tile[kMaxRounds];
    long long warp_units[12], warp_items[12];
};

// ------------------------------------------------------------------------------------------------------ the work
struct Seq {
    int row0, tokens, keys;
};
// Lengths and row starts as far as the buffers go: whatever they hold, no access leaves them.
__device__ __forceinline__ Seq load_seq(const PagedAttnParams& p, int s) {
    Seq q;
    q.row0 = min(max(p.row_starts[s], 0), p.n_tokens);
    q.tokens = min(max(p.row_starts[s + 1], q.row0), p.n_tokens) - q.row0;
    q.keys = (int)min((long long)max(p.lengths[s], 0), min((long long)p.pages_per_sequence * p.page_size, 1ll << 30));
    return q;
}
// First and one past the last key that the token at position pos sees.
__device__ __forceinline__ int sees_end(const PagedAttnParams& p, int keys, int pos) {
    if (p.group == 0) return keys;
    if (pos < 0) return 0;
    return (int)min((long long)keys, (long long)(pos / p.group + 1) * p.group);
}
__device__ __forceinline__ int sees_begin(const PagedAttnParams& p, int pos) {
    if (p.window == 0 || pos < 0) return 0;
    return (int)max(0ll, (long long)(pos / p.group - p.window + 1) * p.group);
}
struct Item {
    int rows, lo, hi, first_tile, n_tiles;
};
__device__ __forceinline__ int item_tiles(const PagedAttnParams& p, const Seq& q) { return (q.tokens * p.share + kPagedRows - 1) / kPagedRows; }
__device__ __forceinline__ Item load_item(const PagedAttnParams& p, const Seq& q, int tile) {
    Item it;
    const int r0 = tile * kPagedRows;
    it.rows = min(kPagedRows, q.tokens * p.share - r0);
    const int at = q.keys - q.tokens;                        // position of the sequence's first new token
    it.lo = sees_begin(p, at + r0 / p.share);
    it.hi = sees_end(p, q.keys, at + (r0 + it.rows - 1) / p.share);
    if (it.lo >= it.hi) it.lo = it.hi = 0;                   // no row sees anything: one tile, all of it masked
    it.first_tile = it.lo / 128;
    it.n_tiles = it.hi > it.lo ? (it.hi + 127) / 128 - it.first_tile : 1;
    return it;
}

// A thread block's stretch of one item.
struct Segment {
    Seq q;
    int seq, tile, head, rows, lo, hi, kt0, n;   // key tiles kt0 .. kt0 + n - 1
    bool starts, ends;
};
struct Walk {
    int round, rounds, seq, head, tile, off;
    long long left;
    Seq q;
    int loaded;   // sequence that q holds
    __device__ __forceinline__ Walk(const Control& c) : round(0), rounds(c.rounds), seq(c.seq), head(c.head), tile(c.tile), off(c.off),
                                                        left(c.left), loaded(-1) {}
    __device__ __forceinline__ bool next(const PagedAttnParams& p, const Control& c, Segment& g) {
        int s, take;
        if (round < rounds) {
            s = c.item_seq[round];
            g.head = c.item_head[round];
            g.tile = c.item_tile[round];
            ++round;
            if (s != loaded) q = load_seq(p, loaded = s);
            const Item it = load_item(p, q, g.tile);
            g.q = q, g.seq = s;
            g.rows = it.rows, g.lo = it.lo, g.hi = it.hi, g.kt0 = it.first_tile, g.n = it.n_tiles;
            g.starts = g.ends = true;
            return true;
        }
        if (left <= 0) return false;
        if (seq != loaded) q = load_seq(p, loaded = seq);
        const Item it = load_item(p, q, tile);
        take = (int)min((long long)(it.n_tiles - off), left);
        if (take < 1) return false;                          // (cannot be: the part was cut from the same lengths)
        g.q = q, g.seq = seq;
        g.head = head, g.tile = tile, g.rows = it.rows, g.lo = it.lo, g.hi = it.hi;
        g.kt0 = it.first_tile + off, g.n = take;
        g.starts = off == 0;
        g.ends = off + take == it.n_tiles;
        left -= take;
        off += take;
        if (g.ends) {
            off = 0;
            if (++tile >= item_tiles(p, q)) {
                tile = 0;
                if (++head >= p.n_k_heads) {
                    head = 0;
                    if (left > 0) {
                        do {
                            if (++seq >= p.n_sequences) {
                                left = 0;
                                break;
                            }
                            q = load_seq(p, loaded = seq);
                        } while (q.tokens == 0);
                    }
                }
            }
        }
        return true;
    }
};

// Number of ring entries before V(j) and K(j) of a segment: the copies come as K(0) .. K(ahead - 1), then V(j), K(j + ahead)
// in turn, in the order in which the products want them.
__device__ __forceinline__ int ring_of_v(int j, int n, int ahead) { return ahead + j + min(j, n - ahead); }
__device__ __forceinline__ int ring_of_k(int j, int ahead) { return j < ahead ? j : 2 * j - ahead + 1; }

__device__ __forceinline__ void plan_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kPgThreads) : "memory"); }

// Exclusive prefix over the thread block of two sums.
__device__ __forceinline__ void block_scan(Control& c, long long& units, long long& items, long long& all_units, long long& all_items) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long u0 = units, i0 = items;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, units, o), i = __shfl_up_sync(0xffffffffu, items, o);
        if (lane >= o) units += u, items += i;
    }
    plan_barrier();
    if (lane == 31) c.warp_units[warp] = units, c.warp_items[warp] = items;
    plan_barrier();
    units -= u0, items -= i0;
    all_units = all_items = 0;
#pragma unroll
    for (int w = 0; w < kPgThreads / 32; ++w) {
        if (w < warp) units += c.warp_units[w], items += c.warp_items[w];
        all_units += c.warp_units[w], all_items += c.warp_items[w];
    }
}

// This thread block's part of the work.  scratch: at least 16 bytes per sequence + 2 KB of shared memory.
__device__ void plan_work(const PagedAttnParams& p, Control& c, uint8_t* scratch) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n_seq = p.n_sequences;
    long long* unit0 = reinterpret_cast<long long*>(scratch);        // [n_seq + 1] units of a sequence, then before it
    int* item0 = reinterpret_cast<int*>(scratch + (size_t)(n_seq + 1) * 8);   // [n_seq + 1] tiles of rows, then items before it
    for (int s = tid; s < n_seq; s += kPgThreads) {
        const Seq q = load_seq(p, s);
        const int tiles = item_tiles(p, q);
        long long units = 0;
        if (p.group == 0) units = tiles ? (long long)tiles * load_item(p, q, 0).n_tiles : 0;
        else if (tiles <= 8)
            for (int t = 0; t < tiles; ++t) units += load_item(p, q, t).n_tiles;
        else units = -1;                                     // the warps below
        unit0[s] = units;
        item0[s] = tiles;
        if (blockIdx.x == 0) {
            const bool good = p.row_starts[s] >= 0 && p.row_starts[s + 1] >= p.row_starts[s] && p.row_starts[s + 1] <= p.n_tokens &&
                              p.lengths[s] >= 0 && p.lengths[s] <= (long long)p.pages_per_sequence * p.page_size;
            if (!good) atomicCAS(p.status, 0, kStatusRange);
        }
    }
    plan_barrier();
    for (int s = warp; s < n_seq; s += kPgThreads / 32) {
        if (unit0[s] >= 0) continue;
        const Seq q = load_seq(p, s);
        long long units = 0;
        for (int t = lane; t < item0[s]; t += 32) units += load_item(p, q, t).n_tiles;
#pragma unroll
        for (int o = 16; o; o >>= 1) units += __shfl_xor_sync(0xffffffffu, units, o);
        __syncwarp();
        if (lane == 0) unit0[s] = units;
    }
    plan_barrier();
    // prefixes over the sequences, a stretch of them per thread
    const int per = (n_seq + kPgThreads - 1) / kPgThreads, s0 = min(n_seq, tid * per), s1 = min(n_seq, s0 + per);
    long long units = 0, items = 0, all_units, all_items;
    for (int s = s0; s < s1; ++s) units += unit0[s] * p.n_k_heads, items += (long long)item0[s] * p.n_k_heads;
    block_scan(c, units, items, all_units, all_items);
    for (int s = s0; s < s1; ++s) {
        const long long u = unit0[s] * p.n_k_heads;
        const int i = item0[s] * p.n_k_heads;
        unit0[s] = units;
        item0[s] = (int)items;
        units += u, items += i;
    }
    if (tid == 0) unit0[n_seq] = all_units, item0[n_seq] = (int)all_items;
    plan_barrier();
    // parts: one per item or per four units, whichever are more
    const int grid = gridDim.x;
    const long long wanted = max(all_items, (all_units + 3) / 4);
    const int parts = (int)min((long long)grid, max(wanted, 1ll));
    int rounds = 0;
    long long start, count;
    const int me = blockIdx.x;
    if (p.rounds && parts == grid) {
        const long long fair = all_units / grid;
        long long mine = 0;
        while (rounds < kMaxRounds && (long long)(rounds + 1) * grid <= all_items) {
            int tiles = 0, s = 0, head = 0, tile = 0;
            if (tid < grid) {
                const int item = rounds * grid + tid;
                int lo = 0, hi = n_seq;                      // the last sequence whose items start at or before it
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (item0[mid] <= item) lo = mid;
                    else hi = mid;
                }
                s = lo;
                const Seq q = load_seq(p, s);
                const int each = item_tiles(p, q);
                head = (item - item0[s]) / each;
                tile = item - item0[s] - head * each;
                tiles = load_item(p, q, tile).n_tiles;
            }
            int over;
            asm volatile(
                "{\n\t.reg .pred a, b;\n\tsetp.ne.u32 a, %1, 0;\n\tbar.red.or.pred b, 1, %2, a;\n\tselp.u32 %0, 1, 0, b;\n\t}"
                : "=r"(over)
                : "r"((uint32_t)(tid < grid && mine + tiles > fair)), "n"(kPgThreads)
                : "memory");
            if (over) break;
            mine += tiles;
            if (tid == me) c.item_seq[rounds] = s, c.item_head[rounds] = head, c.item_tile[rounds] = tile;
            ++rounds;
        }
        // the rest is cut so that every thread block has the same in all
        long long share = tid < grid ? (tid + 1) * all_units / grid - tid * all_units / grid - mine : 0;
        const long long own = share;
        long long done = mine, all_share, all_done;
        block_scan(c, share, done, all_share, all_done);
        if (tid == me) {
            c.left = own;
            unit0[n_seq] = all_done + share;                 // where the part starts on the line
        }
        plan_barrier();
        start = unit0[n_seq];
        count = c.left;
    } else {
        start = me < parts ? me * all_units / parts : 0;
        count = me < parts ? (me + 1) * all_units / parts - start : 0;
    }
    if (warp == 0) {
        int lo = 0, hi = n_seq;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (unit0[mid] <= start) lo = mid;
            else hi = mid;
        }
        int head = 0, tile = 0, off = 0;
        if (count > 0) {
            const Seq q = load_seq(p, lo);
            const int tiles = item_tiles(p, q);
            long long rest = start - unit0[lo];
            long long each = 0;                              // units of one head
            for (int t0 = 0; t0 < tiles; t0 += 32) each += __reduce_add_sync(0xffffffffu, t0 + lane < tiles ? load_item(p, q, t0 + lane).n_tiles : 0);
            head = (int)(rest / each);
            rest -= head * each;
            for (int t0 = 0; t0 < tiles; t0 += 32) {
                const int n = t0 + lane < tiles ? load_item(p, q, t0 + lane).n_tiles : 0;
                int before = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int u = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += u;
                }
                const int all = __shfl_sync(0xffffffffu, before, 31);
                if (rest < all) {
                    const uint32_t here = __ballot_sync(0xffffffffu, rest < before);
                    const int at = __ffs(here) - 1;          // the first tile that ends behind the start
                    tile = t0 + at;
                    off = (int)rest - __shfl_sync(0xffffffffu, before - n, at);
                    break;
                }
                rest -= all;
            }
        }
        if (lane == 0) {
            c.rounds = rounds;
            c.seq = lo, c.head = head, c.tile = tile, c.off = off;
            c.left = count;
        }
    }
}

// ------------------------------------------------------------------------------------------------------ small pieces
__device__ __forceinline__ void streams_barrier() { asm volatile("bar.sync 2, %0;" ::"n"(kPgSoftmax) : "memory"); }

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* map, int x, int slot, int head, int page, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(slot), "r"(head), "r"(page), "r"(bar)
        : "memory");
}

template <bool F16>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
    return F16 ? pack_f16x2(a, b) : pack_bf16x2(a, b);
}

// 32 scores of a row -> 16 packed probability pairs 2^(s scale - m), their fp32 sum added to two packed partial sums.  Bit
// (c % 8) of kMask set: pair c takes the polynomial 2^x on the FMA pipe instead of the special-function unit.
constexpr uint32_t kPagedPoly = 0x24;
template <bool F16>
__device__ __forceinline__ void probabilities(const uint32_t* s, uint64_t scale2, uint64_t negm2, uint32_t* pr, uint64_t& sum_a,
                                              uint64_t& sum_b) {
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        const uint64_t x2 = fma2(pack2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), scale2, negm2);
        uint64_t p2;
        if ((kPagedPoly >> (c & 7)) & 1u) {
            p2 = exp2_poly2(x2);
        } else {
            float x0, x1;
            unpack2(x2, x0, x1);
            p2 = pack2(ex2_approx(x0), ex2_approx(x1));
        }
        if (c & 1) sum_b = add2(sum_b, p2);
        else sum_a = add2(sum_a, p2);
        float p0, p1;
        unpack2(p2, p0, p1);
        pr[c] = pack_pair<F16>(p0, p1);
    }
}

template <int D, bool F16>
__device__ constexpr uint32_t idesc_qk() {
    return F16 ? umma_idesc_f16_f32acc(128, 128) : umma_idesc_bf16_f32acc(128, 128);
}
template <int D, bool F16>
__device__ constexpr uint32_t idesc_pv() {
    return (F16 ? umma_idesc_f16_f32acc(128, D) : umma_idesc_bf16_f32acc(128, D)) | (1u << 16);   // V: MN-major
}
// V's tile as an MN-major operand: the 64 columns of a block are one 128-byte row per key, eight keys to 1024 bytes; the
// next 64 columns lie a block of 16 KB on.
__device__ __forceinline__ uint64_t desc_v(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(16384 >> 4) << 16) |
           (static_cast<uint64_t>(1024 >> 4) << 32) | (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}
template <int D, bool F16>
__device__ __forceinline__ void products_qk(uint32_t s_tmem, uint32_t q, uint32_t k) {
    const uint64_t a = umma_smem_desc_k_sw128(q), b = umma_smem_desc_k_sw128(k);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const uint64_t off = (i >> 2) * (16384 >> 4) + (i & 3) * 2;
        umma_ss(s_tmem, a + off, b + off, idesc_qk<D, F16>(), i > 0);
    }
}
template <int D, bool F16>
__device__ __forceinline__ void products_pv(uint32_t o_tmem, uint32_t p_tmem, uint32_t v, bool accumulate) {
    const uint64_t b = desc_v(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) umma_ts(o_tmem, p_tmem + i * 8, b + i * (2048 >> 4), idesc_pv<D, F16>(), accumulate || i > 0);
}

template <int D>
constexpr uint32_t paged_smem() {
    return 2 * Shape<D>::kTileB + Shape<D>::kRing + 1024 + (uint32_t)((sizeof(Control) + 127) / 128 * 128);
}
static_assert(paged_smem<128>() <= 232448 && paged_smem<64>() <= 232448, "shared memory");
static_assert((kPagedMaxSequences + 1) * 12 <= Shape<128>::kRing && (kPagedMaxSequences + 1) * 12 <= Shape<64>::kRing, "plan's scratch");
static_assert(kPagedMaxGrid <= kPgThreads, "a thread per part in the plan");

// ------------------------------------------------------------------------------------------------------ the kernel
template <int D, bool F16>
__global__ void __launch_bounds__(kPgThreads, 1)
paged_attn_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ CUtensorMap map_k_page, const __grid_constant__ CUtensorMap map_v_page,
                  const __grid_constant__ PagedAttnParams p) {
    using S = Shape<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sQ = base;
    uint8_t* ring = base + 2 * S::kTileB;
    Control* c = reinterpret_cast<Control*>(ring + S::kRing);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const WaitCtl ctl{&c->abort_flag, p.status, kStatusTimeout, kWaitLimitNs};

    if (tid == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(smem_u32(&c->kv_full[i]), 1);
            mbar_init(smem_u32(&c->kv_empty[i]), 1);
        }
        mbar_init(smem_u32(&c->q_full), kPgSoftmax);
        for (int t = 0; t < 2; ++t) {
            mbar_init(smem_u32(&c->s_full[t]), 1);
            mbar_init(smem_u32(&c->p_full[t]), 128);
            mbar_init(smem_u32(&c->o_full[t]), 1);
        }
        c->abort_flag = (*reinterpret_cast<volatile int*>(p.status) != 0) ? 1 : 0;
        fence_mbar_init();
        p.pieces[2 * blockIdx.x].valid = 0;
        p.pieces[2 * blockIdx.x + 1].valid = 0;
    }
    if (warp == kPgMmaWarp) {
        tmem_alloc(smem_u32(&c->tmem_base), 512);
        tmem_relinquish();
    }
    if (warp == kPgTmaWarp && lane == 0) {
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
        if (p.one_page_box) {
            tma_prefetch_desc(&map_k_page);
            tma_prefetch_desc(&map_v_page);
        }
    }
    __syncwarp();
    plan_work(p, *c, ring);
    fence_proxy_async_smem();                                // the plan's scratch is the copies' ring
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem_base = c->tmem_base;

    if (warp >= kPgMmaWarp) {
        setmaxnreg_dec<kPgControlRegs>();
        if (warp == kPgTmaWarp) {
            // ------------------------------------------------------------------------------------- copies
            Walk walk(*c);
            Segment g;
            bool ok = true;
            uint32_t slot = 0, phase = 1;                    // ring slot; the parity of its last release (none in the first round)
            bool first_round = true;
            while (ok && walk.next(p, *c, g)) {
                const int ahead = min(g.rows > 128 ? 1 : 2, g.n), pairs = 2 * (g.n - ahead);
                const int* pages = p.table + g.seq * p.table_stride;
                for (int i = 0; i < 2 * g.n; ++i) {
                    // entry i: a K tile for i < ahead, then V and K in turn while K tiles are left, then V tiles
                    const int b = i - ahead;
                    const bool is_v = b >= 0 && (b >= pairs || (b & 1) == 0);
                    const int j = b < 0 ? i : (b >= pairs ? b - (g.n - ahead) : (b >> 1) + (is_v ? 0 : ahead));
                    const int key0 = (g.kt0 + j) * 128;
                    const bool whole = p.one_page_box && key0 / p.page_size == (key0 + 127) / p.page_size;
                    const int rows = whole ? 128 : p.box_rows, key = key0 + lane * rows;
                    const bool mine = lane * rows < 128 && key < g.hi && key + rows > g.lo;
                    int page = -1, at = 0;
                    if (mine) {
                        const int n = key / p.page_size;
                        at = key - n * p.page_size;
                        page = pages[n];
                        if (page < 0 || page >= p.n_pages) {   // not there: its rows arrive as zeros
                            page = -1;
                            atomicCAS(p.status, 0, kStatusRange);
                        }
                    }
                    const int boxes = __popc(__ballot_sync(0xffffffffu, mine));
                    if (!first_round) ok = mbar_wait(smem_u32(&c->kv_empty[slot]), phase, ctl);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    const uint32_t full = smem_u32(&c->kv_full[slot]);
                    if (lane == 0) {
                        if (boxes) mbar_expect_tx(full, (uint32_t)(boxes * rows * D * 2));
                        else mbar_arrive(full);
                    }
                    __syncwarp();
                    if (mine) {
                        const void* map = is_v ? (whole ? &map_v_page : &map_v) : (whole ? &map_k_page : &map_k);
                        const uint32_t dst = smem_u32(ring) + slot * S::kTileB + lane * rows * 128;
#pragma unroll
                        for (int x = 0; x < S::kBlocks; ++x) tma_load_4d(dst + x * 16384, map, x * 64, at, g.head, page, full);
                    }
                    __syncwarp();
                    if (++slot == S::kStages) {
                        slot = 0;
                        phase ^= 1;
                        first_round = false;
                    }
                }
            }
        } else if (warp == kPgMmaWarp) {
            // ------------------------------------------------------------------------------------- products
            if (elect_one()) {
                Walk walk(*c);
                Segment g;
                bool ok = true;
                uint32_t entry = 0, segment = 0, visit[2] = {0, 0};
                const uint32_t q_addr = smem_u32(sQ), ring_addr = smem_u32(ring);
                auto wait_full = [&](uint32_t e) {
                    return mbar_wait(smem_u32(&c->kv_full[e % S::kStages]), (e / S::kStages) & 1, ctl);
                };
                auto tile_at = [&](uint32_t e) { return ring_addr + (e % S::kStages) * S::kTileB; };
                auto release = [&](uint32_t e) { umma_commit(smem_u32(&c->kv_empty[e % S::kStages])); };
                while (ok && walk.next(p, *c, g)) {
                    const bool two = g.rows > 128;
                    const int ahead = min(two ? 1 : 2, g.n);
                    ok = mbar_wait(smem_u32(&c->q_full), segment & 1, ctl);
                    ++segment;
                    for (int j = 0; ok && j < ahead; ++j) {
                        const uint32_t ek = entry + ring_of_k(j, ahead);
                        ok = wait_full(ek);
                        if (!ok) break;
                        tc_fence_after();
                        for (int t = two ? 0 : j; t < (two ? 2 : j + 1); ++t) {
                            products_qk<D, F16>(tmem_base + t * 128, q_addr + (two ? t * S::kTileB : 0), tile_at(ek));
                            umma_commit(smem_u32(&c->s_full[t]));
                        }
                        release(ek);
                    }
                    for (int j = 0; ok && j < g.n; ++j) {
                        const uint32_t ev = entry + ring_of_v(j, g.n, ahead);
                        const bool more = j + ahead < g.n;
                        const uint32_t ek = entry + ring_of_k(j + ahead, ahead);
                        ok = wait_full(ev);
                        for (int t = two ? 0 : (j & 1); ok && t < (two ? 2 : (j & 1) + 1); ++t) {
                            ok = mbar_wait(smem_u32(&c->p_full[t]), visit[t] & 1, ctl);
                            ++visit[t];
                            if (!ok) break;
                            tc_fence_after();
                            products_pv<D, F16>(tmem_base + 256 + t * 128, tmem_base + t * 128, tile_at(ev), two ? j > 0 : j > 1);
                            umma_commit(smem_u32(&c->o_full[t]));
                            if (t == 1 || !two) release(ev);
                            if (more) {
                                ok = wait_full(ek);
                                if (!ok) break;
                                products_qk<D, F16>(tmem_base + t * 128, q_addr + (two ? t * S::kTileB : 0), tile_at(ek));
                                umma_commit(smem_u32(&c->s_full[t]));
                                if (t == 1 || !two) release(ek);
                            }
                        }
                    }
                    entry += 2 * g.n;
                }
            }
        }
    } else {
        // ----------------------------------------------------------------------------------------- softmax
        setmaxnreg_inc<kPgSoftmaxRegs>();
        const int t = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t t_S = lane_base + t * 128, t_O = lane_base + 256 + t * 128;
        const float scale = p.scale_log2;
        const uint64_t scale2 = pack2(scale, scale);
        Walk walk(*c);
        Segment g;
        bool ok = true;                                      // false once a wait ran out: barriers go on, work does not
        uint32_t entry = 0, visit = 0;
        while (walk.next(p, *c, g)) {
            const bool two = g.rows > 128;
            const int ahead = min(two ? 1 : 2, g.n), first = two ? t * 128 : 0;
            streams_barrier();                               // the last segment's queries and tensor memory are done with
            {
                const int loaders = two ? 128 : 256, id = two ? (tid & 127) : tid;
                uint8_t* dst = sQ + (two ? t * S::kTileB : 0);
                const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q) + g.q.row0 * p.q_token;
#pragma unroll 8
                for (int i = id; i < 128 * (D / 8); i += loaders) {
                    const int r = i / (D / 8), ch = i % (D / 8), in_seq = g.tile * kPagedRows + first + r;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (first + r < g.rows) {
                        const int token = in_seq / p.share, h = g.head * p.share + in_seq - token * p.share;
                        v = *reinterpret_cast<const uint4*>(q + token * p.q_token + h * p.q_head + ch * 8);
                    }
                    *reinterpret_cast<uint4*>(dst + (ch >> 3) * 16384 + sw128_offset(r, ch & 7)) = v;
                }
                fence_proxy_async_smem();
                mbar_arrive(smem_u32(&c->q_full));
            }
            const int in_seq = g.tile * kPagedRows + first + row, token = in_seq / p.share;
            const bool valid = first + row < g.rows, busy = first + (warp & 3) * 32 < g.rows;   // busy: any row of the warp
            int lo = 0, hi = 1 << 30;                        // keys that this row sees
            if (valid) {
                const int pos = g.q.keys - g.q.tokens + token;
                lo = sees_begin(p, pos);
                hi = sees_end(p, g.q.keys, pos);
            }
            float m = -INFINITY, l = 0.0f;
            int done = 0;                                    // tiles of this stream
            for (int j = two ? 0 : t; j < g.n; j += two ? 1 : 2) {
                const int key0 = (g.kt0 + j) * 128;
                if (ok) ok = mbar_wait(smem_u32(&c->s_full[t]), visit & 1, ctl);
                ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
                if (ok && busy) {
                    uint32_t s[128];
#pragma unroll
                    for (int b = 0; b < 4; ++b) tmem_ld32(t_S + 32 * b, s + 32 * b);
                    tmem_wait_ld();
                    const int from = lo - key0, to = hi - key0;
                    if (__any_sync(0xffffffffu, from > 0 || to < 128)) {
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (i < from || i >= to) s[i] = 0xff800000u;   // -inf, whatever was there
                    }
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < 128; i += 8)
#pragma unroll
                        for (int b = 0; b < 4; ++b) mx[b] = max3(mx[b], __uint_as_float(s[i + 2 * b]), __uint_as_float(s[i + 2 * b + 1]));
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                    const bool raise = top > m + kRaise;     // (m is -inf until the row has seen a key)
                    if (__any_sync(0xffffffffu, raise)) {
                        const float alpha = raise ? ex2_approx(m - top) : 1.0f;
                        if (raise) m = top;
                        l *= alpha;
                        if (done > 0) {
                            ok = mbar_wait(smem_u32(&c->o_full[t]), (visit - 1) & 1, ctl);
                            ok = __all_sync(0xffffffffu, ok);
                            tc_fence_after();
                            if (ok) {
#pragma unroll 1
                                for (int b = 0; b < D / 32; ++b) {
                                    uint32_t o[32];
                                    tmem_ld32(t_O + b * 32, o);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                    tmem_st32(t_O + b * 32, o);
                                }
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : m;
                    const uint64_t negm2 = pack2(-ref, -ref);
                    uint64_t sum_a = 0, sum_b = 0;
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        uint32_t pr[16];
                        probabilities<F16>(s + 32 * b, scale2, negm2, pr, sum_a, sum_b);
                        tmem_st16(t_S + 16 * b, pr);
                    }
                    float s0, s1;
                    unpack2(add2(sum_a, sum_b), s0, s1);
                    l += s0 + s1;
                }
                if ((key0 < g.lo || key0 + 128 > g.hi) && (!two || t == 0)) {
                    // rows of V that no row of the item sees; with two tiles of rows stream 0 does it for both (its products
                    // are issued first)
                    const uint32_t e = entry + ring_of_v(j, g.n, ahead);
                    if (ok) ok = mbar_wait(smem_u32(&c->kv_full[e % S::kStages]), (e / S::kStages) & 1, ctl);
                    ok = __all_sync(0xffffffffu, ok);
                    const int key = key0 + row;
                    if (ok && (key < g.lo || key >= g.hi)) {
                        uint8_t* v = ring + (e % S::kStages) * S::kTileB + row * 128;
#pragma unroll
                        for (int x = 0; x < S::kBlocks; ++x)
#pragma unroll
                            for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(v + x * 16384 + ((i + row) & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&c->p_full[t]));
                ++visit;
                ++done;
            }
            entry += 2 * g.n;

            // ------------------------------------------------------------------------------------- results
            if (done > 0) {
                if (ok) ok = mbar_wait(smem_u32(&c->o_full[t]), (visit - 1) & 1, ctl);
                ok = __all_sync(0xffffffffu, ok);
                tc_fence_after();
            }
            float a[2] = {1.0f, 1.0f};                       // weights of the two streams' sums
            if (!two) {
                float2* ml = reinterpret_cast<float2*>(sQ + S::kTileB);   // (the second tile of queries is not in use)
                ml[t * 128 + row] = make_float2(m, l);
                tc_fence_before();
                streams_barrier();
                tc_fence_after();
                const float2 ml0 = ml[row], ml1 = ml[128 + row];
                const float m0 = ml0.x, m1 = ml1.x;
                m = fmaxf(m0, m1);
                a[0] = m0 == -INFINITY ? 0.0f : ex2_approx(m0 - m);
                a[1] = m1 == -INFINITY ? 0.0f : ex2_approx(m1 - m);
                l = a[0] * ml0.y + a[1] * ml1.y;
            } else if (m == -INFINITY) {
                a[t] = 0.0f;
            }
            if (m == -INFINITY) l = 0.0f;
            const bool alone = g.starts && g.ends;
            const int piece = 2 * blockIdx.x + (g.starts ? 1 : 0);
            const int part_row = first + row;
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            const long long out_row = g.q.row0 + token;
            const int h = g.head * p.share + in_seq - token * p.share;
            uint16_t* out = reinterpret_cast<uint16_t*>(p.out) + out_row * p.out_token + h * p.out_head;
            // this thread's columns: all of its stream's row, or half of the joined row
            const int col0 = two ? 0 : t * (D / 2), cols = two ? D : D / 2;
            if (ok && busy) {
#pragma unroll 1
                for (int b = 0; b < cols; b += 32) {
                    uint32_t o[32];
                    if (two) {
                        tmem_ld32(t_O + b, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = a[t] == 0.0f ? 0u : o[i];
                    } else {
                        uint32_t o1[32];
                        tmem_ld32(lane_base + 256 + col0 + b, o);
                        tmem_ld32(lane_base + 384 + col0 + b, o1);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float x = a[0] == 0.0f ? 0.0f : a[0] * __uint_as_float(o[i]);
                            o[i] = __float_as_uint(a[1] == 0.0f ? x : fmaf(a[1], __uint_as_float(o1[i]), x));
                        }
                    }
                    if (!valid) continue;
                    if (alone) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t w[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                w[k] = pack_pair<F16>(__uint_as_float(o[8 * i + 2 * k]) * inv, __uint_as_float(o[8 * i + 2 * k + 1]) * inv);
                            *reinterpret_cast<uint4*>(out + col0 + b + 8 * i) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    } else {
                        float4* to = p.part_o + (size_t)piece * (D / 4) * kPagedRows + (size_t)((col0 + b) / 4) * kPagedRows + part_row;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            to[(size_t)i * kPagedRows] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                                     __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
                    }
                }
                if (valid && (two || t == 0)) {
                    if (!alone) p.part_ml[(size_t)piece * kPagedRows + part_row] = make_float2(m, l);
                    else if (p.lse) p.lse[out_row * p.n_q_heads + h] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
                }
            }
            if (!alone && tid == 0) {
                PagedPiece d;
                d.valid = 1, d.ends = g.ends;
                d.seq_row0 = g.q.row0, d.first_row = g.tile * kPagedRows, d.rows = g.rows, d.head = g.head;
                p.pieces[piece] = d;
            }
            tc_fence_before();
        }
    }

    // --------------------------------------------------------------------------------------------- tear-down
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kPgMmaWarp) {
        __syncwarp();
        if (c->abort_flag) {
            // a wait ran out: copies and products that may still be in flight get time to land
            const uint64_t t0 = global_timer_ns();
            while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
        }
        __syncwarp();
        tmem_dealloc(tmem_base, 512);
    }
}

// Joins the pieces of an item: block (x, y) the item that thread block x of the attention began and did not end, a share of
// its rows.  The pieces are this one and the ones that the following thread blocks left in their slot 0, up to the one that
// ends the item, in that order.
template <int D, bool F16>
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedAttnParams p, const int grid) {
    constexpr int kRowsHere = 256 / (D / 4);
    __shared__ int slots[kPagedMaxGrid + 1];
    __shared__ int end_at, n_pieces;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const PagedPiece first = p.pieces[2 * blockIdx.x + 1];
    const int row0 = blockIdx.y * kRowsHere;
    if (!first.valid || row0 >= first.rows) return;
    if (threadIdx.x == 0) end_at = grid;
    __syncthreads();
    const int next = blockIdx.x + 1 + threadIdx.x;
    int valid = 0, ends = 0;
    if (next < grid) {
        valid = p.pieces[2 * next].valid;
        ends = p.pieces[2 * next].ends;
        if (valid && ends) atomicMin(&end_at, next);
    }
    __syncthreads();
    if (threadIdx.x < 32) {                                  // the valid ones up to the end, in order
        int n = 1;
        if (threadIdx.x == 0) slots[0] = 2 * blockIdx.x + 1;
        for (int b = blockIdx.x + 1; b <= end_at && b < grid; b += 32) {
            const int k = b + threadIdx.x;
            const bool in = k <= end_at && k < grid && p.pieces[2 * k].valid;
            const uint32_t all = __ballot_sync(0xffffffffu, in);
            if (in) slots[n + __popc(all & ((1u << threadIdx.x) - 1))] = 2 * k;
            n += __popc(all);
        }
        if (threadIdx.x == 0) n_pieces = n;
    }
    __syncthreads();
    const int n = n_pieces, row = row0 + threadIdx.x % kRowsHere, c4 = threadIdx.x / kRowsHere;
    if (row >= first.rows) return;
    float m = -INFINITY;
    for (int i = 0; i < n; ++i) m = fmaxf(m, p.part_ml[(size_t)slots[i] * kPagedRows + row].x);
    float l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float2 ml = p.part_ml[(size_t)slots[i] * kPagedRows + row];
        const float4 v = p.part_o[(size_t)slots[i] * (D / 4) * kPagedRows + (size_t)c4 * kPagedRows + row];
        if (ml.x == -INFINITY) continue;
        const float a = ex2_approx(ml.x - m);
        l += a * ml.y;
        o.x += a * v.x, o.y += a * v.y, o.z += a * v.z, o.w += a * v.w;
    }
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    const int in_seq = first.first_row + row, token = in_seq / p.share;
    const long long out_row = first.seq_row0 + token;
    const int h = first.head * p.share + in_seq - token * p.share;
    uint2 w = make_uint2(pack_pair<F16>(o.x * inv, o.y * inv), pack_pair<F16>(o.z * inv, o.w * inv));
    *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p.out) + out_row * p.out_token + h * p.out_head + c4 * 4) = w;
    if (p.lse && c4 == 0) p.lse[out_row * p.n_q_heads + h] = l > 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

template <int D, bool F16>
cudaError_t configure_one_paged() {
    cudaFuncAttributes attr;
    const cudaError_t e = cudaFuncGetAttributes(&attr, paged_attn_kernel<D, F16>);
    if (e != cudaSuccess) return e;
    if (attr.numRegs != kPgLaunchRegs) return cudaErrorInvalidConfiguration;   // the register hand-over counts on it
    return cudaFuncSetAttribute(paged_attn_kernel<D, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)paged_smem<D>());
}

template <int D, bool F16>
cudaError_t launch_one(const PagedMaps& maps, const PagedAttnParams& p, int grid, int* launches, cudaStream_t stream) {
    paged_attn_kernel<D, F16><<<grid, kPgThreads, paged_smem<D>(), stream>>>(maps.k, maps.v, maps.k_page, maps.v_page, p);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    *launches = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid, (unsigned)(kPagedRows / (256 / (D / 4))));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, paged_join_kernel<D, F16>, p, grid);
    if (e == cudaSuccess) *launches = 2;
    return e;
}

}  // namespace

size_t paged_attn_workspace_bytes(int head_dim) {
    return (size_t)kPagedMaxGrid * 2 * (kPagedRows * ((size_t)head_dim * sizeof(float) + sizeof(float2)) + sizeof(PagedPiece));
}

cudaError_t configure_paged_attn() {
    cudaError_t e = configure_one_paged<128, false>();
    if (e == cudaSuccess) e = configure_one_paged<128, true>();
    if (e == cudaSuccess) e = configure_one_paged<64, false>();
    if (e == cudaSuccess) e = configure_one_paged<64, true>();
    return e;
}

cudaError_t launch_paged_attn(const PagedMaps& maps, const PagedAttnParams& p, int head_dim, bool f16, int sm_count,
                              int* launches, cudaStream_t stream) {
    const int grid = sm_count < kPagedMaxGrid ? sm_count : kPagedMaxGrid;
    *launches = 0;
    if (head_dim == 128)
        return f16 ? launch_one<128, true>(maps, p, grid, launches, stream) : launch_one<128, false>(maps, p, grid, launches, stream);
    return f16 ? launch_one<64, true>(maps, p, grid, launches, stream) : launch_one<64, false>(maps, p, grid, launches, stream);
}

}  // namespace regenvc
