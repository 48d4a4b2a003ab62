// Attention of chunks of new tokens over a paged key/value cache, ragged over sequences.
//
//     out[i] = sum_j softmax_j(q_i k_j scale) v_j       over the cached tokens j that token i's position sees
//
// Rows: the new tokens of a sequence times the query heads that share a head of the cache, (token, head) in order, so that
// a chunk of few tokens still fills a tile.  An item is one sequence, one head of the cache and up to 256 rows; it walks over
// the tiles of 128 keys that any of its rows sees.  One thread block per SM:
//   warps 0-3, 4-7  two streams of softmax, a thread per row (TMEM lane): scores from tensor memory, running reference and
//                   sum in registers, probabilities back to tensor memory
//   warp  8         issues the products (one lane) and owns the tensor memory
//   warps 9, 11     copies of K and of V: look the pages up (a lane per box) and fetch the tiles into a ring each by TMA
//   warp  10        walks over this thread block's work and hands it to the others, stretch by stretch
// More than 128 rows: each stream has 128 rows of its own and both take every tile of keys.  At most 128 rows (single
// tokens): both streams have the same rows and take every other tile of keys, and their results are joined in tensor memory
// at the end.  Either way one stream's products run under the other's exponentials.
//
// Bound: single tokens by HBM (64 streams with 16-token pages, 2.77 GB: 463 us, 6.0 TB/s of 6.44 measured; half the bytes at 64
// columns take 371 us, which is not HBM's and was not looked into).  Chunks by the round a stream's tile takes through softmax
// and products, which one buffer of scores does not hide: 128 exponentials a row (1100 cycles alone, 2000 beside the other
// stream's), the products (1024 and some 400 of hand-over), loads and hand-over (500) (a window of 10920 tokens over 31200, 40
// heads: 4.65 ms, 1.05 PFLOP/s; without exponentials 4.2 ms, without products 4.0).
//
// Tensor memory: tiles of scores from column 0 on, two of them beside O0 and O1 of 128 columns, three beside 64 columns; the
// probabilities (16-bit pairs) lie over the scores.  With three, a stream's next scores are formed under its exponentials.
// K comes as [keys][64 columns] blocks with the 128-byte swizzle, which is a K-major operand of Q K^T, V in the same form,
// which is an MN-major operand of P V: neither is rewritten.
//
// Softmax: a row's reference is set by its maximum over the first tile in which it sees a key.  No later maximum is taken: a
// tile's probabilities are formed against the reference, and only if their sum leaves the range of the probabilities' type
// (fp16: 65504) or reaches 1 (bf16) the reference is raised, O rescaled and the tile done again.  A larger probability costs no
// precision, it has as many bits as one below 1.
// Scores, sums, O are fp32; probabilities are rounded to the cache's type, which the product P V takes both operands in: off
// by up to 2^-8 (bf16) or 2^-11 (fp16) of one, independent from key to key.  fp16 ends at steps of 2^-24, where errors are not
// independent: many keys alike far below the reference all lose, or gain, the same.  Its reference lies 2^8 below the maximum
// (128 such probabilities sum to 2^15), so that what vanishes is below 2^-33 of the largest weight: 10^6 such keys weigh 1.2e-4
// of it (3 % with the maximum as reference).  Time as with the maximum (nine chunks and tokens: 214.8 and 214.4 us).
// bf16 has fp32's range: its reference lies 2^32 above the maximum, so that probabilities and their sums stay below 1 and O is
// finite for whatever finite values, up to bf16's largest (formed against the maximum itself, with 2^32 for scores to rise, it
// overflowed from 2^95 on).  What pays are values below 2^-85, whose products leave fp32's normal range.
// Keys that no row of the item sees (behind the length, before the window) are zeroed in V's tile, so that what lies there does
// not reach a sum as 0 * NaN.
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

constexpr int kPgSoftmax = 256, kPgThreads = kPgSoftmax + 128;
// 168 registers a thread fill the SM's; the others hand most of theirs to the softmax warps.  ptxas spills 72 bytes of a build and
// does not say in which role.
constexpr int kPgLaunchRegs = 168, kPgControlRegs = 64;
constexpr int kPgSoftmaxRegs = ((kPgLaunchRegs * kPgThreads - kPgControlRegs * 128) / kPgSoftmax) / 8 * 8;
static_assert(kPgSoftmaxRegs * kPgSoftmax + kPgControlRegs * 128 <= kPgLaunchRegs * kPgThreads, "register budget");
constexpr int kPgMmaWarp = 8, kPgKeyWarp = 9, kPgWalkWarp = 10, kPgValueWarp = 11;
constexpr int kSegments = 4;      // stretches of work handed to the warps ahead
constexpr int kMaxRounds = 64;
// Sums of 128 probabilities from which on a row's reference is set anew.
template <bool F16>
__device__ constexpr float raise_at() { return F16 ? 65504.0f : 1.0f; }
// Powers of two by which a row's reference lies below the maximum that sets it.
template <bool F16>
__device__ constexpr float below_top() { return F16 ? 8.0f : -32.0f; }
// Natural logarithm of a row's sum l against its reference m; both are brought near to the maximum first, where their parts
// are small.
template <bool F16>
__device__ __forceinline__ float log_sum(float m, float l) {
    constexpr float back = F16 ? 1.0f / 256.0f : 4294967296.0f;   // 2^-below_top
    return l > 0.0f ? ((m + below_top<F16>()) + log2f(l * back)) * 0.6931471805599453f : (l == 0.0f ? -INFINITY : l);
}

template <int D>
struct Shape {
    static constexpr int kTileB = 128 * D * 2;               // one tile of Q, K or V
    static constexpr int kKeySlots = D == 128 ? 3 : 5, kValueSlots = D == 128 ? 2 : 5;   // rings of K and of V tiles
    static constexpr int kRing = (kKeySlots + kValueSlots) * kTileB;
    static constexpr int kBlocks = D / 64;                    // 64-column blocks of a tile, 16 KB each
    // Tensor memory (512 columns): as many tiles of scores as fit beside the two streams' O
    static constexpr int kScores = D == 128 ? 2 : 3, kOut = kScores * 128;
};

// The bounded wait of ptx.cuh with its clock out of line (the kernel waits in some twenty places, and its loops have to stay
// in the instruction cache) and a long time given to the hardware's own wait: a warp that polls takes issue slots from the
// exponentials of the others.
constexpr uint32_t kWaitHintNs = 200000;
__device__ __noinline__ uint64_t wait_clock(volatile int* abort_flag, int* status, uint64_t since) {
    if (*abort_flag) return 0;
    const uint64_t now = global_timer_ns();
    if (since == 1) return now;
    if (now - since <= kWaitLimitNs) return since;
    *abort_flag = 1;
    atomicCAS(status, 0, kStatusTimeout);
    return 0;
}
__device__ __forceinline__ bool try_wait_long(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(kWaitHintNs)
        : "memory");
    return ok != 0;
}
struct Waiter {
    volatile int* abort_flag;
    int* status;
    __device__ __forceinline__ bool operator()(const uint64_t* bar, uint32_t parity) const {
        const uint32_t addr = smem_u32(bar);
        uint64_t since = 1;                                  // 1: the clock has not been read yet
        while (!try_wait_long(addr, parity & 1))
            if ((since = wait_clock(abort_flag, status, since)) == 0) return false;
        return true;
    }
};

// ------------------------------------------------------------------------------------------------------ the work
struct Seq {
    int row0, tokens, keys;
};
// Lengths and row starts as far as the buffers go: whatever they hold, no access leaves them.
__device__ __noinline__ Seq load_seq(const PagedAttnParams& p, int s) {
    Seq q;
    q.row0 = min(max(p.row_starts[s], 0), p.n_tokens);
    q.tokens = min(max(p.row_starts[s + 1], q.row0), p.n_tokens) - q.row0;
    q.keys = (int)min((long long)max(p.lengths[s], 0), min((long long)p.pages_per_sequence * p.page_size, kMaxCachedTokens));
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
__device__ __noinline__ Item load_item(const PagedAttnParams& p, const Seq& q, int tile) {
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
    int starts, ends;                       // n = 0: no more work
};
struct Control {
    uint64_t k_full[5], k_empty[5], v_full[5], v_empty[5], q_full, s_full[3], p_full[3], o_full[2][2];
    uint64_t seg_full[kSegments], seg_empty[kSegments], together;
    uint32_t tmem_base;
    int abort_flag;
    Segment seg[kSegments];
    // this thread block's part of the work: whole items of the rounds, then a stretch of the line
    int rounds;
    long long start, left;
    int item_seq[kMaxRounds], item_head[kMaxRounds], item_tile[kMaxRounds];
    // the plan's sums
    long long warp_cost[kPgThreads / 32], warp_items[kPgThreads / 32], taken, before;
    int most;
};

__device__ __forceinline__ void plan_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kPgThreads) : "memory"); }

// The line of work: sequences, in them heads of the cache, in them tiles of rows, in them tiles of keys.  A tile of keys
// counts two for an item of two tiles of rows, one for an item of one, which is about what they take.
__device__ __forceinline__ int weight(const Item& it) { return it.rows > 128 ? 2 : 1; }
// Where part i of n begins on a line of `all`.
__device__ __forceinline__ long long bound(long long all, int n, int i) {
    return i >= n ? all : (long long)((double)all * (double)__fdividef((float)i, (float)n));
}
// Parts: one per item or per four units, whichever are more, as far as there are thread blocks.
__device__ __forceinline__ int parts_of(long long all, long long items) {
    const long long most = max(items, (all + 3) / 4);
    return (int)min((long long)gridDim.x, max(most, 1ll));
}

struct Walk {
    int round, seq, head, tile;
    long long at, left;                     // on the line: place within the item, what is still to be done
    Seq q;
    int loaded;                             // sequence that q holds
    __device__ __forceinline__ bool next(const PagedAttnParams& p, const Control& c, Segment& g) {
#pragma unroll 1
        while (true) {
            const bool whole = round < c.rounds;
            if (!whole && left <= 0) return false;
            const int s = whole ? c.item_seq[round] : seq;
            if (s != loaded) q = load_seq(p, loaded = s);
            g.q = q, g.seq = s;
            g.head = whole ? c.item_head[round] : head;
            g.tile = whole ? c.item_tile[round] : tile;
            const Item it = load_item(p, q, g.tile);
            g.rows = it.rows, g.lo = it.lo, g.hi = it.hi;
            if (whole) {
                ++round;
                g.kt0 = it.first_tile, g.n = it.n_tiles;
                g.starts = g.ends = 1;
                return true;
            }
            const int w = weight(it), cost = it.n_tiles * w;
            const int from = (int)at, to = (int)min((long long)cost, at + left);
            const int a = (from + w - 1) / w, b = (to + w - 1) / w;
            left -= to - from;
            at = to;
            if (to == cost) {
                at = 0;
                if (++tile >= item_tiles(p, q)) {
                    tile = 0;
                    if (++head >= p.n_k_heads) {
                        head = 0;
#pragma unroll 1
                        while (left > 0 && ++seq < p.n_sequences) {
                            q = load_seq(p, loaded = seq);
                            if (q.tokens > 0) break;
                        }
                        if (seq >= p.n_sequences) left = 0;
                    }
                }
            }
            g.kt0 = it.first_tile + a, g.n = b - a;
            g.starts = a == 0, g.ends = b == it.n_tiles;
            if (b > a) return true;
        }
    }
};

// Cost of a sequence's items of one head, a sequence per lane; `most`: the largest item's.  Lanes with many items are helped
// by the whole warp.
__device__ __noinline__ long long cost_of(const PagedAttnParams& p, const Seq& q, int tiles, int& most) {
    const int lane = threadIdx.x & 31;
    long long cost = 0;
    most = 0;
    const bool alike = p.group == 0 && tiles > 2;            // all items but the last are alike
    const int mine = alike ? 2 : (tiles <= 8 ? tiles : 0);
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        const Item it = load_item(p, q, alike && i == 1 ? tiles - 1 : i);
        const int c = it.n_tiles * weight(it);
        cost += alike && i == 0 ? (long long)c * (tiles - 1) : c;
        most = max(most, c);
    }
    uint32_t many = __ballot_sync(0xffffffffu, tiles > 0 && mine == 0);
#pragma unroll 1
    while (many) {
        const int l = __ffs(many) - 1;
        many &= many - 1;
        Seq o;
        o.row0 = __shfl_sync(0xffffffffu, q.row0, l);
        o.tokens = __shfl_sync(0xffffffffu, q.tokens, l);
        o.keys = __shfl_sync(0xffffffffu, q.keys, l);
        const int n = __shfl_sync(0xffffffffu, tiles, l);
        long long sum = 0;
        int top = 0;
#pragma unroll 1
        for (int i = lane; i < n; i += 32) {
            const Item it = load_item(p, o, i);
            const int c = it.n_tiles * weight(it);
            sum += c;
            top = max(top, c);
        }
#pragma unroll 1
        for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == l) cost = sum, most = top;
    }
    return cost;
}

__device__ __forceinline__ void check_seq(const PagedAttnParams& p, int s) {
    const bool good = p.row_starts[s] >= 0 && p.row_starts[s + 1] >= p.row_starts[s] && p.row_starts[s + 1] <= p.n_tokens &&
                      p.lengths[s] >= 0 && p.lengths[s] <= min((long long)p.pages_per_sequence * p.page_size, kMaxCachedTokens);
    if (!good) atomicCAS(p.status, 0, kStatusRange);
}

// Sum over the lanes before this one; `all`: over the warp.
__device__ __forceinline__ long long lanes_before(long long v, long long& all) {
    const int lane = threadIdx.x & 31;
    long long sum = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += u;
    }
    all = __shfl_sync(0xffffffffu, sum, 31);
    return sum - v;
}

// Where `rest` units into a sequence lie: head, tile of rows, place in the item.  One warp.
__device__ __forceinline__ void place(const PagedAttnParams& p, Walk& w, long long rest, long long each) {   // each: of one head, or 0
    const int lane = threadIdx.x & 31, tiles = item_tiles(p, w.q);
    w.head = w.tile = 0;
    bool found = false;
#pragma unroll 1
    for (int pass = each > 0; pass < 2 && !found; ++pass) {
        if (pass == 1) {
            w.head = (int)__fdividef((float)rest, (float)each);   // a quotient below 2^16: off by one at most
            if ((long long)w.head * each > rest) --w.head;
            else if ((long long)(w.head + 1) * each <= rest) ++w.head;
            rest -= w.head * each;
            w.at = rest;
            if (tiles == 1) return;
        }
#pragma unroll 1
        for (int t0 = 0; t0 < tiles; t0 += 32) {
            long long c = 0;
            if (t0 + lane < tiles) {
                const Item it = load_item(p, w.q, t0 + lane);
                c = it.n_tiles * weight(it);
            }
            long long all;
            const long long before = lanes_before(c, all);
            if (pass == 0) {
                each += all;
                continue;
            }
            const uint32_t here = __ballot_sync(0xffffffffu, before <= rest && rest < before + c);
            if (here) {
                const int l = __ffs(here) - 1;
                w.tile = t0 + l;
                w.at = rest - __shfl_sync(0xffffffffu, before, l);
                found = true;
                break;
            }
            rest -= all;
        }
    }
}

// At most 32 sequences and no rounds: the walking warp finds this thread block's part alone, a lane per sequence (a call of
// a few tokens would wait longer for barriers than for its keys).
__device__ __noinline__ void plan_few(const PagedAttnParams& p, Control& c, Walk& w) {
    const int lane = threadIdx.x & 31;
    Seq q{0, 0, 0};
    int tiles = 0, most;
    if (lane < p.n_sequences) {
        q = load_seq(p, lane);
        tiles = item_tiles(p, q);
        if (blockIdx.x == 0) check_seq(p, lane);
    }
    const long long each = cost_of(p, q, tiles, most), mine = each * p.n_k_heads;
    long long all = __shfl_sync(0xffffffffu, mine, 0), before = 0;
    if (p.n_sequences > 1) before = lanes_before(mine, all);
    const int items = __reduce_add_sync(0xffffffffu, tiles) * p.n_k_heads;
    const int parts = parts_of(all, items), me = blockIdx.x;
    const long long start = bound(all, parts, me);
    w.left = me < parts ? bound(all, parts, me + 1) - start : 0;
    const uint32_t at = __ballot_sync(0xffffffffu, mine > 0 && before <= start);
    w.seq = at ? 31 - __clz(at) : 0;                         // the last sequence with work that starts at or before it
    w.loaded = w.seq;
    w.q.row0 = __shfl_sync(0xffffffffu, q.row0, w.seq);
    w.q.tokens = __shfl_sync(0xffffffffu, q.tokens, w.seq);
    w.q.keys = __shfl_sync(0xffffffffu, q.keys, w.seq);
    if (lane == 0) c.rounds = 0;
    const long long rest = start - __shfl_sync(0xffffffffu, before, w.seq);
    __syncwarp();
    const long long its = __shfl_sync(0xffffffffu, each, w.seq);
    if (w.left > 0) place(p, w, rest, its);
}

// Any number: all threads, a thread per sequence.  line: units before each sequence, first_item: items before each.
__device__ __noinline__ void plan_many(const PagedAttnParams& p, Control& c, long long* line, int* first_item) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n_seq = p.n_sequences, grid = gridDim.x, me = blockIdx.x;
    long long all = 0, items = 0;
    int most = 0;
    if (tid == 0) c.most = 0, c.taken = c.before = 0;
#pragma unroll 1
    for (int s0 = 0; s0 < n_seq; s0 += kPgThreads) {
        const int s = s0 + tid;
        Seq q{0, 0, 0};
        int tiles = 0, top;
        if (s < n_seq) {
            q = load_seq(p, s);
            tiles = item_tiles(p, q);
            if (me == 0) check_seq(p, s);
        }
        const long long cost = cost_of(p, q, tiles, top) * p.n_k_heads;
        most = max(most, top);
        long long warp_cost, warp_items;
        long long before = lanes_before(cost, warp_cost);
        long long items_before = lanes_before((long long)tiles * p.n_k_heads, warp_items);
        if (lane == 0) c.warp_cost[warp] = warp_cost, c.warp_items[warp] = warp_items;
        plan_barrier();
        before += all, items_before += items;
#pragma unroll 1
        for (int w = 0; w < kPgThreads / 32; ++w) {
            if (w < warp) before += c.warp_cost[w], items_before += c.warp_items[w];
            all += c.warp_cost[w], items += c.warp_items[w];
        }
        // (rounds take items from the first on: numbers past a few thousand are only compared)
        if (s < n_seq) line[s] = before, first_item[s] = (int)min(items_before, 1ll << 30);
        plan_barrier();
    }
    const int parts = parts_of(all, items);
    int rounds = 0;
    long long start = bound(all, parts, me), count = me < parts ? bound(all, parts, me + 1) - start : 0;
    if (p.rounds && items >= grid) {
        // whole items in rounds, as many as no part can be too small for
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) atomicMax(&c.most, most);
        plan_barrier();
        const long long fair = bound(all, grid, 1) - 2 - (all >> 20);
        rounds = (int)min(min((long long)kMaxRounds, items / grid), (long long)((float)fair / (float)c.most * 0.9999f));
        rounds = max(rounds, 0);
        long long mine = 0;
        if (tid < grid) {
#pragma unroll 1
            for (int r = 0; r < rounds; ++r) {
                const int item = r * grid + tid;
                int lo = 0, hi = n_seq;                      // the last sequence whose items start at or before it
#pragma unroll 1
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (first_item[mid] <= item) lo = mid;
                    else hi = mid;
                }
                const Seq q = load_seq(p, lo);
                const int each = item_tiles(p, q), head = (item - first_item[lo]) / each, tile = item - first_item[lo] - head * each;
                const Item it = load_item(p, q, tile);
                mine += it.n_tiles * weight(it);
                if (tid == me) c.item_seq[r] = lo, c.item_head[r] = head, c.item_tile[r] = tile;
            }
            // the rest of the line is cut so that every thread block has the same in all
            const long long share = bound(all, grid, tid + 1) - bound(all, grid, tid) - mine;
            atomicAdd(reinterpret_cast<unsigned long long*>(&c.taken), (unsigned long long)mine);
            if (tid < me) atomicAdd(reinterpret_cast<unsigned long long*>(&c.before), (unsigned long long)share);
            if (tid == me) c.left = share;
        }
        plan_barrier();
        start = c.taken + c.before;
        count = c.left;
    }
    if (tid == kPgWalkWarp * 32) c.rounds = rounds, c.start = start, c.left = count;
}
// ... and where it begins, by the walking warp.
__device__ __noinline__ void plan_start(const PagedAttnParams& p, const Control& c, const long long* line, Walk& w) {
    int lo = 0, hi = p.n_sequences;
#pragma unroll 1
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (line[mid] <= c.start) lo = mid;
        else hi = mid;
    }
    w.seq = w.loaded = lo;
    w.q = load_seq(p, lo);
    w.left = c.left;
    if (w.left > 0) place(p, w, c.start - line[lo], 0);
}

// ------------------------------------------------------------------------------------------------------ small pieces
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* map, int x, int slot, int head, int page, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(slot), "r"(head), "r"(page), "r"(bar)
        : "memory");
}

__device__ __forceinline__ bool wait_segment(const Control& c, uint32_t segment, const Waiter& wait) {
    return wait(&c.seg_full[segment % kSegments], segment / kSegments);
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

template <bool F16>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
    return F16 ? pack_f16x2(a, b) : pack_bf16x2(a, b);
}

// 32 scores of a row -> 16 packed probability pairs 2^(s scale - m), their fp32 sum added to two packed partial sums.  All
// powers on the special-function unit: the loop is bound by issue slots and latencies, and a polynomial on the FMA pipe for
// every fourth pair, as the attention over a whole window has it, costs more of them (a latent frame: 140 -> 144 us).
template <bool F16>
__device__ __forceinline__ void probabilities(const uint32_t* s, uint64_t scale2, uint64_t negm2, uint32_t* pr, uint64_t& sum_a,
                                              uint64_t& sum_b) {
#pragma unroll
    for (int c = 0; c < 16; ++c) {
        const uint64_t x2 = fma2(pack2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), scale2, negm2);
        float x0, x1;
        unpack2(x2, x0, x1);
        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
        if (c & 1) sum_b = add2(sum_b, pack2(p0, p1));
        else sum_a = add2(sum_a, pack2(p0, p1));
        pr[c] = pack_pair<F16>(p0, p1);
    }
}

// Items of at most 16 rows (single tokens) have products of 64 rows instead of 128: the first 16 lie in lanes 0-15 of both
// forms, and what the other lanes hold is nobody's.  They take the same time but less power, which is what holds long runs of
// such calls: 64 streams at 600 calls in a row 528 -> 496 us, another GPU 495 -> 466 (the SM clock falls to 1.8 instead of
// 1.65 GHz; the first ten calls take 462 us either way).  At 64 columns the form stays in the instructions: chosen at run time
// it costs chunks 2 % (215 -> 220 us).
constexpr int kFewRows = 16;
template <int D, bool F16, int M>
__device__ constexpr uint32_t idesc_qk() {
    return F16 ? umma_idesc_f16_f32acc(M, 128) : umma_idesc_bf16_f32acc(M, 128);
}
template <int D, bool F16, int M>
__device__ constexpr uint32_t idesc_pv() {
    return (F16 ? umma_idesc_f16_f32acc(M, D) : umma_idesc_bf16_f32acc(M, D)) | (1u << 16);   // V: MN-major
}
// V's tile as an MN-major operand: the 64 columns of a block are one 128-byte row per key, eight keys to 1024 bytes; the
// next 64 columns lie a block of 16 KB on.
__device__ __forceinline__ uint64_t desc_v(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(16384 >> 4) << 16) |
           (static_cast<uint64_t>(1024 >> 4) << 32) | (static_cast<uint64_t>(1) << 46) | (static_cast<uint64_t>(2) << 61);
}
template <int D, bool F16>
__device__ __forceinline__ void products_qk(uint32_t s_tmem, uint32_t q, uint32_t k, uint32_t idesc, uint32_t elected) {
    const uint64_t a = umma_smem_desc_k_sw128(q), b = umma_smem_desc_k_sw128(k);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const uint64_t off = (i >> 2) * (16384 >> 4) + (i & 3) * 2;
        umma_ss_elect(s_tmem, a + off, b + off, idesc, i > 0, elected);
    }
}
template <int D, bool F16>
__device__ __forceinline__ void products_pv(uint32_t o_tmem, uint32_t p_tmem, uint32_t v, uint32_t idesc, bool accumulate, uint32_t elected) {
    const uint64_t b = desc_v(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) umma_ts_elect(o_tmem, p_tmem + i * 8, b + i * (2048 >> 4), idesc, accumulate || i > 0, elected);
}

template <int D>
constexpr uint32_t paged_smem() {
    return 2 * Shape<D>::kTileB + Shape<D>::kRing + 1024 + (uint32_t)((sizeof(Control) + 127) / 128 * 128);
}
static_assert(paged_smem<128>() <= 232448 && paged_smem<64>() <= 232448, "shared memory");
static_assert(kPagedMaxSequences * 12 <= Shape<128>::kRing && kPagedMaxSequences * 12 <= Shape<64>::kRing, "plan's scratch");
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
    const Waiter wait{&c->abort_flag, p.status};

    if (tid == kPgValueWarp * 32) {
#pragma unroll 1
        for (int i = 0; i < 5; ++i) {
            mbar_init(smem_u32(&c->k_full[i]), 1);
            mbar_init(smem_u32(&c->k_empty[i]), 1);
            mbar_init(smem_u32(&c->v_full[i]), 1);
            mbar_init(smem_u32(&c->v_empty[i]), 1);
        }
        mbar_init(smem_u32(&c->q_full), kPgSoftmax / 32);
        mbar_init(smem_u32(&c->together), kPgSoftmax / 32);
#pragma unroll 1
        for (int i = 0; i < kSegments; ++i) {
            mbar_init(smem_u32(&c->seg_full[i]), 1);
            mbar_init(smem_u32(&c->seg_empty[i]), 3 + kPgSoftmax / 32);   // both copying warps, products, softmax warps
        }
#pragma unroll 1
        for (int i = 0; i < 3; ++i) {
            mbar_init(smem_u32(&c->s_full[i]), 1);
            mbar_init(smem_u32(&c->p_full[i]), 4);
        }
#pragma unroll 1
        for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&c->o_full[i >> 1][i & 1]), 1);
        c->abort_flag = (*reinterpret_cast<volatile int*>(p.status) != 0) ? 1 : 0;
        fence_mbar_init();
        p.pieces[2 * blockIdx.x].valid = 0;
        p.pieces[2 * blockIdx.x + 1].valid = 0;
    }
    if (warp == kPgMmaWarp) {
        tmem_alloc(smem_u32(&c->tmem_base), 512);
        tmem_relinquish();
    }
    if (warp == kPgKeyWarp && lane == 0) {
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
        if (p.one_page_box) {
            tma_prefetch_desc(&map_k_page);
            tma_prefetch_desc(&map_v_page);
        }
    }
    __syncwarp();
    const bool few = p.n_sequences <= 32 && !p.rounds;
    long long* line = reinterpret_cast<long long*>(ring);
    Walk walk;
    if (few) {
        if (warp == kPgWalkWarp) plan_few(p, *c, walk);
    } else {
        plan_many(p, *c, line, reinterpret_cast<int*>(line + p.n_sequences));
        fence_proxy_async_smem();                            // the plan's scratch is the copies' ring
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem_base = c->tmem_base;

    if (warp >= kPgMmaWarp) {
        setmaxnreg_dec<kPgControlRegs>();
        if (warp == kPgKeyWarp || warp == kPgValueWarp) {
            // ------------------------------------------------------------------------------------- copies
            // One warp for the keys, one for the values.  A lane looks up the page of its box of a tile, a tile ahead; the
            // copies are issued by one lane, box by box, with operands that are the same in the whole warp (a copy per lane
            // costs a turn of the warp each).
            const bool values = warp == kPgValueWarp;
            const CUtensorMap *map = values ? &map_v : &map_k, *page_map = values ? &map_v_page : &map_k_page;
            uint64_t *full = values ? c->v_full : c->k_full, *empty = values ? c->v_empty : c->k_empty;
            const uint32_t slots = values ? S::kValueSlots : S::kKeySlots;
            const uint32_t ring_addr = smem_u32(ring) + (values ? S::kKeySlots * S::kTileB : 0);
            const uint32_t elected = elect_one();
            bool ok = true, first_round = true;              // (of the ring: nothing to wait for)
            uint32_t slot = 0, phase = 1;                    // the parity of the slot's last release
#pragma unroll 1
            for (uint32_t segment = 0; ok; ++segment) {
                ok = __all_sync(0xffffffffu, wait_segment(*c, segment, wait));
                if (!ok) break;
                const Segment* g = &c->seg[segment % kSegments];
                const int n = g->n, head = g->head, lo = g->lo, hi = g->hi, kt0 = g->kt0;
                const int* pages = p.table + g->seq * p.table_stride;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->seg_empty[segment % kSegments]));
                if (n == 0) break;
                // this lane's box of the next tile to look up; and the tile as a whole, where it lies within a page
                int key = kt0 * 128 + lane * p.box_rows;
                int entry0 = kt0 * 128 / p.page_size, at0 = kt0 * 128 - entry0 * p.page_size;
                int entry = key / p.page_size, at = key - entry * p.page_size;
                int page, page_at;
                uint32_t which, whole;
                auto look_up = [&]() {
                    whole = p.one_page_box && at0 + 128 <= p.page_size;
                    const bool mine = key < hi && (whole ? lane == 0 : lane * p.box_rows < 128 && key + p.box_rows > lo);
                    page = mine ? pages[whole ? entry0 : entry] : 0;
                    page_at = whole ? at0 : at;
                    which = __ballot_sync(0xffffffffu, mine);
                    key += 128, at0 += 128, at += 128;
#pragma unroll 1
                    while (at0 >= p.page_size) at0 -= p.page_size, ++entry0;
#pragma unroll 1
                    while (at >= p.page_size) at -= p.page_size, ++entry;
                };
                look_up();
#pragma unroll 1
                for (int j = 0; j < n; ++j) {
                    int my_page = page;
                    const int my_at = page_at;
                    uint32_t left = which;
                    const int rows = whole ? 128 : p.box_rows;
                    const CUtensorMap* m = whole ? page_map : map;
                    if (j + 1 < n) look_up();
                    if (!first_round) ok = __all_sync(0xffffffffu, wait(&empty[slot], phase));
                    if (!ok) break;
                    if (my_page < 0 || my_page >= p.n_pages) {   // not there: its rows arrive as zeros
                        my_page = -1;
                        atomicCAS(p.status, 0, kStatusRange);
                    }
                    const uint32_t bar = smem_u32(&full[slot]), dst = ring_addr + slot * S::kTileB;
                    if (elected) {
                        if (left) mbar_expect_tx(bar, (uint32_t)(__popc(left) * rows * D * 2));
                        else mbar_arrive(bar);
                    }
                    __syncwarp();
#pragma unroll 1
                    while (left) {
                        const int b = __ffs(left) - 1;
                        left &= left - 1;
                        const int box_page = __shfl_sync(0xffffffffu, my_page, b), box_at = __shfl_sync(0xffffffffu, my_at, b);
                        if (elected) {
#pragma unroll
                            for (int x = 0; x < S::kBlocks; ++x) tma_load_4d(dst + b * rows * 128 + x * 16384, m, x * 64, box_at, head, box_page, bar);
                        }
                    }
                    __syncwarp();
                    if (++slot == slots) {
                        slot = 0;
                        phase ^= 1;
                        first_round = false;
                    }
                }
            }
        } else if (warp == kPgMmaWarp) {
            // ------------------------------------------------------------------------------------- products
            // (the whole warp goes through the loop and one lane issues: operands that are the same in every lane stay in
            // uniform registers)
            {
                const uint32_t elected = elect_one();
                bool ok = true;
                const uint32_t q_addr = smem_u32(sQ), ring_addr = smem_u32(ring);
                uint32_t k_next = 0, k_phase = 0, v_next = 0, v_phase = 0;
                auto take_k = [&](uint32_t& mine) {
                    mine = k_next;
                    const bool got = __all_sync(0xffffffffu, wait(&c->k_full[k_next], k_phase));
                    if (++k_next == S::kKeySlots) k_next = 0, k_phase ^= 1;
                    return got;
                };
                auto take_v = [&](uint32_t& mine) {
                    mine = v_next;
                    const bool got = __all_sync(0xffffffffu, wait(&c->v_full[v_next], v_phase));
                    if (++v_next == S::kValueSlots) v_next = 0, v_phase ^= 1;
                    return got;
                };
                auto release_k = [&](uint32_t e) { umma_commit_elect(smem_u32(&c->k_empty[e]), elected); };
                auto release_v = [&](uint32_t e) { umma_commit_elect(smem_u32(&c->v_empty[e]), elected); };
                // Steps: stream 0 and 1 in turn.  Step i's scores go to buffer i % kScores, as soon as the probabilities of
                // the step that had it are used up.
                uint32_t put = 0, used = 0, phase = 0;   // next buffer to fill, to use; its parity
                uint32_t idesc_s = 0, idesc_o = 0;
                auto scores = [&](uint32_t q, uint32_t k_slot) {
                    products_qk<D, F16>(tmem_base + put * 128, q, ring_addr + k_slot * S::kTileB, idesc_s, elected);
                    umma_commit_elect(smem_u32(&c->s_full[put]), elected);
                    if (++put == S::kScores) put = 0;
                };
                auto output = [&](uint32_t t, uint32_t v_slot, bool accumulate) {
                    if (!__all_sync(0xffffffffu, wait(&c->p_full[used], phase))) return false;
                    tc_fence_after();
                    products_pv<D, F16>(tmem_base + S::kOut + t * D, tmem_base + used * 128,
                                        ring_addr + (S::kKeySlots + v_slot) * S::kTileB, idesc_o, accumulate, elected);
                    if (++used == S::kScores) used = 0, phase ^= 1;
                    return true;
                };
                uint32_t visit0 = 0, visit1 = 0;
#pragma unroll 1
                for (uint32_t segment = 0; ok; ++segment) {
                    ok = __all_sync(0xffffffffu, wait_segment(*c, segment, wait));
                    if (!ok) break;
                    const Segment* at = &c->seg[segment % kSegments];
                    const bool two = at->rows > 128;
                    const int n = at->n, steps = two ? 2 * n : n;
                    const bool few_rows = D == 128 && at->rows <= kFewRows;
                    idesc_s = few_rows ? idesc_qk<D, F16, 64>() : idesc_qk<D, F16, 128>();
                    idesc_o = few_rows ? idesc_pv<D, F16, 64>() : idesc_pv<D, F16, 128>();
                    __syncwarp();
                    if (elected) mbar_arrive(smem_u32(&c->seg_empty[segment % kSegments]));
                    if (n == 0) break;
                    uint32_t k = 0, v = 0;
                    ok = __all_sync(0xffffffffu, wait(&c->q_full, segment));
                    // with two tiles of rows a tile of keys is taken by an even step and released by the odd one behind it
#pragma unroll 1
                    for (int i = -S::kScores; ok && i < steps; ++i) {
                        // what does not depend on the probabilities first; behind them only the products and, last, what
                        // others wait for less urgently
                        const bool odd = i & 1;
                        const int ahead = i + S::kScores;
                        const bool second = ahead & 1, more = ahead < steps;
                        if (i >= 0 && (!two || !odd)) ok = take_v(v);
                        if (ok && more && two && !second) ok = take_k(k);
                        if (ok && i >= 0) ok = output(odd, v, i > 1);
                        if (ok && i >= 0) {
                            // with two tiles of scores a stream's scores come behind its products so far: only the last need telling
                            if (S::kScores == 3 || ahead >= steps) {
                                const uint32_t visit = odd ? visit1++ : visit0++;
                                umma_commit_elect(smem_u32(&c->o_full[odd][visit & 1]), elected);
                            }
                            if (!two || odd) release_v(v);
                        }
                        if (ok && more && !two) ok = take_k(k);   // (single tokens wait for keys, not for probabilities)
                        if (!ok) break;
                        if (more) {
                            tc_fence_after();
                            scores(q_addr + (two && second ? S::kTileB : 0), k);
                            if (!two || second) release_k(k);
                        }
                    }
                }
            }
        } else if (warp == kPgWalkWarp) {
            // ------------------------------------------------------------------------------------- the work, stretch by stretch
            walk.round = 0;
            if (!few) {
                plan_start(p, *c, line, walk);
                fence_proxy_async_smem();
                __syncwarp();
            }
            if (lane == 0) {
                bool more = true, ok = true;
#pragma unroll 1
                for (uint32_t segment = 0; ok && more; ++segment) {
                    Segment g;
                    more = walk.next(p, *c, g);
                    if (!more) g.n = 0;
                    const uint32_t slot = segment % kSegments, round = segment / kSegments;
                    if (round > 0) ok = wait(&c->seg_empty[slot], round - 1);
                    if (!ok) break;
                    c->seg[slot] = g;
                    mbar_arrive(smem_u32(&c->seg_full[slot]));
                }
            }
        }
    } else {
        // ----------------------------------------------------------------------------------------- softmax
        setmaxnreg_inc<kPgSoftmaxRegs>();
        const int t = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t t_O = lane_base + S::kOut + t * D;
        const float scale = p.scale_log2;
        const uint64_t scale2 = pack2(scale, scale);
        uint32_t entry = 0, steps = 0, visit = 0, met = 0;
        // all softmax warps have come here (with a limit, like every wait: a wait that runs out ends the warp's work)
        auto meet_all = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c->together));
            return __all_sync(0xffffffffu, wait(&c->together, met++));
        };
        bool ok = true;
#pragma unroll 1
        for (uint32_t segment = 0; ok; ++segment) {
            ok = __all_sync(0xffffffffu, wait_segment(*c, segment, wait));
            if (!ok) break;
            const Segment& g = c->seg[segment % kSegments];
            const int n = g.n;
            if (n == 0) break;
            const bool two = g.rows > 128;
            const int first = two ? t * 128 : 0;
            ok = meet_all();                                 // the last segment's queries and tensor memory are done with
            if (!ok) break;
            {
                // a thread has one 16-byte piece of every kStep-th row, and loads them all before it stores the first
                constexpr int kPer = D / 8, kRowsAtOnce = 128 / kPer, kMost = 128 / kRowsAtOnce;
                const int step = two ? kRowsAtOnce : 2 * kRowsAtOnce, mine = two ? kMost : kMost / 2;
                const int id = two ? (tid & 127) : tid, ch = id % kPer, r0 = id / kPer;
                uint8_t* dst = sQ + (two ? t * S::kTileB : 0) + (ch >> 3) * 16384;
                const int in_seq = g.tile * kPagedRows + first + r0;
                int token = in_seq / p.share, h = in_seq - token * p.share;
                const int step_token = step / p.share, step_h = step - step_token * p.share;
                const uint16_t* q = reinterpret_cast<const uint16_t*>(p.q) + g.q.row0 * p.q_token + g.head * p.share * p.q_head + ch * 8;
                const int rows = g.rows - first;
                uint4 v[kMost];
#pragma unroll
                for (int i = 0; i < kMost; ++i) {
                    v[i] = make_uint4(0, 0, 0, 0);
                    if (i < mine && r0 + i * step < rows) v[i] = *reinterpret_cast<const uint4*>(q + token * p.q_token + h * p.q_head);
                    token += step_token, h += step_h;
                    if (h >= p.share) h -= p.share, ++token;
                }
#pragma unroll
                for (int i = 0; i < kMost; ++i)
                    if (i < mine) *reinterpret_cast<uint4*>(dst + sw128_offset(r0 + i * step, ch & 7)) = v[i];
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->q_full));
            }
            const int in_seq = g.tile * kPagedRows + first + row, token = in_seq / p.share;
            const bool valid = first + row < g.rows, busy = first + (warp & 3) * 32 < g.rows;   // busy: any row of the warp
            const int key_first = g.kt0 * 128, all_lo = g.lo - key_first, all_hi = g.hi - key_first;
            int lo = all_lo, hi = all_hi;                    // keys that this row sees, from key_first on (not a row: any)
            if (valid) {
                const int pos = g.q.keys - g.q.tokens + token;
                lo = sees_begin(p, pos) - key_first;
                hi = sees_end(p, g.q.keys, pos) - key_first;
            }
            // tiles that all rows of the warp see whole
            const int open0 = (__reduce_max_sync(0xffffffffu, max(lo, 0)) + 127) / 128, open1 = __reduce_min_sync(0xffffffffu, max(hi, 0)) / 128;
            float m = valid ? -INFINITY : 0.0f, l = 0.0f;    // (what is not a row never asks for another reference)
            bool fresh = true;                               // some row of the warp has not seen a key yet
            int done = 0;                                    // tiles of this stream
#pragma unroll 1
            for (int j = two ? 0 : t; j < n; j += two ? 1 : 2) {
                const uint32_t step = steps + (two ? 2 * j + t : j), buffer = step % S::kScores, t_S = lane_base + buffer * 128;
                ok = __all_sync(0xffffffffu, wait(&c->s_full[buffer], step / S::kScores));
                if (!ok) break;
                tc_fence_after();
                const int from = lo - 128 * j, to = hi - 128 * j;
                const bool masked = j < open0 || j >= open1;
                if (masked) {
                    if ((128 * j < all_lo || 128 * j + 128 > all_hi) && (!two || t == 0)) {
                        // rows of V that no row of the item sees; with two tiles of rows stream 0 does it for both (its products
                        // are issued first)
                        const uint32_t e = entry + j;
                        ok = __all_sync(0xffffffffu, wait(&c->v_full[e % S::kValueSlots], e / S::kValueSlots));
                        if (!ok) break;
                        const int key = 128 * j + row;
                        if (key < all_lo || key >= all_hi) {
                            uint8_t* v = ring + (S::kKeySlots + e % S::kValueSlots) * S::kTileB + row * 128;
#pragma unroll
                            for (int x = 0; x < S::kBlocks; ++x)
#pragma unroll
                                for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(v + x * 16384 + ((i + row) & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async_smem();
                    }
                }
                uint32_t s[128];
                if (busy) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) tmem_ld32(t_S + 32 * b, s + 32 * b);
                    tmem_wait_ld();
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 128; ++i)
                            if (i < from || i >= to) s[i] = 0xff800000u;   // -inf, whatever was there
                    }
                    auto highest = [&]() {
                        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int i = 0; i < 128; i += 8)
#pragma unroll
                            for (int b = 0; b < 4; ++b) mx[b] = max3(mx[b], __uint_as_float(s[i + 2 * b]), __uint_as_float(s[i + 2 * b + 1]));
                        return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                    };
                    // rows that have not seen a key yet take their reference from the tile's maximum
                    bool again;
                    if (fresh) {
                        const float top = highest() - below_top<F16>();
                        if (m == -INFINITY) m = top;
                        fresh = __any_sync(0xffffffffu, m == -INFINITY);
                    }
                    float sum;
#pragma unroll 1
                    while (true) {
                        const float ref = m == -INFINITY ? 0.0f : m;
                        uint64_t sum_a = 0, sum_b = 0;
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            uint32_t pr[16];
                            probabilities<F16>(s + 32 * b, scale2, pack2(-ref, -ref), pr, sum_a, sum_b);
                            tmem_st16(t_S + 16 * b, pr);
                        }
                        float s0, s1;
                        unpack2(add2(sum_a, sum_b), s0, s1);
                        sum = s0 + s1;
                        again = valid && !(sum < raise_at<F16>());
                        if (!__any_sync(0xffffffffu, again)) break;
                        // Rare: scores far above the reference.  O and the sum are brought to the new reference, and the tile
                        // is done again.
                        const float top = highest() - below_top<F16>();
                        again = again && top > m;            // (a NaN among the scores stays one)
                        if (!__any_sync(0xffffffffu, again)) break;
                        const float alpha = again ? ex2_approx(ref - top) : 1.0f;
                        if (again) m = top;
                        l *= alpha;
                        if (done > 0) {
                            // (with two tiles of scores these came behind the stream's products so far)
                            if (S::kScores == 3) {
                                ok = __all_sync(0xffffffffu, wait(&c->o_full[t][(visit - 1) & 1], (visit - 1) >> 1));
                                tc_fence_after();
                            }
#pragma unroll 1
                            for (int b = 0; ok && b < D; b += 16) {
                                uint32_t o[16];
                                tmem_ld16(t_O + b, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tmem_st16(t_O + b, o);
                            }
                        }
                    }
                    l += sum;
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&c->p_full[buffer]));
                if (!ok) break;
                if (S::kScores == 3) ++visit;
                ++done;
            }
            if (!ok) break;
            entry += n;                                      // V tiles so far
            steps += two ? 2 * n : n;

            // ------------------------------------------------------------------------------------- results
            if (done > 0) {
                if (S::kScores == 2) ++visit;                // (told once, at the end)
                ok = __all_sync(0xffffffffu, wait(&c->o_full[t][(visit - 1) & 1], (visit - 1) >> 1));
                if (!ok) break;
                tc_fence_after();
            }
            float a[2] = {1.0f, 1.0f};                       // weights of the two streams' sums
            if (!two) {
                float2* ml = reinterpret_cast<float2*>(sQ + S::kTileB);   // (the second tile of queries is not in use)
                ml[t * 128 + row] = make_float2(m, l);
                tc_fence_before();
                ok = meet_all();
                if (!ok) break;
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
            const bool alone = g.starts && g.ends;
            const int piece = 2 * blockIdx.x + (g.starts ? 1 : 0);
            const int part_row = first + row;
            const float inv = l > 0.0f ? 1.0f / l : l;       // 0: sees nothing; NaN: a score was NaN, and so is the row
            const long long out_row = g.q.row0 + token;
            const int h = g.head * p.share + in_seq - token * p.share;
            uint16_t* out = reinterpret_cast<uint16_t*>(p.out) + out_row * p.out_token + h * p.out_head;
            // this thread's columns: all of its stream's row, or half of the joined row
            const int col0 = two ? 0 : t * (D / 2), cols = two ? D : D / 2;
            if (busy) {
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
                        tmem_ld32(lane_base + S::kOut + col0 + b, o);
                        tmem_ld32(lane_base + S::kOut + D + col0 + b, o1);
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
                    else if (p.lse) p.lse[out_row * p.n_q_heads + h] = log_sum<F16>(m, l);
                }
            }
            if (!alone && tid == 0) {
                PagedPiece d;
                d.valid = 1, d.ends = g.ends;
                d.seq_row0 = g.q.row0, d.first_row = g.tile * kPagedRows, d.rows = g.rows, d.head = g.head;
                p.pieces[piece] = d;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&c->seg_empty[segment % kSegments]));
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
#pragma unroll 1
            while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
        }
        __syncwarp();
        tmem_dealloc(tmem_base, 512);
    }
}

// Joins the pieces of an item: block (x, y) the item that thread block x of the attention began and did not end, 32 of its
// rows.  The pieces are this one and the ones that the following thread blocks left in their slot 0, up to the one that ends
// the item, in that order.  Bound by latencies (the blocks start when the attention's have left the SMs, whose registers are
// all taken): the descriptions of all pieces are read at once, and the pieces of four rows side by side.
constexpr int kJoinRows = 32, kJoinThreads = 256;
template <int D, bool F16>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const PagedAttnParams p, const int grid) {
    constexpr int kRowsAtOnce = kJoinThreads / (D / 4), kTurns = kJoinRows / kRowsAtOnce;
    constexpr int kWarps = kJoinThreads / 32;
    static_assert(kPagedMaxGrid <= 32 * kWarps, "a thread per piece");
    __shared__ int slots[kPagedMaxGrid + 1];
    __shared__ uint32_t valid_at[kWarps], ends_at[kWarps];
    __shared__ int n_pieces;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row0 = blockIdx.y * kJoinRows, next = blockIdx.x + 1 + threadIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const PagedPiece first = p.pieces[2 * blockIdx.x + 1];
    int valid = 0, ends = 0;
    if (next < grid) valid = p.pieces[2 * next].valid, ends = p.pieces[2 * next].ends;
    if (!first.valid || row0 >= first.rows) return;
    const uint32_t v = __ballot_sync(0xffffffffu, valid), e = __ballot_sync(0xffffffffu, valid && ends);
    if (lane == 0) valid_at[warp] = v, ends_at[warp] = e;
    if (threadIdx.x == 0) n_pieces = 0;
    __syncthreads();
    {   // this thread's piece, if it is one of the item's: the valid ones before it, and none of those ends the item
        int before = 0;
        bool in = valid;
        for (int w = 0; w < warp; ++w) before += __popc(valid_at[w]), in = in && !ends_at[w];
        const uint32_t below = (1u << lane) - 1;
        before += __popc(v & below);
        in = in && !(e & below);
        if (in) slots[1 + before] = 2 * next;
        if (in && ends) n_pieces = 2 + before;
        if (threadIdx.x == 0) slots[0] = 2 * blockIdx.x + 1;
    }
    __syncthreads();
    const int n = n_pieces, c4 = threadIdx.x / kRowsAtOnce;
    if (n == 0) return;                                      // (a thread block gave up on a wait: the end is not there)
    float m[kTurns], l[kTurns];
    float4 o[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) m[t] = -INFINITY, l[t] = 0.0f, o[t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
    for (int i = 0; i < n; ++i) {
        const float2* ml = p.part_ml + (size_t)slots[i] * kPagedRows + row0 + threadIdx.x % kRowsAtOnce;
        const float4* po = p.part_o + ((size_t)slots[i] * (D / 4) + c4) * kPagedRows + row0 + threadIdx.x % kRowsAtOnce;
        float2 x[kTurns];
        float4 y[kTurns];
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {                   // (rows behind the last are in the workspace too, whatever they hold)
            x[t] = ml[t * kRowsAtOnce];
            y[t] = po[t * kRowsAtOnce];
        }
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const float top = fmaxf(m[t], x[t].x);
            const float a = m[t] == -INFINITY ? 0.0f : ex2_approx(m[t] - top), b = x[t].x == -INFINITY ? 0.0f : ex2_approx(x[t].x - top);
            m[t] = top;
            l[t] = a * l[t] + b * x[t].y;
            o[t].x = a * o[t].x + (b == 0.0f ? 0.0f : b * y[t].x);
            o[t].y = a * o[t].y + (b == 0.0f ? 0.0f : b * y[t].y);
            o[t].z = a * o[t].z + (b == 0.0f ? 0.0f : b * y[t].z);
            o[t].w = a * o[t].w + (b == 0.0f ? 0.0f : b * y[t].w);
        }
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int row = row0 + t * kRowsAtOnce + threadIdx.x % kRowsAtOnce;
        if (row >= first.rows) continue;
        const float inv = l[t] > 0.0f ? 1.0f / l[t] : l[t];
        const int in_seq = first.first_row + row, token = in_seq / p.share;
        const long long out_row = first.seq_row0 + token;
        const int h = first.head * p.share + in_seq - token * p.share;
        const uint2 w = make_uint2(pack_pair<F16>(o[t].x * inv, o[t].y * inv), pack_pair<F16>(o[t].z * inv, o[t].w * inv));
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p.out) + out_row * p.out_token + h * p.out_head + c4 * 4) = w;
        if (p.lse && c4 == 0) p.lse[out_row * p.n_q_heads + h] = log_sum<F16>(m[t], l[t]);
    }
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
    cfg.gridDim = dim3((unsigned)grid, (unsigned)(kPagedRows / kJoinRows));
    cfg.blockDim = dim3(kJoinThreads);
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
    const int grid = paged_attn_grid(sm_count);
    *launches = 0;
    if (head_dim == 128)
        return f16 ? launch_one<128, true>(maps, p, grid, launches, stream) : launch_one<128, false>(maps, p, grid, launches, stream);
    return f16 ? launch_one<64, true>(maps, p, grid, launches, stream) : launch_one<64, false>(maps, p, grid, launches, stream);
}

}  // namespace regenvc
