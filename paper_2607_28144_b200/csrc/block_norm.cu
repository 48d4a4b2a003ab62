// Norms before and after a transformer block, fused with the block's gate and residual scale, and their gradients.
//
//     z  = N2(y) pw  (or y pw)       x' = a x + g z          h = (N1(x') w + b) (1 + s) + t
//
// N is layer norm ((v - mean) r, r = 1 / sqrt(var + eps)) or RMS norm (v r, r = 1 / sqrt(mean v^2 + eps)); g, s, t are
// rows of a modulation table shared by tokens_per_mod consecutive tokens.  With xhat = N1(x'), yhat = N2(y):
//
//     d  = dh (1 + s) w                                dx' = r (d - [layer] mean(d) - xhat mean(d xhat)) + dx'_in
//     dt = S0,  ds = w S1 + b S0,                      dw = sum_rows (1 + s) S1,  db = sum_rows (1 + s) S0
//     dz = g dx',  dy = N2's gradient of dz pw         dg = pw S2,  dpw = sum_rows g S2,    dx = a dx'
//     S0 = sum dh,  S1 = sum dh xhat,  S2 = sum dx' yhat  over the tokens of one modulation row
//
// Bound: HBM (every tensor is read or written once; 8 bytes per element forward in bf16).  A thread block owns a
// contiguous range of tokens and a thread sixteen fixed columns, for two reasons: the modulation, weight and bias values
// of a column stay in registers over all tokens that share them (read per token they would be 12 bytes of fp32 against
// 8 bytes of tokens), and the backward pass can sum over tokens in registers too, without atomics, in an order that
// depends on the shape and the device alone.  Statistics take two passes over registers (mean, then centred squares) in fp32.
//
// What a row costs beside its bytes is instructions: with eight columns per thread and plain fp32 the forward kernel
// issued 299 per warp and row and kept the schedulers busy for two thirds of its 41 us (10920 x 1536 bf16, HBM at 0.27).
// Hence sixteen columns per thread, which halves the share of the sums' exchanges, arithmetic on pairs (f32x2), and
// asynchronous copies of the rows ahead into a ring in shared memory, which takes no registers: 16-bit rows by the thread
// that reads them (no barrier), fp32 rows by its warp, rows of odd width or address as images of 16-byte words by the block.
// Measured: 10920 x 1536 bf16 with residual, gate and modulation 28.7 us (4.7 TB/s of 6.45 measured), 31200 x 5120 with an
// fp32 stream and RMS norms on both sides 324 us in bursts and 331 under the power cap (5.9 and 5.8 TB/s); gradients
// 49.1 us (4.1 TB/s) and, at 12480 x 5120, 279 us (4.1 TB/s): there the three sums per column take the registers that more
// rows in flight would need.
#include "block_norm.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kCols = 16;            // columns per thread
constexpr int kPairs = kCols / 2;
typedef uint64_t f32x2;

__device__ __forceinline__ f32x2 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float low(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return a;
}
__device__ __forceinline__ float join(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

// 16 bytes, or 16 zeros without a read where bytes is 0 (dead columns).
__device__ __forceinline__ void copy_async16(uint32_t smem, const void* global, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(global), "r"(bytes) : "memory");
}
__device__ __forceinline__ void store16_if(bool on, void* p, uint4 v) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %0, 0;\n\t@q st.global.v4.b32 [%1], {%2, %3, %4, %5};\n\t}"
                 ::"r"((uint32_t)on), "l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until at most `stages` - 1 of this thread's groups are under way.
__device__ __forceinline__ void copy_wait(int stages) {
    if (stages == 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// Where a thread's columns are.  VEC: two groups of eight neighbouring ones, `threads` groups apart (16-byte accesses of
// neighbouring threads are neighbours).  Otherwise, where sizes, strides or addresses do not allow that: sixteen columns
// `threads` apart.
template <bool VEC>
struct Place {
    int tid, threads;
    unsigned live;   // VEC: bit per group, else bit per column
    __device__ __forceinline__ explicit Place(int channels) : tid(threadIdx.x), threads(blockDim.x), live(0) {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < 2; ++j) live |= (col(8 * j) < channels ? 1u : 0u) << j;
        } else {
#pragma unroll
            for (int i = 0; i < kCols; ++i) live |= (col(i) < channels ? 1u : 0u) << i;
        }
    }
    __device__ __forceinline__ int col(int i) const {
        return VEC ? ((i >> 3) * threads + tid) * 8 + (i & 7) : i * threads + tid;
    }
    __device__ __forceinline__ bool on(int i) const { return live >> (VEC ? i >> 3 : i) & 1; }
    // v in the live columns, 0 in the others
    __device__ __forceinline__ f32x2 masked(int pair, float v) const {
        if constexpr (VEC) return both(on(2 * pair) ? v : 0.0f);
        else return pack2(on(2 * pair) ? v : 0.0f, on(2 * pair + 1) ? v : 0.0f);
    }
};

// Bytes of a row's image: the row and what 16-byte words add at its ends.
__host__ __device__ __forceinline__ uint32_t image_bytes(int channels, size_t size) {
    return ((uint32_t)(channels * size) + 15) / 16 * 16 + 16;
}
// Bytes of one thread's columns of a row of T.
template <typename T>
constexpr uint32_t kMine = kCols * sizeof(T);

// One tensor's rows, taken in order.  Where rows allow 16-byte accesses they are copied ahead into this warp's part of a ring stage (16-byte words of
// neighbouring lanes are neighbours in global and in shared memory: word w of a warp's data is lane w % 32's copy
// number w / 32).  A 16-bit lane reads back its own words.  An fp32 group of eight columns is two words: lane l reads
// words 2l and 2l + 1, which other lanes of its warp copied, so a warp synchronises behind its waits; the words of every
// other eight are swapped in pairs, which keeps those reads off each other's banks.
template <typename T, bool VEC, uint32_t AT, int MAXT>
struct Rows;
template <typename T, uint32_t AT, int MAXT>
struct Rows<T, true, AT, MAXT> {
    enum { kWords = (int)sizeof(T) / 2 };   // 16-byte words per lane and group
    const T* next;        // this thread's first word of the row to fetch next
    long long stride;
    uint32_t bytes;       // what each of the copies moves, a byte of this number for each (16, or 0 in dead columns)
    __device__ __forceinline__ Rows(const void* base, long long row_stride, int row0, const Place<true>& at, const BlockNormParams& p, uint32_t&)
        : next(nullptr), stride(row_stride), bytes(0) {
        if (!base) return;
        const T* row = reinterpret_cast<const T*>(base) + row0 * row_stride;
        const int first = word_column(at, 0, 0);
        next = row + (first < p.channels ? first : 0);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int k = 0; k < kWords; ++k)
                bytes |= (word_column(at, j, k) < p.channels ? 16u : 0u) << (j * kWords + k) * 8;
    }
    // First column of the word that this lane copies as its k-th of group j.
    static __device__ __forceinline__ int word_column(const Place<true>& at, int j, int k) {
        return ((j * at.threads + (at.tid & ~31)) * kWords + k * 32 + (at.tid & 31)) * (16 / (int)sizeof(T));
    }
    static __device__ __forceinline__ uint32_t word_place(uint32_t w) { return kWords == 1 ? w : w ^ (w >> 3 & 1); }
    // `stage`: the stage's address plus this warp's share, 16 bytes per lane (the part of group j, copy k is a constant on)
    __device__ __forceinline__ void fetch(const Place<true>& at, uint32_t stage) {
        {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < kWords; ++k) {
                    const uint32_t size = bytes >> (j * kWords + k) * 8 & 0xFFu;
                    copy_async16(stage + AT * MAXT + j * (MAXT * kWords * 16) + (at.tid >> 5) * (kWords * 512) +
                                     word_place(k * 32 + (at.tid & 31)) * 16,
                                 next + (size ? j * at.threads * 8 + k * (32 * 16 / (int)sizeof(T)) : 0), size);
                }
            next += stride;
        }
    }
    __device__ __forceinline__ void read(const Place<true>& at, uint32_t stage, f32x2* v) {
        {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                Raw8<T> r;
#pragma unroll
                for (int k = 0; k < kWords; ++k)
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(r.w[k].x), "=r"(r.w[k].y), "=r"(r.w[k].z), "=r"(r.w[k].w)
                                 : "r"(stage + AT * MAXT + j * (MAXT * kWords * 16) + (at.tid >> 5) * (kWords * 512) +
                                       word_place((at.tid & 31) * kWords + k) * 16) : "memory");
                float e[8];
                widen8(r, e);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * j + i] = pack2(e[2 * i], e[2 * i + 1]);
            }
        }
    }
    __device__ __forceinline__ void done() {}
};
// The other rows (odd widths, strides or addresses): every 16-byte word that a row touches is copied into an image of the
// row in the stage, by whichever thread comes to it, and the elements are read from there wherever they fall.  Words are
// whole 16-byte words of global memory, cut off at the tensor's last element; the one that would begin before its first
// element goes element by element.
template <typename T, uint32_t AT, int MAXT>
struct Rows<T, false, AT, MAXT> {
    uintptr_t first, end, next, here;   // the tensor's ends, the row to fetch next and the one to read
    long long step;
    uint32_t place, width;
    __device__ __forceinline__ Rows(const void* base, long long row_stride, int row0, const Place<false>&, const BlockNormParams& p,
                                    uint32_t& used)
        : first((uintptr_t)base), step(row_stride * (long long)sizeof(T)), place(used), width(p.channels * (uint32_t)sizeof(T)) {
        end = first + (uintptr_t)(p.n_tokens - 1) * (uintptr_t)step + width;
        next = here = first + (uintptr_t)row0 * (uintptr_t)step;
        if (base) used += image_bytes(p.channels, sizeof(T));
    }
    __device__ __forceinline__ void fetch(const Place<false>& at, uint32_t stage) {
        const uintptr_t from = next & ~(uintptr_t)15, to = next + width;
        for (uint32_t w = at.tid; from + 16 * w < to; w += at.threads) {
            const uintptr_t g = from + 16 * w;
            const uint32_t s = stage + place + 16 * w;
            if (g >= first) {
                copy_async16(s, reinterpret_cast<const void*>(g), end - g < 16 ? (uint32_t)(end - g) : 16u);
            } else {
                for (uintptr_t e = first; e < g + 16 && e < end; e += sizeof(T)) store_shared(s + (uint32_t)(e - g), *reinterpret_cast<const T*>(e));
            }
        }
        next += (uintptr_t)step;
    }
    static __device__ __forceinline__ void store_shared(uint32_t a, T v) {
        if constexpr (sizeof(T) == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(__float_as_uint(v)) : "memory");
        else asm volatile("st.shared.u16 [%0], %1;" ::"r"(a), "h"(*reinterpret_cast<const uint16_t*>(&v)) : "memory");
    }
    static __device__ __forceinline__ float load_shared(uint32_t a) {
        if constexpr (sizeof(T) == 4) {
            uint32_t u;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(u) : "r"(a) : "memory");
            return __uint_as_float(u);
        } else {
            uint16_t u;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(a) : "memory");
            return to_f32(*reinterpret_cast<const T*>(&u));
        }
    }
    __device__ __forceinline__ void read(const Place<false>& at, uint32_t stage, f32x2* v) {
        const uint32_t a = stage + place + (uint32_t)(here & 15) + at.tid * (uint32_t)sizeof(T);
        float e[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i) e[i] = at.on(i) ? load_shared(a + i * at.threads * (uint32_t)sizeof(T)) : 0.0f;
#pragma unroll
        for (int i = 0; i < kPairs; ++i) v[i] = pack2(e[2 * i], e[2 * i + 1]);
    }
    __device__ __forceinline__ void done() { here += (uintptr_t)step; }   // with the row that read() reads
};
// A result's rows, written in order.
template <typename T, bool VEC>
struct Results {
    T* next;
    long long stride;
    __device__ __forceinline__ Results(void* base, long long row_stride, int row0, const Place<VEC>& at)
        : next(reinterpret_cast<T*>(base) + (base ? row0 * row_stride + at.col(0) : 0)), stride(row_stride) {}
    __device__ __forceinline__ void write(const Place<VEC>& at, const f32x2* v) {
        float e[kCols];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) unpack2(v[i], e[2 * i], e[2 * i + 1]);
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                T* to = next + j * at.threads * 8;
                const float* x = e + 8 * j;
                if constexpr (sizeof(T) == 4) {
                    store16_if(at.on(8 * j), to, make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])));
                    store16_if(at.on(8 * j), to + 4, make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])));
                } else {
                    const T* tag = nullptr;
                    store16_if(at.on(8 * j), to, make_uint4(narrow2(x[0], x[1], tag), narrow2(x[2], x[3], tag), narrow2(x[4], x[5], tag), narrow2(x[6], x[7], tag)));
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kCols; ++i)
                if (at.on(i)) from_f32(e[i], next[i * at.threads]);
        }
        next += stride;
    }
};
// A vector of parameters at this thread's columns; `absent` without one and in dead columns.
template <bool VEC>
__device__ __forceinline__ void read_vector(const float* base, float absent, const Place<VEC>& at, f32x2* v) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = both(absent);
    if (base == nullptr) return;
    if constexpr (VEC) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (at.on(8 * j))
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float4 q = __ldg(reinterpret_cast<const float4*>(base + at.col(8 * j)) + k);
                    v[4 * j + 2 * k] = pack2(q.x, q.y);
                    v[4 * j + 2 * k + 1] = pack2(q.z, q.w);
                }
    } else {
#pragma unroll
        for (int i = 0; i < kPairs; ++i)
            v[i] = pack2(at.on(2 * i) ? __ldg(base + at.col(2 * i)) : absent, at.on(2 * i + 1) ? __ldg(base + at.col(2 * i + 1)) : absent);
    }
}

// Sums over the thread block, the same value in every thread, in a fixed order.  Two buffers used in turn make one
// barrier per sum enough: a buffer is written again only behind the next sum's barrier.  WARPS: the build's most; the
// warps' parts are read back without a loop, all in flight (as a loop over the launched warps every value waited for shared
// memory two or three times: 31200 x 5120 forward 358 us instead of 324, 12480 x 5120 gradients 340 instead of 279).
template <int WARPS>
struct BlockSum {
    float (*buf)[4][16];   // [2 buffers][4 values][warp]
    int warps, turn;
    template <int N>
    __device__ __forceinline__ void run(float* v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
        if (warps == 1) return;
        float (*b)[16] = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) b[n][threadIdx.x >> 5] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float4 q = *reinterpret_cast<const float4*>(&b[n][0]);
            float s = (q.x + q.y) + (q.z + q.w);
#pragma unroll
            for (int w = 4; w < WARPS; w += 4) {   // (no such warp: 0)
                const float4 r = *reinterpret_cast<const float4*>(&b[n][w]);
                s += (r.x + r.y) + (r.z + r.w);
            }
            v[n] = s;
        }
    }
};
template <int WARPS>
__device__ __forceinline__ BlockSum<WARPS> block_sum_init(float (*buf)[4][16]) {
    for (int i = threadIdx.x; i < 128; i += blockDim.x) (&buf[0][0][0])[i] = 0.0f;   // entries past the last warp stay 0
    __syncthreads();
    return BlockSum<WARPS>{buf, (int)(blockDim.x + 31) / 32, 0};
}

// s / channels with one step of residual correction (Markstein's): exact where the quotient is an fp32 value, as a constant
// row's mean is, which the product with the reciprocal alone may miss by an ulp.  An infinite s stays infinite (the residual
// would be inf - inf): a row whose sum of squares passes fp32's range then has r = 0 and normalises to 0.
struct Channels {
    float n, inverse;
    __device__ __forceinline__ explicit Channels(int channels) : n((float)channels), inverse(1.0f / (float)channels) {}
    __device__ __forceinline__ float mean(float s) const {
        const float q = s * inverse;
        return fabsf(q) < __uint_as_float(0x7F800000u) ? fmaf(fmaf(-q, n, s), inverse, q) : q;
    }
};

// This thread's share of a row's sum, and of the sum of its squares.
__device__ __forceinline__ float total(const f32x2* v) {
    f32x2 t = add2(v[0], v[1]), u = add2(v[2], v[3]);
#pragma unroll
    for (int i = 4; i < kPairs; i += 2) {
        t = add2(t, v[i]);
        u = add2(u, v[i + 1]);
    }
    return join(add2(t, u));
}
__device__ __forceinline__ float total_squares(const f32x2* v) {
    f32x2 t = mul2(v[0], v[0]), u = mul2(v[1], v[1]);
#pragma unroll
    for (int i = 2; i < kPairs; i += 2) {
        t = fma2(v[i], v[i], t);
        u = fma2(v[i + 1], v[i + 1], u);
    }
    return join(add2(t, u));
}
// v - mean in the live columns (dead ones hold and keep 0)
template <bool VEC>
__device__ __forceinline__ void subtract(f32x2* v, float mean, const Place<VEC>& at) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = add2(v[i], at.masked(i, -mean));
}
// Layer norm's mean carries the rounding of its sum, up to 24 u of the row's magnitude, which counts where that magnitude is
// far above the deviation (a constant fp32 row of 12345.678 came out as +-0.7 at eps 1e-6 instead of 0).  The centred values'
// mean is that error: it goes out of the values, and its square out of their squares' mean.
__device__ __forceinline__ float variance(float mean_squares, float error) {
    const float v = fmaf(-error, error, mean_squares);
    return v < 0.0f ? 0.0f : v;
}
// v -> normalised v
template <bool VEC, typename SUM>
__device__ __forceinline__ void normalise(f32x2* v, int kind, float eps, const Channels& ch, const Place<VEC>& at, SUM& sum) {
    float s[2], var;
    if (kind == kNormLayer) {
        s[0] = total(v);
        sum.template run<1>(s);
        subtract<VEC>(v, ch.mean(s[0]), at);
        s[0] = total_squares(v);
        s[1] = total(v);
        sum.template run<2>(s);
        const float error = ch.mean(s[1]);
        subtract<VEC>(v, error, at);
        var = variance(ch.mean(s[0]), error);
    } else {
        s[0] = total_squares(v);
        sum.template run<1>(s);
        var = ch.mean(s[0]);
    }
    const f32x2 r = both(rsqrtf(var + eps));
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = mul2(v[i], r);
}

// A vector of this thread's columns that the gradients' rows share: in shared memory (only this thread reads and writes
// it), or in registers in the build of 160 to 320 threads, which has one block per SM, registers to spare and, without
// these 40 KB, room for a third row ahead (12480 x 5120 sandwich: 333 -> 321 us).
template <int MAXT, bool REGS>
struct Kept {
    float4* mem;
    __device__ __forceinline__ void set(const f32x2* v) {
#pragma unroll
        for (int i = 0; i < kPairs / 2; ++i) {
            float4 q;
            unpack2(v[2 * i], q.x, q.y);
            unpack2(v[2 * i + 1], q.z, q.w);
            mem[i * MAXT + threadIdx.x] = q;
        }
    }
    __device__ __forceinline__ void get(int i, f32x2* a, f32x2* b) const {   // pairs 2i and 2i + 1
        const float4 q = mem[i * MAXT + threadIdx.x];
        *a = pack2(q.x, q.y);
        *b = pack2(q.z, q.w);
    }
};
template <int MAXT>
struct Kept<MAXT, true> {
    f32x2 r[kPairs];
    __device__ __forceinline__ void set(const f32x2* v) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) r[i] = v[i];
    }
    __device__ __forceinline__ void get(int i, f32x2* a, f32x2* b) const {
        *a = r[2 * i];
        *b = r[2 * i + 1];
    }
};
// The rows of up to four tensors copied ahead: `stages` rows' worth of shared memory in turn.  A stage is filled again one
// row after it was read, behind that row's barriers.
struct Ring {
    int stages;
    uint32_t bytes;      // of a stage
};

// Starts the copies into the stage that was read last (`before`) and makes this row's ones visible to whoever reads them:
// the thread itself (OWN), its warp, or, for images, the whole thread block.
template <bool VEC, bool OWN, typename F>
__device__ __forceinline__ void next_row(F& fetch, uint32_t before, int stages) {
    if constexpr (VEC) {
        if constexpr (!OWN) __syncwarp();   // all lanes have read what is filled again
        fetch(before);
        copy_wait(stages);
        if constexpr (!OWN) __syncwarp();
    } else {
        if (stages == 1) {
            __syncthreads();
            fetch(before);
            copy_wait(1);
            __syncthreads();
        } else {
            copy_wait(stages - 1);
            __syncthreads();                // this row has arrived, and everyone has read the one before
            fetch(before);
        }
    }
}

template <typename TX, typename TIO, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 128 ? 4 : 1) block_norm_forward_kernel(const BlockNormParams p, const Ring ring) {
    __shared__ alignas(16) float buf[2][4][16];
    extern __shared__ uint4 ring_mem[];
    BlockSum<MAXT / 32> sum = block_sum_init<MAXT / 32>(buf);
    const Place<VEC> at(p.channels);
    const Channels ch(p.channels);
    const int row0 = blockIdx.x * p.rows_per_cta;
    const int row1 = min(p.n_tokens, row0 + p.rows_per_cta);
    const bool residual = p.y != nullptr;
    const uint32_t mine = smem_u32(ring_mem), ring_end = mine + ring.stages * ring.bytes;
    uint32_t used = 0;
    Rows<TX, VEC, 0, MAXT> xs(p.x, p.x_stride, row0, at, p, used);
    Rows<TIO, VEC, kMine<TX>, MAXT> ys(p.y, p.y_stride, row0, at, p, used);
    Results<TX, VEC> xo(p.x_out, p.x_out_stride, row0, at);
    Results<TIO, VEC> ho(p.h, p.h_stride, row0, at);
    int ahead = row0;     // next row to fetch
    auto fetch = [&](uint32_t record) {
        if (ahead++ < row1) {
            xs.fetch(at, record);
            if (residual) ys.fetch(at, record);
        }
        copy_commit();
    };
    for (int s = 0; s < ring.stages - 1; ++s) fetch(mine + s * ring.bytes);

    int mod_end = row0;   // first token behind the modulation row held in registers
    f32x2 w[kPairs], b[kPairs], g[kPairs];
    const f32x2 alpha = both(p.residual_scale);
    uint32_t here = mine, before = ring_end - ring.bytes;   // this row's record, and the one to fill again
    for (int row = row0; row < row1; ++row) {
        if (row >= mod_end) {
            const int mod = row / p.tokens_per_mod;
            mod_end = p.tokens_per_mod < p.n_tokens - mod * p.tokens_per_mod ? (mod + 1) * p.tokens_per_mod : p.n_tokens;
            const long long from = mod * p.mod_stride;
            f32x2 t[kPairs];
            read_vector<VEC>(p.weight, 1.0f, at, w);
            read_vector<VEC>(p.bias, 0.0f, at, b);
            read_vector<VEC>(p.scale ? p.scale + from : nullptr, 0.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                w[i] = fma2(w[i], t[i], w[i]);
                b[i] = fma2(b[i], t[i], b[i]);
            }
            read_vector<VEC>(p.shift ? p.shift + from : nullptr, 0.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) b[i] = add2(b[i], t[i]);
            read_vector<VEC>(p.gate ? p.gate + from : nullptr, 1.0f, at, g);
            read_vector<VEC>(p.post_weight, 1.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) g[i] = mul2(g[i], t[i]);
        }
        next_row<VEC, sizeof(TX) + sizeof(TIO) <= 4>(fetch, before, ring.stages);
        f32x2 v[kPairs];
        xs.read(at, here, v);
        if (residual) {
            f32x2 z[kPairs];
            ys.read(at, here, z);
            if (p.post_norm) normalise<VEC>(z, p.post_norm, p.post_eps, ch, at, sum);
            // (dead columns: z and x are 0, so x' is)
            if (p.residual_scale != 1.0f)
#pragma unroll
                for (int i = 0; i < kPairs; ++i) v[i] = mul2(v[i], alpha);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) v[i] = fma2(g[i], z[i], v[i]);
            if (p.x_out) xo.write(at, v);
        }
        if (p.norm) {   // on x' before its rounding to the residual stream's type
            normalise<VEC>(v, p.norm, p.eps, ch, at, sum);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) v[i] = fma2(v[i], w[i], b[i]);
            ho.write(at, v);
        }
        xs.done();
        ys.done();
        before = here;
        here += ring.bytes;
        if (here == ring_end) here = mine;
    }
}

// Results of a modulation row from its three sums, for one column.
__device__ __forceinline__ void write_mod_grads(const BlockNormParams& p, long long mod, int c, float s0, float s1, float s2) {
    const long long at = mod * p.channels + c;
    if (p.dshift) p.dshift[at] = s0;
    if (p.dscale) p.dscale[at] = fmaf(p.weight ? p.weight[c] : 1.0f, s1, (p.bias ? p.bias[c] : 0.0f) * s0);
    if (p.dgate) p.dgate[at] = (p.post_weight ? p.post_weight[c] : 1.0f) * s2;
}

// `N` neighbouring fp32 values (16-byte aligned where N is 4).
template <int N>
__device__ __forceinline__ void read_run(const float* from, float absent, float* v) {
    if (from == nullptr) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = absent;
    } else if constexpr (N == 4) {
        const float4 q = *reinterpret_cast<const float4*>(from);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = from[k];
    }
}
template <int N>
__device__ __forceinline__ void write_run(float* to, const float* v) {
    if constexpr (N == 4) {
        *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) to[k] = v[k];
    }
}

// Workspace: per thread block two slots of [3][channels] sums (its first modulation row, and its last one where that is
// another) that are not complete inside the block, then [3][channels] of sums for the weights' gradients.
__device__ __forceinline__ float* slot_of(const BlockNormParams& p, int cta, int which) {
    return p.partials + ((long long)cta * 9 + which * 3) * p.channels;
}

// w = weight (1 + scale), g = gate post_weight; the registers hold three sums per column.
template <typename TX, typename TIO, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 96 ? 5 : (MAXT == 128 ? 4 : 1)) block_norm_backward_kernel(const BlockNormParams p, const Ring ring) {
    __shared__ alignas(16) float buf[2][4][16];
    extern __shared__ uint4 shared_mem[];
    constexpr bool kRegs = MAXT == 320;
    // Rows of fp32 have the error of a layer norm's mean taken out (see variance()).  x's takes the place of y's squares in
    // the second exchange: those go with the means or, where y has a mean itself, into an exchange of their own (12480 x
    // 5120 with an fp32 stream: 279 us, 296 us with a fifth sum).  Rows of 16-bit types do without: a sum of values of one
    // binade is exact in fp32, and values of several leave a deviation that such an error does not touch.
    constexpr bool kSharpX = sizeof(TX) == 4, kSharpY = sizeof(TIO) == 4;
    Kept<MAXT, kRegs> w_kept, g_kept;
    uint4* ring_mem = shared_mem;
    if constexpr (!kRegs) {
        w_kept.mem = reinterpret_cast<float4*>(shared_mem);
        g_kept.mem = w_kept.mem + kCols / 4 * MAXT;
        ring_mem += 2 * (kCols / 4) * MAXT;
    }
    BlockSum<MAXT / 32> sum = block_sum_init<MAXT / 32>(buf);
    const Place<VEC> at(p.channels);
    const Channels ch(p.channels);
    const int row0 = blockIdx.x * p.rows_per_cta;
    const int row1 = min(p.n_tokens, row0 + p.rows_per_cta);
    const int first_mod = row0 / p.tokens_per_mod;
    const bool want_w = p.dweight || p.dbias || p.dpost_weight;
    const bool want_mod = p.dscale || p.dshift || p.dgate;
    const bool normed = p.norm != 0, branch = p.y != nullptr, more = p.dx_out != nullptr;
    const uint32_t mine = smem_u32(ring_mem), ring_end = mine + ring.stages * ring.bytes;
    uint32_t used = 0;
    Rows<TX, VEC, 0, MAXT> xs(p.x, p.x_stride, row0, at, p, used);
    Rows<TIO, VEC, kMine<TX>, MAXT> hs(p.dh, p.h_stride, row0, at, p, used);
    Rows<TX, VEC, kMine<TX> + kMine<TIO>, MAXT> ds(p.dx_out, p.dx_out_stride, row0, at, p, used);
    Rows<TIO, VEC, 2 * kMine<TX> + kMine<TIO>, MAXT> ys(p.y, p.y_stride, row0, at, p, used);
    Results<TX, VEC> dxo(p.dx, p.dx_stride, row0, at);
    Results<TIO, VEC> dyo(p.dy, p.dy_stride, row0, at);
    int ahead = row0;     // next row to fetch
    auto fetch = [&](uint32_t record) {
        if (ahead++ < row1) {
            if (normed) {
                xs.fetch(at, record);
                hs.fetch(at, record);
            }
            if (more) ds.fetch(at, record);
            if (branch) ys.fetch(at, record);
        }
        copy_commit();
    };
    for (int s = 0; s < ring.stages - 1; ++s) fetch(mine + s * ring.bytes);

    f32x2 s0[kPairs], s1[kPairs], s2[kPairs];
    const f32x2 alpha = both(p.residual_scale);
    uint32_t here = mine, before = ring_end - ring.bytes;   // this row's record, and the one to fill again
    bool first_flush = true;
    for (int row = row0; row < row1;) {
        const int mod = row / p.tokens_per_mod;
        const int begin = mod * p.tokens_per_mod;
        const int whole_end = p.tokens_per_mod < p.n_tokens - begin ? begin + p.tokens_per_mod : p.n_tokens;
        const int end = min(row1, whole_end);
        const bool complete = row == begin && end == whole_end;
        const long long from = mod * p.mod_stride;
        {
            f32x2 t[kPairs], w[kPairs];
            read_vector<VEC>(p.weight, 1.0f, at, w);
            read_vector<VEC>(p.scale ? p.scale + from : nullptr, 0.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) w[i] = fma2(w[i], t[i], w[i]);
            w_kept.set(w);
            read_vector<VEC>(p.gate ? p.gate + from : nullptr, 1.0f, at, w);
            read_vector<VEC>(p.post_weight, 1.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                w[i] = mul2(w[i], t[i]);
                s0[i] = s1[i] = s2[i] = 0ull;
            }
            g_kept.set(w);
        }
        for (; row < end; ++row) {
            next_row<VEC, sizeof(TX) + sizeof(TIO) <= 4>(fetch, before, ring.stages);
            f32x2 d[kPairs], v[kPairs];
            float y_mean = 0.0f, y_r = 1.0f;
            if (normed || p.post_norm) {
                // All sums of the row that do not need dx' take two barriers: the means, then the centred squares of x' and
                // y and the sums of d = dh (1 + s) w and of d against the centred x' (one barrier where both are RMS norms).
                const bool sharp = kSharpX && p.norm == kNormLayer;
                const bool y_early = kSharpX && (sharp || p.post_norm == kNormLayer);   // y's squares before the second exchange
                float m[2] = {0.0f, 0.0f}, q[4];
                if (normed) xs.read(at, here, v);
                if (p.norm == kNormLayer) m[0] = total(v);
                if (p.post_norm == kNormLayer) {
                    ys.read(at, here, d);
                    m[1] = total(d);
                } else if (sharp && p.post_norm) {
                    ys.read(at, here, d);
                    m[1] = total_squares(d);
                }
                if (p.norm == kNormLayer || p.post_norm == kNormLayer) sum.template run<2>(m);
                if (!kSharpX || p.post_norm == kNormLayer) y_mean = ch.mean(m[1]);
                float y_squares = m[1], y_error = 0.0f;
                q[2] = 0.0f;
                if (p.post_norm && (!y_early || p.post_norm == kNormLayer)) {
                    ys.read(at, here, d);
                    if (p.post_norm == kNormLayer) subtract<VEC>(d, y_mean, at);
                    q[2] = total_squares(d);
                }
                if (kSharpX && p.post_norm == kNormLayer) {
                    float e[2] = {q[2], kSharpY ? total(d) : 0.0f};
                    sum.template run<kSharpY ? 2 : 1>(e);
                    y_squares = e[0];
                    if (kSharpY) {
                        y_error = ch.mean(e[1]);
                        y_mean += y_error;   // (the columns are read again below)
                    }
                }
                if (normed) {
                    if (p.norm == kNormLayer) subtract<VEC>(v, ch.mean(m[0]), at);
                    q[3] = total_squares(v);
                    if (sharp) q[2] = total(v);
                    hs.read(at, here, d);
                    f32x2 ta = 0ull, tb = 0ull;
#pragma unroll
                    for (int i = 0; i < kPairs; i += 2) {
                        f32x2 w0, w1;
                        w_kept.get(i / 2, &w0, &w1);
                        w0 = mul2(d[i], w0);
                        w1 = mul2(d[i + 1], w1);
                        ta = add2(ta, add2(w0, w1));
                        tb = fma2(w1, v[i + 1], fma2(w0, v[i], tb));
                    }
                    q[0] = join(ta);
                    q[1] = join(tb);
                    sum.template run<4>(q);
                    float var = ch.mean(q[3]);
                    if (kSharpX) {
                        const float error = sharp ? ch.mean(q[2]) : 0.0f;
                        var = variance(var, error);
                        q[1] = fmaf(-error, q[0], q[1]);
#pragma unroll
                        for (int i = 0; i < kPairs; ++i) v[i] = add2(v[i], both(-error));   // (dead columns are not used below)
                    }
                    const float r = rsqrtf(var + p.eps);
                    // dx' = r (d - m0 - xhat m1), xhat = r times the centred x' (r = 0: nothing comes through, even where
                    // the sum against the centred x' is infinite)
                    const f32x2 r2 = both(r), m0 = both(p.norm == kNormLayer ? -r * ch.mean(q[0]) : 0.0f),
                                m1 = both(r == 0.0f ? 0.0f : -(r * (r * (r * ch.mean(q[1])))));
#pragma unroll
                    for (int i = 0; i < kPairs; i += 2) {
                        f32x2 wi[2];
                        w_kept.get(i / 2, &wi[0], &wi[1]);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            s0[i + k] = add2(s0[i + k], d[i + k]);
                            s1[i + k] = fma2(mul2(d[i + k], r2), v[i + k], s1[i + k]);
                            d[i + k] = fma2(v[i + k], m1, fma2(mul2(d[i + k], wi[k]), r2, m0));
                        }
                    }
                } else if (!y_early) {
                    sum.template run<1>(q + 2);
                }
                if (!y_early) y_squares = q[2];
                if (p.post_norm) y_r = rsqrtf((kSharpY ? variance(ch.mean(y_squares), y_error) : ch.mean(y_squares)) + p.post_eps);
            }
            if (!normed) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) d[i] = 0ull;
            }
            if (more) {
                ds.read(at, here, v);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) d[i] = add2(d[i], v[i]);
            }
            if (p.dx) {
                if (p.residual_scale != 1.0f) {
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) v[i] = mul2(d[i], alpha);
                    dxo.write(at, v);
                } else {
                    dxo.write(at, d);
                }
            }
            if (branch) {
                ys.read(at, here, v);
                if (p.post_norm == kNormLayer) subtract<VEC>(v, y_mean, at);
                if (p.post_norm)
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) v[i] = mul2(v[i], both(y_r));
                f32x2 ta = 0ull, tb = 0ull;
#pragma unroll
                for (int i = 0; i < kPairs; i += 2) {
                    f32x2 g0, g1;
                    g_kept.get(i / 2, &g0, &g1);
                    s2[i] = fma2(d[i], v[i], s2[i]);
                    s2[i + 1] = fma2(d[i + 1], v[i + 1], s2[i + 1]);
                    d[i] = mul2(d[i], g0);
                    d[i + 1] = mul2(d[i + 1], g1);
                }
                if (p.post_norm) {
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        // (dead columns of d hold -m0 r: their terms stay out of the mean)
                        ta = add2(ta, VEC || (at.on(2 * i) && at.on(2 * i + 1)) ? (at.on(2 * i) ? d[i] : 0ull)
                                                                               : (at.on(2 * i) ? pack2(low(d[i]), 0.0f) : 0ull));
                        tb = fma2(d[i], v[i], tb);   // v is 0 there
                    }
                    float t[2] = {join(ta), join(tb)};
                    sum.template run<2>(t);
                    const f32x2 m0 = both(p.post_norm == kNormLayer ? -y_r * ch.mean(t[0]) : 0.0f), m1 = both(-y_r * ch.mean(t[1])), r2 = both(y_r);
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) d[i] = fma2(v[i], m1, fma2(d[i], r2, m0));
                }
                if (p.dy) dyo.write(at, d);
            }
            xs.done();
            hs.done();
            ds.done();
            ys.done();
            before = here;
            here += ring.bytes;
            if (here == ring_end) here = mine;
        }
        // the modulation row's sums: final where all of its tokens are this block's, else a slot of the workspace
        if (want_w || want_mod) {
            float* slot = slot_of(p, blockIdx.x, mod == first_mod ? 0 : 1);
            float* wslot = slot_of(p, blockIdx.x, 2);
            constexpr int kRun = VEC ? 4 : 1;   // neighbouring columns written at a time
#pragma unroll
            for (int i = 0; i < kCols; i += kRun) {
                if (!at.on(i)) continue;
                const int c = at.col(i);
                float e0[kRun], e1[kRun], e2[kRun];
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    float lo, hi;
                    unpack2(s0[(i + k) / 2], lo, hi);
                    e0[k] = (i + k) % 2 ? hi : lo;
                    unpack2(s1[(i + k) / 2], lo, hi);
                    e1[k] = (i + k) % 2 ? hi : lo;
                    unpack2(s2[(i + k) / 2], lo, hi);
                    e2[k] = (i + k) % 2 ? hi : lo;
                }
                if (want_w) {   // this thread's own columns of this block's own slot
                    float s[kRun], gate[kRun], o0[kRun], o1[kRun], o2[kRun];
                    read_run<kRun>(p.scale ? p.scale + from + c : nullptr, 0.0f, s);
                    read_run<kRun>(p.gate ? p.gate + from + c : nullptr, 1.0f, gate);
                    read_run<kRun>(first_flush ? nullptr : wslot + c, 0.0f, o0);
                    read_run<kRun>(first_flush ? nullptr : wslot + p.channels + c, 0.0f, o1);
                    read_run<kRun>(first_flush ? nullptr : wslot + 2 * p.channels + c, 0.0f, o2);
#pragma unroll
                    for (int k = 0; k < kRun; ++k) {
                        o0[k] += fmaf(s[k], e1[k], e1[k]);
                        o1[k] += fmaf(s[k], e0[k], e0[k]);
                        o2[k] = fmaf(gate[k], e2[k], o2[k]);
                    }
                    write_run<kRun>(wslot + c, o0);
                    write_run<kRun>(wslot + p.channels + c, o1);
                    write_run<kRun>(wslot + 2 * p.channels + c, o2);
                }
                if (!want_mod) continue;
                if (complete) {
                    const long long to = (long long)mod * p.channels + c;
                    float w[kRun], b[kRun], pw[kRun];
                    read_run<kRun>(p.weight ? p.weight + c : nullptr, 1.0f, w);
                    read_run<kRun>(p.bias ? p.bias + c : nullptr, 0.0f, b);
                    read_run<kRun>(p.post_weight ? p.post_weight + c : nullptr, 1.0f, pw);
                    if (p.dshift) write_run<kRun>(p.dshift + to, e0);
#pragma unroll
                    for (int k = 0; k < kRun; ++k) {
                        e1[k] = fmaf(w[k], e1[k], b[k] * e0[k]);
                        e2[k] *= pw[k];
                    }
                    if (p.dscale) write_run<kRun>(p.dscale + to, e1);
                    if (p.dgate) write_run<kRun>(p.dgate + to, e2);
                } else {
                    write_run<kRun>(slot + c, e0);
                    write_run<kRun>(slot + p.channels + c, e1);
                    write_run<kRun>(slot + 2 * p.channels + c, e2);
                }
            }
            first_flush = false;
        }
    }
}

// Joins the slots.  Thread block (32 columns, job): 16 lanes of threads take every 16th slot each, then one of them
// adds the 16 sums.  Jobs below n_jobs are modulation rows that no single thread block of the first kernel held whole;
// job n_jobs is the weights' gradients.
constexpr int kJoinLanes = 16;
__global__ void __launch_bounds__(32 * kJoinLanes, 2) block_norm_join_kernel(const BlockNormParams p, const int n_ctas, const int n_jobs,
                                                              const int by_boundary) {
    __shared__ float part[3][kJoinLanes][33];
    const int c = blockIdx.x * 32 + threadIdx.x, lane = threadIdx.y, job = blockIdx.y;
    const bool weights = job == n_jobs;
    int mod = job, a = 0, b = n_ctas;
    if (!weights) {
        if (by_boundary) {
            // the modulation row, if any, that runs over the end of thread block `job` (rows shorter than a block's
            // range: at most two blocks hold one)
            const long long token = (long long)(job + 1) * p.rows_per_cta;
            mod = (int)(token / p.tokens_per_mod);
            if (token % p.tokens_per_mod == 0) return;
        }
        const long long t0 = (long long)mod * p.tokens_per_mod;
        const long long t1 = t0 + p.tokens_per_mod < p.n_tokens ? t0 + p.tokens_per_mod : p.n_tokens;
        a = (int)(t0 / p.rows_per_cta);
        b = (int)((t1 - 1) / p.rows_per_cta) + 1;
        if (b - a < 2) return;   // complete already
    }
    float s[3] = {0.0f, 0.0f, 0.0f};
    if (c < p.channels)
#pragma unroll 4
        for (int cta = a + lane; cta < b; cta += kJoinLanes) {
            const int which = weights ? 2 : ((long long)cta * p.rows_per_cta / p.tokens_per_mod == mod ? 0 : 1);
            const float* slot = slot_of(p, cta, which) + c;
#pragma unroll
            for (int k = 0; k < 3; ++k) s[k] += slot[(long long)k * p.channels];
        }
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][lane][threadIdx.x] = s[k];
    __syncthreads();
    if (lane != 0 || c >= p.channels) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        s[k] = 0.0f;
        for (int i = 0; i < kJoinLanes; ++i) s[k] += part[k][i][threadIdx.x];
    }
    if (weights) {
        if (p.dweight) p.dweight[c] = s[0];
        if (p.dbias) p.dbias[c] = s[1];
        if (p.dpost_weight) p.dpost_weight[c] = s[2];
    } else {
        write_mod_grads(p, mod, c, s[0], s[1], s[2]);
    }
}

constexpr uint32_t kMostShared = 228000;   // dynamic shared memory of a thread block, at most (plan_ring)

int threads_for(int channels) { return (channels + 32 * kCols - 1) / (32 * kCols) * 32; }

// A persistent grid: as many thread blocks as the device holds at a time (more would run as a second, mostly empty wave:
// 41 us instead of 33 at the window), each with an equal share of the rows; at most `cap`.
template <typename K>
cudaError_t plan(BlockNormParams* p, K kernel, int threads, size_t smem, int sm_count, int cap, int* ctas) {
    if (smem > 40000) {   // static and dynamic shared memory together past the default limit of 48 KB
        // The limit belongs to the kernel, not to the call, and other host threads launch the same kernel at other widths:
        // it is always set to the most that any width takes, so that no call lowers it under another one's launch.
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared);
        if (e != cudaSuccess) return e;
    }
    int most = p->n_tokens;
    if (most > sm_count) {
        int per_sm = 1;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem);
        if (e != cudaSuccess) return e;
        if (per_sm < 1) per_sm = 1;
        if (most > per_sm * sm_count) most = per_sm * sm_count;
        if (most > cap) most = cap;
    }
    p->rows_per_cta = (p->n_tokens + most - 1) / most;
    *ctas = (p->n_tokens + p->rows_per_cta - 1) / p->rows_per_cta;
    return cudaSuccess;
}

// Stages: as many as fit a share of the SM's shared memory (for about `threads_wanted` threads on it), two to four; one
// where two rows do not fit an SM: gradients with an fp32 stream from 5128 channels on (rows read as images: from 5073, or
// 6761 with 16-bit branches).  Every row then waits for its copies in full.
Ring plan_ring(uint32_t stage_bytes, uint32_t other_bytes, int threads, int threads_wanted) {
    const int blocks = threads_wanted / threads > 1 ? threads_wanted / threads : 1;
    int stages = (int)((224000u / blocks - other_bytes) / stage_bytes);
    if (stages < 2) stages = 2 * stage_bytes + other_bytes <= kMostShared ? 2 : 1;
    if (stages > 4) stages = 4;
    return Ring{stages, stage_bytes};
}

template <typename TX, typename TIO, bool VEC, int MAXT>
cudaError_t forward_one(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    const int threads = threads_for(p.channels);
    const Ring ring = plan_ring(VEC ? MAXT * (kMine<TX> + kMine<TIO>) : image_bytes(p.channels, sizeof(TX)) + image_bytes(p.channels, sizeof(TIO)), 0, threads, MAXT == 128 ? 480 : 320);
    const size_t smem = (size_t)ring.stages * ring.bytes;
    const cudaError_t e = plan(&p, block_norm_forward_kernel<TX, TIO, VEC, MAXT>, threads, smem, sm_count, 1 << 30, ctas);
    if (e != cudaSuccess) return e;
    block_norm_forward_kernel<TX, TIO, VEC, MAXT><<<*ctas, threads, smem, stream>>>(p, ring);
    return cudaGetLastError();
}
template <typename TX, typename TIO, bool VEC, int MAXT>
cudaError_t backward_one(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    const int threads = threads_for(p.channels);
    constexpr uint32_t kept = MAXT == 320 ? 0 : 2 * kMine<float> * MAXT;
    const Ring ring = plan_ring(VEC ? MAXT * 2 * (kMine<TX> + kMine<TIO>) : 2 * (image_bytes(p.channels, sizeof(TX)) + image_bytes(p.channels, sizeof(TIO))), kept, threads, MAXT == 96 ? 480 : 384);
    const size_t smem = (size_t)ring.stages * ring.bytes + kept;
    const cudaError_t e = plan(&p, block_norm_backward_kernel<TX, TIO, VEC, MAXT>, threads, smem, sm_count, kNormMaxCtas, ctas);
    if (e != cudaSuccess) return e;
    block_norm_backward_kernel<TX, TIO, VEC, MAXT><<<*ctas, threads, smem, stream>>>(p, ring);
    return cudaGetLastError();
}
// Builds by the registers and the shared memory that a row's threads leave: up to 1536 channels (gradients: five blocks
// per SM instead of four), 2048, 5120, 8192; rows read as images: 2048 and 8192.
template <typename TX, typename TIO, bool VEC>
cudaError_t forward_sized(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    if (threads_for(p.channels) <= 128) return forward_one<TX, TIO, VEC, 128>(p, sm_count, ctas, stream);
    if constexpr (VEC)
        if (threads_for(p.channels) <= 320) return forward_one<TX, TIO, VEC, 320>(p, sm_count, ctas, stream);
    return forward_one<TX, TIO, VEC, 512>(p, sm_count, ctas, stream);
}
template <typename TX, typename TIO, bool VEC>
cudaError_t backward_sized(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    if constexpr (VEC)
        if (threads_for(p.channels) <= 96) return backward_one<TX, TIO, VEC, 96>(p, sm_count, ctas, stream);
    if (threads_for(p.channels) <= 128) return backward_one<TX, TIO, VEC, 128>(p, sm_count, ctas, stream);
    if constexpr (VEC)
        if (threads_for(p.channels) <= 320) return backward_one<TX, TIO, VEC, 320>(p, sm_count, ctas, stream);
    return backward_one<TX, TIO, VEC, 512>(p, sm_count, ctas, stream);
}

}  // namespace

#define REGENVC_BY_TYPE(call)                                                                           \
    if (x_type == kTypeBf16) return vec ? call<__nv_bfloat16, __nv_bfloat16, true> : call<__nv_bfloat16, __nv_bfloat16, false>; \
    if (x_type == kTypeF16) return vec ? call<__half, __half, true> : call<__half, __half, false>;        \
    if (io_type == kTypeBf16) return vec ? call<float, __nv_bfloat16, true> : call<float, __nv_bfloat16, false>; \
    if (io_type == kTypeF16) return vec ? call<float, __half, true> : call<float, __half, false>;         \
    return vec ? call<float, float, true> : call<float, float, false>;

typedef cudaError_t (*NormLaunch)(BlockNormParams&, int, int*, cudaStream_t);
static NormLaunch pick_forward(int x_type, int io_type, bool vec) { REGENVC_BY_TYPE(forward_sized) }
static NormLaunch pick_backward(int x_type, int io_type, bool vec) { REGENVC_BY_TYPE(backward_sized) }

cudaError_t launch_block_norm_forward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count,
                                      cudaStream_t stream) {
    int ctas = 0;
    return pick_forward(x_type, io_type, vec)(p, sm_count, &ctas, stream);
}

cudaError_t launch_block_norm_backward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count, int* launches,
                                       cudaStream_t stream) {
    int ctas = 0;
    *launches = 0;
    cudaError_t e = pick_backward(x_type, io_type, vec)(p, sm_count, &ctas, stream);
    if (e != cudaSuccess) return e;
    *launches = 1;
    const bool want_w = p.dweight || p.dbias || p.dpost_weight;
    const bool want_mod = p.dscale || p.dshift || p.dgate;
    const bool by_boundary = p.tokens_per_mod < p.rows_per_cta;
    const int n_mods = (int)(((long long)p.n_tokens + p.tokens_per_mod - 1) / p.tokens_per_mod);
    const int jobs = !want_mod || ctas == 1 ? 0 : (by_boundary ? ctas - 1 : n_mods);   // at most `ctas` either way
    if (jobs + (want_w ? 1 : 0) == 0) return cudaSuccess;
    block_norm_join_kernel<<<dim3((p.channels + 31) / 32, jobs + (want_w ? 1 : 0)), dim3(32, kJoinLanes), 0, stream>>>(p, ctas, jobs,
                                                                                                          by_boundary ? 1 : 0);
    e = cudaGetLastError();
    if (e == cudaSuccess) *launches = 2;
    return e;
}

}  // namespace regenvc
