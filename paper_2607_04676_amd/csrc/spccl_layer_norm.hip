// Layer norm over the rows of a matrix, forward and backward, with the
// reduction of the weight's and the bias's gradient over the rows.
//
//   forward    mean = sum x / C, rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),
//              y = (x - mean) rstd w + b
//   backward   h = (x - mean) rstd, g = dy w:
//              dx = rstd (g - sum g / C - h sum(g h) / C)
//              dw = sum over rows of dy h,  db = sum over rows of dy
//
// Every sum is held in fp32; x, y and dx are rounded once, to their own type.
// Both directions are bound by memory: forward reads x and writes y, backward
// reads dy and x and writes dx, each once, so a row stays in the registers of
// the lanes that loaded it between its statistics and its result.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "spccl_internal.h"
#include "../../include/spccl.h"

namespace spccl {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// element types: 16-byte vectors of either

struct F32 {
    using raw = uint32_t;
    typedef u32x4 __attribute__((aligned(4))) vec_any;           // at any element's address
    static constexpr int vec = 4;
    static __device__ __forceinline__ float get(const u32x4& v, int j) { return __uint_as_float(v[j]); }
    static __device__ __forceinline__ float one(raw r) { return __uint_as_float(r); }
    static __device__ __forceinline__ raw round(float f) { return __float_as_uint(f); }
    static __device__ __forceinline__ u32x4 pack(const float* f) {
        return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
};
struct BF16 {
    using raw = uint16_t;
    typedef u32x4 __attribute__((aligned(2))) vec_any;
    static constexpr int vec = 8;
    static __device__ __forceinline__ float get(const u32x4& v, int j) {
        return __uint_as_float(j & 1 ? v[j / 2] & 0xFFFF0000u : v[j / 2] << 16);
    }
    static __device__ __forceinline__ float one(raw r) { return __uint_as_float((uint32_t)r << 16); }
    static __device__ __forceinline__ uint32_t two(float a, float b) {      // nearest, ties to even
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    }
    static __device__ __forceinline__ raw round(float f) { return (raw)two(f, f); }
    static __device__ __forceinline__ u32x4 pack(const float* f) {
        return u32x4{two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7])};
    }
};

// A row's vector of `E::vec` elements from column c on, of which `rem` exist
// (the others read 0).  Rows start at any element: the vector accesses ask
// for no more than the element's alignment.
template <class E>
__device__ __forceinline__ u32x4 load_vec(const uint8_t* row, uint32_t c, uint32_t rem) {
    using raw = typename E::raw;
    const raw* p = reinterpret_cast<const raw*>(row) + c;
    if (rem >= (uint32_t)E::vec) return *reinterpret_cast<const typename E::vec_any*>(p);
    u32x4 v{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < E::vec - 1; j++)
        if ((uint32_t)j < rem) v[j * sizeof(raw) / 4] |= (uint32_t)p[j] << (8 * (j * sizeof(raw) % 4));
    return v;
}

template <class E>
__device__ __forceinline__ void store_vec(uint8_t* row, uint32_t c, uint32_t rem, const float* f) {
    using raw = typename E::raw;
    raw* p = reinterpret_cast<raw*>(row) + c;
    if (rem >= (uint32_t)E::vec) {
        *reinterpret_cast<typename E::vec_any*>(p) = E::pack(f);
        return;
    }
#pragma unroll
    for (int j = 0; j < E::vec - 1; j++)
        if ((uint32_t)j < rem) p[j] = E::round(f[j]);
}

// N elements of a weight or bias from column c on (0 beyond `rem`, and
// `absent` for a null array).
template <class W, int N>
__device__ __forceinline__ void load_param(const uint8_t* base, uint32_t c, uint32_t rem, float absent, float* f) {
    if (!base) {
#pragma unroll
        for (int j = 0; j < N; j++) f[j] = absent;
        return;
    }
    if constexpr (N >= W::vec) {
#pragma unroll
        for (int h = 0; h < N / W::vec; h++) {
            const uint32_t at = h * W::vec;
            const u32x4 v = load_vec<W>(base, c + at, rem > at ? rem - at : 0);
#pragma unroll
            for (int j = 0; j < W::vec; j++) f[h * W::vec + j] = W::get(v, j);
        }
    } else {                                              // fp32 rows, bf16 weights: half a vector
        static_assert(N * 2 == W::vec, "half a vector");
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        typedef u32x2 __attribute__((aligned(2))) halfu;
        const uint16_t* p = reinterpret_cast<const uint16_t*>(base) + c;
        if (rem >= (uint32_t)N) {
            const u32x2 v = *reinterpret_cast<const halfu*>(p);
#pragma unroll
            for (int j = 0; j < N; j++) f[j] = __uint_as_float(j & 1 ? v[j / 2] & 0xFFFF0000u : v[j / 2] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < N; j++) f[j] = (uint32_t)j < rem ? W::one(p[j]) : 0.f;
        }
    }
}

// A lane's vector of a row that lies whole in registers: columns [a, a + vec),
// of which those before `first` are another lane's or do not exist.  Every
// load is one full vector inside the row, without a branch (a load in a branch
// is waited for at the branch's end, before the next can issue): a lane past
// the end reads the row's last vector for nothing, and where the row's length
// is no multiple of vec (Ragged), its last vector is read from vec columns
// before its end.
template <class E, bool Ragged>
struct Place {
    uint32_t a, first;
    __device__ __forceinline__ Place(uint32_t c, uint32_t cols) {
        if constexpr (Ragged) {
            a = c + E::vec <= cols ? c : cols - E::vec;
            first = c + E::vec <= cols ? 0 : (c >= cols ? E::vec : c + E::vec - cols);
            asm volatile("" : "+v"(first));         // masks of its values are made where they are used, not kept
        } else {
            a = c < cols ? c : cols - E::vec;
            first = c < cols ? 0 : E::vec;
        }
    }
    __device__ __forceinline__ bool any() const { return first < (uint32_t)E::vec; }
    // zeros in the elements before `first`
    __device__ __forceinline__ void clear(u32x4& v) const {
        constexpr int per = 4 / sizeof(typename E::raw);
#pragma unroll
        for (int q = 0; q < 4; q++) {
            if constexpr (!Ragged)
                v[q] = any() ? v[q] : 0u;
            else if constexpr (per == 2)
                v[q] = first >= (uint32_t)(2 * q + 2) ? 0u : (first == (uint32_t)(2 * q + 1) ? v[q] & 0xFFFF0000u : v[q]);
            else
                v[q] = first > (uint32_t)q ? 0u : v[q];
        }
    }
    __device__ __forceinline__ void store(uint8_t* row, const float* f) const {
        using raw = typename E::raw;
        if (first == 0) {
            __builtin_nontemporal_store(E::pack(f), reinterpret_cast<typename E::vec_any*>(row + a * (uint32_t)sizeof(raw)));
            return;
        }
        if constexpr (Ragged) {
            raw* p = reinterpret_cast<raw*>(row) + a;
#pragma unroll
            for (int j = 1; j < E::vec; j++)
                if ((uint32_t)j >= first) p[j] = E::round(f[j]);
        }
    }
};
template <class E, bool Stream>
__device__ __forceinline__ u32x4 load_row(const uint8_t* row, uint32_t a) {
    const auto* p = reinterpret_cast<const typename E::vec_any*>(row + a * (uint32_t)sizeof(typename E::raw));
    if constexpr (Stream) return __builtin_nontemporal_load(p);
    else return *p;
}

// A row's weights or biases at a lane's places, as they are stored: all loads
// issue before the first is converted.  absent: the bits of a null array.
template <class E, class W, int K>
struct Params {
    static constexpr int D = E::vec * sizeof(typename W::raw) / 4;     // words per vector: 2, 4 or 8
    uint32_t r[K][D];
    __device__ __forceinline__ void load(const uint8_t* base, const uint32_t (&a)[K], float absent) {
        if (base) {
#pragma unroll
            for (int k = 0; k < K; k++) {
                const uint8_t* p = base + a[k] * (uint32_t)sizeof(typename W::raw);
                if constexpr (D == 2) {
                    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                    typedef u32x2 __attribute__((aligned(2))) half_any;
                    const u32x2 v = *reinterpret_cast<const half_any*>(p);
                    r[k][0] = v[0];
                    r[k][1] = v[1];
                } else {
#pragma unroll
                    for (int q = 0; q < D / 4; q++) {
                        const u32x4 v = reinterpret_cast<const typename W::vec_any*>(p)[q];
#pragma unroll
                        for (int z = 0; z < 4; z++) r[k][4 * q + z] = v[z];
                    }
                }
            }
        } else {
            const uint32_t one = sizeof(typename W::raw) == 4 ? W::round(absent) : W::round(absent) * 0x10001u;
#pragma unroll
            for (int k = 0; k < K; k++)
#pragma unroll
                for (int z = 0; z < D; z++) r[k][z] = one;
        }
    }
    __device__ __forceinline__ void pin(int k) {
#pragma unroll
        for (int z = 0; z < D; z++) asm volatile("" : "+v"(r[k][z]));
    }
    __device__ __forceinline__ float get(int k, int j) const {
        if constexpr (sizeof(typename W::raw) == 4) return __uint_as_float(r[k][j]);
        else return __uint_as_float(j & 1 ? r[k][j / 2] & 0xFFFF0000u : r[k][j / 2] << 16);
    }
};

// ---------------------------------------------------------------------------
// sums over the lanes of a row

template <int Ctrl>
__device__ __forceinline__ float dpp(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), Ctrl, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float x, int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane));
}

// The sum over groups of L consecutive lanes, in every lane of the group:
// partners at distance 1 and 2 (quad permutations), then the mirrored lane of
// 8 and of 16 (whose quads and halves hold one value by then), then the four
// rows of 16.
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
    constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;
    x += dpp<kXor1>(x);
    x += dpp<kXor2>(x);
    x += dpp<kMirror8>(x);
    if constexpr (L >= 16) x += dpp<kMirror16>(x);
    if constexpr (L == 32) x += __shfl_xor(x, 16);
    if constexpr (L == 64) x = (lane_of(x, 0) + lane_of(x, 16)) + (lane_of(x, 32) + lane_of(x, 48));
    return x;
}

// How a row lies over lanes: L lanes of one wave (Waves = 1) or all lanes of
// Waves waves, K vectors each; vector k of lane i is vector k * lanes + i.
template <class E, int L, int Waves, int K, uint32_t Threads = 256>
struct Row {
    static_assert(Waves == 1 || L == 64, "a row is part of a wave, or whole waves");
    static constexpr uint32_t lanes = L * Waves;
    static constexpr uint32_t cap = lanes * K * E::vec;           // columns that fit
    static constexpr uint32_t threads = 64 * Waves > Threads ? 64 * Waves : Threads;
    static constexpr uint32_t rows = threads / lanes;             // rows of a block at a time
    static constexpr uint32_t waves = threads / 64;
    // whether vector k lies past the row's end in every lane, or in some
    static __device__ __forceinline__ bool beyond(int k, uint32_t cols) { return k * lanes * E::vec >= cols; }
    static __device__ __forceinline__ bool edge(int k, uint32_t cols) { return (k + 1) * lanes * E::vec > cols; }
    // the thread's row of the block; whole waves know it as a scalar
    static __device__ __forceinline__ uint32_t group() {
        if constexpr (L == 64) return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) / Waves;
        else return threadIdx.x / lanes;
    }
};

struct LnArgs {
    const uint8_t* x;
    const uint8_t* w;
    const uint8_t* b;
    uint8_t* y;
    float* mean;
    float* rstd;
    uint64_t ldx, ldy;        // bytes between rows
    uint64_t rows;
    uint32_t cols;
    float eps;
};

// One row per group of lanes.  The deviations are summed about the mean in a
// second pass over the registers, so a large mean costs no precision; where a
// row spans waves, each takes the mean and the squared deviations of its own
// columns and the waves' are joined (n1 m1 + n2 m2; the squared distance of a
// part's mean from the whole's counts for each of its columns), so a row
// meets one barrier.  A row of one wave reads its weights along with x; a
// longer one afterwards, as their registers would cost it waves (32768 x 8192
// bf16: 181 us against 194; 16384 x 1024: 11.3 early, 12.1 late).  Stores
// are non-temporal, loads are not (10007 x 1600 fp32: 20.3 us; 27.1 with
// ordinary stores, 25.4 with non-temporal loads too: 6.3 TB/s; 32768 x 8192 bf16
// runs at 5.9 TB/s).
template <class E, class W, int L, int Waves, int K, bool Ragged>
__global__ void __launch_bounds__((Row<E, L, Waves, K>::threads)) k_layer_norm(LnArgs g) {
    using R = Row<E, L, Waves, K>;
    using At = Place<E, Ragged>;
    constexpr int V = E::vec;
    const uint32_t i = threadIdx.x % R::lanes;                    // lane of the row
    const uint32_t group = R::group();
    const uint64_t row = (uint64_t)blockIdx.x * R::rows + group;
    const bool mine = row < g.rows;
    const uint8_t* src = g.x + (mine ? row : 0) * g.ldx;
    uint32_t a[K];
    u32x4 v[K];
#pragma unroll
    for (int k = 0; k < K; k++) {
        a[k] = At((k * R::lanes + i) * V, g.cols).a;
        v[k] = load_row<E, false>(src, a[k]);
    }
    Params<E, W, K> w, b;
    if constexpr (Waves == 1) {
        w.load(g.w, a, 1.f);
        b.load(g.b, a, 0.f);
    }
    // masks of single elements are worth a branch around them
    constexpr bool Branch = Ragged && K > 2;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; k++) {
        if (Branch && R::beyond(k, g.cols)) break;
        if (!Branch || R::edge(k, g.cols)) At((k * R::lanes + i) * V, g.cols).clear(v[k]);
#pragma unroll
        for (int j = 0; j < V; j++) sum += E::get(v[k], j);
    }
    // the columns whose mean is taken first: the row's, or this wave's part
    uint32_t n = g.cols;
    if constexpr (Waves > 1) {
        n = 0;
#pragma unroll
        for (int k = 0; k < K; k++) {
            const uint32_t c0 = (k * R::lanes + (i & ~63u)) * V;
            n += c0 < g.cols ? (g.cols - c0 < 64u * V ? g.cols - c0 : 64u * V) : 0;
        }
    }
    float mean = lanes_sum<L>(sum) / (float)(n ? n : 1);
    float dev = 0.f;
#pragma unroll
    for (int k = 0; k < K; k++) {
        if (Branch && R::beyond(k, g.cols)) break;
        float part = 0.f;
        if (!Branch || R::edge(k, g.cols)) {
            const At at((k * R::lanes + i) * V, g.cols);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float d = !Ragged || (uint32_t)j >= at.first ? E::get(v[k], j) - mean : 0.f;
                part = fmaf(d, d, part);
            }
            part = at.any() ? part : 0.f;
        } else {
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float d = E::get(v[k], j) - mean;
                part = fmaf(d, d, part);
            }
        }
        dev += part;
    }
    dev = lanes_sum<L>(dev);
    if constexpr (Waves > 1) {
        __shared__ float s_n[R::waves], s_mean[R::waves], s_dev[R::waves];
        const uint32_t wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63u) == 0) {
            s_n[wave] = (float)n;
            s_mean[wave] = mean;
            s_dev[wave] = dev;
        }
        __syncthreads();
        const uint32_t first = group * Waves;
        float total = 0.f;
#pragma unroll
        for (int q = 0; q < Waves; q++) total += s_n[first + q] * s_mean[first + q];
        mean = total / (float)g.cols;
        dev = 0.f;
#pragma unroll
        for (int q = 0; q < Waves; q++) {
            const float d = s_mean[first + q] - mean;
            dev += fmaf(s_n[first + q], d * d, s_dev[first + q]);
        }
    }
    if (!mine) return;
    const float rstd = 1.0f / sqrtf(dev / (float)g.cols + g.eps);
    if (i == 0) {
        if (g.mean) g.mean[row] = mean;
        if (g.rstd) g.rstd[row] = rstd;
    }
    uint8_t* dst = g.y + row * g.ldy;
    if constexpr (Waves > 1) {
#pragma unroll
        for (int k = 0; k < K; k++) asm volatile("" : "+v"(a[k]));    // not earlier
        w.load(g.w, a, 1.f);
        b.load(g.b, a, 0.f);
    }
#pragma unroll
    for (int k = 0; k < K; k++) {
        if (Branch && R::beyond(k, g.cols)) break;
        float y[V];
#pragma unroll
        for (int j = 0; j < V; j++) y[j] = fmaf((E::get(v[k], j) - mean) * rstd, w.get(k, j), b.get(k, j));
        At((k * R::lanes + i) * V, g.cols).store(dst, y);
    }
}

// Rows too long for the registers of a block, or shorter than a vector: the
// block reads its row three times (the L2 holds it from the first), for the
// mean, the deviations and y.
template <class E, class W>
__global__ void __launch_bounds__(1024) k_layer_norm_long(LnArgs g) {
    constexpr int V = E::vec;
    __shared__ float s_part[2][16];
    const uint8_t* src = g.x + (uint64_t)blockIdx.x * g.ldx;
    uint8_t* dst = g.y + (uint64_t)blockIdx.x * g.ldy;
    const uint32_t wave = threadIdx.x >> 6;
    const auto block_sum = [&](float x, int which) {
        x = lanes_sum<64>(x);
        if ((threadIdx.x & 63u) == 0) s_part[which][wave] = x;
        __syncthreads();
        float t = 0.f;
#pragma unroll
        for (int q = 0; q < 16; q++) t += s_part[which][q];
        return t;
    };
    float sum = 0.f;
    for (uint32_t c = threadIdx.x * V; c < g.cols; c += 1024 * V) {
        const u32x4 v = load_vec<E>(src, c, g.cols - c);
#pragma unroll
        for (int j = 0; j < V; j++) sum += E::get(v, j);
    }
    const float mean = block_sum(sum, 0) / (float)g.cols;
    float dev = 0.f;
    for (uint32_t c = threadIdx.x * V; c < g.cols; c += 1024 * V) {
        const uint32_t rem = g.cols - c;
        const u32x4 v = load_vec<E>(src, c, rem);
#pragma unroll
        for (int j = 0; j < V; j++) {
            const float d = (uint32_t)j < rem ? E::get(v, j) - mean : 0.f;
            dev = fmaf(d, d, dev);
        }
    }
    const float rstd = 1.0f / sqrtf(block_sum(dev, 1) / (float)g.cols + g.eps);
    if (threadIdx.x == 0) {
        if (g.mean) g.mean[blockIdx.x] = mean;
        if (g.rstd) g.rstd[blockIdx.x] = rstd;
    }
    for (uint32_t c = threadIdx.x * V; c < g.cols; c += 1024 * V) {
        const uint32_t rem = g.cols - c;
        const u32x4 v = load_vec<E>(src, c, rem);
        float w[V], b[V], y[V];
        load_param<W, V>(g.w, c, rem, 1.f, w);
        load_param<W, V>(g.b, c, rem, 0.f, b);
#pragma unroll
        for (int j = 0; j < V; j++) y[j] = fmaf((E::get(v, j) - mean) * rstd, w[j], b[j]);
        store_vec<E>(dst, c, rem, y);
    }
}

// ---------------------------------------------------------------------------
// backward

struct LnBackArgs {
    const uint8_t* dy;
    const uint8_t* x;
    const uint8_t* w;
    const float* mean;
    const float* rstd;
    uint8_t* dx;              // null: only the weight's and bias's gradient
    float* part;              // [blocks][2][cols]: the blocks' sums of dy h and of dy (null: not wanted)
    uint64_t lddy, ldx, lddx; // bytes between rows
    uint64_t rows;
    uint32_t cols;
};

constexpr uint32_t kBackThreads = 512, kShortThreads = 512;
__device__ const float kNoRow = 0.f;          // the mean and rstd of a group without a row

// Each group of lanes walks over rows, keeping its columns' sums of dy h and
// dy in registers; a block joins its groups' through LDS, in their order, and
// leaves one pair of sums per column for k_layer_norm_grads, so no sum depends
// on which block comes first.  Rows of whole vectors are read non-temporally
// (65536 x 4096 bf16, 1.6 GB: 266 us, 6.0 TB/s; 288 with ordinary loads).
template <class E, class W, int L, int Waves, int K, bool Ragged>
__global__ void __launch_bounds__((Row<E, L, Waves, K, kBackThreads>::threads)) k_layer_norm_back(LnBackArgs g) {
    using R = Row<E, L, Waves, K, kBackThreads>;
    using At = Place<E, Ragged>;
    constexpr int V = E::vec;
    __shared__ __attribute__((aligned(16))) float s_sum[R::rows > 1 ? R::rows * R::cap : 1];
    __shared__ float s_row[2][2][R::waves];
    const uint32_t i = threadIdx.x % R::lanes;
    const uint32_t group = R::group();
    const uint32_t wave = threadIdx.x >> 6;
    float dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; k++)
#pragma unroll
        for (int j = 0; j < V; j++) dw[k][j] = db[k][j] = 0.f;
    uint32_t a[K];
#pragma unroll
    for (int k = 0; k < K; k++) a[k] = At((k * R::lanes + i) * V, g.cols).a;
    Params<E, W, K> w;
    w.load(g.w, a, 1.f);
    const float inv = 1.0f / (float)g.cols;
    // a row's data; a group past the last row reads the start of its block's
    // first row instead, a line a load (600 x 12000 fp32: 30.7 us; 33.2 where
    // every block's groups read the whole last row, 8192 x 12288 220 and 222)
    struct Data {
        u32x4 x[K], dy[K];
        float mean, rstd;
    };
    // (its mean and rstd are zeros: the deviation of a zero from another row's mean
    // may be infinite, and 0 times that is NaN)
    struct Source {
        uint64_t row;
        uint32_t mask;
        const float* mean;
        const float* rstd;
    };
    const uint64_t first = (uint64_t)blockIdx.x * R::rows;
    const auto source = [&](uint64_t r0) {
        const bool mine = r0 + group < g.rows;
        const uint64_t row = mine ? r0 + group : first;
        const bool stats = mine || R::rows == 1;                     // a lone group ends with its last row
        return Source{row, mine ? ~0u : 0u, stats ? g.mean + row : &kNoRow, stats ? g.rstd + row : &kNoRow};
    };
    const auto fetch = [&](const Source& s, Data& d) {
        const uint8_t* px = g.x + s.row * g.ldx;
        const uint8_t* pdy = g.dy + s.row * g.lddy;
#pragma unroll
        for (int k = 0; k < K; k++) {
            d.x[k] = load_row<E, !Ragged>(px, a[k] & s.mask);
            d.dy[k] = load_row<E, !Ragged>(pdy, a[k] & s.mask);
        }
        d.mean = *s.mean;
        d.rstd = *s.rstd;
    };
    // the next row is on its way while this one is worked on, where the
    // registers for it are there (not for 32 fp32 elements a lane; there, loading
    // each of its vectors as soon as this row's is stored took 8192 x 16384 from
    // 310 us to 302, but 3001 x 12289 from 98 to 101 and 600 x 16384 from 42 to 43)
    constexpr bool Ahead = K <= 6;
    const uint64_t step = (uint64_t)gridDim.x * R::rows;
    uint32_t turn = 0;
    Data next;
    if constexpr (Ahead) fetch(source(first), next);
    for (uint64_t r0 = first; r0 < g.rows; r0 += step, turn ^= 1) {
        Data now;
        if constexpr (Ahead) {
            now = next;
            fetch(source(r0 + step), next);
        } else {
            fetch(source(r0), now);
        }
        const bool mine = R::rows == 1 || r0 + group < g.rows;
        const uint64_t row = r0 + group;
        auto& x = now.x;
        auto& dy = now.dy;
        const float mean = now.mean, rstd = now.rstd;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; k++) {
            w.pin(k);
            At((k * R::lanes + i) * V, mine ? g.cols : 0).clear(dy[k]);
            // (in place, the block's first row is already written over)
            if (R::rows > 1) x[k] = mine ? x[k] : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float d = E::get(dy[k], j);
                const float h = (E::get(x[k], j) - mean) * rstd;
                const float t = d * w.get(k, j);
                s1 = fmaf(t, h, s1);
                s2 += t;
                dw[k][j] = fmaf(d, h, dw[k][j]);
                db[k][j] += d;
                asm volatile("" : "+v"(dw[k][j]), "+v"(db[k][j]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        s1 = lanes_sum<L>(s1);
        s2 = lanes_sum<L>(s2);
        if constexpr (Waves > 1) {
            // two buffers in turn: a wave that is a row ahead writes the other
            if ((threadIdx.x & 63u) == 0) {
                s_row[turn][0][wave] = s1;
                s_row[turn][1][wave] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int q = 0; q < Waves; q++) {
                s1 += s_row[turn][0][group * Waves + q];
                s2 += s_row[turn][1][group * Waves + q];
            }
        }
        s1 *= inv;
        s2 *= inv;
        // converted again below: what the first pass made of x and dy would
        // otherwise stay in registers, four times what they take as stored
#pragma unroll
        for (int k = 0; k < K; k++) asm volatile("" : "+v"(x[k]), "+v"(dy[k]));
        uint8_t* dst = g.dx + row * g.lddx;
#pragma unroll
        for (int k = 0; k < K; k++) {
            float o[V];
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float h = (E::get(x[k], j) - mean) * rstd;
                o[j] = fmaf(-h, s1, fmaf(E::get(dy[k], j), w.get(k, j), -s2)) * rstd;
            }
            const At at((k * R::lanes + i) * V, g.cols);
            if (mine && g.dx && at.any()) at.store(dst, o);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (!g.part) return;
    float* part = g.part + (uint64_t)blockIdx.x * 2 * g.cols;
    if constexpr (R::rows == 1) {
#pragma unroll
        for (int k = 0; k < K; k++) {
            const At at((k * R::lanes + i) * V, g.cols);
#pragma unroll
            for (int j = 0; j < V; j++)
                if ((uint32_t)j >= at.first) {
                    part[at.a + j] = dw[k][j];
                    part[g.cols + at.a + j] = db[k][j];
                }
        }
        return;
    }
    // every group leaves its sums in LDS, then each thread adds up columns
#pragma unroll
    for (int which = 0; which < 2; which++) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; k++) {
            const At at((k * R::lanes + i) * V, g.cols);
#pragma unroll
            for (int j = 0; j < V; j++)
                if ((uint32_t)j >= at.first) s_sum[group * R::cap + at.a + j] = which ? db[k][j] : dw[k][j];
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < g.cols; c += R::threads) {
            float t = 0.f;
#pragma unroll 8
            for (uint32_t q = 0; q < R::rows; q++) t += s_sum[q * R::cap + c];
            part[which * g.cols + c] = t;
        }
    }
}

// dx of one row by a whole block, reading the row twice.
template <class E, class W, uint32_t Threads>
__device__ __forceinline__ void back_row(const LnBackArgs& g, uint64_t row) {
    constexpr int V = E::vec;
    constexpr uint32_t waves = Threads / 64;
    __shared__ float s_part[2][waves];
    const uint8_t* px = g.x + row * g.ldx;
    const uint8_t* pdy = g.dy + row * g.lddy;
    const float mean = g.mean[row], rstd = g.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (uint32_t c = threadIdx.x * V; c < g.cols; c += Threads * V) {
        const uint32_t rem = g.cols - c;
        const u32x4 x = load_vec<E>(px, c, rem), dy = load_vec<E>(pdy, c, rem);
        float w[V];
        load_param<W, V>(g.w, c, rem, 1.f, w);
        float h[V];
#pragma unroll
        for (int j = 0; j < V; j++) h[j] = (E::get(x, j) - mean) * rstd;
        // places past the row's end hold zeros, whose deviation may be infinite
        if (rem < (uint32_t)V) {
#pragma unroll
            for (int j = 0; j < V; j++) h[j] = (uint32_t)j < rem ? h[j] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < V; j++) {
            const float t = E::get(dy, j) * w[j];
            s1 = fmaf(t, h[j], s1);
            s2 += t;
        }
    }
    s1 = lanes_sum<64>(s1);
    s2 = lanes_sum<64>(s2);
    if ((threadIdx.x & 63u) == 0) {
        s_part[0][threadIdx.x >> 6] = s1;
        s_part[1][threadIdx.x >> 6] = s2;
    }
    __syncthreads();
    s1 = s2 = 0.f;
#pragma unroll
    for (uint32_t q = 0; q < waves; q++) {
        s1 += s_part[0][q];
        s2 += s_part[1][q];
    }
    s1 /= (float)g.cols;
    s2 /= (float)g.cols;
    uint8_t* dst = g.dx + row * g.lddx;
    for (uint32_t c = threadIdx.x * V; c < g.cols; c += Threads * V) {
        const uint32_t rem = g.cols - c;
        const u32x4 x = load_vec<E>(px, c, rem), dy = load_vec<E>(pdy, c, rem);
        float w[V], o[V];
        load_param<W, V>(g.w, c, rem, 1.f, w);
#pragma unroll
        for (int j = 0; j < V; j++)
            o[j] = fmaf(-((E::get(x, j) - mean) * rstd), s1, fmaf(E::get(dy, j), w[j], -s2)) * rstd;
        store_vec<E>(dst, c, rem, o);
    }
}

// Long or very short rows.
template <class E, class W>
__global__ void __launch_bounds__(1024) k_layer_norm_back_long(LnBackArgs g) {
    back_row<E, W, 1024>(g, blockIdx.x);
}

// A backward pass of few rows in one launch: the first blocks take 256 columns
// and a strip of the rows each (8 waves every 8th row, then their sums in
// order), the others write a row of dx each.  Every element is read twice, the
// second time from the caches; in return a column has as many sums to join as
// there are strips, not as there are CUs (a single strip's are final).  In
// place, dx would be written over what a column block has yet to read: then the
// two kinds of blocks are two launches (first_block picks them), with the same
// bits.
struct LnSmallArgs {
    uint32_t columns, strips, first_block;    // column blocks: columns of them per strip
    void* dw;
    void* db;
    int accumulate;
};
constexpr uint32_t kSmallThreads = 512;
template <class E, class W, class G>
__global__ void __launch_bounds__(kSmallThreads) k_layer_norm_back_small(LnBackArgs g, LnSmallArgs o) {
    const uint32_t block = blockIdx.x + o.first_block;
    if (block >= o.columns * o.strips) {
        back_row<E, W, kSmallThreads>(g, block - o.columns * o.strips);
        return;
    }
    const uint32_t strip = block / o.columns, column = block % o.columns;
    const uint32_t per = ((uint32_t)g.rows + o.strips - 1) / o.strips, first = strip * per;
    const uint32_t end = first + per < (uint32_t)g.rows ? first + per : (uint32_t)g.rows;
    constexpr uint32_t waves = kSmallThreads / 64;
    __shared__ float s_sum[2][waves][256];
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
    const uint32_t c = column * 256 + lane * 4;
    const uint32_t rem = c < g.cols ? (g.cols - c < 4 ? g.cols - c : 4) : 0;
    float dw[4] = {0.f, 0.f, 0.f, 0.f}, db[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (uint32_t row = first + wave; row < end; row += waves) {
        float x[4], dy[4];
        load_param<E, 4>(g.x + row * g.ldx, c, rem, 0.f, x);
        load_param<E, 4>(g.dy + row * g.lddy, c, rem, 0.f, dy);
        const float mean = g.mean[row], rstd = g.rstd[row];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            dw[j] = fmaf(dy[j], (x[j] - mean) * rstd, dw[j]);
            db[j] += dy[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; j++) {
        s_sum[0][wave][lane * 4 + j] = dw[j];
        s_sum[1][wave][lane * 4 + j] = db[j];
    }
    __syncthreads();
    const uint32_t which = threadIdx.x >> 8, col = threadIdx.x & 255u;
    typename G::raw* out = static_cast<typename G::raw*>(which ? o.db : o.dw);
    const uint32_t at = column * 256 + col;
    if (at >= g.cols) return;
    float t = 0.f;
#pragma unroll
    for (uint32_t q = 0; q < waves; q++) t += s_sum[which][q][col];
    if (o.strips > 1) {
        g.part[((uint64_t)strip * 2 + which) * g.cols + at] = t;
        return;
    }
    if (!out) return;
    if (o.accumulate) t += G::one(out[at]);
    out[at] = G::round(t);
}

// Sums of dy h and dy over a strip of rows (grid y), a vector of columns per
// thread: k_layer_norm_back's second result for long rows.
template <class E>
__global__ void __launch_bounds__(64) k_layer_norm_columns(LnBackArgs g) {
    constexpr int V = E::vec;
    const uint32_t c = (blockIdx.x * 64 + threadIdx.x) * V;
    if (c >= g.cols) return;
    const uint32_t rem = g.cols - c;
    float dw[V], db[V];
#pragma unroll
    for (int j = 0; j < V; j++) dw[j] = db[j] = 0.f;
    for (uint64_t row = blockIdx.y; row < g.rows; row += gridDim.y) {
        const u32x4 x = load_vec<E>(g.x + row * g.ldx, c, rem), dy = load_vec<E>(g.dy + row * g.lddy, c, rem);
        const float mean = g.mean[row], rstd = g.rstd[row];
#pragma unroll
        for (int j = 0; j < V; j++) {
            const float d = E::get(dy, j);
            dw[j] = fmaf(d, (E::get(x, j) - mean) * rstd, dw[j]);
            db[j] += d;
        }
    }
    float* part = g.part + (uint64_t)blockIdx.y * 2 * g.cols + c;
#pragma unroll
    for (int j = 0; j < V; j++)
        if ((uint32_t)j < rem) {
            part[j] = dw[j];
            part[g.cols + j] = db[j];
        }
}

// The same for rows shorter than a vector, of which there may be 2^31: a row
// per thread and every 2^17th after it (256 blocks), so the chains of additions
// stay short (64 strips of a lane each had 2^25 rows, and a sum of ones stopped
// at 2^24); then the lanes, and the waves through LDS, in order.  70,000 x 5 bf16
// with dx: 498 us, 1940 with the strips.
template <class E>
__global__ void __launch_bounds__(kShortThreads) k_layer_norm_columns_short(LnBackArgs g) {
    constexpr int C = E::vec - 1;                                 // columns at most
    constexpr uint32_t waves = kShortThreads / 64;
    __shared__ float s_sum[2][waves][C];
    float dw[C], db[C];
#pragma unroll
    for (int j = 0; j < C; j++) dw[j] = db[j] = 0.f;
    const uint64_t step = (uint64_t)gridDim.x * kShortThreads;
#pragma unroll 2
    for (uint64_t row = (uint64_t)blockIdx.x * kShortThreads + threadIdx.x; row < g.rows; row += step) {
        const u32x4 x = load_vec<E>(g.x + row * g.ldx, 0, g.cols), dy = load_vec<E>(g.dy + row * g.lddy, 0, g.cols);
        const float mean = g.mean[row], rstd = g.rstd[row];
#pragma unroll
        for (int j = 0; j < C; j++) {
            const float d = E::get(dy, j);
            dw[j] = fmaf(d, (E::get(x, j) - mean) * rstd, dw[j]);
            db[j] += d;
        }
    }
    const uint32_t wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < C; j++) {
        dw[j] = lanes_sum<64>(dw[j]);
        db[j] = lanes_sum<64>(db[j]);
        if ((threadIdx.x & 63u) == 0) {
            s_sum[0][wave][j] = dw[j];
            s_sum[1][wave][j] = db[j];
        }
    }
    __syncthreads();
    if (threadIdx.x >= 2 * g.cols) return;
    const uint32_t which = threadIdx.x >= g.cols, c = threadIdx.x - which * g.cols;
    float t = 0.f;
#pragma unroll
    for (uint32_t q = 0; q < waves; q++) t += s_sum[which][q][c];
    g.part[(uint64_t)blockIdx.x * 2 * g.cols + threadIdx.x] = t;
}

// The weight's and the bias's gradient: the sums of `parts` blocks (at most
// kBackBlocks), 16 waves taking every 16th each with all their loads in
// flight, then the waves' sums in order, onto what is there where they
// accumulate.
constexpr uint32_t kBackBlocks = 256;
template <class G>
__global__ void __launch_bounds__(1024) k_layer_norm_grads(const float* part, uint32_t parts, uint32_t cols,
                                                           typename G::raw* dw, typename G::raw* db, int accumulate) {
    __shared__ float s_sum[16][64];
    const uint32_t wave = threadIdx.x >> 6, l = threadIdx.x & 63u;
    const uint64_t c = (uint64_t)blockIdx.x * 64 + l;             // column of [dw | db]
    const uint64_t width = 2ull * cols;
    const float* p = part + (c < width ? c : width - 1);
    float v[kBackBlocks / 16];
#pragma unroll
    for (uint32_t u = 0; u < kBackBlocks / 16; u++) {
        const uint32_t q = wave + 16 * u;
        v[u] = p[(uint64_t)(q < parts ? q : 0) * width];
    }
    float sum = 0.f;
#pragma unroll
    for (uint32_t u = 0; u < kBackBlocks / 16; u++) sum += wave + 16 * u < parts ? v[u] : 0.f;
    s_sum[wave][l] = sum;
    __syncthreads();
    if (wave || c >= width) return;
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 16; q++) t += s_sum[q][l];
    typename G::raw* out = c < cols ? dw : db;
    if (!out) return;
    const uint64_t at = c < cols ? c : c - cols;
    if (accumulate) t += G::one(out[at]);
    out[at] = G::round(t);
}

// No rows: the sums are zero.
template <class G>
__global__ void __launch_bounds__(256) k_layer_norm_no_grads(uint32_t cols, typename G::raw* dw, typename G::raw* db) {
    const uint64_t c = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= cols) return;
    if (dw) dw[c] = G::round(0.f);
    if (db) db[c] = G::round(0.f);
}

// ---------------------------------------------------------------------------
// host side

inline bool dtype_ok(int32_t dt) { return dt == kF32 || dt == kBF16; }
inline bool aligned(const void* p, int32_t dt) { return (reinterpret_cast<uintptr_t>(p) & (elem_bytes(dt) - 1)) == 0; }
inline spccl_status_t launch_status() { return hipGetLastError() == hipSuccess ? SPCCL_OK : SPCCL_ERR_HIP; }

// Whether two matrices of `rows` x `cols` elements share one.  Rows of the
// same pitch may interleave (column ranges of one buffer).
struct Rows {
    const void* p;
    uint64_t ld;              // elements between rows
};
bool rows_overlap(const Rows& a, const Rows& b, uint64_t rows, uint64_t cols, uint64_t s) {
    if (!rows || !cols) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const uint64_t an = ((rows - 1) * a.ld + cols) * s, bn = ((rows - 1) * b.ld + cols) * s;
    if (x + an <= y || y + bn <= x) return false;
    if (a.ld != b.ld) return true;
    const uint64_t pitch = a.ld * s;
    const uint64_t d = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;
    return d < cols * s || pitch - d < cols * s;
}
bool span_overlap(const void* p, uint64_t pn, const Rows& m, uint64_t rows, uint64_t cols, uint64_t s) {
    if (!p || !m.p || !pn || !rows || !cols) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(m.p);
    return x < y + ((rows - 1) * m.ld + cols) * s && y < x + pn;
}
// Whether an array that is written shares a byte with another of the call.
struct Span {
    const void* p;
    uint64_t bytes;
};
template <size_t Written, size_t Read>
bool spans_overlap(const Span (&w)[Written], const Span (&r)[Read]) {
    const auto meet = [](const Span& a, const Span& b) {
        return a.p && b.p && span_overlap(a.p, a.bytes, Rows{b.p, b.bytes}, 1, b.bytes, 1);
    };
    for (size_t i = 0; i < Written; i++) {
        for (size_t j = 0; j < i; j++)
            if (meet(w[i], w[j])) return true;
        for (const Span& b : r)
            if (meet(w[i], b)) return true;
    }
    return false;
}

// Columns of any call stay below 2^26: k_layer_norm_grads takes 1024 threads for
// 32 of them, k_layer_norm_back_small up to 16 strips of 512 for 256, and a grid
// has fewer than 2^32 threads.
constexpr uint64_t kColsLimit = 1ull << 26;

// The layout of a row: lanes of a wave, or waves, and vectors per lane; calls
// fn with the three as constants.  Each step keeps the lanes two thirds full or
// better where that pays, since a row's fixed instructions count as much as its
// elements' (12952 x 8309 bf16 forward: 86 us in 4 waves of 40, 161 in 8 of 32;
// 16384 x 1600: 16.5 in a wave of 32, 17.3 in two of 16; 16384 x 1024: 11.3 in a
// wave of 16, 13.8 in one of 32).  The backward pass holds two sums for each
// element, so its rows take 16 and spread over waves sooner (32: 65536 x 1024 88
// us against 74, 65536 x 4096 283 against 268); 24 between the powers of two, in
// bf16 only (16384 x 2056: 46 us, 56 without; 16384 x 4099 fp32: 159 and 142).
constexpr uint32_t kMaxCols = 32768, kMaxBackCols = 16384;       // beyond: the long forms

template <int N>
using Int = std::integral_constant<int, N>;

template <class E, bool Back, class Fn>
auto with_row(uint32_t cols, Fn fn) {
    const auto go = [&](auto l, auto waves, auto elements) { return fn(l, waves, Int<elements() / E::vec>{}); };
    if (cols <= 64) return go(Int<8>{}, Int<1>{}, Int<8>{});
    if (cols <= 128) return go(Int<16>{}, Int<1>{}, Int<8>{});
    if (cols <= 256) return go(Int<16>{}, Int<1>{}, Int<16>{});
    if (cols <= 512) return go(Int<32>{}, Int<1>{}, Int<16>{});
    if (cols <= 1024) return go(Int<64>{}, Int<1>{}, Int<16>{});
    if constexpr (Back) {
        constexpr bool bf16 = E::vec == 8;
        if (bf16 && cols <= 1536) return go(Int<64>{}, Int<1>{}, Int<24>{});
        if (cols <= 2048) return go(Int<64>{}, Int<2>{}, Int<16>{});
        if (bf16 && cols <= 3072) return go(Int<64>{}, Int<2>{}, Int<24>{});
        if (cols <= 4096) return go(Int<64>{}, Int<4>{}, Int<16>{});
        if (bf16 && cols <= 6144) return go(Int<64>{}, Int<4>{}, Int<24>{});
        if (cols <= 8192) return go(Int<64>{}, Int<8>{}, Int<16>{});
        if (cols <= 12288) return go(Int<64>{}, Int<8>{}, Int<24>{});
        return go(Int<64>{}, Int<8>{}, Int<32>{});
    } else {
        if (cols <= 1536) return go(Int<64>{}, Int<1>{}, Int<24>{});
        if (cols <= 2048) return go(Int<64>{}, Int<1>{}, Int<32>{});
        if (cols <= 3072) return go(Int<64>{}, Int<2>{}, Int<24>{});
        if (cols <= 4096) return go(Int<64>{}, Int<2>{}, Int<32>{});
        if (cols <= 6144) return go(Int<64>{}, Int<4>{}, Int<24>{});
        if (cols <= 8192) return go(Int<64>{}, Int<4>{}, Int<32>{});
        if (cols <= 10240) return go(Int<64>{}, Int<4>{}, Int<40>{});
        if (cols <= 12288) return go(Int<64>{}, Int<4>{}, Int<48>{});
        if (cols <= 16384) return go(Int<64>{}, Int<8>{}, Int<32>{});
        if (cols <= 24576) return go(Int<64>{}, Int<8>{}, Int<48>{});
        return go(Int<64>{}, Int<16>{}, Int<32>{});
    }
}

// Launches fn(first, count) over rows, as many at a time as one grid may have
// threads for (2^32).
template <class Fn>
spccl_status_t by_rows(uint64_t rows, uint32_t rows_per_block, uint32_t threads, Fn fn) {
    const uint64_t most = (uint64_t)(0xFFFFFFFFu / threads) * rows_per_block;
    for (uint64_t first = 0; first < rows; first += most) {
        fn(first, rows - first < most ? rows - first : most);
        if (launch_status() != SPCCL_OK) return SPCCL_ERR_HIP;
    }
    return SPCCL_OK;
}

LnArgs rows_of(LnArgs g, uint64_t first, uint64_t count) {
    g.x += first * g.ldx;
    g.y += first * g.ldy;
    if (g.mean) g.mean += first;
    if (g.rstd) g.rstd += first;
    g.rows = count;
    return g;
}
LnBackArgs rows_of(LnBackArgs g, uint64_t first, uint64_t count) {
    g.x += first * g.ldx;
    g.dy += first * g.lddy;
    g.dx += first * g.lddx;
    g.mean += first;
    g.rstd += first;
    g.rows = count;
    return g;
}

template <class E, class W>
spccl_status_t launch_forward(const LnArgs& g, hipStream_t st) {
    if (g.cols > kMaxCols || g.cols < (uint32_t)E::vec)
        return by_rows(g.rows, 1, 1024, [&](uint64_t first, uint64_t count) {
            hipLaunchKernelGGL((k_layer_norm_long<E, W>), dim3((uint32_t)count), dim3(1024), 0, st, rows_of(g, first, count));
        });
    return with_row<E, false>(g.cols, [&](auto l, auto waves, auto k) {
        using R = Row<E, l(), waves(), k()>;
        return by_rows(g.rows, R::rows, R::threads, [&](uint64_t first, uint64_t count) {
            const dim3 grid((uint32_t)((count + R::rows - 1) / R::rows)), block(R::threads);
            const LnArgs part = rows_of(g, first, count);
            if (g.cols % E::vec) hipLaunchKernelGGL((k_layer_norm<E, W, l(), waves(), k(), true>), grid, block, 0, st, part);
            else hipLaunchKernelGGL((k_layer_norm<E, W, l(), waves(), k(), false>), grid, block, 0, st, part);
        });
    });
}

// Blocks of a backward pass, each of which leaves two sums per column: one per
// CU, as every further block's sums are written and read again (65536 x 4096
// bf16: 268 us; with 512 blocks of 256 threads 277, with 1024 blocks 353), and
// none for less than two rounds of rows (307 x 11622: 25 us; one round 36, four
// 29).
constexpr uint32_t kStrips = 64;
static_assert(kStrips <= kBackBlocks, "k_layer_norm_grads adds up to kBackBlocks parts");
uint32_t back_blocks(uint64_t rows, uint32_t rows_per_block) {
    const uint64_t b = (rows + 2 * rows_per_block - 1) / (2 * rows_per_block);
    return (uint32_t)(b < kBackBlocks ? b : kBackBlocks);
}
uint32_t strips(uint64_t rows) { return (uint32_t)(rows < kStrips ? rows : kStrips); }
// blocks of k_layer_norm_columns_short
uint32_t short_blocks(uint64_t rows) {
    const uint64_t b = (rows + kShortThreads - 1) / kShortThreads;
    return (uint32_t)(b < kBackBlocks ? b : kBackBlocks);
}

// Backward passes of up to 1024 rows in bf16, 512 in fp32, are taken by
// k_layer_norm_back_small at any width: reading their rows twice moves less
// than a pair of sums per column and CU (us with the host's part, so / by
// k_layer_norm_back, bf16: 64 x 1024 9.7 / 12.9, 256 x 8192 12.3 / 17.1, 512 x
// 16384 22 / 40, 1024 x 8192 19 / 26, 1536 x 16384 60 / 55; fp32: 512 x 4096
// 12.1 / 13.2, 1024 x 4096 18.6 / 16.5).  Narrow rows leave most lanes of its
// blocks idle and are much the same either way (the kernels alone, 256 x 256 bf16
// 7.6 / 9.0, 256 x 128 8.1 / 7.1, 256 x 64 8.1 / 7.4; fp32 6.0 / 9.4, 6.5 / 6.6,
// 6.4 / 7.1); a call of 129 rows and more takes 11-12 with either.  Strips of 64
// rows beyond 128.
template <class E>
bool small_backward(uint64_t rows) {
    return rows * sizeof(typename E::raw) <= 2048;
}
inline uint32_t small_strips(uint64_t rows) { return rows <= 128 ? 1 : (uint32_t)((rows + 63) / 64); }

template <class E>
uint32_t back_parts(uint64_t rows, uint32_t cols) {
    if (small_backward<E>(rows)) return small_strips(rows);
    if (cols > kMaxBackCols) return strips(rows);
    if (cols < (uint32_t)E::vec) return short_blocks(rows);
    return with_row<E, true>(cols, [&](auto l, auto waves, auto k) {
        return back_blocks(rows, Row<E, l(), waves(), k(), kBackThreads>::rows);
    });
}

template <class E, class W>
spccl_status_t launch_small(const LnBackArgs& g, int32_t gdtype, void* dw, void* db, int32_t accumulate, bool in_place,
                            hipStream_t st) {
    LnSmallArgs o{(g.cols + 255) / 256, g.part ? small_strips(g.rows) : 0, 0, dw, db, accumulate};
    const uint32_t rows = g.dx ? (uint32_t)g.rows : 0, sums = o.columns * o.strips;
    const auto go = [&](uint32_t first, uint32_t count) {
        if (!count) return SPCCL_OK;
        o.first_block = first;
        if (gdtype == kBF16)
            hipLaunchKernelGGL((k_layer_norm_back_small<E, W, BF16>), dim3(count), dim3(kSmallThreads), 0, st, g, o);
        else
            hipLaunchKernelGGL((k_layer_norm_back_small<E, W, F32>), dim3(count), dim3(kSmallThreads), 0, st, g, o);
        return launch_status();
    };
    if (!in_place) return go(0, sums + rows);
    const spccl_status_t st1 = go(0, sums);
    return st1 == SPCCL_OK ? go(sums, rows) : st1;
}

spccl_status_t launch_grads(const float* part, uint32_t parts, uint32_t cols, int32_t gdtype, void* dw, void* db,
                            int32_t accumulate, hipStream_t st) {
    const dim3 grid((uint32_t)((2ull * cols + 63) / 64)), block(1024);
    if (gdtype == kBF16)
        hipLaunchKernelGGL(k_layer_norm_grads<BF16>, grid, block, 0, st, part, parts, cols, static_cast<uint16_t*>(dw),
                           static_cast<uint16_t*>(db), accumulate);
    else
        hipLaunchKernelGGL(k_layer_norm_grads<F32>, grid, block, 0, st, part, parts, cols, static_cast<uint32_t*>(dw),
                           static_cast<uint32_t*>(db), accumulate);
    return launch_status();
}

template <class E, class W>
spccl_status_t launch_backward(const LnBackArgs& g, int32_t gdtype, void* dw, void* db, int32_t accumulate,
                               hipStream_t st) {
    if (small_backward<E>(g.rows)) {
        const bool in_place = g.dx && (g.dx == g.x || g.dx == g.dy);
        const spccl_status_t st1 = launch_small<E, W>(g, gdtype, dw, db, accumulate, in_place, st);
        if (st1 != SPCCL_OK || !g.part || small_strips(g.rows) == 1) return st1;
        return launch_grads(g.part, small_strips(g.rows), g.cols, gdtype, dw, db, accumulate, st);
    }
    if (g.cols > kMaxBackCols || g.cols < (uint32_t)E::vec) {
        // the columns' sums first: dx may be written over dy or x
        if (g.part) {
            if (g.cols < (uint32_t)E::vec)
                hipLaunchKernelGGL(k_layer_norm_columns_short<E>, dim3(short_blocks(g.rows)), dim3(kShortThreads), 0, st, g);
            else
                hipLaunchKernelGGL(k_layer_norm_columns<E>,
                                   dim3((g.cols + 64 * E::vec - 1) / (64 * E::vec), strips(g.rows)), dim3(64), 0, st, g);
            if (launch_status() != SPCCL_OK) return SPCCL_ERR_HIP;
        }
        if (g.dx) {
            const spccl_status_t st1 = by_rows(g.rows, 1, 1024, [&](uint64_t first, uint64_t count) {
                hipLaunchKernelGGL((k_layer_norm_back_long<E, W>), dim3((uint32_t)count), dim3(1024), 0, st,
                                   rows_of(g, first, count));
            });
            if (st1 != SPCCL_OK) return st1;
        }
    } else {
        with_row<E, true>(g.cols, [&](auto l, auto waves, auto k) {
            using R = Row<E, l(), waves(), k(), kBackThreads>;
            const dim3 grid(back_blocks(g.rows, R::rows)), block(R::threads);
            // a misaligned row's vectors lie across lines, which streaming
            // loads would fetch twice: it takes the ordinary ones (7434 x
            // 5760 bf16, pitch 5761: 60 us, 81 streamed)
            const bool odd = g.cols % E::vec || ((reinterpret_cast<uintptr_t>(g.x) | reinterpret_cast<uintptr_t>(g.dy) |
                                                  g.ldx | g.lddy) & 15u);
            if (odd) hipLaunchKernelGGL((k_layer_norm_back<E, W, l(), waves(), k(), true>), grid, block, 0, st, g);
            else hipLaunchKernelGGL((k_layer_norm_back<E, W, l(), waves(), k(), false>), grid, block, 0, st, g);
        });
    }
    if (launch_status() != SPCCL_OK) return SPCCL_ERR_HIP;
    if (!g.part) return SPCCL_OK;
    return launch_grads(g.part, back_parts<E>(g.rows, g.cols), g.cols, gdtype, dw, db, accumulate, st);
}

}  // namespace
}  // namespace spccl

using namespace spccl;

extern "C" {

spccl_status_t spccl_layer_norm(const void* x, uint64_t ldx, const void* weight, const void* bias, void* y, uint64_t ldy,
                                float* mean, float* rstd, uint64_t rows, uint64_t cols, int32_t dtype, int32_t wdtype,
                                double eps, void* stream) {
    if (!dtype_ok(dtype) || !dtype_ok(wdtype)) return SPCCL_ERR_UNSUPPORTED;
    if (rows >= (1ull << 31) || cols >= kColsLimit) return SPCCL_ERR_UNSUPPORTED;
    if (cols == 0 || ldx < cols || ldy < cols || !(eps >= 0.0)) return SPCCL_ERR_INVALID_ARG;
    if (rows == 0) return SPCCL_OK;
    if (!x || !y || !aligned(x, dtype) || !aligned(y, dtype) || !aligned(weight, wdtype) || !aligned(bias, wdtype) ||
        !aligned(mean, kF32) || !aligned(rstd, kF32))
        return SPCCL_ERR_INVALID_ARG;
    const uint64_t s = elem_bytes(dtype), ws = elem_bytes(wdtype);
    const Rows rx{x, ldx}, ry{y, ldy};
    if (!(x == y && ldx == ldy) && rows_overlap(rx, ry, rows, cols, s)) return SPCCL_ERR_INVALID_ARG;
    for (const Rows& m : {rx, ry})
        if (span_overlap(mean, 4 * rows, m, rows, cols, s) || span_overlap(rstd, 4 * rows, m, rows, cols, s))
            return SPCCL_ERR_INVALID_ARG;
    if (span_overlap(weight, ws * cols, ry, rows, cols, s) || span_overlap(bias, ws * cols, ry, rows, cols, s))
        return SPCCL_ERR_INVALID_ARG;
    const Span statistics[2] = {{mean, 4 * rows}, {rstd, 4 * rows}}, params[2] = {{weight, ws * cols}, {bias, ws * cols}};
    if (spans_overlap(statistics, params)) return SPCCL_ERR_INVALID_ARG;
    const LnArgs g{static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(weight), static_cast<const uint8_t*>(bias),
                   static_cast<uint8_t*>(y), mean, rstd, ldx * s, ldy * s, rows, (uint32_t)cols, (float)eps};
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (dtype == kF32) return wdtype == kF32 ? launch_forward<F32, F32>(g, st) : launch_forward<F32, BF16>(g, st);
    return wdtype == kF32 ? launch_forward<BF16, F32>(g, st) : launch_forward<BF16, BF16>(g, st);
}

uint64_t spccl_layer_norm_scratch_bytes(uint64_t rows, uint64_t cols) {
    if (rows == 0 || rows >= (1ull << 31) || cols == 0 || cols >= kColsLimit) return 0;
    const uint32_t a = back_parts<F32>(rows, (uint32_t)cols), b = back_parts<BF16>(rows, (uint32_t)cols);
    return 8ull * cols * (a > b ? a : b);
}

spccl_status_t spccl_layer_norm_backward(const void* dy, uint64_t lddy, const void* x, uint64_t ldx, const void* weight,
                                         const float* mean, const float* rstd, void* dx, uint64_t lddx, void* dweight,
                                         void* dbias, uint64_t rows, uint64_t cols, int32_t dtype, int32_t wdtype,
                                         int32_t gdtype, int32_t accumulate, void* scratch, uint64_t scratch_bytes,
                                         void* stream) {
    if (!dtype_ok(dtype) || !dtype_ok(wdtype) || !dtype_ok(gdtype)) return SPCCL_ERR_UNSUPPORTED;
    if (rows >= (1ull << 31) || cols >= kColsLimit) return SPCCL_ERR_UNSUPPORTED;
    if (cols == 0 || lddy < cols || ldx < cols || (dx && lddx < cols)) return SPCCL_ERR_INVALID_ARG;
    if (!aligned(dweight, gdtype) || !aligned(dbias, gdtype)) return SPCCL_ERR_INVALID_ARG;
    const bool grads = dweight || dbias;
    if (rows && (!dy || !x || !mean || !rstd || !aligned(dy, dtype) || !aligned(x, dtype) || !aligned(dx, dtype) ||
                 !aligned(weight, wdtype) || !aligned(mean, kF32) || !aligned(rstd, kF32)))
        return SPCCL_ERR_INVALID_ARG;
    const uint64_t s = elem_bytes(dtype), gs = elem_bytes(gdtype);
    const uint64_t need = grads ? spccl_layer_norm_scratch_bytes(rows, cols) : 0;
    if (need) {
        if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 15u)) return SPCCL_ERR_INVALID_ARG;
        if (scratch_bytes < need) return SPCCL_ERR_WORKSPACE;
    }
    const Rows rdy{dy, lddy}, rx{x, ldx}, rdx{dx, lddx};
    if (rows && dx) {
        if (!(dx == dy && lddx == lddy) && rows_overlap(rdx, rdy, rows, cols, s)) return SPCCL_ERR_INVALID_ARG;
        if (!(dx == x && lddx == ldx) && rows_overlap(rdx, rx, rows, cols, s)) return SPCCL_ERR_INVALID_ARG;
        if (span_overlap(weight, elem_bytes(wdtype) * cols, rdx, rows, cols, s) ||
            span_overlap(mean, 4 * rows, rdx, rows, cols, s) || span_overlap(rstd, 4 * rows, rdx, rows, cols, s))
            return SPCCL_ERR_INVALID_ARG;
    }
    const Rows d[3] = {rdy, rx, rdx};
    for (const Rows& m : d)
        if (span_overlap(dweight, gs * cols, m, rows, cols, s) || span_overlap(dbias, gs * cols, m, rows, cols, s) ||
            (need && span_overlap(scratch, need, m, rows, cols, s)))
            return SPCCL_ERR_INVALID_ARG;
    const Span sums[3] = {{dweight, gs * cols}, {dbias, gs * cols}, {need ? scratch : nullptr, need}};
    const Span read[3] = {{weight, elem_bytes(wdtype) * cols}, {mean, 4 * rows}, {rstd, 4 * rows}};
    if (spans_overlap(sums, read)) return SPCCL_ERR_INVALID_ARG;
    const LnBackArgs g{static_cast<const uint8_t*>(dy), static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(weight),
                       mean, rstd, static_cast<uint8_t*>(dx), grads ? static_cast<float*>(scratch) : nullptr,
                       lddy * s, ldx * s, lddx * s, rows, (uint32_t)cols};
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (rows == 0) {
        // no rows: the sums are zero
        if (!grads || accumulate) return SPCCL_OK;
        const dim3 grid((uint32_t)((cols + 255) / 256)), block(256);
        if (gdtype == kBF16)
            hipLaunchKernelGGL(k_layer_norm_no_grads<BF16>, grid, block, 0, st, (uint32_t)cols,
                               static_cast<uint16_t*>(dweight), static_cast<uint16_t*>(dbias));
        else
            hipLaunchKernelGGL(k_layer_norm_no_grads<F32>, grid, block, 0, st, (uint32_t)cols,
                               static_cast<uint32_t*>(dweight), static_cast<uint32_t*>(dbias));
        return launch_status();
    }
    if (!dx && !grads) return SPCCL_OK;
    if (dtype == kF32)
        return wdtype == kF32 ? launch_backward<F32, F32>(g, gdtype, dweight, dbias, accumulate, st)
                              : launch_backward<F32, BF16>(g, gdtype, dweight, dbias, accumulate, st);
    return wdtype == kF32 ? launch_backward<BF16, F32>(g, gdtype, dweight, dbias, accumulate, st)
                          : launch_backward<BF16, BF16>(g, gdtype, dweight, dbias, accumulate, st);
}

}  // extern "C"
