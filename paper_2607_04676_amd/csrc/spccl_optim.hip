// The two ends of a data-parallel step around the collectives: pruning a
// gradient with error feedback (Sec. VI-B), and the AdamW step over many
// tensors at once that consumes the reduced gradient.
//
//   prune   a = g + leak r;  out = a where |a| >= threshold, else 0;
//           r = a - out
//   AdamW   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//           p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Both are bound by memory: every array is read and written once and nothing is
// kept for a second pass.  All arithmetic is fp32, each operation rounded by
// itself (no contraction), so equal inputs give equal bits wherever it is
// computed.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <algorithm>

#include "spccl_internal.h"
#include "../../include/spccl.h"

namespace spccl {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// vectors at any element's address
typedef u32x4 __attribute__((aligned(4))) u32x4_any;
typedef u32x2 __attribute__((aligned(2))) u32x2_any;
typedef uint32_t __attribute__((aligned(1))) u32_any;

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {         // nearest, ties to even
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// A pair whose zeros have no sign: rounding made them of small negative values.
__device__ __forceinline__ uint32_t no_minus_zero(uint32_t p) {
    if ((p & 0x7FFFu) == 0) p &= 0xFFFF0000u;
    if ((p & 0x7FFF0000u) == 0) p &= 0x0000FFFFu;
    return p;
}

// A place in global memory, as a base that the whole block shares (scalar
// registers) and a lane's offset in bytes.  A table's addresses are numbers to
// the compiler; without the address space it would take generic accesses, which
// count against the LDS as well and kept an 8-bit step of 10^8 elements at 485
// us instead of 299.
template <class T>
__device__ __forceinline__ T __attribute__((address_space(1))) * at(uint64_t base, uint32_t offset) {
    return (T __attribute__((address_space(1)))*)(base + offset);
}

// Four consecutive elements from element o of a chunk on, `rem` of which exist
// (Full: all; the others read 0 and are not written).  Every array is read
// once and written once a call, so all accesses are non-temporal: an fp32 step
// of 2^28 elements takes 1338 us so and 1455 through the caches, an 8-bit one
// of 10^8 263 and 291 (at 2^22 elements, which the caches hold from call to
// call, 20.7 and 19.2).
struct Quad {
    float f[4];
};
template <int DT, bool Full>
__device__ __forceinline__ Quad get4(uint64_t base, uint32_t o, uint32_t rem) {
    Quad q{{0.f, 0.f, 0.f, 0.f}};
    if constexpr (DT == kF32) {
        if (Full || rem >= 4) {
            const u32x4 v = __builtin_nontemporal_load(at<const u32x4_any>(base, 4 * o));
#pragma unroll
            for (int j = 0; j < 4; j++) q.f[j] = __uint_as_float(v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 3; j++)
                if ((uint32_t)j < rem) q.f[j] = __uint_as_float(at<const uint32_t>(base, 4 * o)[j]);
        }
    } else {
        if (Full || rem >= 4) {
            const u32x2 v = __builtin_nontemporal_load(at<const u32x2_any>(base, 2 * o));
#pragma unroll
            for (int j = 0; j < 4; j++) q.f[j] = __uint_as_float(j & 1 ? v[j / 2] & 0xFFFF0000u : v[j / 2] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < 3; j++)
                if ((uint32_t)j < rem) q.f[j] = __uint_as_float((uint32_t)at<const uint16_t>(base, 2 * o)[j] << 16);
        }
    }
    return q;
}
template <bool Full>
__device__ __forceinline__ void put4_f32(uint64_t base, uint32_t o, uint32_t rem, const float* f) {
    if (Full || rem >= 4) {
        const u32x4 v{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
        __builtin_nontemporal_store(v, at<u32x4_any>(base, 4 * o));
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; j++)
        if ((uint32_t)j < rem) at<uint32_t>(base, 4 * o)[j] = __float_as_uint(f[j]);
}
template <bool Full>
__device__ __forceinline__ void put4_16(uint64_t base, uint32_t o, uint32_t rem, u32x2 v) {
    if (Full || rem >= 4) {
        __builtin_nontemporal_store(v, at<u32x2_any>(base, 2 * o));
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; j++)
        if ((uint32_t)j < rem) at<uint16_t>(base, 2 * o)[j] = (uint16_t)(v[j / 2] >> (16 * (j & 1)));
}
template <bool Full>
__device__ __forceinline__ uint32_t get4_8(uint64_t base, uint32_t o, uint32_t rem) {
    if (Full || rem >= 4) return __builtin_nontemporal_load(at<const u32_any>(base, o));
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 3; j++)
        if ((uint32_t)j < rem) w |= (uint32_t)at<const uint8_t>(base, o)[j] << (8 * j);
    return w;
}
template <bool Full>
__device__ __forceinline__ void put4_8(uint64_t base, uint32_t o, uint32_t rem, uint32_t w) {
    if (Full || rem >= 4) {
        __builtin_nontemporal_store(w, at<u32_any>(base, o));
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; j++)
        if ((uint32_t)j < rem) at<uint8_t>(base, o)[j] = (uint8_t)(w >> (8 * j));
}

inline spccl_status_t launch_status() { return hipGetLastError() == hipSuccess ? SPCCL_OK : SPCCL_ERR_HIP; }
inline bool dtype_ok(int32_t dt) { return dt == kF32 || dt == kBF16; }
inline bool aligned_to(const void* p, uint64_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool overlaps(const void* a, uint64_t an, const void* b, uint64_t bn) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return an && bn && x < y + bn && y < x + an;
}

// ---------------------------------------------------------------------------
// pruning with error feedback

constexpr uint32_t kThreads = 256;
// Quads of a thread and elements of a block (fp32 at 2^26 elements with 4, 2 and
// 1 quads 170, 180 and 178 us: 6.3 TB/s with 4; bf16 at 10^8 191, 191 and 188).
constexpr uint32_t kPruneQuads = 4, kPruneChunk = kThreads * kPruneQuads * 4;

struct PruneArgs {
    const uint8_t* grad;
    uint8_t* residual;
    uint8_t* out;
    const float* threshold;
    uint64_t n;
    float leak;
};

// What is not finite is sent, never kept: a NaN or an infinity that stayed
// behind would spoil its element for good and no rank would see it.  A sum
// that overflows bf16 is sent as the infinity it rounds to, likewise without
// a residual.
template <int DT, bool Full>
__device__ __forceinline__ void prune_chunk(const PruneArgs& g, uint64_t e0, uint32_t end) {
    constexpr uint32_t size = DT == kF32 ? 4 : 2;
    const uint64_t grad = (uint64_t)g.grad + e0 * size, out = (uint64_t)g.out + e0 * size;
    const uint64_t residual = (uint64_t)g.residual + e0 * 4;
    const float tau = *g.threshold;
    const auto exists = [&](uint32_t i) -> uint32_t { return Full ? 4u : (i >= end ? 0u : (end - i < 4 ? end - i : 4u)); };
    Quad x[kPruneQuads], r[kPruneQuads];
#pragma unroll
    for (uint32_t k = 0; k < kPruneQuads; k++) {
        const uint32_t i = (k * kThreads + threadIdx.x) * 4;
        x[k] = get4<DT, Full>(grad, i, exists(i));
        r[k] = get4<kF32, Full>(residual, i, exists(i));
    }
#pragma unroll
    for (uint32_t k = 0; k < kPruneQuads; k++) {
        const uint32_t i = (k * kThreads + threadIdx.x) * 4, rem = exists(i);
        if (!Full && !rem) continue;
        float sent[4], back[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float a = x[k].f[j] + g.leak * r[k].f[j];
            // a zero is absent, whatever its sign (bf16's own zeros: below)
            const bool stays = fabsf(a) < tau || a == 0.f;
            sent[j] = stays ? 0.f : a;
            back[j] = a;
        }
        u32x2 pairs;
        if constexpr (DT == kBF16) {
            pairs = u32x2{no_minus_zero(bf16_pair(sent[0], sent[1])), no_minus_zero(bf16_pair(sent[2], sent[3]))};
#pragma unroll
            for (int j = 0; j < 4; j++)
                sent[j] = __uint_as_float(j & 1 ? pairs[j / 2] & 0xFFFF0000u : pairs[j / 2] << 16);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) back[j] = __builtin_isfinite(sent[j]) ? back[j] - sent[j] : 0.f;
        put4_f32<Full>(residual, i, rem, back);
        if constexpr (DT == kBF16) put4_16<Full>(out, i, rem, pairs);
        else put4_f32<Full>(out, i, rem, sent);
    }
}

template <int DT>
__global__ void __launch_bounds__(kThreads) k_prune(PruneArgs g) {
    const uint64_t e0 = (uint64_t)blockIdx.x * kPruneChunk;
    if (g.n - e0 >= kPruneChunk) prune_chunk<DT, true>(g, e0, kPruneChunk);
    else prune_chunk<DT, false>(g, e0, (uint32_t)(g.n - e0));
}

// ---------------------------------------------------------------------------
// AdamW

constexpr uint32_t kBlock = 32;             // 8-bit states: elements that share a scale


// One tensor as the kernel sees it, in the plan's table.
struct AdamTensor {
    uint8_t* param;
    uint8_t* model;
    uint8_t* m;
    uint8_t* v;
    uint8_t* ms;
    uint8_t* vs;
    const uint8_t* grad;      // the array, or the message
    uint64_t grad_cap;
    uint64_t grad_n;          // elements of the message
    uint64_t grad_offset;     // the tensor's first element in it
    uint64_t n;
    uint64_t counter;         // its first element's place in the random sequence
    uint64_t first;           // its first chunk
    uint64_t chunks;
    double decay;             // weight decay
    uint64_t pad;
};
static_assert(sizeof(AdamTensor) == 128, "a table entry is 128 bytes");

constexpr int kTableBatch = 24;             // entries that travel in one launch's arguments
struct TableArgs {
    AdamTensor t[kTableBatch];
    AdamTensor* table;
    uint32_t* chunk;          // tensor of every chunk
    uint32_t first, count;
};

// Writes a batch of table entries (block b: entry b) and their chunks' words.
__global__ void __launch_bounds__(kThreads) k_adamw_table(TableArgs a) {
    const AdamTensor& t = a.t[blockIdx.x];
    if (threadIdx.x == 0) a.table[a.first + blockIdx.x] = t;
    for (uint64_t c = threadIdx.x; c < t.chunks; c += kThreads) a.chunk[t.first + c] = a.first + blockIdx.x;
}

struct AdamArgs {
    const AdamTensor* table;
    const uint32_t* chunk;
    const float* grad_scale;  // null: 1
    WsCtrl* ctrl;
    uint64_t chunk0;          // of this launch's first block
    double lr;
    float b1, c1, b2, c2;     // beta and 1 - beta
    float root, rate, eps;    // 1 / sqrt(1 - b2^t), lr / (1 - b1^t)
    uint32_t key;             // of the random sequence
};

// Random bits: a multiplicative hash (Knuth's golden-ratio multiplier and one
// from the square root of 2, each between shifted exclusive ors) of the place
// of four elements under a key drawn from the seed; the four take it a
// golden-ratio stride apart, which spreads them evenly over the range.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x9E3779B1u;
    x ^= x >> 15;
    x *= 0x6A09E667u;
    return x ^ (x >> 16);
}
constexpr uint32_t kStride = 0x9E3779B9u, kSecond = 0x6A09E667u;

// x to bf16, rounded up with the probability of the part cut off (16 random
// bits): nearest-even would lose every update below half a unit of a 16-bit
// parameter.
__device__ __forceinline__ uint32_t bf16_stochastic(float x, uint32_t r) {
    const uint32_t b = __float_as_uint(x);
    return ((b & 0x7F800000u) == 0x7F800000u ? b : b + (r >> 16)) >> 16;
}

// The largest magnitude's bits over the 8 lanes (32 elements) of a block.
template <int Ctrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, Ctrl, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t block_max(uint32_t x) {
    constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141;
    x = max(x, dpp<kXor1>(x));
    x = max(x, dpp<kXor2>(x));
    return max(x, dpp<kMirror8>(x));
}

// 8-bit states: E4M3 values times a power of two that a block of 32 shares
// (its exponent in one byte, biased by 127).  The scale brings the block's
// largest magnitude into [2^7, 2^8), so the values' 448 is never passed; it
// is exact, and so is a stored value's product with it.  What is stored is
// rounded stochastically: beta2 = 0.999 moves a second moment by a thousandth
// of itself a step, which rounding to nearest would never let happen at three
// bits of mantissa.  A second moment above zero stays above zero (2^-9 is the
// smallest value), so no update divides by eps alone.  A block with a NaN or
// an infinity has the scale 255 and stands for NaN.
struct Scale {
    uint32_t byte;
    float up;                 // 2^-(its exponent); 0 for a block that is not finite
};
__device__ __forceinline__ Scale scale_of(uint32_t top) {
    uint32_t e = top >> 23;
    const bool finite = e != 255u;
    e = max(e, 32u);
    return Scale{finite ? e - 7u : 255u, finite ? __uint_as_float((261u - e) << 23) : 0.f};
}
__device__ __forceinline__ uint32_t encode4(const float* x, float up, uint32_t h, int left, bool second) {
    int word = 0;
    const float least = second && up != 0.f ? 0x1p-9f : 0.f;
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
        y[j] = x[j] * up;
        if (second) y[j] = x[j] > 0.f ? fmaxf(y[j], least) : y[j];
    }
    word = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], (h + 0 * kStride) << left, word, 0);
    word = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], (h + 1 * kStride) << left, word, 1);
    word = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], (h + 2 * kStride) << left, word, 2);
    word = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], (h + 3 * kStride) << left, word, 3);
    return (uint32_t)word;
}
__device__ __forceinline__ Quad decode4(uint32_t word, uint32_t scale) {
    const float s = __uint_as_float(scale == 255u ? 0x7FC00000u : scale << 23);    // 255: NaN, whatever the values
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true);
    return Quad{{a[0] * s, a[1] * s, b[0] * s, b[1] * s}};
}
// A gradient message: its header, checked like every reader's (each offset is
// the one that the layout implies, so a passing header bounds every read).
struct Message {
    bool ok, pici;
    uint64_t nnz;
};
__device__ __forceinline__ Message check_message(const uint8_t* msg, uint64_t cap, uint64_t n, int dtype) {
    const uint64_t* w = reinterpret_cast<const uint64_t*>(msg);
    const uint32_t fmt = (uint32_t)(w[0] >> 32) & 0xFFFFu;
    const uint64_t nnz = w[2], total = w[5];
    bool ok = (uint32_t)w[0] == kMagic && (uint32_t)(w[0] >> 48) == (uint32_t)dtype && w[1] == n && total <= cap;
    if (fmt == (uint32_t)kFmtPici)
        ok = ok && w[3] == off_I(n) && w[4] == off_A(n) && nnz <= n && total == pici_bytes(n, dtype, nnz);
    else
        ok = ok && fmt == (uint32_t)kFmtDense && w[4] == kHeaderBytes && total == dense_msg_bytes(n, dtype);
    return Message{ok, fmt == (uint32_t)kFmtPici, nnz};
}

__device__ __forceinline__ uint32_t wave_incl_scan(uint32_t x) {
    constexpr int kRowShr = 0x110, kRowBcast15 = 0x142, kRowBcast31 = 0x143;
    int v = (int)x;
    v += __builtin_amdgcn_update_dpp(0, v, kRowShr + 1, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, kRowShr + 2, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, kRowShr + 4, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, kRowShr + 8, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, kRowBcast15, 0xa, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, kRowBcast31, 0xc, 0xf, false);
    return (uint32_t)v;
}

// Expands tile t of a checked Pici message into LDS, row by row: lane c of
// wave w walks rows [16w, 16w + 16) of column c.  A tile whose counts disagree
// with its index or that sets a bit past the end is empty and flagged.
template <int GT>
__device__ __forceinline__ void expand_tile(const uint8_t* msg, uint64_t nnz, uint64_t n, uint64_t t, float* tile,
                                            WsCtrl* ctrl) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t word = reinterpret_cast<const uint64_t*>(msg + kHeaderBytes)[t * 64 + lane];
    const uint32_t* I = reinterpret_cast<const uint32_t*>(msg + off_I(n));
    const uint32_t base = I[t], next = I[t + 1];
    u32x4* zero = reinterpret_cast<u32x4*>(tile);
#pragma unroll
    for (uint32_t k = 0; k < kTileElems / (4 * kThreads); k++) zero[k * kThreads + threadIdx.x] = u32x4{0, 0, 0, 0};
    const uint32_t cnt = (uint32_t)__popcll(word);
    const uint32_t incl = wave_incl_scan(cnt);
    const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    // rows of this column below n
    const uint64_t left = n - t * kTileElems;
    const uint32_t rows = left >= kTileElems ? 64u : (left > lane ? (uint32_t)((left - lane + 63) / 64) : 0u);
    const bool past = rows < 64 && (word >> rows) != 0;
    const bool bad = __any(past) || next < base || next - base != total || next > nnz;
    __syncthreads();
    if (bad) {
        if (threadIdx.x == 0) atomicCAS(&ctrl->status, 0u, (uint32_t)SPCCL_ERR_CORRUPT_STREAM);
    } else {
        const uint32_t r0 = wave * 16;
        uint32_t bits = (uint32_t)(word >> r0) & 0xFFFFu;
        uint64_t rank = (uint64_t)base + (incl - cnt) + (uint32_t)__popcll(word & ((1ull << r0) - 1));
        const uint8_t* A = msg + off_A(n);
        while (bits) {
            const uint32_t r = (uint32_t)__builtin_ctz(bits);
            bits &= bits - 1;
            float f;
            if constexpr (GT == kF32) f = __uint_as_float(reinterpret_cast<const uint32_t*>(A)[rank]);
            else f = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(A)[rank] << 16);
            tile[(r0 + r) * 64 + lane] = f;
            rank++;
        }
    }
    __syncthreads();
}

// Quads of a thread and elements of a chunk: a stream's chunk is a tile of the
// message; an array's is a quad a thread.  More in flight per block is no
// faster (2, 4 and 8 quads at 2^28 elements: 1384, 1354 and 1327 us against
// 1338, but 274, 272 and 290 against 263 in 8 bits, and 78, 82 and 84 against
// 77 at 2^24).
constexpr uint32_t chunk_quads(bool stream) { return stream ? kTileElems / (kThreads * 4) : 1; }
constexpr uint32_t chunk_elems(bool stream) { return kThreads * chunk_quads(stream) * 4; }
static_assert(chunk_elems(true) == kTileElems, "a stream's chunk is a tile");

// What a block works on: a tensor's arrays from the chunk's first element on,
// `lead` places before which (a stream's first chunk) and `end` places after
// which the tensor has none.
struct Chunk {
    uint64_t param, model, m, v, ms, vs, grad;
    uint32_t lead, end;
    uint32_t random;          // place of the first element in the random sequence, over 4
    bool pici;
    uint64_t nnz, tile;
};

template <int PT, int GT, bool Eight, bool Stream, bool Full>
__device__ __forceinline__ void adamw_chunk(const AdamArgs& a, const AdamTensor& t, const Chunk& c, float* tile) {
    constexpr uint32_t kQuads = chunk_quads(Stream);
    const uint32_t i0 = threadIdx.x * 4;
    const auto exists = [&](uint32_t i) -> uint32_t {          // how many of the four places at i
        return Full ? 4u : (i < c.lead || i >= c.end ? 0u : (c.end - i < 4 ? c.end - i : 4u));
    };
    Quad p[kQuads], g[kQuads], m[kQuads], v[kQuads];
    uint32_t mc[kQuads], vc[kQuads], ms[kQuads], vs[kQuads];
#pragma unroll
    for (uint32_t k = 0; k < kQuads; k++) {
        const uint32_t i = i0 + k * kThreads * 4, rem = exists(i);
        p[k] = get4<PT, Full>(c.param, i, rem);
        if (!Stream || !c.pici) g[k] = get4<GT, Full>(c.grad, i, rem);
        if constexpr (Eight) {
            mc[k] = get4_8<Full>(c.m, i, rem);
            vc[k] = get4_8<Full>(c.v, i, rem);
            ms[k] = Full || rem ? *at<const uint8_t>(c.ms, i / kBlock) : 0;
            vs[k] = Full || rem ? *at<const uint8_t>(c.vs, i / kBlock) : 0;
        } else {
            m[k] = get4<kF32, Full>(c.m, i, rem);
            v[k] = get4<kF32, Full>(c.v, i, rem);
        }
    }
    if constexpr (Stream) {
        if (c.pici) {
            expand_tile<GT>(t.grad, c.nnz, t.grad_n, c.tile, tile, a.ctrl);
#pragma unroll
            for (uint32_t k = 0; k < kQuads; k++) {
                const u32x4 x = reinterpret_cast<const u32x4*>(tile)[k * kThreads + threadIdx.x];
#pragma unroll
                for (int j = 0; j < 4; j++) g[k].f[j] = __uint_as_float(x[j]);
            }
        }
    }
    const float scale = a.grad_scale ? *a.grad_scale : 1.0f;
    const float keep = (float)(1.0 - a.lr * t.decay);
#pragma unroll
    for (uint32_t k = 0; k < kQuads; k++) {
        const uint32_t i = i0 + k * kThreads * 4, rem = exists(i);
        if constexpr (Eight) {
            m[k] = decode4(mc[k], ms[k]);
            v[k] = decode4(vc[k], vs[k]);
        }
        float pn[4], mn[4], vn[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float d = g[k].f[j] * scale;
            mn[j] = m[k].f[j] * a.b1 + d * a.c1;
            vn[j] = v[k].f[j] * a.b2 + (d * d) * a.c2;
            pn[j] = p[k].f[j] * keep - (mn[j] / (sqrtf(vn[j]) * a.root + a.eps)) * a.rate;
        }
        uint32_t h = 0;
        if constexpr (Eight || PT == kBF16) h = mix((c.random + i / 4) ^ a.key);
        if constexpr (Eight) {
            // places past the end hold zeros: they do not move a block's scale
            uint32_t mt = 0, vt = 0;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const bool in = Full || (uint32_t)j < rem;
                mt = max(mt, in ? __float_as_uint(mn[j]) & 0x7FFFFFFFu : 0u);
                vt = max(vt, in ? __float_as_uint(vn[j]) & 0x7FFFFFFFu : 0u);
            }
            const Scale sm = scale_of(block_max(mt)), sv = scale_of(block_max(vt));
            if (Full || rem) {
                put4_8<Full>(c.m, i, rem, encode4(mn, sm.up, h, 0, false));
                put4_8<Full>(c.v, i, rem, encode4(vn, sv.up, h, 12, true));
                if (i % kBlock == 0) {
                    *at<uint8_t>(c.ms, i / kBlock) = (uint8_t)sm.byte;
                    *at<uint8_t>(c.vs, i / kBlock) = (uint8_t)sv.byte;
                }
            }
        }
        if (!Full && !rem) continue;
        if constexpr (!Eight) {
            put4_f32<Full>(c.m, i, rem, mn);
            put4_f32<Full>(c.v, i, rem, vn);
        }
        if constexpr (PT == kF32) {
            put4_f32<Full>(c.param, i, rem, pn);
            if (c.model) put4_16<Full>(c.model, i, rem, u32x2{bf16_pair(pn[0], pn[1]), bf16_pair(pn[2], pn[3])});
        } else {
            const uint32_t h2 = h * kSecond;
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; j++) b[j] = bf16_stochastic(pn[j], h2 + (uint32_t)j * kStride);
            put4_16<Full>(c.param, i, rem, u32x2{b[0] | (b[1] << 16), b[2] | (b[3] << 16)});
        }
    }
}

// One chunk of one tensor per block, found through the plan's table.  Stream:
// the chunk is what the tensor has of one 4096-element tile of the message,
// whose gradient is expanded into LDS while the states are on their way.
template <int PT, int GT, bool Eight, bool Stream>
__global__ void __launch_bounds__(kThreads) k_adamw(AdamArgs a) {
    __shared__ __attribute__((aligned(16))) float tile[Stream ? kTileElems : 4];
    constexpr uint32_t kChunk = chunk_elems(Stream);
    const uint64_t id = a.chunk0 + blockIdx.x;
    const AdamTensor t = a.table[a.chunk[id]];
    const uint64_t nth = id - t.first;
    Chunk c{};
    c.lead = Stream && nth == 0 ? (uint32_t)(t.grad_offset % kTileElems) : 0u;
    // the tensor's element at the chunk's first place; a stream's chunks follow
    // the message's tiles, so its first may begin before the tensor
    const int64_t e0 = (int64_t)(nth * kChunk) - (Stream ? (int64_t)(t.grad_offset % kTileElems) : 0);
    const int64_t left = (int64_t)t.n - e0;
    c.end = left < (int64_t)kChunk ? (uint32_t)left : kChunk;
    c.param = (uint64_t)t.param + e0 * (PT == kF32 ? 4 : 2);
    c.model = t.model ? (uint64_t)t.model + e0 * 2 : 0;
    c.m = (uint64_t)t.m + e0 * (Eight ? 1 : 4);
    c.v = (uint64_t)t.v + e0 * (Eight ? 1 : 4);
    c.ms = (uint64_t)t.ms + e0 / (int64_t)kBlock;
    c.vs = (uint64_t)t.vs + e0 / (int64_t)kBlock;
    c.grad = (uint64_t)t.grad + e0 * (GT == kF32 ? 4 : 2);
    c.random = (uint32_t)((t.counter + (uint64_t)e0) >> 2);
    if constexpr (Stream) {
        const Message msg = check_message(t.grad, t.grad_cap, t.grad_n, GT);
        if (!msg.ok) {
            if (threadIdx.x == 0) atomicCAS(&a.ctrl->status, 0u, (uint32_t)SPCCL_ERR_CORRUPT_STREAM);
            return;
        }
        c.pici = msg.pici;
        c.nnz = msg.nnz;
        c.tile = t.grad_offset / kTileElems + nth;
        if (!c.pici) c.grad += kHeaderBytes + t.grad_offset * (GT == kF32 ? 4 : 2);
    }
    if (c.lead == 0 && c.end == kChunk) adamw_chunk<PT, GT, Eight, Stream, true>(a, t, c, tile);
    else adamw_chunk<PT, GT, Eight, Stream, false>(a, t, c, tile);
}

// ---------------------------------------------------------------------------
// host side

constexpr uint32_t kPlanMagic = 0x4D414441u;      // "ADAM"

inline bool is_stream(const spccl_adamw_tensor_t& t) { return t.grad.kind == SPCCL_STREAM; }

// Chunks of a tensor; a stream's are cut where the message's tiles are.
uint64_t chunks_of(const spccl_adamw_tensor_t& t) {
    if (!t.n) return 0;
    const uint64_t lead = is_stream(t) ? t.grad_offset % kTileElems : 0;
    const uint64_t chunk = chunk_elems(is_stream(t));
    return (lead + t.n + chunk - 1) / chunk;
}

uint64_t table_bytes(int32_t count, uint64_t chunks) {
    return (uint64_t)count * sizeof(AdamTensor) + (chunks * 4 + 15) / 16 * 16;
}
uint64_t table_bytes(const spccl_adamw_tensor_t* t, int32_t count, uint64_t* arrays, uint64_t* streams) {
    *arrays = *streams = 0;
    for (int32_t i = 0; i < count; i++) (is_stream(t[i]) ? *streams : *arrays) += chunks_of(t[i]);
    return table_bytes(count, *arrays + *streams);
}

spccl_status_t check_tensor(const spccl_adamw_tensor_t& t, int32_t pdt, int32_t gdt, int32_t state) {
    if (t.n >= (1ull << 32)) return SPCCL_ERR_UNSUPPORTED;
    if (!(t.weight_decay >= 0.0)) return SPCCL_ERR_INVALID_ARG;
    if (t.grad.kind != SPCCL_ARRAY && t.grad.kind != SPCCL_STREAM) return SPCCL_ERR_INVALID_ARG;
    if (!t.n) return SPCCL_OK;
    const uint64_t ss = state == SPCCL_STATE_F8 ? 1 : 4;
    if (!t.param || !t.m || !t.v || !t.grad.ptr) return SPCCL_ERR_INVALID_ARG;
    if (!aligned_to(t.param, elem_bytes(pdt)) || !aligned_to(t.m, ss) || !aligned_to(t.v, ss) || !aligned_to(t.model, 2))
        return SPCCL_ERR_INVALID_ARG;
    if (t.model && pdt != kF32) return SPCCL_ERR_INVALID_ARG;
    if ((state == SPCCL_STATE_F8) != (t.m_scale && t.v_scale) || (state != SPCCL_STATE_F8 && (t.m_scale || t.v_scale)))
        return SPCCL_ERR_INVALID_ARG;
    if (is_stream(t)) {
        if (t.grad_n >= (1ull << 32)) return SPCCL_ERR_UNSUPPORTED;
        if (t.grad.fmt == SPCCL_FMT_COO) return SPCCL_ERR_UNSUPPORTED;
        if (t.grad.fmt != SPCCL_FMT_PICI && t.grad.fmt != SPCCL_FMT_DENSE) return SPCCL_ERR_INVALID_ARG;
        if (!aligned_to(t.grad.ptr, 16) || t.grad_offset % 64 || t.grad_offset > t.grad_n || t.n > t.grad_n - t.grad_offset)
            return SPCCL_ERR_INVALID_ARG;
        if (t.grad.bytes < kHeaderBytes) return SPCCL_ERR_CAPACITY;
    } else {
        if (!aligned_to(t.grad.ptr, elem_bytes(gdt))) return SPCCL_ERR_INVALID_ARG;
        if (t.grad.bytes < t.n * elem_bytes(gdt)) return SPCCL_ERR_CAPACITY;
    }
    return SPCCL_OK;
}

// Whether a written range meets any other range (gradients are only read, and
// may be shared).
struct Span {
    uintptr_t lo, hi;
    bool write;
};
spccl_status_t check_spans(const spccl_adamw_tensor_t* t, int32_t count, int32_t pdt, int32_t state, const void* table,
                           uint64_t bytes) {
    Span* s = static_cast<Span*>(malloc(sizeof(Span) * (7ull * (uint64_t)count + 1)));
    if (!s) return SPCCL_ERR_CAPACITY;
    uint64_t k = 0;
    const auto add = [&](const void* p, uint64_t n, bool write) {
        if (p && n) s[k++] = Span{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + n, write};
    };
    const uint64_t ss = state == SPCCL_STATE_F8 ? 1 : 4;
    add(table, bytes, true);
    for (int32_t i = 0; i < count; i++) {
        if (!t[i].n) continue;
        const uint64_t scales = (t[i].n + kBlock - 1) / kBlock;
        add(t[i].param, t[i].n * elem_bytes(pdt), true);
        add(t[i].model, t[i].n * 2, true);
        add(t[i].m, t[i].n * ss, true);
        add(t[i].v, t[i].n * ss, true);
        add(t[i].m_scale, scales, true);
        add(t[i].v_scale, scales, true);
        add(t[i].grad.ptr, t[i].grad.bytes, false);
    }
    std::sort(s, s + k, [](const Span& a, const Span& b) { return a.lo < b.lo; });
    uintptr_t written = 0, any = 0;
    spccl_status_t st = SPCCL_OK;
    for (uint64_t i = 0; i < k && st == SPCCL_OK; i++) {
        if (s[i].lo < (s[i].write ? any : written)) st = SPCCL_ERR_INVALID_ARG;
        if (s[i].hi > any) any = s[i].hi;
        if (s[i].write && s[i].hi > written) written = s[i].hi;
    }
    free(s);
    return st;
}

// Whether the runtime knows both ends of a range as memory that a kernel can
// reach (also true inside an allocation).  The failed query is taken out of the
// runtime's last error.
bool reachable(const void* p, uint64_t bytes) {
    for (const uint64_t at : {uint64_t{0}, bytes - 1}) {
        hipPointerAttribute_t a{};
        if (hipPointerGetAttributes(&a, static_cast<const uint8_t*>(p) + at) != hipSuccess) {
            (void)hipGetLastError();
            return false;
        }
        if (a.type == hipMemoryTypeUnregistered) return false;
    }
    return true;
}

template <int PT, int GT, bool Eight>
spccl_status_t launch_adamw(const spccl_adamw_plan_t& plan, AdamArgs a, hipStream_t st) {
    constexpr uint64_t most = 0xFFFFFFFFu / kThreads;            // a grid has fewer than 2^32 threads
    const uint64_t ends[2] = {plan.array_chunks, plan.array_chunks + plan.stream_chunks};
    for (int stream = 0; stream < 2; stream++)
        for (a.chunk0 = stream ? ends[0] : 0; a.chunk0 < ends[stream]; a.chunk0 += most) {
            const dim3 grid((uint32_t)std::min(most, ends[stream] - a.chunk0));
            if (stream) hipLaunchKernelGGL((k_adamw<PT, GT, Eight, true>), grid, dim3(kThreads), 0, st, a);
            else hipLaunchKernelGGL((k_adamw<PT, GT, Eight, false>), grid, dim3(kThreads), 0, st, a);
            if (launch_status() != SPCCL_OK) return SPCCL_ERR_HIP;
        }
    return SPCCL_OK;
}

}  // namespace
}  // namespace spccl

using namespace spccl;

extern "C" {

spccl_status_t spccl_prune(const void* grad, float* residual, const float* threshold, double leak, void* out, uint64_t n,
                           int32_t dtype, void* stream) {
    if (!dtype_ok(dtype)) return SPCCL_ERR_UNSUPPORTED;
    if (n >= (1ull << 36)) return SPCCL_ERR_UNSUPPORTED;          // a grid has fewer than 2^32 threads
    if (!(leak >= 0.0 && leak <= 1.0)) return SPCCL_ERR_INVALID_ARG;
    if (!threshold || !aligned_to(threshold, 4)) return SPCCL_ERR_INVALID_ARG;
    if (n == 0) return SPCCL_OK;
    const uint64_t s = elem_bytes(dtype);
    if (!grad || !residual || !out || !aligned_to(grad, s) || !aligned_to(out, s) || !aligned_to(residual, 4))
        return SPCCL_ERR_INVALID_ARG;
    if (out != grad && overlaps(grad, n * s, out, n * s)) return SPCCL_ERR_INVALID_ARG;
    if (overlaps(residual, 4 * n, grad, n * s) || overlaps(residual, 4 * n, out, n * s)) return SPCCL_ERR_INVALID_ARG;
    if (overlaps(threshold, 4, out, n * s) || overlaps(threshold, 4, residual, 4 * n)) return SPCCL_ERR_INVALID_ARG;
    const PruneArgs g{static_cast<const uint8_t*>(grad), reinterpret_cast<uint8_t*>(residual), static_cast<uint8_t*>(out),
                      threshold, n, (float)leak};
    const dim3 grid((uint32_t)((n + kPruneChunk - 1) / kPruneChunk)), block(kThreads);
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (dtype == kF32) hipLaunchKernelGGL(k_prune<kF32>, grid, block, 0, st, g);
    else hipLaunchKernelGGL(k_prune<kBF16>, grid, block, 0, st, g);
    return launch_status();
}

uint64_t spccl_adamw_plan_bytes(const spccl_adamw_tensor_t* tensors, int32_t count) {
    if (count < 0 || (count && !tensors)) return 0;
    uint64_t a, s;
    return table_bytes(tensors, count, &a, &s);
}

spccl_status_t spccl_adamw_plan(const spccl_adamw_tensor_t* tensors, int32_t count, int32_t param_dtype, int32_t grad_dtype,
                                int32_t state, void* table, uint64_t bytes, spccl_adamw_plan_t* plan, void* stream) {
    if (!dtype_ok(param_dtype) || !dtype_ok(grad_dtype)) return SPCCL_ERR_UNSUPPORTED;
    if (state != SPCCL_STATE_F32 && state != SPCCL_STATE_F8) return SPCCL_ERR_UNSUPPORTED;
    if (count < 0 || (count && !tensors) || !plan) return SPCCL_ERR_INVALID_ARG;
    for (int32_t i = 0; i < count; i++) {
        const spccl_status_t st = check_tensor(tensors[i], param_dtype, grad_dtype, state);
        if (st != SPCCL_OK) return st;
    }
    uint64_t arrays, streams;
    const uint64_t need = table_bytes(tensors, count, &arrays, &streams);
    if (count && (!table || !aligned_to(table, 16))) return SPCCL_ERR_INVALID_ARG;
    if (bytes < need) return SPCCL_ERR_WORKSPACE;
    spccl_status_t st = check_spans(tensors, count, param_dtype, state, table, need);
    if (st != SPCCL_OK) return st;
    // the kernels below write the table at once: an address that is none of the
    // device's would fault there
    if (need && !reachable(table, need)) return SPCCL_ERR_HIP;
    AdamTensor* entries = static_cast<AdamTensor*>(table);
    uint32_t* chunk = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(table) + (uint64_t)count * sizeof(AdamTensor));
    uint64_t next[2] = {0, arrays}, counter = 0;
    for (int32_t first = 0; first < count; first += kTableBatch) {
        TableArgs a{};
        a.table = entries;
        a.chunk = chunk;
        a.first = (uint32_t)first;
        a.count = (uint32_t)(count - first < kTableBatch ? count - first : kTableBatch);
        for (uint32_t i = 0; i < a.count; i++) {
            const spccl_adamw_tensor_t& t = tensors[first + (int32_t)i];
            const uint64_t chunks = chunks_of(t);
            uint64_t& at = next[is_stream(t) ? 1 : 0];
            a.t[i] = AdamTensor{static_cast<uint8_t*>(t.param), static_cast<uint8_t*>(t.model), static_cast<uint8_t*>(t.m),
                                static_cast<uint8_t*>(t.v), static_cast<uint8_t*>(t.m_scale),
                                static_cast<uint8_t*>(t.v_scale), static_cast<const uint8_t*>(t.grad.ptr), t.grad.bytes,
                                t.grad_n, is_stream(t) ? t.grad_offset : 0, t.n, counter, at, chunks, t.weight_decay, 0};
            at += chunks;
            counter += (t.n + 63) / 64 * 64;
        }
        hipLaunchKernelGGL(k_adamw_table, dim3(a.count), dim3(kThreads), 0, reinterpret_cast<hipStream_t>(stream), a);
        if ((st = launch_status()) != SPCCL_OK) return st;
    }
    *plan = spccl_adamw_plan_t{kPlanMagic, param_dtype, grad_dtype, state, count, 0, arrays, streams, table};
    return SPCCL_OK;
}

spccl_status_t spccl_adamw_step(const spccl_adamw_plan_t* plan, const spccl_adamw_t* hyper, const float* grad_scale,
                                void* ws, uint64_t ws_bytes, void* stream) {
    if (!plan || plan->magic != kPlanMagic || !hyper) return SPCCL_ERR_INVALID_ARG;
    const spccl_adamw_t& h = *hyper;
    if (!(h.beta1 >= 0.0 && h.beta1 < 1.0) || !(h.beta2 >= 0.0 && h.beta2 < 1.0) || !(h.eps >= 0.0) || !(h.lr >= 0.0) ||
        h.step < 1)
        return SPCCL_ERR_INVALID_ARG;
    if (!aligned_to(grad_scale, 4) || !ws || !aligned_to(ws, 16)) return SPCCL_ERR_INVALID_ARG;
    if (ws_bytes < sizeof(WsCtrl)) return SPCCL_ERR_WORKSPACE;
    const uint64_t table = table_bytes(plan->count, plan->array_chunks + plan->stream_chunks);
    if (overlaps(ws, sizeof(WsCtrl), plan->table, table)) return SPCCL_ERR_INVALID_ARG;
    const double t = (double)h.step;
    AdamArgs a{};
    a.table = static_cast<const AdamTensor*>(plan->table);
    a.chunk = reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(plan->table) +
                                                (uint64_t)plan->count * sizeof(AdamTensor));
    a.grad_scale = grad_scale;
    a.ctrl = static_cast<WsCtrl*>(ws);
    a.lr = h.lr;
    a.b1 = (float)h.beta1;
    a.c1 = (float)(1.0 - h.beta1);
    a.b2 = (float)h.beta2;
    a.c2 = (float)(1.0 - h.beta2);
    a.root = (float)(1.0 / sqrt(1.0 - pow(h.beta2, t)));
    a.rate = (float)(h.lr / (1.0 - pow(h.beta1, t)));
    a.eps = (float)h.eps;
    a.key = mix(mix((uint32_t)h.seed) ^ (uint32_t)(h.seed >> 32));
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const bool eight = plan->state == SPCCL_STATE_F8;
    if (plan->param_dtype == kF32) {
        if (plan->grad_dtype == kF32)
            return eight ? launch_adamw<kF32, kF32, true>(*plan, a, st) : launch_adamw<kF32, kF32, false>(*plan, a, st);
        return eight ? launch_adamw<kF32, kBF16, true>(*plan, a, st) : launch_adamw<kF32, kBF16, false>(*plan, a, st);
    }
    if (plan->grad_dtype == kF32)
        return eight ? launch_adamw<kBF16, kF32, true>(*plan, a, st) : launch_adamw<kBF16, kF32, false>(*plan, a, st);
    return eight ? launch_adamw<kBF16, kBF16, true>(*plan, a, st) : launch_adamw<kBF16, kBF16, false>(*plan, a, st);
}

}  // extern "C"
