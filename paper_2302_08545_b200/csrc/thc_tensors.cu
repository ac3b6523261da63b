// Lists of tensors around a round: global norm, clipping, the ways into and out of the flat vector, the Adam step.
// See include/thc.h for the contract of every entry point.
//
// All of it is streaming: two to twenty operations per element against 2 to 30 bytes, so the loads are what the
// kernels are built around.  A list is cut into pieces of at most 2048 elements of one tensor, and a warp takes a piece
// at a time with all loads of half or all of it in flight.  The table of pieces is made once per list; a piece
// names its flat position, from which every address follows (the table of tensor addresses holds the address that
// flat position 0 would have).
//
// Clipping needs the norm of everything before the first product.  Short lists take one launch, a cluster of CTAs per worker
// that keeps what it reads in shared memory.  The others take two: sums of squares, whose last CTA forms norm and factor, then
// products, eight pieces to a CTA and the last pieces first, which are still in L2.  (One launch for them too, with a barrier
// of all CTAs in its middle, was not faster: a cooperative launch waits some 2 us longer for the one before it, and CTAs that stay
// take their pieces further apart than the scheduler deals them out.  DRAM minds when reads and writes mix: 256 MiB fp32 to
// another buffer 92 us with pieces in a fixed stride, 82 us with a CTA for each eight.)
#include "thc_host.h"

#include <algorithm>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <new>
#include <type_traits>
#include <vector>

namespace thc {

constexpr uint32_t kPiece = 2048;              // elements of a piece: eight units of eight per lane
constexpr uint32_t kUnit = 8;                  // consecutive elements of a lane: 16 bytes of a 16-bit type, 32 of fp32
constexpr int kListThreads = 256, kListWarps = kListThreads / 32;
constexpr uint32_t kNormCtasPerSm = 4, kNormMostRows = 8, kNormLeastRounds = 6;
constexpr int kClusterThreads = 512, kClusterWarps = kClusterThreads / 32;
constexpr uint32_t kClusterCtas = 8;
constexpr uint32_t kHeldBytes = 4096;          // per warp: half a piece of fp32, which is the most that a warp of the cluster takes at a time

// {flat position (64 bits), tensor, length (16 bits) and type}
struct Piece { uint64_t flat; uint32_t tensor, len_type; };
static_assert(sizeof(Piece) == 16, "one load");

struct ListTable {
    const Piece *pieces;
    const uint64_t *base;        // [n][count]: address of the tensor less its flat position, in bytes
    uint32_t count, pieces_n;
};

// The factor c of the products as two: c x = factor (x scale).  Where c is an fp32 denormal (gradients near fp32's end)
// scale is 2^-126 and factor keeps all its bits: x scale is exact wherever c x is not itself a denormal.  Else scale is 1.
struct Factor { float factor, scale; };
__device__ __forceinline__ float times(const Factor &c, float x) { return c.factor * (x * c.scale); }
__device__ __forceinline__ Factor factor_of(double norm, double max_norm)
{
    if (isinf(max_norm)) return Factor{1.0f, 1.0f};
    const double c = max_norm / (norm + 1e-6);
    if (c < 0x1p-126) return Factor{(float)(c * 0x1p126), 0x1p-126f};
    return Factor{c > 1.0 ? 1.0f : (float)c, 1.0f};    // NaN stays
}

// What the norm leaves for the products.
struct alignas(16) NormResult { Factor c; float step_size, inv_sqrt_by2; uint32_t stop, pad_[3]; };

__device__ __forceinline__ Piece load_piece(const Piece *p)
{
    const uint4 q = __ldg(reinterpret_cast<const uint4 *>(p));
    return Piece{(uint64_t)q.x | (uint64_t)q.y << 32, q.z, q.w};
}
__device__ __forceinline__ uint64_t load_base(const uint64_t *p)
{
    uint64_t v;
    asm volatile("ld.global.u64 %0, [%1];" : "=l"(v) : "l"(p));
    return v;
}

// ------------------------------------------------------------------------------ elements
// A unit as it is loaded (4 or 8 registers), and its values.
template <uint32_t T> struct Raw { uint32_t w[T == THC_F32 ? 8 : 4]; };
template <uint32_t T> __host__ __device__ constexpr uint32_t size_of() { return T == THC_F32 ? 4u : 2u; }

template <uint32_t T>
__device__ __forceinline__ Raw<T> load_unit8(uint64_t a)
{
    Raw<T> r;
    if constexpr (T == THC_F32)
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "l"(a));
    else
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(a));
    return r;
}

template <uint32_t T>
__device__ __forceinline__ float widen16(uint32_t v)
{
    return T == THC_BF16 ? __uint_as_float(v << 16) : __half2float(__ushort_as_half((unsigned short)v));
}
template <uint32_t T>
__device__ __forceinline__ float value(const Raw<T> &r, int e)
{
    if constexpr (T == THC_F32) return __uint_as_float(r.w[e]);
    const uint32_t w = r.w[e >> 1];
    if (T == THC_BF16) return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    return widen16<T>(e & 1 ? w >> 16 : w & 0xFFFFu);
}
template <uint32_t T>
__device__ __forceinline__ float load_one(uint64_t a)
{
    if (T == THC_F32) return ld_global(reinterpret_cast<const float *>(a));
    return widen16<T>(ld_global(reinterpret_cast<const uint16_t *>(a)));
}
// The only rounding of a result: to nearest, ties to even.
template <uint32_t T>
__device__ __forceinline__ uint32_t narrow16(float v)
{
    return T == THC_BF16 ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v)) : (uint32_t)__half_as_ushort(__float2half_rn(v));
}
template <uint32_t T>
__device__ __forceinline__ void store_one(uint64_t a, float v)
{
    if (T == THC_F32) *reinterpret_cast<float *>(a) = v;
    else *reinterpret_cast<uint16_t *>(a) = (uint16_t)narrow16<T>(v);
}
template <uint32_t T>
__device__ __forceinline__ void store_unit8(uint64_t a, const float (&v)[8])
{
    if (T == THC_F32) {
        asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     :: "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "l"(a) : "memory");
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = narrow16<T>(v[2 * i]) | narrow16<T>(v[2 * i + 1]) << 16;
        asm volatile("st.global.v4.b32 [%4], {%0, %1, %2, %3};" :: "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "l"(a) : "memory");
    }
}

// Elements before the first one on a unit boundary.
template <uint32_t T>
__device__ __forceinline__ uint32_t head_of(uint64_t a) { return (uint32_t)((0ull - a) / size_of<T>()) & (kUnit - 1u); }

// ---------------------------------------------------------------------------------- held units
// Units of the item that a warp of the cluster has read, in its part of shared memory (at address `held`); a lane reads what it wrote
// itself.
// 16 bytes of a lane next to its neighbours': no bank conflicts.
template <uint32_t T>
__device__ __forceinline__ void hold_unit(uint32_t held, uint32_t b, uint32_t lane, const Raw<T> &r)
{
    constexpr uint32_t kParts = T == THC_F32 ? 2 : 1;
#pragma unroll
    for (uint32_t i = 0; i < kParts; ++i)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                     :: "r"(held + (b * kParts + i) * 512u + lane * 16u), "r"(r.w[4 * i]), "r"(r.w[4 * i + 1]), "r"(r.w[4 * i + 2]), "r"(r.w[4 * i + 3]) : "memory");
}
template <uint32_t T>
__device__ __forceinline__ Raw<T> held_unit(uint32_t held, uint32_t b, uint32_t lane)
{
    constexpr uint32_t kParts = T == THC_F32 ? 2 : 1;
    Raw<T> r;
#pragma unroll
    for (uint32_t i = 0; i < kParts; ++i)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r.w[4 * i]), "=r"(r.w[4 * i + 1]), "=r"(r.w[4 * i + 2]), "=r"(r.w[4 * i + 3])
                     : "r"(held + (b * kParts + i) * 512u + lane * 16u));
    return r;
}

// ---------------------------------------------------------------------------------- norm
// s + the squares of a unit.  fp32: each square in fp64, which no value leaves.  16 bits: the squares are exact in fp32, eight
// of them are added there in three levels (3 x 2^-24 off at most, as all are positive) and the sum in fp64: a conversion and an fp64
// operation per unit instead of eight, which were what bounded it (355M bf16 again and again: 125 us, now 106).  fp16's squares and their sums
// stay within fp32; for bf16 a sum outside [2^-100, 2^126] (a square may have left fp32's range) is formed as for fp32, in a loop
// (unrolled it takes the registers of the ordinary case: 111 us).
template <uint32_t T>
__device__ __forceinline__ void add_squares(double (&s)[2], const Raw<T> &r)
{
    if constexpr (T != THC_F32) {
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = fmaf(value<T>(r, 2 * i), value<T>(r, 2 * i), value<T>(r, 2 * i + 1) * value<T>(r, 2 * i + 1));
        const float sum = (q[0] + q[1]) + (q[2] + q[3]);
        if (T == THC_F16 || (sum >= 0x1p-100f && sum <= 0x1p126f)) {
            s[0] += (double)sum;
            return;
        }
        if (((r.w[0] | r.w[1] | r.w[2] | r.w[3]) & 0x7FFF7FFFu) == 0u) return;
#pragma unroll 1
        for (int e = 0; e < 4; ++e) {
            const uint32_t w = e == 0 ? r.w[0] : e == 1 ? r.w[1] : e == 2 ? r.w[2] : r.w[3];
            const double lo = (double)__uint_as_float(w << 16), hi = (double)__uint_as_float(w & 0xFFFF0000u);
            s[0] = fma(lo, lo, s[0]);
            s[1] = fma(hi, hi, s[1]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double v = (double)value<T>(r, e);
        s[e & 1] = fma(v, v, s[e & 1]);
    }
}

// Sum of squares of a piece, in a lane; HOLD: its units go to `held`.
template <uint32_t T, bool HOLD>
__device__ __forceinline__ double squares_of_piece(uint64_t a, uint32_t len, uint32_t lane, uint32_t held)
{
    constexpr int kBatch = 4;
    double s[2] = {0.0, 0.0};
    const uint32_t head = min(head_of<T>(a), len), units = (len - head) / kUnit, tail = head + units * kUnit;
    // lanes 0..7 the elements before the units, lanes 8..15 those behind
    const uint32_t single = lane < 8u ? lane : tail + lane - 8u;
    float edge = 0.0f;
    if (lane < 8u ? single < head : lane < 16u && single < len) edge = load_one<T>(a + (uint64_t)single * size_of<T>());
    uint64_t at = a + head * size_of<T>();
    uint32_t first = 0;                                // unit of the batch, in rows of 32
    // a whole batch, or what is left: lanes without a unit load the last one again and add nothing
    const auto batch = [&](auto whole, uint32_t left) {
        constexpr bool kWhole = decltype(whole)::value;
        Raw<T> r[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            r[b] = load_unit8<T>(at + (kWhole ? lane + 32u * b : min(lane + 32u * b, left - 1u)) * (kUnit * size_of<T>()));
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (HOLD) hold_unit<T>(held, first + b, lane, r[b]);
            if (!kWhole && lane + 32u * b >= left) r[b] = Raw<T>{};
            add_squares<T>(s, r[b]);
        }
        at += 32u * kBatch * kUnit * size_of<T>();
        first += kBatch;
    };
    uint32_t u = 0;
#pragma unroll 1
    for (; u + 32u * kBatch <= units; u += 32u * kBatch) batch(std::true_type{}, 0u);
    if (u < units) batch(std::false_type{}, units - u);
    const double v = (double)edge;
    return fma(v, v, s[0]) + s[1];
}

template <bool HOLD>
__device__ __forceinline__ double squares(const Piece &p, const uint64_t *base, uint64_t flat, uint32_t lane, uint32_t held = 0)
{
    const uint32_t len = p.len_type & 0xFFFFu, type = p.len_type >> 16;
    if (flat != 0) return squares_of_piece<THC_F32, HOLD>(flat + p.flat * 4u, len, lane, held);
    const uint64_t b = load_base(base + p.tensor);
    if (type == THC_F32) return squares_of_piece<THC_F32, HOLD>(b + p.flat * 4u, len, lane, held);
    if (type == THC_BF16) return squares_of_piece<THC_BF16, HOLD>(b + p.flat * 2u, len, lane, held);
    return squares_of_piece<THC_F16, HOLD>(b + p.flat * 2u, len, lane, held);
}

// Sum over the CTA's threads, in thread 0.
template <int WARPS>
__device__ __forceinline__ double sum_of_cta(double s, double (&red)[WARPS])
{
    for (int off = 16; off > 0; off >>= 1) s += __shfl_down_sync(0xFFFFFFFFu, s, off);
    if ((threadIdx.x & 31u) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < WARPS; ++w) t += red[w];
    return t;
}

// ---------------------------------------------------------------------------------- products
// y = c x (+ e) for a piece, whose units are in `held` (HELD) or in memory; zeros (or e) from its end up to dst_len.
template <uint32_t S, uint32_t D, bool EF, bool HELD>
__device__ __forceinline__ void move_piece(uint64_t src, uint64_t dst, uint64_t ef, uint32_t len, uint32_t dst_len, const Factor &c, uint32_t lane, uint32_t held)
{
    const auto product = [&c](float x, float e) { return EF ? fmaf(c.factor, x * c.scale, e) : times(c, x); };
    const uint32_t h = min(head_of<S>(src), len);
    if (head_of<S>(src) == head_of<D>(dst) && (!EF || head_of<S>(src) == head_of<THC_F32>(ef))) {
        constexpr int kBatch = EF ? 2 : S == THC_F32 ? 4 : 8;
        const uint32_t units = (len - h) / kUnit;
        uint64_t s = src + h * size_of<S>(), d = dst + h * size_of<D>(), q = ef + h * 4u;
        uint32_t first = 0;
        // a whole batch, or what is left: lanes without a unit load the last one again and store nothing
        const auto batch = [&](auto whole, uint32_t left) {
            constexpr bool kWhole = decltype(whole)::value;
            Raw<S> x[kBatch];
            Raw<THC_F32> r[EF ? kBatch : 1];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const uint32_t v = (kWhole ? lane + 32u * b : min(lane + 32u * b, left - 1u)) * kUnit;
                x[b] = HELD ? held_unit<S>(held, first + b, lane) : load_unit8<S>(s + v * size_of<S>());
                if constexpr (EF) r[b] = load_unit8<THC_F32>(q + v * 4u);
            }
            first += kBatch;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (!kWhole && lane + 32u * b >= left) break;
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = product(value<S>(x[b], e), EF ? value<THC_F32>(r[EF ? b : 0], e) : 0.0f);
                store_unit8<D>(d + (lane + 32u * b) * (kUnit * size_of<D>()), y);
            }
            s += 32u * kBatch * kUnit * size_of<S>();
            d += 32u * kBatch * kUnit * size_of<D>();
            q += 32u * kBatch * kUnit * 4u;
        };
        uint32_t u = 0;
#pragma unroll 1
        for (; u + 32u * kBatch <= units; u += 32u * kBatch) batch(std::true_type{}, 0u);
        if (u < units) batch(std::false_type{}, units - u);
        // lanes 0..7 the elements before the units, lanes 8..15 those behind
        const uint32_t i = lane < 8u ? lane : h + units * kUnit + lane - 8u;
        if (lane < 8u ? i < h : lane < 16u && i < len) {
            const float e = EF ? load_one<THC_F32>(ef + i * 4u) : 0.0f;
            store_one<D>(dst + i * size_of<D>(), product(load_one<S>(src + i * size_of<S>()), e));
        }
    } else {
        constexpr int kBatch = EF ? 8 : 16;
        uint64_t s = src, d = dst, q = ef;
        const auto batch = [&](auto whole, uint32_t left) {
            constexpr bool kWhole = decltype(whole)::value;
            float x[kBatch], r[EF ? kBatch : 1];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                const uint32_t v = kWhole ? lane + 32u * b : min(lane + 32u * b, left - 1u);
                x[b] = load_one<S>(s + v * size_of<S>());
                if constexpr (EF) r[b] = load_one<THC_F32>(q + v * 4u);
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (!kWhole && lane + 32u * b >= left) break;
                store_one<D>(d + (lane + 32u * b) * size_of<D>(), product(x[b], EF ? r[EF ? b : 0] : 0.0f));
            }
            s += 32u * kBatch * size_of<S>();
            d += 32u * kBatch * size_of<D>();
            q += 32u * kBatch * 4u;
        };
        uint32_t j = 0;
#pragma unroll 1
        for (; j + 32u * kBatch <= len; j += 32u * kBatch) batch(std::true_type{}, 0u);
        if (j < len) batch(std::false_type{}, len - j);
    }
    for (uint32_t j = len + lane; j < dst_len; j += 32u)
        store_one<D>(dst + j * size_of<D>(), EF ? load_one<THC_F32>(ef + j * 4u) : 0.0f);
}

// ---------------------------------------------------------------------------------- Adam
struct AdamParams {
    const float *grad;
    float *master, *m, *v;       // master null: the tensors are the weights
    const float *lr, *decay;     // decay null: weight_decay
    int64_t *step;
    double beta1, beta2, eps, weight_decay;
};

struct AdamStep { Factor c; float b1, b2, a1, a2, eps, step_size, inv_sqrt_by2, keep; };

// m and v in place; the new weight.
__device__ __forceinline__ float adam(const AdamStep &k, float g, float &m, float &v, float w)
{
    g = times(k.c, g);
    m = fmaf(k.b1, m, k.a1 * g);
    v = fmaf(k.b2, v, k.a2 * g * g);
    const float move = m / fmaf(sqrtf(v), k.inv_sqrt_by2, k.eps);
    return fmaf(-k.step_size, move, w * k.keep);
}

// Where an item's operands are.  The tensor itself is read and written in units if it is aligned for them, else by element.
struct AdamPlace { uint64_t g, m, v, w, out; uint32_t len, units; bool w_units; };
template <bool MASTER>
__device__ __forceinline__ AdamPlace adam_place(const AdamParams &P, const Piece &p, uint64_t tensor)
{
    const uint64_t at = p.flat * 4u;
    AdamPlace a;
    a.g = reinterpret_cast<uint64_t>(P.grad) + at;
    a.m = reinterpret_cast<uint64_t>(P.m) + at;
    a.v = reinterpret_cast<uint64_t>(P.v) + at;
    a.out = tensor + p.flat * ((p.len_type >> 16) == THC_F32 ? 4u : 2u);
    a.w = MASTER ? reinterpret_cast<uint64_t>(P.master) + at : a.out;
    a.len = p.len_type & 0xFFFFu;
    a.w_units = (a.w & 31u) == 0;
    a.units = ((a.g | a.m | a.v) & 31u) == 0 && (!MASTER || a.w_units) ? a.len / kUnit : 0u;
    return a;
}

struct AdamUnit { Raw<THC_F32> g, m, v, w; };
template <bool MASTER, bool HELD>
__device__ __forceinline__ AdamUnit adam_load(const AdamPlace &a, uint32_t u, uint32_t held, uint32_t lane)
{
    const uint64_t o = (uint64_t)u * (kUnit * 4u);
    AdamUnit r;
    r.m = load_unit8<THC_F32>(a.m + o);
    r.v = load_unit8<THC_F32>(a.v + o);
    if (MASTER || a.w_units) r.w = load_unit8<THC_F32>(a.w + o);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w.w[e] = ld_global(reinterpret_cast<const uint32_t *>(a.w + o + 4u * e));
    r.g = HELD ? held_unit<THC_F32>(held, u / 32u, lane) : load_unit8<THC_F32>(a.g + o);
    return r;
}

// The step of an item; `cur` is the lane's first unit, if it has one.
template <uint32_t T, bool MASTER, bool HELD>
__device__ __forceinline__ void adam_item(const AdamPlace &a, const AdamStep &k, AdamUnit cur, uint32_t lane, uint32_t held)
{
    const bool whole = head_of<T>(a.out) == 0u;
#pragma unroll 1
    for (uint32_t u = lane; u < a.units; u += 32u) {
        const uint64_t o = (uint64_t)u * (kUnit * 4u), to = a.out + (uint64_t)u * (kUnit * size_of<T>());
        AdamUnit next{};
        if (u + 32u < a.units) next = adam_load<MASTER, HELD>(a, u + 32u, held, lane);
        float ym[8], yv[8], yw[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            ym[e] = value<THC_F32>(cur.m, e);
            yv[e] = value<THC_F32>(cur.v, e);
            yw[e] = adam(k, value<THC_F32>(cur.g, e), ym[e], yv[e], value<THC_F32>(cur.w, e));
        }
        store_unit8<THC_F32>(a.m + o, ym);
        store_unit8<THC_F32>(a.v + o, yv);
        if (MASTER) store_unit8<THC_F32>(a.w + o, yw);
        if (whole) store_unit8<T>(to, yw);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) store_one<T>(to + size_of<T>() * e, yw[e]);
        cur = next;
    }
    for (uint32_t j = a.units * kUnit + lane; j < a.len; j += 32u) {
        const uint64_t o = (uint64_t)j * 4u;
        float ym = load_one<THC_F32>(a.m + o), yv = load_one<THC_F32>(a.v + o);
        const float yw = adam(k, load_one<THC_F32>(a.g + o), ym, yv, load_one<THC_F32>(a.w + o));
        store_one<THC_F32>(a.m + o, ym);
        store_one<THC_F32>(a.v + o, yv);
        if (MASTER) store_one<THC_F32>(a.w + o, yw);
        store_one<T>(a.out + (uint64_t)j * size_of<T>(), yw);
    }
}

// ---------------------------------------------------------------------------------- the calls
enum ClipKind { kClip, kGatherF32, kGatherBf16, kGatherResidual, kScatter, kAdam, kAdamMaster, kNorm };
__host__ __device__ constexpr bool is_adam(ClipKind k) { return k == kAdam || k == kAdamMaster; }
// CTAs of list_product_kernel on an SM, by registers.  us with 2, 3, 4: 8 x 25.6M fp32 gathered 243, 242, 249; 355M scattered to
// bf16 306, 305, 312; 138M bf16 clipped -, 141, 135; Adam step of 138M (two units at a time only with 2) 735, 806, -.
__host__ __device__ constexpr int product_ctas_per_sm(ClipKind k) { return is_adam(k) ? 2 : k == kClip ? 4 : 3; }

struct ListParams {
    ListTable L;                 // whose pieces are walked
    uint32_t n;
    uint32_t split_log2;         // a warp takes a 2^-split_log2 of a piece at a time: an item
    uint64_t src_flat;           // kScatter, kAdam*: what is read (else the tensors of L)
    const uint64_t *dst_base;    // kClip: addresses of the tensors that are written
    double max_norm;
    float *norms;                // or null: no norm, factor 1
    double *partial;             // workspace: a sum per CTA
    uint32_t row, rounds;        // list_norm_kernel: see there
    uint32_t partials;           // sums per worker that list_product_kernel adds itself, or 0: it finds the result
    NormResult *result;          // workspace: one per worker
    DeviceBlock *dev;
    AdamParams adam;
};
struct GatherParams : ListParams { uint64_t dst_flat[THC_MAX_WORKERS], ef[THC_MAX_WORKERS]; };
// (1 KB less to hand over where it is not needed)
template <ClipKind K> using ParamsOf = std::conditional_t<K == kGatherF32 || K == kGatherBf16 || K == kGatherResidual, GatherParams, ListParams>;

// Part `item` of all parts of the pieces; length 0 where a piece is too short to have it.
__device__ __forceinline__ Piece load_item(const ListTable &L, uint32_t item, uint32_t split_log2)
{
    Piece p = load_piece(L.pieces + (item >> split_log2));
    const uint32_t part = kPiece >> split_log2, from = (item & ((1u << split_log2) - 1u)) * part, len = p.len_type & 0xFFFFu;
    p.flat += from;
    p.len_type = (p.len_type & 0xFFFF0000u) | (len > from ? min(len - from, part) : 0u);
    return p;
}

// The addresses that the products of an item need from the tables.
struct ItemBase { uint64_t tensor, dst; };
template <ClipKind K>
__device__ __forceinline__ ItemBase load_item_base(const ListParams &P, const Piece &p, uint32_t worker)
{
    const uint64_t i = (uint64_t)worker * P.L.count + p.tensor;
    return ItemBase{load_base(P.L.base + i), K == kClip ? load_base(P.dst_base + i) : 0};
}

template <ClipKind K, uint32_t T, bool HELD>
__device__ __forceinline__ void move_typed(const ParamsOf<K> &P, const Piece &p, const ItemBase &base, uint32_t worker, const Factor &c, uint32_t lane,
                                           uint32_t held)
{
    const uint32_t len = p.len_type & 0xFFFFu;
    const uint64_t at = p.flat * size_of<T>(), tensor = base.tensor + at;
    if constexpr (K == kClip) {
        move_piece<T, T, false, HELD>(tensor, base.dst + at, 0, len, len, c, lane, held);
    } else if constexpr (K == kScatter) {
        move_piece<THC_F32, T, false, HELD>(P.src_flat + p.flat * 4u, tensor, 0, len, len, c, lane, held);
    } else {
        constexpr uint32_t D = K == kGatherBf16 ? THC_BF16 : THC_F32;
        const uint32_t full = (len + THC_TENSOR_ALIGN - 1u) / THC_TENSOR_ALIGN * THC_TENSOR_ALIGN;
        move_piece<T, D, K == kGatherResidual, HELD>(tensor, P.dst_flat[worker] + p.flat * size_of<D>(),
                                                     K == kGatherResidual ? P.ef[worker] + p.flat * 4u : 0, len, full, c, lane, held);
    }
}

// What can be loaded of an item's products before the norm is known (Adam step: the lanes' first units).
template <ClipKind K>
struct Early {};
template <>
struct Early<kAdam> { AdamPlace place; AdamUnit first; float decay; };
template <>
struct Early<kAdamMaster> : Early<kAdam> {};

template <ClipKind K, bool HELD>
__device__ __forceinline__ Early<K> load_early(const ListParams &P, const Piece &p, const ItemBase &base, uint32_t lane, uint32_t held = 0)
{
    Early<K> r{};
    if constexpr (is_adam(K)) {
        r.place = adam_place<K == kAdamMaster>(P.adam, p, base.tensor);
        if (lane < r.place.units) r.first = adam_load<K == kAdamMaster, HELD>(r.place, lane, held, lane);
        if (P.adam.decay != nullptr) r.decay = ld_global(P.adam.decay + p.tensor);
    }
    return r;
}

template <ClipKind K, bool HELD>
__device__ __forceinline__ void products(const ParamsOf<K> &P, const Piece &p, const ItemBase &base, const Early<K> &early, uint32_t worker, AdamStep &k,
                                         float lr, uint32_t lane, uint32_t held = 0)
{
    const uint32_t type = p.len_type >> 16;
    if constexpr (is_adam(K)) {
        constexpr bool kMaster = K == kAdamMaster;
        k.keep = (float)(1.0 - (double)lr * (P.adam.decay != nullptr ? (double)early.decay : P.adam.weight_decay));
        if (!kMaster || type == THC_F32) adam_item<THC_F32, kMaster, HELD>(early.place, k, early.first, lane, held);
        else if (type == THC_BF16) adam_item<THC_BF16, kMaster, HELD>(early.place, k, early.first, lane, held);
        else adam_item<THC_F16, kMaster, HELD>(early.place, k, early.first, lane, held);
    } else {
        if (type == THC_F32) move_typed<K, THC_F32, HELD>(P, p, base, worker, k.c, lane, held);
        else if (type == THC_BF16) move_typed<K, THC_BF16, HELD>(P, p, base, worker, k.c, lane, held);
        else move_typed<K, THC_F16, HELD>(P, p, base, worker, k.c, lane, held);
    }
}

// The constants of the Adam step that do not depend on the norm.
__device__ __forceinline__ void adam_constants(const AdamParams &a, AdamStep &k)
{
    k.b1 = (float)a.beta1;
    k.b2 = (float)a.beta2;
    k.a1 = (float)(1.0 - a.beta1);
    k.a2 = (float)(1.0 - a.beta2);
    k.eps = (float)a.eps;
}
// beta^t by squaring.  Each product's rounding counts t times at most: t beta^t 2^-53 <= 2^-53 / (e (1 - beta)) off.  (pow() was
// a third of a small step's time.)
__device__ __forceinline__ double power(double beta, uint64_t t)
{
    double r = 1.0;
#pragma unroll 1
    for (; t != 0u; t >>= 1, beta *= beta)
        if (t & 1u) r *= beta;
    return r;
}
// Those that depend on the step count t (in the norm's result: step_size, inv_sqrt_by2).
__device__ __forceinline__ float adam_step_size(const AdamParams &a, float lr, int64_t t) { return (float)((double)lr / (1.0 - power(a.beta1, (uint64_t)t))); }
__device__ __forceinline__ float adam_inv_sqrt(const AdamParams &a, int64_t t) { return (float)(1.0 / sqrt(1.0 - power(a.beta2, (uint64_t)t))); }

// Sums of squares, grid (CTAs of a worker, workers).  A warp's pieces are fixed by the grid: `row` CTAs, as many as run at a
// time, go side by side through `rounds` rounds of pieces, the next row of CTAs through the next rounds.  (One row for all of
// it drifts apart, which DRAM minds while the last launch's writes still leave L2: 355M scattered 526 us, in eight rows 507;
// eight workers gathered 380, 366.)  The sums are added in a fixed order; a worker's last CTA does that and forms what the products
// need (ADAM: also the step count, unless the norm is not finite), or the products' warps do.
template <bool ADAM>
__global__ void __launch_bounds__(kListThreads, kNormCtasPerSm)
list_norm_kernel(const __grid_constant__ ListParams P)
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, worker = blockIdx.y;
    const uint32_t stride = P.row * kListWarps, from = blockIdx.x / P.row * P.rounds * stride;
    const uint32_t end = min(P.L.pieces_n << P.split_log2, from + P.rounds * stride);
    uint32_t c = from + blockIdx.x % P.row * kListWarps + warp;
    Piece p{};
    if (c < end) p = load_item(P.L, c, P.split_log2);       // written before any launch
    depend_on_previous();
    const uint64_t *base = P.L.base + (uint64_t)worker * P.L.count;
    double s = 0.0;
#pragma unroll 1
    while (c < end) {
        const Piece now = p;
        c += stride;
        if (c < end) p = load_item(P.L, c, P.split_log2);
        s += squares<false>(now, base, P.src_flat, lane);
    }
    __shared__ double red[kListWarps];
    __shared__ NormResult s_result;
    __shared__ uint32_t last;
    double sum = sum_of_cta(s, red);
    if (threadIdx.x == 0) {
        __stcg(P.partial + (uint64_t)worker * gridDim.x + blockIdx.x, sum);
        last = ADAM && blockIdx.x == 0 ? 1u : 0u;      // (for the two sizes)
        if (P.partials == 0u) {
            __threadfence();
            last = atomicInc(P.dev->norm_counters + worker, gridDim.x - 1u) == gridDim.x - 1u;
        }
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    int64_t t = 0;
    if (ADAM && lane == 0u && warp < 3u) {             // three threads of three warps at a time
        t = (int64_t)load_base(reinterpret_cast<const uint64_t *>(P.adam.step)) + 1;
        if (warp == 1u) s_result.step_size = adam_step_size(P.adam, ld_global(P.adam.lr), t);
        if (warp == 2u) s_result.inv_sqrt_by2 = adam_inv_sqrt(P.adam, t);
    }
    sum = 0.0;
    if (P.partials == 0u)
#pragma unroll 4
        for (uint32_t i = threadIdx.x; i < gridDim.x; i += kListThreads) sum += __ldcg(P.partial + (uint64_t)worker * gridDim.x + i);
    sum = sum_of_cta(sum, red);                        // (with a barrier: the two sizes are there)
    if (threadIdx.x != 0) return;
    if (P.partials == 0u) {
        const double norm = sqrt(sum);
        P.norms[worker] = (float)norm;
        s_result.c = factor_of(norm, P.max_norm);
        s_result.stop = isfinite(norm) ? 0u : 1u;
        if (!isfinite(norm)) atomicOr(&P.dev->status, THC_STATUS_NONFINITE);
        else if (ADAM) *P.adam.step = t;
    }
    if (P.result != nullptr) P.result[worker] = s_result;
}

// Products of eight items to a CTA, over all workers; the last ones first.
template <ClipKind K>
__global__ void __launch_bounds__(kListThreads, product_ctas_per_sm(K))
list_product_kernel(const __grid_constant__ ParamsOf<K> P)
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t items = P.L.pieces_n << P.split_log2, all = items * P.n, j = blockIdx.x * kListWarps + warp;
    if (j >= all) return;
    const uint32_t at = all - 1u - j, worker = at / items;
    const Piece p = load_item(P.L, at % items, P.split_log2);
    depend_on_previous();
    const ItemBase base = load_item_base<K>(P, p, worker);
    AdamStep k{};
    k.c = Factor{1.0f, 1.0f};
    float lr = 0.0f;
    uint4 q{};
    uint32_t stop = 0u;
    double sum = 0.0;
    if (P.norms != nullptr) {
        if (is_adam(K) || P.partials == 0u) q = ld_global(reinterpret_cast<const uint4 *>(P.result + worker));
        if (is_adam(K)) stop = ld_global(&P.result[worker].stop);
        for (uint32_t i = lane; i < P.partials; i += 32u)
            sum += __longlong_as_double((long long)load_base(reinterpret_cast<const uint64_t *>(P.partial + (uint64_t)worker * P.partials + i)));
    }
    if (is_adam(K)) lr = ld_global(P.adam.lr);
    const Early<K> early = load_early<K, false>(P, p, base, lane);
    if (P.norms != nullptr) {
        k.c = Factor{__uint_as_float(q.x), __uint_as_float(q.y)};
        k.step_size = __uint_as_float(q.z);
        k.inv_sqrt_by2 = __uint_as_float(q.w);
        if (P.partials != 0u) {                        // the warp adds the worker's sums itself, all warps in the same order
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
            const double norm = sqrt(sum);
            k.c = factor_of(norm, P.max_norm);
            stop = isfinite(norm) ? 0u : 1u;
            if (at % items == 0u && lane == 0u) {      // one warp per worker
                P.norms[worker] = (float)norm;
                if (stop != 0u) atomicOr(&P.dev->status, THC_STATUS_NONFINITE);
                else if (is_adam(K)) *P.adam.step = *P.adam.step + 1;
            }
        }
        if (is_adam(K) && stop != 0u) return;          // the norm is not finite
    }
    if (is_adam(K)) adam_constants(P.adam, k);
    products<K, false>(P, p, base, early, worker, k, lr, lane);
}

// Lists of at most this many pieces a worker take the cluster: as long as it is faster.  us, cluster / two launches:
// (captured launches in a row; beyond 64 a warp would have a second item)
//   pieces            16          32          48          64
//   gather        3.7 / 4.3   4.0 / 4.3   4.6 / 4.7   4.6 / 4.7
//   Adam step     5.8 / 6.4   7.3 / 6.2  10.0 / 6.7  10.1 / 6.8
__host__ __device__ constexpr uint32_t cluster_most_pieces(ClipKind k) { return is_adam(k) ? 16u : 64u; }

// Both in one launch, grid (8 CTAs, workers), a cluster per worker.  The CTAs' sums are written to all CTAs' shared memory;
// each adds them in the same order and forms norm and factor itself.  A warp has one item at most (cluster_most_pieces), whose products come
// from its shared memory.
// A chain of latencies: 4 x 65,536 fp32 gathered in 4.9 us, of which an empty launch of clusters is 2.1.
template <ClipKind K>
__global__ void __launch_bounds__(kClusterThreads, 1)
list_cluster_kernel(const __grid_constant__ ParamsOf<K> P)
{
    static_assert(cluster_most_pieces(K) * 2 <= kClusterCtas * kClusterWarps && kPiece / 2 * 4 <= kHeldBytes, "an item, half a piece at most, per warp");
    extern __shared__ __align__(16) unsigned char held_bytes[];
    __shared__ double red[kClusterWarps], sums[kClusterCtas];
    __shared__ NormResult s_result;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, worker = blockIdx.y;
    const uint32_t held = (uint32_t)__cvta_generic_to_shared(held_bytes) + warp * kHeldBytes;
    const uint32_t item = blockIdx.x * kClusterWarps + warp;
    const bool busy = item < P.L.pieces_n << P.split_log2;
    Piece p{};
    ItemBase item_base{};
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this CTA runs: the others may write to it
    if (busy) p = load_item(P.L, item, P.split_log2);       // written before any launch
    depend_on_previous();
    const uint64_t *base = P.L.base + (uint64_t)worker * P.L.count;
    AdamStep k{};
    int64_t t = 0;
    float lr = 0.0f;
    if (is_adam(K)) {
        adam_constants(P.adam, k);
        lr = ld_global(P.adam.lr);
        t = (int64_t)load_base(reinterpret_cast<const uint64_t *>(P.adam.step)) + 1;
    }
    // by the CTA's last warps, which have no item in the shortest lists
    if (is_adam(K) && threadIdx.x == kClusterThreads - 32) s_result.step_size = adam_step_size(P.adam, lr, t);
    if (is_adam(K) && threadIdx.x == kClusterThreads - 64) s_result.inv_sqrt_by2 = adam_inv_sqrt(P.adam, t);
    double s = 0.0;
    Early<K> early{};
    if (busy) {
        if constexpr (K != kNorm) item_base = load_item_base<K>(P, p, worker);
        s = squares<K != kNorm>(p, base, P.src_flat, lane, held);
        if constexpr (K != kNorm) early = load_early<K, true>(P, p, item_base, lane, held);
    }
    const double sum = sum_of_cta(s, red);
    __syncwarp();
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");             // all CTAs run
    if (threadIdx.x == 0) {
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(&sums[blockIdx.x]);
#pragma unroll
        for (uint32_t r = 0; r < kClusterCtas; ++r)
            asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f64 [a], %2;\n\t}" :: "r"(to), "r"(r), "d"(sum) : "memory");
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x == 0) {
        double total = 0.0;
#pragma unroll
        for (uint32_t r = 0; r < kClusterCtas; ++r) total += sums[r];
        const double norm = sqrt(total);
        s_result.c = factor_of(norm, P.max_norm);
        s_result.stop = isfinite(norm) ? 0u : 1u;
        if (blockIdx.x == 0) {
            P.norms[worker] = (float)norm;
            if (!isfinite(norm)) atomicOr(&P.dev->status, THC_STATUS_NONFINITE);
            else if (is_adam(K)) *P.adam.step = t;     // every CTA has read it before the barrier
        }
    }
    if constexpr (K != kNorm) {
        __syncthreads();
        if (is_adam(K)) {
            if (s_result.stop != 0u) return;
            k.step_size = s_result.step_size;
            k.inv_sqrt_by2 = s_result.inv_sqrt_by2;
        }
        k.c = s_result.c;
        if (busy) products<K, true>(P, p, item_base, early, worker, k, lr, lane, held);
    }
}

// ---------------------------------------------------------------------------------- void rounds
struct VoidParams {
    const float *norms;
    float *scales, *out;
    uint64_t d, scales_n;
    uint32_t n, residuals;       // residuals: n or 0
    float most;                  // a larger norm, or a NaN, makes the round void
    DeviceBlock *dev;
    float *grads[THC_MAX_WORKERS];
    const float *ef[THC_MAX_WORKERS];
};

// Writes what a void round leaves (see thc.h), or, as nearly always, reads n numbers and ends: 1.0 to 1.1 us of a round of 28 us
// (4 x 65,536 elements), of one of 38 us with residuals.  A launch of its own, so that the transform kernels do not change; a void round of
// 8 x 25.6M with residuals takes 456 us here, 4 bytes written per element of the average and 8 moved per element of a residual.
// d is a multiple of 64, every vector aligned to 16 bytes.
__global__ void __launch_bounds__(kListThreads)
void_round_kernel(const __grid_constant__ VoidParams P)
{
    depend_on_previous();
    const bool bad = threadIdx.x < P.n && !(ld_global(P.norms + threadIdx.x) <= P.most);
    if (!__syncthreads_or(bad)) return;
    const uint64_t first = (uint64_t)blockIdx.x * kListThreads + threadIdx.x, stride = (uint64_t)gridDim.x * kListThreads;
    const float nan = __uint_as_float(0x7FFFFFFFu);
    for (uint64_t j = first; j < P.d / 4u; j += stride) {
        reinterpret_cast<float4 *>(P.out)[j] = make_float4(nan, nan, nan, nan);
        for (uint32_t i = 0; i < P.residuals; ++i)
            reinterpret_cast<uint4 *>(P.grads[i])[j] = ld_global(reinterpret_cast<const uint4 *>(P.ef[i]) + j);
    }
    for (uint64_t j = first; j < P.scales_n; j += stride) P.scales[j] = 0.0f;
    if (first == 0) atomicOr(&P.dev->status, THC_STATUS_NONFINITE);
}

// ---------------------------------------------------------------------------------- tables
// The pieces of a list, made on the device (a list of 355M elements in 290 tensors: 0.35 ms, with the table from the host 1.6).
// `first` is the number of a tensor's first piece; tensors without elements have none.
struct TensorRow { uint64_t numel, flat; uint32_t first, type; };
__global__ void list_pieces_kernel(const TensorRow *rows, uint32_t count, Piece *pieces, uint32_t pieces_n)
{
    depend_on_previous();
    const uint32_t i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= pieces_n) return;
    uint32_t lo = 0, hi = count;                       // the last tensor whose first piece is at most i
    while (hi - lo > 1u) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (rows[mid].first <= i) lo = mid;
        else hi = mid;
    }
    const TensorRow r = rows[lo];
    const uint64_t from = (uint64_t)(i - r.first) * kPiece;
    pieces[i] = Piece{r.flat + from, lo, (uint32_t)min((uint64_t)kPiece, r.numel - from) | r.type << 16};
}

constexpr uint32_t kAssignMost = 448;
struct AssignParams { uint64_t *to; uint32_t n; uint64_t base[kAssignMost]; };
__global__ void list_assign_kernel(const __grid_constant__ AssignParams P)
{
    depend_on_previous();
    if (threadIdx.x < P.n) P.to[threadIdx.x] = P.base[threadIdx.x];
}

}  // namespace thc

// =========================================================================== host side
using namespace thc;

struct thc_tensors {
    int device;                                // -1: host only
    uint32_t n, count, pieces_n, sm_count;
    uint64_t d, elements;
    bool all_f32;                              // the tensors that are not empty
    std::vector<uint64_t> numel, offset;
    std::vector<uint32_t> dtype;
    std::vector<uint64_t> address;             // [n][count]
    struct Range { uint64_t lo, hi; uint32_t index; };
    std::vector<Range> ranges;                 // of the tensors that are not empty, by address
    bool overlapping;                          // tensors of the list overlap each other
    bool torn;                                 // an assignment failed when part of the device's table had been set
    uint64_t *base;                            // the allocation; pieces are in it
    Piece *pieces;
};

static uint32_t size_of_type(uint32_t t) { return t == THC_F32 ? 4u : 2u; }

// Addresses into the list: checked, sorted for the overlap checks.
static int take_addresses(thc_tensors *h, const void *const *tensors)
{
    const size_t total = (size_t)h->n * h->count;
    for (size_t i = 0; i < total; ++i) {
        const uint64_t a = reinterpret_cast<uint64_t>(tensors[i]);
        const uint32_t t = (uint32_t)(i % h->count);
        if (h->numel[t] == 0) continue;
        if (a == 0 || a % size_of_type(h->dtype[t]) != 0) return THC_EINVAL;
    }
    h->ranges.clear();
    for (size_t i = 0; i < total; ++i) {
        const uint32_t t = (uint32_t)(i % h->count);
        h->address[i] = reinterpret_cast<uint64_t>(tensors[i]);
        if (h->numel[t] != 0)
            h->ranges.push_back({h->address[i], h->address[i] + h->numel[t] * size_of_type(h->dtype[t]), (uint32_t)i});
    }
    std::sort(h->ranges.begin(), h->ranges.end(), [](const thc_tensors::Range &a, const thc_tensors::Range &b) {
        return a.lo != b.lo ? a.lo < b.lo : a.index < b.index;
    });
    h->overlapping = false;
    uint64_t reach = 0;
    for (const auto &r : h->ranges) {
        if (r.lo < reach) h->overlapping = true;
        reach = std::max(reach, r.hi);
    }
    return THC_OK;
}

static uint64_t base_of(const thc_tensors *h, size_t i)
{
    const uint32_t t = (uint32_t)(i % h->count);
    return h->address[i] - h->offset[t] * size_of_type(h->dtype[t]);
}

int thc_tensors_create(const thc_ctx *ctx, const void *const *tensors, const uint64_t *numel, const uint32_t *dtype,
                       uint32_t n, uint32_t count, thc_tensors **list)
{
    if (list == nullptr) return THC_EINVAL;
    *list = nullptr;
    if (ctx == nullptr || tensors == nullptr || numel == nullptr || dtype == nullptr) return THC_EINVAL;
    if (n == 0 || n > THC_MAX_WORKERS || count == 0 || count > (1u << 20)) return THC_EINVAL;
    const CtxView view = view_of(ctx);
    if (view.device >= 0) {
        const int rc = check_launch_ctx(ctx);
        if (rc != THC_OK) return rc;
    }
    uint64_t d = 0, elements = 0, pieces_n = 0;
    for (uint32_t t = 0; t < count; ++t) {
        if (dtype[t] != THC_F32 && dtype[t] != THC_BF16 && dtype[t] != THC_F16) return THC_EINVAL;
        if (numel[t] > (1ull << 40)) return THC_EINVAL;
        elements += numel[t];
        d += (numel[t] + THC_TENSOR_ALIGN - 1) / THC_TENSOR_ALIGN * THC_TENSOR_ALIGN;
        pieces_n += (numel[t] + kPiece - 1) / kPiece;
        if (d > (1ull << 40)) return THC_EINVAL;
    }
    if (elements == 0) return THC_EINVAL;
    if (pieces_n * n > 0x7FFFFFFFull) return THC_EUNSUPPORTED;
    thc_tensors *h = nullptr;
    try {
        h = new thc_tensors;
        h->device = view.device;
        h->n = n;
        h->count = count;
        h->pieces_n = (uint32_t)pieces_n;
        h->sm_count = (uint32_t)view.sm_count;
        h->d = d;
        h->elements = elements;
        h->all_f32 = true;
        h->torn = false;
        h->pieces = nullptr;
        h->base = nullptr;
        h->numel.assign(numel, numel + count);
        h->dtype.assign(dtype, dtype + count);
        h->offset.resize(count);
        h->address.resize((size_t)n * count);
        uint64_t at = 0;
        for (uint32_t t = 0; t < count; ++t) {
            h->offset[t] = at;
            at += (numel[t] + THC_TENSOR_ALIGN - 1) / THC_TENSOR_ALIGN * THC_TENSOR_ALIGN;
            if (numel[t] != 0 && dtype[t] != THC_F32) h->all_f32 = false;
        }
        const int rc = take_addresses(h, tensors);
        if (rc != THC_OK) { delete h; return rc; }
        if (view.device >= 0) {
            // one allocation: addresses, rows, pieces
            const size_t base_bytes = h->address.size() * sizeof(uint64_t), rows_bytes = (size_t)count * sizeof(TensorRow);
            const size_t pieces_at = (base_bytes + rows_bytes + 15) / 16 * 16;
            std::vector<unsigned char> host(base_bytes + rows_bytes);
            for (size_t i = 0; i < h->address.size(); ++i) {
                const uint64_t v = base_of(h, i);
                memcpy(host.data() + i * sizeof v, &v, sizeof v);
            }
            uint32_t first = 0;
            for (uint32_t t = 0; t < count; ++t) {
                const TensorRow r{numel[t], h->offset[t], first, dtype[t]};
                memcpy(host.data() + base_bytes + t * sizeof r, &r, sizeof r);
                first += (uint32_t)((numel[t] + kPiece - 1) / kPiece);
            }
            cudaError_t e = cudaMalloc(reinterpret_cast<void **>(&h->base), pieces_at + (size_t)pieces_n * sizeof(Piece));
            if (e == cudaSuccess) {
                h->pieces = reinterpret_cast<Piece *>(reinterpret_cast<char *>(h->base) + pieces_at);
                e = cudaMemcpy(h->base, host.data(), host.size(), cudaMemcpyHostToDevice);
            }
            if (e == cudaSuccess)
                e = launch_after(list_pieces_kernel, dim3((unsigned)((pieces_n + 255) / 256)), 256, 0, nullptr,
                                 reinterpret_cast<const TensorRow *>(reinterpret_cast<const char *>(h->base) + base_bytes), count, h->pieces, h->pieces_n);
            if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
            if (e != cudaSuccess) {
                thc_tensors_destroy(h);
                return cuda_fail(e);
            }
        }
    } catch (const std::bad_alloc &) {
        thc_tensors_destroy(h);
        return THC_EINVAL;
    }
    *list = h;
    return THC_OK;
}

int thc_tensors_destroy(thc_tensors *h)
{
    if (h == nullptr) return THC_OK;
    if (h->base != nullptr) {
        // (a list may be collected while its thread captures a graph, which a plain cudaFree would spoil)
        cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
        const bool relaxed = cudaThreadExchangeStreamCaptureMode(&mode) == cudaSuccess;
        cudaFree(h->base);
        if (relaxed) cudaThreadExchangeStreamCaptureMode(&mode);
    }
    delete h;
    return THC_OK;
}

// CTAs per worker of the sums: rows of as many as run at a time (see list_norm_kernel), each of them at least six rounds long; one
// row where nothing is written after them, which is then 2 to 5 % faster.
struct NormShape { uint32_t row, rounds, ctas; };
static NormShape norm_shape(const thc_tensors *h, uint32_t split_log2, bool alone)
{
    const uint32_t most = std::max(1u, h->sm_count * kNormCtasPerSm / h->n);
    const uint64_t groups = (((uint64_t)h->pieces_n << split_log2) + kListWarps - 1) / kListWarps;
    NormShape s;
    s.row = (uint32_t)std::min<uint64_t>(most, groups);
    const uint32_t rounds = (uint32_t)((groups + s.row - 1) / s.row), rows = alone ? 1u : std::min(std::max(rounds / kNormLeastRounds, 1u), kNormMostRows);
    s.rounds = (rounds + rows - 1) / rows;
    s.ctas = (rounds + s.rounds - 1) / s.rounds * s.row;
    return s;
}

static uint64_t round_up256(uint64_t v) { return (v + 255) / 256 * 256; }

// Workspace: results of the workers, then the sums' partial results.  The same for every list of a device, so that a program's one buffer
// serves the gradients of n workers as well as the weights: norm_shape gives at most kNormMostRows rows of at most
// max(1, kNormCtasPerSm sm_count / n) CTAs to each of n workers.
static uint64_t results_bytes() { return round_up256(THC_MAX_WORKERS * sizeof(NormResult)); }
static uint64_t workspace_need(const thc_tensors *h)
{
    return results_bytes() + round_up256((uint64_t)kNormMostRows * std::max(h->sm_count * kNormCtasPerSm, THC_MAX_WORKERS) * sizeof(double));
}

int thc_tensors_sizes(const thc_tensors *h, thc_tensors_sizes_t *s)
{
    if (h == nullptr || s == nullptr) return THC_EINVAL;
    memset(s, 0, sizeof *s);
    s->d = h->d;
    s->elements = h->elements;
    s->workspace_bytes = workspace_need(h);
    s->n = h->n;
    s->count = h->count;
    s->device = h->device;
    return THC_OK;
}

int thc_tensors_offsets(const thc_tensors *h, uint64_t *offsets)
{
    if (h == nullptr || offsets == nullptr) return THC_EINVAL;
    std::copy(h->offset.begin(), h->offset.end(), offsets);
    return THC_OK;
}

// A list can be used where its context can launch.
static int check_list_device(const thc_ctx *ctx, const thc_tensors *h)
{
    if (ctx == nullptr || h == nullptr) return THC_EINVAL;
    const int rc = check_launch_ctx(ctx);
    if (rc != THC_OK) return rc;
    return h->device == view_of(ctx).device ? THC_OK : THC_EINVAL;
}

static int check_list(const thc_ctx *ctx, const thc_tensors *h)
{
    const int rc = check_list_device(ctx, h);
    return rc == THC_OK && h->torn ? THC_EINVAL : rc;
}

int thc_tensors_assign(const thc_ctx *ctx, thc_tensors *h, const void *const *tensors, void *stream)
{
    int rc = check_list_device(ctx, h);
    if (rc != THC_OK) return rc;
    if (tensors == nullptr) return THC_EINVAL;
    try {
        std::vector<uint64_t> old_address = h->address;
        std::vector<thc_tensors::Range> old_ranges = h->ranges;
        const bool old_overlapping = h->overlapping;
        rc = take_addresses(h, tensors);
        size_t set = 0;
        while (rc == THC_OK && set < h->address.size()) {
            AssignParams P;
            P.to = h->base + set;
            P.n = (uint32_t)std::min<size_t>(kAssignMost, h->address.size() - set);
            for (uint32_t j = 0; j < P.n; ++j) P.base[j] = base_of(h, set + j);
            const cudaError_t e = launch_after(list_assign_kernel, dim3(1), (kAssignMost + 31) / 32 * 32, 0, static_cast<cudaStream_t>(stream), P);
            if (e != cudaSuccess) rc = cuda_fail(e);
            else set += P.n;
        }
        if (rc != THC_OK) {                    // the checks of later calls go by what the device's table holds
            h->address.swap(old_address);
            h->ranges.swap(old_ranges);
            h->overlapping = old_overlapping;
        }
        if (rc == THC_OK || set != 0) h->torn = rc != THC_OK;
    } catch (const std::bad_alloc &) {
        return THC_EINVAL;
    }
    return rc;
}

static ListTable table_of(const thc_tensors *h) { return ListTable{h->pieces, h->base, h->count, h->pieces_n}; }

static int check_workspace(const thc_tensors *h, const void *workspace, uint64_t bytes)
{
    if (workspace == nullptr || !aligned16(workspace)) return THC_EINVAL;
    return bytes < workspace_need(h) ? THC_EWORKSPACE : THC_OK;
}

static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Whether [lo, hi) overlaps a tensor of the list.  Tensors that overlap each other make the answer "yes" at most
// more often than it is.
static bool overlaps(const thc_tensors *h, uint64_t lo, uint64_t hi)
{
    if (h->overlapping) {
        for (const auto &r : h->ranges) if (r.lo < hi && lo < r.hi) return true;
        return false;
    }
    const auto it = std::lower_bound(h->ranges.begin(), h->ranges.end(), lo, [](const thc_tensors::Range &r, uint64_t a) { return r.hi <= a; });
    return it != h->ranges.end() && it->lo < hi;
}

// A piece is eight units of a lane, one after the other or four at a time: few pieces are cut so that more warps share them.
static uint32_t split_of(const thc_tensors *h, uint64_t warps)
{
    uint32_t split = 0;
    while (split < 3 && ((uint64_t)h->pieces_n << (split + 1)) <= warps) ++split;
    return split;
}

static void fill_params(ListParams &P, const thc_ctx *ctx, const thc_tensors *h, double max_norm, float *norms, void *workspace)
{
    P.L = table_of(h);
    P.n = h->n;
    P.max_norm = max_norm;
    P.norms = norms;
    P.result = static_cast<NormResult *>(workspace);
    P.partial = reinterpret_cast<double *>(static_cast<char *>(workspace) + results_bytes());
    P.dev = view_of(ctx).dev;
}

static uint32_t split_of_norm(const thc_tensors *h) { return split_of(h, (uint64_t)h->sm_count * kListWarps / h->n); }

template <bool ADAM>
static int launch_norm(ListParams &P, const thc_tensors *h, bool alone, cudaStream_t st)
{
    P.split_log2 = split_of_norm(h);
    const NormShape shape = norm_shape(h, P.split_log2, alone);
    P.row = shape.row;
    P.rounds = shape.rounds;
    const dim3 grid(shape.ctas, h->n);
    THC_CUDA(launch_after(list_norm_kernel<ADAM>, grid, kListThreads, 0, st, static_cast<const ListParams &>(P)));
    return THC_OK;
}

template <ClipKind K>
static int launch_cluster(ParamsOf<K> &P, const thc_tensors *h, cudaStream_t st)
{
    P.split_log2 = std::max(1u, split_of(h, kClusterCtas * kClusterWarps));   // (1: see kHeldBytes)
    const size_t smem = K == kNorm ? 0 : kHeldBytes * kClusterWarps;
    if (smem != 0) {
        const int rc = ensure_dynamic_smem(reinterpret_cast<const void *>(list_cluster_kernel<K>));
        if (rc != THC_OK) return rc;
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kClusterCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(kClusterCtas, h->n);
    cfg.blockDim = dim3(kClusterThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    THC_CUDA(cudaLaunchKernelEx(&cfg, list_cluster_kernel<K>, P));
    return THC_OK;
}

// Up to so many pieces over all workers the products' warps add the sums themselves, which leaves out the last CTA's turn.  us,
// so / by the last CTA: 1024 pieces of bf16 gathered 7.4 / 8.1, 4096 13.5 / 14.1; beyond them too many warps would.
constexpr uint32_t kOwnSumsMostPieces = 4096;

template <ClipKind K>
static int launch_call(ParamsOf<K> &P, const thc_ctx *ctx, const thc_tensors *h, double max_norm, float *norms, void *workspace, void *stream)
{
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    fill_params(P, ctx, h, max_norm, norms, workspace);
    if (norms != nullptr && h->pieces_n <= cluster_most_pieces(K)) return launch_cluster<K>(P, h, st);
    if (norms != nullptr) {
        if ((uint64_t)h->pieces_n * h->n <= kOwnSumsMostPieces) P.partials = norm_shape(h, split_of_norm(h), false).ctas;
        const int rc = launch_norm<is_adam(K)>(P, h, false, st);
        if (rc != THC_OK) return rc;
    }
    P.split_log2 = split_of(h, (uint64_t)h->sm_count * product_ctas_per_sm(K) * kListWarps / h->n);
    const uint64_t items = ((uint64_t)h->pieces_n << P.split_log2) * h->n;
    THC_CUDA(launch_after(list_product_kernel<K>, dim3((unsigned)((items + kListWarps - 1) / kListWarps)), kListThreads, 0, st, P));
    return THC_OK;
}

int thc_grad_norm(thc_ctx *ctx, const thc_tensors *list, float *norms, void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_list(ctx, list);
    if (rc != THC_OK) return rc;
    if (norms == nullptr || !aligned4(norms)) return THC_EINVAL;
    if ((rc = check_workspace(list, workspace, workspace_bytes)) != THC_OK) return rc;
    ListParams P;
    memset(&P, 0, sizeof P);
    fill_params(P, ctx, list, INFINITY, norms, workspace);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (list->pieces_n <= cluster_most_pieces(kNorm)) return launch_cluster<kNorm>(P, list, st);
    P.result = nullptr;
    return launch_norm<false>(P, list, true, st);
}

// max_norm, norms and workspace of a call that clips.
static int check_clip(const thc_tensors *h, double max_norm, const float *norms, bool need_norms, const void *workspace, uint64_t bytes)
{
    if (!(max_norm >= 0.0) || !aligned4(norms)) return THC_EINVAL;
    if (norms == nullptr) return need_norms || !isinf(max_norm) ? THC_EINVAL : THC_OK;
    return check_workspace(h, workspace, bytes);
}

int thc_clip_grads(thc_ctx *ctx, const thc_tensors *list, double max_norm, const thc_tensors *out_or_null, float *norms,
                   void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_list(ctx, list);
    if (rc != THC_OK) return rc;
    const thc_tensors *out = out_or_null != nullptr ? out_or_null : list;
    if ((rc = check_list(ctx, out)) != THC_OK) return rc;
    if ((rc = check_clip(list, max_norm, norms, true, workspace, workspace_bytes)) != THC_OK) return rc;
    if (out->n != list->n || out->numel != list->numel || out->dtype != list->dtype || out->overlapping) return THC_EINVAL;
    if (out != list) {
        // both sorted by address; those of `out` do not overlap each other
        size_t j = 0;
        for (const auto &r : list->ranges) {
            while (j < out->ranges.size() && out->ranges[j].hi <= r.lo) ++j;
            if (j == out->ranges.size()) break;
            const auto &w = out->ranges[j];
            if (w.lo < r.hi && !(w.lo == r.lo && w.index == r.index)) return THC_EINVAL;
        }
    }
    ListParams P;
    memset(&P, 0, sizeof P);
    P.dst_base = out->base;
    return launch_call<kClip>(P, ctx, list, max_norm, norms, workspace, stream);
}

int thc_gather_grads(thc_ctx *ctx, const thc_tensors *list, double max_norm, const float *const *ef_or_null, void *const *flats,
                     float *norms, void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_list(ctx, list);
    if (rc != THC_OK) return rc;
    if ((rc = check_clip(list, max_norm, norms, false, workspace, workspace_bytes)) != THC_OK) return rc;
    const bool bf16 = view_of(ctx).in_dtype == THC_BF16;
    if (bf16 && ef_or_null != nullptr) return THC_EUNSUPPORTED;
    if (flats == nullptr) return THC_EINVAL;
    const uint64_t bytes = list->d * (bf16 ? 2u : 4u);
    GatherParams P;
    memset(&P, 0, sizeof P);
    for (uint32_t i = 0; i < list->n; ++i) {
        if (flats[i] == nullptr || !aligned16(flats[i])) return THC_EINVAL;
        P.dst_flat[i] = reinterpret_cast<uint64_t>(flats[i]);
        if (ef_or_null != nullptr) {
            if (ef_or_null[i] == nullptr || !aligned16(ef_or_null[i])) return THC_EINVAL;
            P.ef[i] = reinterpret_cast<uint64_t>(ef_or_null[i]);
        }
    }
    const auto apart = [bytes](uint64_t a, uint64_t b) { return a + bytes <= b || b + bytes <= a; };
    for (uint32_t i = 0; i < list->n; ++i) {
        if (overlaps(list, P.dst_flat[i], P.dst_flat[i] + bytes)) return THC_EINVAL;
        for (uint32_t j = 0; j < list->n; ++j) {
            if (j != i && !apart(P.dst_flat[i], P.dst_flat[j])) return THC_EINVAL;
            if (ef_or_null != nullptr && !(j == i && P.ef[j] == P.dst_flat[i]) && !apart(P.dst_flat[i], P.ef[j])) return THC_EINVAL;
        }
    }
    if (ef_or_null != nullptr) return launch_call<kGatherResidual>(P, ctx, list, max_norm, norms, workspace, stream);
    if (bf16) return launch_call<kGatherBf16>(P, ctx, list, max_norm, norms, workspace, stream);
    return launch_call<kGatherF32>(P, ctx, list, max_norm, norms, workspace, stream);
}

// Norms up to here pass a block of the context.  A rotation adds up to sqrt(B) |x| before it is scaled, the one back B times M = t_p |x| / sqrt(B): with
// 2^126 for either the fourfold is left for residuals and roundings.
static double transform_limit(const CtxView &view)
{
    return 0x1p126 / (sqrt((double)(1ull << view.log2_block)) * std::max(1.0, view.t_p));
}

int thc_void_round(thc_ctx *ctx, const thc_tensors *list, double max_norm, const float *norms, float *scales, float *out,
                   float *const *grads_or_null, const float *const *ef_or_null, void *stream)
{
    int rc = check_list(ctx, list);
    if (rc != THC_OK) return rc;
    if (!(max_norm >= 0.0) || norms == nullptr || !aligned4(norms) || scales == nullptr || !aligned16(scales) || out == nullptr || !aligned16(out)) return THC_EINVAL;
    if ((grads_or_null == nullptr) != (ef_or_null == nullptr)) return THC_EINVAL;
    if (ef_or_null != nullptr && view_of(ctx).in_dtype != THC_F32) return THC_EUNSUPPORTED;
    thc_sizes_t sz;
    if ((rc = thc_sizes(ctx, list->d, 1, &sz)) != THC_OK) return rc;
    VoidParams P;
    memset(&P, 0, sizeof P);
    P.norms = norms;
    P.scales = scales;
    P.out = out;
    P.d = list->d;
    P.scales_n = sz.scales_count;
    P.n = list->n;
    const CtxView view = view_of(ctx);
    P.dev = view.dev;
    P.most = max_norm <= transform_limit(view) ? 0x1.fffffep127f : (float)transform_limit(view);   // (clipped: any finite norm)
    struct Span { uint64_t lo, bytes; };
    Span written[THC_MAX_WORKERS + 2], read[THC_MAX_WORKERS + 1];
    uint32_t writes = 0, reads = 0;
    written[writes++] = {reinterpret_cast<uint64_t>(out), list->d * 4u};
    written[writes++] = {reinterpret_cast<uint64_t>(scales), P.scales_n * 4u};
    read[reads++] = {reinterpret_cast<uint64_t>(norms), list->n * 4u};
    if (ef_or_null != nullptr) {
        P.residuals = list->n;
        for (uint32_t i = 0; i < list->n; ++i) {
            P.grads[i] = grads_or_null[i];
            P.ef[i] = ef_or_null[i];
            if (P.grads[i] == nullptr || !aligned16(P.grads[i]) || P.ef[i] == nullptr || !aligned16(P.ef[i])) return THC_EINVAL;
            written[writes++] = {reinterpret_cast<uint64_t>(P.grads[i]), list->d * 4u};
            read[reads++] = {reinterpret_cast<uint64_t>(P.ef[i]), list->d * 4u};
        }
    }
    const auto apart = [](const Span &a, const Span &b) { return a.lo + a.bytes <= b.lo || b.lo + b.bytes <= a.lo; };
    for (uint32_t i = 0; i < writes; ++i) {
        for (uint32_t j = 0; j < i; ++j) if (!apart(written[i], written[j])) return THC_EINVAL;
        for (uint32_t j = 0; j < reads; ++j) if (!apart(written[i], read[j])) return THC_EINVAL;
    }
    const uint64_t ctas = std::min<uint64_t>((list->d / 4u + kListThreads - 1) / kListThreads, 2ull * std::max(1u, list->sm_count));
    THC_CUDA(launch_after(void_round_kernel, dim3((unsigned)ctas), kListThreads, 0, static_cast<cudaStream_t>(stream), P));
    return THC_OK;
}

int thc_scatter_grads(thc_ctx *ctx, const float *flat, double max_norm, const thc_tensors *list, float *norms, void *workspace,
                      uint64_t workspace_bytes, void *stream)
{
    int rc = check_list(ctx, list);
    if (rc != THC_OK) return rc;
    if ((rc = check_clip(list, max_norm, norms, false, workspace, workspace_bytes)) != THC_OK) return rc;
    if (flat == nullptr || !aligned16(flat) || list->n != 1 || list->overlapping) return THC_EINVAL;
    const uint64_t lo = reinterpret_cast<uint64_t>(flat), hi = lo + list->d * 4u;
    for (const auto &r : list->ranges)
        if (r.lo < hi && lo < r.hi && !(list->dtype[r.index] == THC_F32 && r.lo == lo + list->offset[r.index] * 4u)) return THC_EINVAL;
    ListParams P;
    memset(&P, 0, sizeof P);
    P.src_flat = lo;
    return launch_call<kScatter>(P, ctx, list, max_norm, norms, workspace, stream);
}

int thc_adamw(thc_ctx *ctx, const thc_adamw_config *cfg, const float *grad, const thc_tensors *list, const float *lr, int64_t *step,
              float *master_or_null, float *m, float *v, const float *decay_or_null, float *norms, void *workspace,
              uint64_t workspace_bytes, void *stream)
{
    int rc = check_list(ctx, list);
    if (rc != THC_OK) return rc;
    if (cfg == nullptr) return THC_EINVAL;
    if ((rc = check_clip(list, cfg->max_norm, norms, true, workspace, workspace_bytes)) != THC_OK) return rc;
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0 && cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return THC_EINVAL;
    if (!(cfg->eps >= 0.0) || isinf(cfg->eps) || !(cfg->weight_decay >= 0.0) || isinf(cfg->weight_decay)) return THC_EINVAL;
    if (list->n != 1 || list->overlapping || (master_or_null == nullptr && !list->all_f32)) return THC_EINVAL;
    if (lr == nullptr || !aligned4(lr) || step == nullptr || (reinterpret_cast<uintptr_t>(step) & 7u) != 0 || !aligned4(decay_or_null)) return THC_EINVAL;
    const void *flat[4] = {grad, m, v, master_or_null};
    const uint64_t bytes = list->d * 4u;
    const int flats = master_or_null != nullptr ? 4 : 3;
    for (int i = 0; i < flats; ++i) {
        if (flat[i] == nullptr || !aligned16(flat[i])) return THC_EINVAL;
        const uint64_t a = reinterpret_cast<uint64_t>(flat[i]);
        if (overlaps(list, a, a + bytes)) return THC_EINVAL;
        for (int j = 0; j < i; ++j) {
            const uint64_t b = reinterpret_cast<uint64_t>(flat[j]);
            if (a < b + bytes && b < a + bytes) return THC_EINVAL;
        }
    }
    ListParams P;
    memset(&P, 0, sizeof P);
    P.src_flat = reinterpret_cast<uint64_t>(grad);
    P.adam = AdamParams{grad, master_or_null, m, v, lr, decay_or_null, step, cfg->beta1, cfg->beta2, cfg->eps, cfg->weight_decay};
    if (master_or_null != nullptr) return launch_call<kAdamMaster>(P, ctx, list, cfg->max_norm, norms, workspace, stream);
    return launch_call<kAdam>(P, ctx, list, cfg->max_norm, norms, workspace, stream);
}
