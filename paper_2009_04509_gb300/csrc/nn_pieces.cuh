// Pieces of eight neighbouring columns of 16-bit rows, at any alignment, and the
// random numbers of dropout: shared by the norms (nn_norm.cu) and dropout (nn_dropout.cu).
//
// The loads are plain ones, not the read-only path's: a call may write the rows that it
// reads (y the residual itself).  At odd alignment a piece lies in two aligned words,
// which hold neighbours' bytes too; those are dropped, whatever their state.
#pragma once

#include "nn_pair.cuh"

namespace emtk {
namespace {

constexpr int kPiece = 8;

struct Rows16 {  // a matrix of 16-bit elements
    uint8_t *p;
    int64_t row_bytes;
    __device__ __forceinline__ uint16_t *row(int64_t r) const { return reinterpret_cast<uint16_t *>(p + r * row_bytes); }
};
inline Rows16 rows16_of(const emtk_matrix &m) { return {static_cast<uint8_t *>(m.d), 2 * m.ld}; }
// Every row starts on 16 bytes (or the matrix is absent).
inline bool on_grid(const emtk_matrix &m, int64_t rows, size_t elem = 2) {
    return !m.d || (reinterpret_cast<uintptr_t>(m.d) % 16 == 0 && (rows <= 1 || m.ld * elem % 16 == 0));
}

struct Eight {  // a piece's values
    float2 v[4];
    __device__ __forceinline__ void fill(float x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = both(x);
    }
};
template <bool F16>
__device__ __forceinline__ Eight values8(const uint32_t *w) {
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) e.v[i] = values_of<F16>(w[i]);
    return e;
}
template <bool F16>
__device__ __forceinline__ void words8(const Eight &e, uint32_t (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack16<F16>(e.v[i].x, e.v[i].y);
}

// Four words out of eight, from half word `halves` on; one case to a row.
template <int FIRST>
__device__ __forceinline__ void funnel(const uint32_t *x, int bits, uint32_t *y) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = __funnelshift_r(x[FIRST + i], FIRST + i + 1 < 8 ? x[FIRST + i + 1] : 0u, bits);
}
__device__ __forceinline__ void shift_words(const uint32_t *x, int halves, uint32_t *y) {
    const int bits = 16 * (halves & 1);
    switch (halves >> 1) {
        case 0: funnel<0>(x, bits, y); break;
        case 1: funnel<1>(x, bits, y); break;
        case 2: funnel<2>(x, bits, y); break;
        default: funnel<3>(x, bits, y);
    }
}

// Columns c .. c + 7 of row r of an m x n matrix; those from n on are 0.  ANY: rows
// start anywhere; else on 16 bytes.  load() starts the loads, words() takes the values.
template <bool ANY>
struct Piece16 {
    uint32_t x[ANY ? 8 : 4];
    int halves;  // 16-bit elements to drop

    __device__ __forceinline__ void load(const Rows16 &a, int64_t r, int c, int m, int n) {
        const uint16_t *const p = a.row(r) + c;
        halves = 0;
        if (ANY ? c + kPiece <= n && (r > 0 || c >= kPiece) && (r < m - 1 || c + 2 * kPiece <= n) : c + kPiece <= n) {
            if (ANY) halves = (int)(reinterpret_cast<uintptr_t>(p) % 16) / 2;
            const uint4 *const q = reinterpret_cast<const uint4 *>(p - halves);
            const uint4 w = *q;
            x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
            if (ANY && halves) {
                const uint4 u = q[1];
                x[4] = u.x, x[5] = u.y, x[6] = u.z, x[7] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = 0u;
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (c + i < n) x[i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
        }
    }
    __device__ __forceinline__ void clear() {
        halves = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = 0u;
    }
    template <bool F16>
    __device__ __forceinline__ Eight values() const {
        if (ANY && halves) {
            uint32_t y[4];
            shift_words(x, halves, y);
            return values8<F16>(y);
        }
        return values8<F16>(x);
    }
};

// Stores a piece a lane, `lanes` neighbouring lanes (4 .. 32) to a run of a row that
// starts at p and has n elements (0 .. 8 lanes).  All lanes of the warp call this
// together.  ANY: each lane stores the 16 aligned bytes that start in its own piece, the
// run's ends go by elements, one a lane: 8 stores of 2 bytes a lane instead, 16 bytes
// apart, write every 32-byte sector twice eight times.
template <bool ANY>
__device__ __forceinline__ void store_run(uint16_t *p, int n, const uint32_t (&w)[4], int lanes, int lane) {
    const int c = kPiece * lane;
    const int head = ANY ? (int)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(p) % 16)) % 16) / 2 : 0;
    if (head == 0) {
        if (c + kPiece <= n) {
            *reinterpret_cast<uint4 *>(p + c) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < kPiece; ++i)
                if (c + i < n) p[c + i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
        }
    }
    if constexpr (ANY) {
        if (!__any_sync(0xffffffffu, head != 0)) return;
        uint32_t x[8];
    #pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = w[i];
            x[4 + i] = __shfl_down_sync(0xffffffffu, w[i], 1, lanes);
        }
        const int whole = head ? max(0, min(lanes - 1, (n - head) / kPiece)) : 0;  // aligned words
        if (lane < whole) {
            uint32_t y[4];
            shift_words(x, head, y);
            *reinterpret_cast<uint4 *>(p + c + head) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        const int tail = head + kPiece * whole;
        for (int e0 = 0; e0 < 16; e0 += lanes) {  // lanes 0 .. 7 the head's elements, 8 .. 15 the tail's
            const int e = e0 + lane;
            const int at = e < 8 ? e : tail + e - 8;
            const int from = (at >> 3) & (lanes - 1), word = (at & 7) >> 1;
            uint32_t y = 0;
    #pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t v = __shfl_sync(0xffffffffu, w[i], from, lanes);
                y = word == i ? v : y;
            }
            if (head && e < 16 && at < (e < 8 ? min(head, n) : n)) p[at] = (uint16_t)(y >> (16 * (at & 1)));
        }
    }
}

// ---- parameters of a row's columns: 16 bits or fp32, vectors at any alignment
struct Param {
    const void *p;
    int f32, vec;  // vec: on 16 bytes
};
inline Param param_of(const void *p, bool f32) { return {p, f32, reinterpret_cast<uintptr_t>(p) % 16 == 0}; }
// Columns c .. of one that is there; those from n on are 0.  whole: none of them.
template <bool F16>
__device__ __forceinline__ Eight param8(const Param &a, int c, int n, bool whole) {
    Eight e;
    if (a.f32) {
        const float *const p = static_cast<const float *>(a.p) + c;
        if (a.vec && whole) {
            const float4 lo = __ldg(reinterpret_cast<const float4 *>(p)), hi = __ldg(reinterpret_cast<const float4 *>(p) + 1);
            e.v[0] = make_float2(lo.x, lo.y), e.v[1] = make_float2(lo.z, lo.w);
            e.v[2] = make_float2(hi.x, hi.y), e.v[3] = make_float2(hi.z, hi.w);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                e.v[i] = make_float2(c + 2 * i < n ? __ldg(p + 2 * i) : 0.f, c + 2 * i + 1 < n ? __ldg(p + 2 * i + 1) : 0.f);
        }
        return e;
    }
    const uint16_t *const p = static_cast<const uint16_t *>(a.p) + c;
    uint32_t w[4] = {};
    if (a.vec && whole) {
        const uint4 q = __ldg(reinterpret_cast<const uint4 *>(p));
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else {
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (c + i < n) w[i / 2] |= (uint32_t)__ldg(p + i) << (16 * (i % 2));
    }
    return values8<F16>(w);
}

// ---- dropout
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3,
// SC 2011): ten rounds of two 32 x 32-bit products, the key raised by a constant in each.
// One call serves a piece: 16 bits an element.  32 bits would cost twice the products,
// and these are already half of what a wide copy has to issue; the share dropped is
// rounded to 2^-16 and the factor made for the rounded share, so the mean stays right.
struct Drop {
    uint64_t seed, offset;
    const uint64_t *d_offset;
    uint32_t below;  // of 65536; 0: nothing is dropped
    float factor;
};
inline Drop drop_of(const emtk_drop &d) {
    const double t = d.p * 65536.0, whole = (double)(int64_t)t, rest = t - whole;
    int64_t below = (int64_t)whole + (rest > 0.5 || (rest == 0.5 && ((int64_t)whole & 1)) ? 1 : 0);
    below = below < 65535 ? below : 65535;
    return {d.seed, d.offset, d.d_offset, (uint32_t)below, (float)(65536.0 / (65536.0 - (double)below))};
}
// The call's offset, as the device has it.
__device__ __forceinline__ uint64_t drop_offset(const Drop &d) { return d.offset + (d.d_offset ? *d.d_offset : 0u); }

// The random numbers of row r, columns 8 g ..
__device__ __forceinline__ void drop_numbers(const Drop &d, uint64_t offset, uint32_t r, uint32_t g, uint32_t *x) {
    x[0] = g, x[1] = r, x[2] = (uint32_t)offset, x[3] = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)d.seed, k1 = (uint32_t)(d.seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)x[0] * 0xD2511F53u, b = (uint64_t)x[2] * 0xCD9E8D57u;
        x[0] = (uint32_t)(b >> 32) ^ x[1] ^ k0;
        x[1] = (uint32_t)b;
        x[2] = (uint32_t)(a >> 32) ^ x[3] ^ k1;
        x[3] = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}
// Eight elements under their numbers.
__device__ __forceinline__ void dropped_by(const Drop &d, const uint32_t *x, Eight &e) {
    const uint32_t high = d.below << 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = e.v[i] * both(d.factor);
        e.v[i] = make_float2((x[i] << 16) >= high ? v.x : 0.f, x[i] >= high ? v.y : 0.f);
    }
}
// The piece's elements under dropout: row r, columns 8 g ..
__device__ __forceinline__ void dropped(const Drop &d, uint64_t offset, uint32_t r, uint32_t g, Eight &e) {
    uint32_t x[4];
    drop_numbers(d, offset, r, g, x);
    dropped_by(d, x, e);
}

}  // namespace
}  // namespace emtk
