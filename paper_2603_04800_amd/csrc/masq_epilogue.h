// Epilogues of the layer's GEMMs and the rows of the experts' layer.
#pragma once

#include "masq_device.h"

namespace masq {
namespace {

// What a tile does past the layer's own result: nothing (kTilePlain); bias,
// activation and residual (kTileEpilogue); the same for output rows sorted by
// expert, each expert with a weight, scales, factors and bias of its own
// (kTileExperts).
enum { kTilePlain = 0, kTileEpilogue = 1, kTileExperts = 2 };

// One tile of rows of one expert.
struct GroupTile {
    int expert, tn;
    int64_t first, end;       // its slots
};

// Edge e of the experts' slot ranges, within [0, n] whatever the array holds.
__device__ __forceinline__ int group_edge(const TileExtra& ex, int e, int64_t n) {
    return static_cast<int>(min(max(static_cast<int64_t>(ex.offsets[min(e, ex.n_experts)]), int64_t{0}), n));
}

// Rows of tiles that run together: those of one expert or two share a weight.
// Groups of 8 / 4 / 3 / 1 rows, us the layer: on 256 x 256 tiles 32768 slots over 64
// experts, 2048 -> 2816 344 / 344 / 332 / 331 and 1408 -> 2048 251 / 258 / 241 / 248,
// 16384 over 8, 3584 -> 8192 584 / 611 / 592 / 628 and 4096 -> 3584 330 / 334 / 338 /
// 336; on smaller ones 8192 over 64, 2048 -> 2048 123 / 124 / 120 / 119 and over 16,
// 2048 -> 4096 143 / 143 / 136 / 133.
constexpr int kExpertGroup = 3;

// The tile of workgroup `block`: every wave counts the experts' tiles of BM
// rows, a lane an expert, places the workgroup among them as tile_coords_at
// does, and finds the expert that holds its row of tiles.  False past the last
// tile (the grid is sized for the most tiles that n slots can make).  Offsets
// that do not ascend can ask for more tiles than that, more than an int counts:
// they get none.
template <int BM>
__device__ __forceinline__ bool group_tile(const TileExtra& ex, int64_t n, int64_t block, int tiles_n,
                                           GroupTile& out) {
    const int lane = threadIdx.x & 63;
    auto count = [&](int e, int& lo, int& hi) __attribute__((always_inline)) {
        lo = group_edge(ex, e, n);
        hi = e < ex.n_experts ? max(group_edge(ex, e + 1, n), lo) : lo;
        return (hi - lo) / BM + ((hi - lo) % BM != 0);
    };
    auto scan = [&](int v) __attribute__((always_inline)) {          // inclusive over the lanes
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int p = __shfl_up(v, o);
            v += lane >= o ? p : 0;
        }
        return v;
    };
    int lo, hi;
    int incl = scan(count(lane, lo, hi));
    // (64 lanes' tiles: at most half of them can start over, 32 n / BM + 64)
    uint32_t total = static_cast<uint32_t>(__builtin_amdgcn_readlane(incl, 63));
    for (int b = 64; b < ex.n_experts; b += 64) {
        int l2, h2;
        total = min(total + static_cast<uint32_t>(__builtin_amdgcn_readlane(scan(count(b + lane, l2, h2)), 63)),
                    0x7FFFFFFFu);
    }
    if (total > static_cast<uint32_t>(expert_tiles(n, ex.n_experts, BM))) return false;
    int tm;
    if (!tile_coords_at<kExpertGroup>(static_cast<int>(block), static_cast<int>(total), tiles_n, tm, out.tn))
        return false;
    int before = 0, b = 0;
    for (;;) {
        const int here = __builtin_amdgcn_readlane(incl, 63);
        if (tm < before + here || b + 64 >= ex.n_experts) break;
        before += here;
        b += 64;
        incl = scan(count(b + lane, lo, hi));
    }
    const unsigned long long past = __ballot(before + incl > tm);
    const int l = past != 0 ? __builtin_ctzll(past) : 63;            // (tm < total: past != 0)
    const int prev = l > 0 ? __builtin_amdgcn_readlane(incl, l - 1) : 0;
    out.expert = min(b + l, ex.n_experts - 1);
    out.first = __builtin_amdgcn_readlane(lo, l) + static_cast<int64_t>(tm - before - prev) * BM;
    out.end = min(out.first + BM, static_cast<int64_t>(__builtin_amdgcn_readlane(hi, l)));
    return true;
}

// The row of x behind a slot (an index outside it reads row 0).
__device__ __forceinline__ int64_t slot_row(const TileExtra& ex, int64_t slot) {
    if (ex.rows == nullptr) return slot;
    const int t = ex.rows[slot];
    return t >= 0 && t < ex.x_rows ? t : 0;
}

// 1 / (1 + exp(-z)) from v_exp_f32 and v_rcp_f32 (one unit in the last place
// each).  Results that are rounded to bf16 take -z log2 e as one product, off by
// |z| 2^-24; fp32 results add the product's own error and the next bits of
// log2 e.  An exponential that overflows has the reciprocal 0, the limit.  The
// correction is a difference, which a product past fp32's range would make
// infinity less infinity, so fp32 results take z within +-128, past which the
// function is 1 or below the smallest normal number whatever z is.
template <bool EXACT>
__device__ __forceinline__ float logistic(float z) {
    constexpr float kL = -1.44269504088896341f, kLo = -1.92596299e-8f, kLn2 = 0.69314718055994531f;
    if constexpr (EXACT) z = __builtin_amdgcn_fmed3f(z, -128.f, 128.f);
    const float t = z * kL;
    float e = __builtin_amdgcn_exp2f(t);
    if constexpr (EXACT) e *= fmaf(fmaf(z, kLo, fmaf(z, kL, -t)), kLn2, 1.f);
    return __builtin_amdgcn_rcpf(1.f + e);
}
template <bool EXACT>
__device__ __forceinline__ float act_silu(float z) { return z * logistic<EXACT>(z); }
// z Phi(z) = z erfc(-z / sqrt 2) / 2: erfc, unlike 1 + erf, keeps its relative
// accuracy for negative z, where it is small.  Results that are rounded to bf16
// take erfc(x) = t 2^(Q(t) - x^2 log2 e), t = 1 / (1 + x / 2), for x >= 0 (the form
// of Press et al., Numerical Recipes, 6.2), Q the degree-9 Chebyshev interpolant
// in t of log2(erfc(x) e^(x^2) / t) over x in [0, 10], off by 1.2e-7 of the value.
// The rounding of x^2 log2 e adds to that where the value is small: in all at most
// (16 + 4 z^2) 2^-24 of it (found: 4.4e-7 up to z = -1, 1.2e-6 to -3, 8.3e-6 to -9,
// 1.9e-5 to -13), and in absolute terms, what a residual that cancels the result
// leaves, about 1e-7 for z < 0.  4096 x 3584 -> 37888 gated: 614 us where erfcf
// takes 709.
template <bool EXACT>
__device__ __forceinline__ float act_gelu(float z) {
    if constexpr (EXACT) {
        return 0.5f * z * erfcf(z * -0.70710678118654752f);
    } else {
        constexpr float kQ[10] = {-1.8256655931472778f, 1.4409384727478027f, 0.5558468103408813f,
                                  0.05972175672650337f, -0.0281441118568182f, -0.057514917105436325f,
                                  -1.0769284963607788f, 1.724493384361267f, -1.0063326358795166f,
                                  0.21358530223369598f};
        const float x = fabsf(z) * 0.70710678118654752f;
        const float t = __builtin_amdgcn_rcpf(fmaf(0.5f, x, 1.f));
        float q = kQ[9];
#pragma unroll
        for (int i = 8; i >= 0; --i) q = fmaf(q, t, kQ[i]);
        const float e = t * __builtin_amdgcn_exp2f(fmaf(x * -1.44269504f, x, q));
        return 0.5f * z * (z > 0.f ? 2.f - e : e);
    }
}
template <bool EXACT>
__device__ __forceinline__ float act_gelu_tanh(float z) {   // (1 + tanh t) / 2 = 1 / (1 + exp(-2 t))
    return z * logistic<EXACT>(1.5957691216057308f * (z + 0.044715f * (z * z * z)));
}
// act on every STEP-th of the N values, one branch for all of them
template <typename YT, int STEP, int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
    constexpr bool kExact = sizeof(YT) == 4;
    switch (act) {                                          // uniform
        case kActSilu:
#pragma unroll
            for (int e = 0; e < N; e += STEP) v[e] = act_silu<kExact>(v[e]);
            break;
        case kActGelu:
#pragma unroll
            for (int e = 0; e < N; e += STEP) v[e] = act_gelu<kExact>(v[e]);
            break;
        case kActGeluTanh:
#pragma unroll
            for (int e = 0; e < N; e += STEP) v[e] = act_gelu_tanh<kExact>(v[e]);
            break;
        default: break;
    }
}

// Bias, activation (times the up channel where gated), residual, rounding and
// store of a row of NJ blocks of one wave (32 tokens x 32 channels each; lane =
// token lane % 32, register 4 g + e = channel 8 g + 4 (lane / 32) + e).  The
// values pass through a per-wave LDS transpose, 16 channels at a time, after
// which a lane holds 8 neighbouring channels of one token: bias and residual
// are read, and the output written, in whole pieces of 8 (gated: 4) elements,
// and the only rounding to the output type follows the last addition.  An
// element of the residual is read by the lane that writes the output's same
// element, so the two may be one array.  LDS operations of one wave execute in
// order, so its buffer (32 rows of kEpiPitch floats) needs no synchronisation.
//
// The loop over the blocks is not unrolled (they move down a block a turn): a
// tile runs through this code once, so that its length is paid in instruction
// fetches.  Fully unrolled, the products and epilogues of 4096 x 3584 -> 37888
// (gated) took 930 us where this form takes 593.
constexpr int kEpiPitch = 20;                               // 16 channels and 16 bytes
template <typename YT, int NJ>
__device__ __forceinline__ void finish_row(v16f (&yb)[NJ], const TileExtra& ex, const float* bias,
                                           float* scr, YT* y, int64_t trow, int64_t rend, int tcol,
                                           int N, int lane) {
    const int width = ex.gated ? N >> 1 : N;                // outputs of a row
    const int64_t t = trow + (lane >> 1);
    const YT* res = static_cast<const YT*>(ex.residual);
    float* wr = scr + (lane & 31) * kEpiPitch + 4 * (lane >> 5);
    const float* rd = scr + (lane >> 1) * kEpiPitch + 8 * (lane & 1);
    // 16 channels from the first 8 registers of y16 on
    auto unit = [&](const v16f& y16, auto half, int c) __attribute__((always_inline)) {
        constexpr int o0 = 8 * decltype(half)::value;
#pragma unroll
        for (int g = 0; g < 2; ++g)
            *reinterpret_cast<v4f*>(wr + 8 * g) = v4f{y16[o0 + 4 * g], y16[o0 + 4 * g + 1], y16[o0 + 4 * g + 2],
                                                      y16[o0 + 4 * g + 3]};
        float v[8];
        load8_f32(rd, v);
        if (t >= rend || c >= N) return;
        if (bias != nullptr) {
            float b[8];
            load8_f32(bias + c, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += b[e];
        }
        if (ex.gated) {
            activate<YT, 2>(ex.act, v);
            float o[4] = {v[0] * v[1], v[2] * v[3], v[4] * v[5], v[6] * v[7]};
            const int64_t at = t * width + (c >> 1);
            if (res != nullptr) {
                float q[4];
                Elem<YT>::load4(res + at, q);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += q[e];
            }
            store4(y + at, o);
        } else {
            activate<YT, 1>(ex.act, v);
            const int64_t at = t * width + c;
            if (res != nullptr) {
                float q[8];
                Elem<YT>::load8(res + at, q);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += q[e];
            }
            store8(y + at, v);
        }
    };
    const int c0 = tcol + 8 * (lane & 1);
#pragma unroll 1
    for (int j = 0; j < NJ; ++j) {
        unit(yb[0], std::integral_constant<int, 0>{}, c0 + 32 * j);
        unit(yb[0], std::integral_constant<int, 1>{}, c0 + 32 * j + 16);
#pragma unroll
        for (int k = 0; k + 1 < NJ; ++k) yb[k] = yb[k + 1];
    }
}

// The same for one channel a lane, neighbouring channels in neighbouring lanes
// (decode GEMM): the lanes of a gate and its up channel are active together,
// and the gate's lane writes their output.
template <typename YT>
__device__ __forceinline__ void finish_one(float v, const TileExtra& ex, YT* y, int t, int ch, int N) {
    if (ex.bias != nullptr) v += ex.bias[ch];
    int o = ch, width = N;
    float z[1] = {v};
    activate<YT, 1>(ex.act, z);
    if (ex.gated) {
        const float up = __shfl_xor(v, 1);
        if (ch & 1) return;
        v = z[0] * up;
        o = ch >> 1;
        width = N >> 1;
    } else {
        v = z[0];
    }
    const int64_t at = static_cast<int64_t>(t) * width + o;
    if (ex.residual != nullptr) v += Elem<YT>::load1(static_cast<const YT*>(ex.residual) + at);
    Elem<YT>::store1(y + at, v);
}

}  // namespace
}  // namespace masq
