// Smoothing and per-token quantisation of one row, by a workgroup or by a wave.
#pragma once

#include "masq_device.h"

namespace masq {
namespace {

// Row t quantised by a workgroup of NT threads keeping NT x 8 x NCH elements
// of the row in registers.
template <typename XT, int NT, int NCH>
__device__ __forceinline__ void sq_row(const XT* __restrict__ x, const int32_t* __restrict__ mod,
                                       const float* __restrict__ inv_s, int K, int n_mod,
                                       int8_t* __restrict__ q, float* __restrict__ x_scale,
                                       int64_t t, bool pair) {
    __shared__ float red[NT / 64];
    const int m = sane_mod(mod[t], n_mod);
    const XT* xr = x + t * static_cast<int64_t>(K);
    const float* sr = inv_s + static_cast<int64_t>(m) * K;
    int8_t* qr = q + code_row(t, K, pair);
    const int nv = K >> 3;

    float xs[NCH][8];
    float amax = 0.f;
    {
        float xv[NCH][8], sv[NCH][8];
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int v = min(static_cast<int>(threadIdx.x) + NT * c, nv - 1);   // clamped
            Elem<XT>::load8(xr + 8 * v, xv[c]);
            load8_f32(sr + 8 * v, sv[c]);
        }
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const bool in = static_cast<int>(threadIdx.x) + NT * c < nv;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                xs[c][j] = xv[c][j] * sv[c][j];
                if (in) amax = fmaxf(amax, fabsf(xs[c][j]));
            }
        }
    }
    for (int v = threadIdx.x + NT * NCH; v < nv; v += NT) {
        float xv[8], sv[8];
        Elem<XT>::load8(xr + 8 * v, xv);
        load8_f32(sr + 8 * v, sv);
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(xv[j] * sv[j]));
    }
    amax = wave_max(amax);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    __syncthreads();
    amax = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) amax = fmaxf(amax, red[w]);

    const bool nz = amax > 0.f;
    const float dx = nz ? amax / 127.0f : 0.f;     // correctly rounded
    const float rq = nz ? 127.0f / amax : 0.f;
    if (threadIdx.x == 0) x_scale[t] = dx;

    auto put8 = [&](int v, const float (&val)[8]) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float c = rintf(val[j] * rq);
            c = fminf(fmaxf(c, -127.0f), 127.0f);
            w[j >> 2] |= (static_cast<uint32_t>(static_cast<int32_t>(c)) & 0xFFu) << (8 * (j & 3));
        }
        v2i out;
        out.x = static_cast<int32_t>(w[0]);
        out.y = static_cast<int32_t>(w[1]);
        *reinterpret_cast<v2i*>(qr + code_col(8 * v, pair)) = out;
    };
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int v = static_cast<int>(threadIdx.x) + NT * c;
        if (v < nv) put8(v, xs[c]);
    }
    for (int v = threadIdx.x + NT * NCH; v < nv; v += NT) {
        float xv[8], sv[8], val[8];
        Elem<XT>::load8(xr + 8 * v, xv);
        load8_f32(sr + 8 * v, sv);
#pragma unroll
        for (int j = 0; j < 8; ++j) val[j] = xv[j] * sv[j];
        put8(v, val);
    }
}

// Chunks of 512 columns a wave holds of a row of K columns, of the instances
// there are.  A chunk past the row's end costs its loads and arithmetic all
// the same: with 8 for every row, 16384 x 256 fp32 took 17.2 us, 65536 x 512
// 63 us, where fitting chunks take 8 and 33.
inline __host__ __device__ int quant_row_chunks(int64_t K) {
    return K <= 512 ? 1 : (K <= 1024 ? 2 : (K <= 2048 ? 4 : (K <= 3072 ? 6 : 8)));
}

// One row t quantised by one wave (lane = this lane), its smoothed values
// kept in registers between the absmax and the codes for rows of up to
// 64 * 8 * NC elements; longer rows stream their remainder twice.  The row's
// NC loads are in flight together, issued before anything that waits for the
// modality id (lanes past the row's end repeat its last piece); `between`
// runs while they are.
template <typename XT, int NC, typename Between>
__device__ __forceinline__ void quant_row_wave(const XT* __restrict__ x, const int32_t* __restrict__ mod,
                                               const float* __restrict__ inv_s, int K, int n_mod,
                                               int8_t* __restrict__ q, float* __restrict__ x_scale,
                                               int64_t t, bool pair, int lane, Between between) {
    const XT* xr = x + t * static_cast<int64_t>(K);
    const int nv = K >> 3;
    Raw8<XT> raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) raw[c].load(xr + 8 * min(lane + 64 * c, nv - 1));
    const int m = sane_mod(mod[t], n_mod);
    const float* sr = inv_s + static_cast<int64_t>(m) * K;
    int8_t* qr = q + code_row(t, K, pair);
    between(m);

    float xs[NC][8];
    float amax = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) load8_f32(sr + 8 * min(lane + 64 * c, nv - 1), xs[c]);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float xv[8];
        raw[c].to_f32(xv);
#pragma unroll
        for (int j = 0; j < 8; ++j) {                 // (repeats do not change the maximum)
            xs[c][j] = xv[j] * xs[c][j];
            amax = fmaxf(amax, fabsf(xs[c][j]));
        }
    }
    for (int v = lane + 64 * NC; v < nv; v += 64) {
        float xv[8], sv[8];
        Elem<XT>::load8(xr + 8 * v, xv);
        load8_f32(sr + 8 * v, sv);
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(xv[j] * sv[j]));
    }
    amax = wave_max(amax);
    const bool nz = amax > 0.f;
    const float dx = nz ? amax / 127.0f : 0.f;     // correctly rounded
    const float rq = nz ? 127.0f / amax : 0.f;
    if (lane == 0) x_scale[t] = dx;

    auto store8 = [&](int v, const float (&vals)[8]) {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float c = rintf(vals[j] * rq);
            c = fminf(fmaxf(c, -127.0f), 127.0f);
            w[j >> 2] |= (static_cast<uint32_t>(static_cast<int32_t>(c)) & 0xFFu) << (8 * (j & 3));
        }
        v2i out;
        out.x = static_cast<int32_t>(w[0]);
        out.y = static_cast<int32_t>(w[1]);
        *reinterpret_cast<v2i*>(qr + code_col(8 * v, pair)) = out;
    };
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int v = lane + 64 * c;
        if (v < nv) store8(v, xs[c]);
    }
    for (int v = lane + 64 * NC; v < nv; v += 64) {
        float xv[8], sv[8], vals[8];
        Elem<XT>::load8(xr + 8 * v, xv);
        load8_f32(sr + 8 * v, sv);
#pragma unroll
        for (int j = 0; j < 8; ++j) vals[j] = xv[j] * sv[j];
        store8(v, vals);
    }
}

}  // namespace
}  // namespace masq
