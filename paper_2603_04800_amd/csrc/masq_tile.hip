// Launchers of the small-tile and the decode GEMM (masq_tile.h).

#include "masq_tile.h"

namespace masq {
namespace {

template <typename YT, typename LT, bool CMC, bool ACC, bool W4>
hipError_t launch_tile_t(const TileGemm& g) {
    const int bm = kTileShapes[g.plan.shape].bm, bn = kTileShapes[g.plan.shape].bn;
    const int tiles_m = static_cast<int>((g.T + bm - 1) / bm);
    const int tiles_n = static_cast<int>((g.N + bn - 1) / bn);
    const int64_t nt = static_cast<int64_t>(tiles_m) * tiles_n * g.plan.S;
#define MASQ_TILE(BM, BN, WM, WN, NST, WPE)                                                         \
    hipLaunchKernelGGL((k_gemm_tile<YT, LT, CMC, ACC, W4, BM, BN, WM, WN, NST, WPE>),               \
                       grid_of(8 * ((nt + 7) / 8), 64 * WM * WN), dim3(64 * WM * WN), 0, g.stream,  \
                       g.q, g.wq, g.x_scale, g.w_scale, g.T, static_cast<int>(g.K),                 \
                       static_cast<int>(g.N), tiles_m, tiles_n, g.mod, g.u, g.u_hl, g.rank,         \
                       g.n_mod, static_cast<const LT*>(g.r_up), g.acc, static_cast<YT*>(g.y),       \
                       g.plan.S, g.part, g.tickets, g.a_pair, TileExtra{})
    switch (g.plan.shape) {
        case 0: MASQ_TILE(32, 64, 1, 2, 3, 2); break;
        case 1: MASQ_TILE(64, 64, 2, 2, 3, 3); break;
        case 2: MASQ_TILE(128, 128, 2, 2, 2, 2); break;
        default: return hipErrorInvalidValue;
    }
#undef MASQ_TILE
    return hipGetLastError();
}

template <typename YT, typename LT, bool CMC, bool ACC>
hipError_t launch_tile_w(const TileGemm& g) {
    return g.w4 ? launch_tile_t<YT, LT, CMC, ACC, true>(g) : launch_tile_t<YT, LT, CMC, ACC, false>(g);
}

template <typename YT, typename LT, bool W4>
hipError_t launch_stream_t(const StreamGemm& g) {
    int ns = 0, sp = 0, groups = 0;
    plan_decode(g.K, g.N, ns, sp, groups);
    const int S = stream_slices(g.K, groups, ns);
    const size_t lds = g.u != nullptr ? static_cast<size_t>((g.T + S - 1) / S) * g.rank * sizeof(float)
                                      : 0;
    hipLaunchKernelGGL((k_gemm_stream<YT, LT, W4>), dim3(static_cast<unsigned>(groups * S)),
                       dim3(kStrThreads), lds, g.stream, g.q, g.wq, g.x_scale, g.w_scale,
                       static_cast<int>(g.T), static_cast<int>(g.K), static_cast<int>(g.N), S, g.mod, g.u,
                       g.u_slices, g.rank, g.n_mod, static_cast<const LT*>(g.r_up), g.part, g.tickets,
                       static_cast<YT*>(g.y), g.only_mod, TileExtra{});
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_stream(const StreamGemm& g) {
    if (!small_path(g.T, g.K) || g.N % 16 != 0 || g.part == nullptr || g.tickets == nullptr)
        return hipErrorInvalidValue;
#define MASQ_STREAM(YT, LT) (g.w4 ? launch_stream_t<YT, LT, true>(g) : launch_stream_t<YT, LT, false>(g))
    if (g.y_dt == DT::BF16) return g.lr_dt == DT::BF16 ? MASQ_STREAM(bf16_t, bf16_t) : MASQ_STREAM(bf16_t, float);
    return g.lr_dt == DT::BF16 ? MASQ_STREAM(float, bf16_t) : MASQ_STREAM(float, float);
#undef MASQ_STREAM
}

hipError_t launch_gemm_tile(const TileGemm& g) {
    if (g.K % 16 != 0 || g.N % 16 != 0 || g.plan.S < 1 || (g.w4 && g.K % 64 != 0) ||
        (g.a_pair && g.K % 64 != 0) || (g.plan.S > 1 && (g.part == nullptr || g.tickets == nullptr)))
        return hipErrorInvalidValue;
    // the int32 accumulator output exists only for the plain product
    if (!g.cmc) {
        if (g.acc != nullptr)
            return g.y_dt == DT::BF16 ? launch_tile_w<bf16_t, bf16_t, false, true>(g)
                                      : launch_tile_w<float, bf16_t, false, true>(g);
        return g.y_dt == DT::BF16 ? launch_tile_w<bf16_t, bf16_t, false, false>(g)
                                  : launch_tile_w<float, bf16_t, false, false>(g);
    }
    if (g.y_dt == DT::BF16)
        return g.lr_dt == DT::BF16 ? launch_tile_w<bf16_t, bf16_t, true, false>(g)
                                   : launch_tile_w<bf16_t, float, true, false>(g);
    return g.lr_dt == DT::BF16 ? launch_tile_w<float, bf16_t, true, false>(g)
                               : launch_tile_w<float, float, true, false>(g);
}

}  // namespace masq
