// The operators around the quantised layer of a decoder block.
//
//   layer epilogue   the layer's GEMMs (masq_tile.h) with bias, activation and
//                    residual: launch_gemm_tile_epilogue, launch_gemm_stream_epilogue
//   k_route_*        the k largest logits of a token, their softmax weights, and
//                    the choices of all tokens sorted by expert
//   k_expert_stage1  u = (x S^-1) L1 of the experts' rows, beside the quantisation
//   k_gemm_tile      (kTileExperts) the layer over rows sorted by expert
//   k_combine        a token's expert rows, weighted and summed

#include "masq_quant.h"
#include "masq_tile.h"

namespace masq {
namespace {

// ================================================================ layer epilogue
template <typename YT, typename LT, bool CMC, bool W4, int MODE>
hipError_t launch_tile_mode(const TileGemm& g, const TileExtra& ex, int tiles_m) {
    const int bn = kTileShapes[g.plan.shape].bn;
    const int tiles_n = static_cast<int>((g.N + bn - 1) / bn);
    const int64_t nt = static_cast<int64_t>(tiles_m) * tiles_n * g.plan.S;
#define MASQ_TILE_WK(BM, BN, WM, WN, NST, WPE, WK)                                                  \
    hipLaunchKernelGGL((k_gemm_tile<YT, LT, CMC, false, W4, BM, BN, WM, WN, NST, WPE, MODE, WK>),   \
                       grid_of(8 * ((nt + 7) / 8), 64 * WM * WN * WK), dim3(64 * WM * WN * WK), 0,  \
                       g.stream,                                                                    \
                       g.q, g.wq, g.x_scale, g.w_scale, g.T, static_cast<int>(g.K),                 \
                       static_cast<int>(g.N), tiles_m, tiles_n, g.mod, g.u, g.u_hl, g.rank,         \
                       g.n_mod, static_cast<const LT*>(g.r_up), nullptr, static_cast<YT*>(g.y),     \
                       g.plan.S, g.part, g.tickets, g.a_pair, ex)
#define MASQ_TILE(BM, BN, WM, WN, NST, WPE) MASQ_TILE_WK(BM, BN, WM, WN, NST, WPE, 1)
    switch (g.plan.shape) {
        case 0:
            // two waves a block, each half of a stage's columns
            if constexpr (MODE == kTileExperts) {
                // past 16 stages a ring of four (us with one wave and three buffers / two
                // and three / two and four: 16 tokens x 8 of 64 experts of 1024
                // -> 2048 32.1 / 30.9 / 32.6, of 4096 -> 2048 130.3 / 124.0 / 110.9; one
                // token 19.0 / 18.4 / 18.4)
                if (g.K > 16 * kTileStageK) MASQ_TILE_WK(32, 64, 1, 2, 4, 2, 2);
                else MASQ_TILE_WK(32, 64, 1, 2, 3, 2, 2);
            } else {
                MASQ_TILE_WK(32, 64, 1, 2, 4, 2, 2);
            }
            break;
        case 1: MASQ_TILE(64, 64, 2, 2, 3, 3); break;
        case 2: MASQ_TILE(128, 128, 2, 2, 2, 2); break;
        default: return hipErrorInvalidValue;
    }
#undef MASQ_TILE
#undef MASQ_TILE_WK
    return hipGetLastError();
}

template <int MODE>
hipError_t launch_tile_any(const TileGemm& g, const TileExtra& ex, int tiles_m) {
#define MASQ_MODE(YT, LT, CMC)                                                                      \
    (g.w4 ? launch_tile_mode<YT, LT, CMC, true, MODE>(g, ex, tiles_m)                               \
          : launch_tile_mode<YT, LT, CMC, false, MODE>(g, ex, tiles_m))
    if (!g.cmc) return g.y_dt == DT::BF16 ? MASQ_MODE(bf16_t, bf16_t, false) : MASQ_MODE(float, bf16_t, false);
    if (g.y_dt == DT::BF16)
        return g.lr_dt == DT::BF16 ? MASQ_MODE(bf16_t, bf16_t, true) : MASQ_MODE(bf16_t, float, true);
    return g.lr_dt == DT::BF16 ? MASQ_MODE(float, bf16_t, true) : MASQ_MODE(float, float, true);
#undef MASQ_MODE
}

template <typename YT, typename LT, bool W4>
hipError_t launch_stream_epi(const StreamGemm& g, const TileExtra& ex) {
    int ns = 0, sp = 0, groups = 0;
    plan_decode(g.K, g.N, ns, sp, groups);
    const int S = stream_slices(g.K, groups, ns);
    const size_t lds = g.u != nullptr ? static_cast<size_t>((g.T + S - 1) / S) * g.rank * sizeof(float)
                                      : 0;
    hipLaunchKernelGGL((k_gemm_stream<YT, LT, W4, kTileEpilogue>), dim3(static_cast<unsigned>(groups * S)),
                       dim3(kStrThreads), lds, g.stream, g.q, g.wq, g.x_scale, g.w_scale,
                       static_cast<int>(g.T), static_cast<int>(g.K), static_cast<int>(g.N), S, g.mod, g.u,
                       g.u_slices, g.rank, g.n_mod, static_cast<const LT*>(g.r_up), g.part, g.tickets,
                       static_cast<YT*>(g.y), -1, ex);
    return hipGetLastError();
}

// ================================================================ routing
// A token's experts: a wave holds its logits, lane l those of experts l, l +
// 64, ..., as unsigned keys in the order of the values (0: -inf and NaN, never
// chosen; -0 and +0 alike).  Each of the k rounds takes the largest key of the
// wave (a chain of lane shifts) and its first holder (a ballot per 64 experts),
// so ties go to the lowest index.
//
// The choices of 32 tokens leave a bit mask per expert (bit t: token t of the
// block chose it; a token never chooses one twice), which is all that sorting
// by expert needs: the count of the block is its population count, and a
// choice's place among the block's the count of the bits below its own.  So
// slots ascend with the token inside an expert, whatever order anything ran in.
//
// What bounds it is latency, not the 5.5 MB of 8192 tokens over 128 experts (1.1
// us): the rounds' chains and two launches.  8192 tokens 13.4 us (choices 8.5,
// places 5) where 16 tokens a wave, one token's logits at a time, and the counts
// summed in a launch of their own took 26.2; 4 tokens of 64 experts 3.9 in one
// launch.
constexpr int kRouteTokens = 32;
constexpr int kRouteOneTokens = 64;       // at most this many: one workgroup does it all
constexpr int kRouteOneThreads = 1024;
constexpr int kRouteChooseThreads = 1024;
constexpr int64_t kRouteFewBlocks = 256;

__device__ __forceinline__ uint32_t logit_key(float f) {
    if (!(f > -INFINITY)) return 0;                          // -inf, NaN
    const uint32_t b = __float_as_uint(f + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

// The largest of the lanes' values, in every lane: lane shifts within rows of
// 16, then the rows' last lanes onto the rows behind them.
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
#define MASQ_DPP_MAX(ctrl, rows)                                                                    \
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), ctrl, rows, 0xf, false)))
    MASQ_DPP_MAX(0x111, 0xf);                                // row_shr:1
    MASQ_DPP_MAX(0x112, 0xf);
    MASQ_DPP_MAX(0x114, 0xf);
    MASQ_DPP_MAX(0x118, 0xf);
    MASQ_DPP_MAX(0x142, 0xa);                                // row_bcast:15
    MASQ_DPP_MAX(0x143, 0xc);                                // row_bcast:31
#undef MASQ_DPP_MAX
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// The keys of token t (a wave; lane l: experts l, l + 64, ...).
template <typename LT, int C>
__device__ __forceinline__ void load_keys(const LT* __restrict__ logits, int64_t t, int E, int lane,
                                          uint32_t (&key)[C]) {
    float f[C];
#pragma unroll
    for (int c = 0; c < C; ++c) f[c] = Elem<LT>::load1(logits + t * E + min(lane + 64 * c, E - 1));
#pragma unroll
    for (int c = 0; c < C; ++c) key[c] = lane + 64 * c < E ? logit_key(f[c]) : 0;
}

// A token's choices by one wave: experts and weights to global memory, the
// experts' mask bits to masks[expert].
template <int C>
__device__ __forceinline__ void route_token(uint32_t (&key)[C], int k, bool renorm,
                                            int32_t* __restrict__ experts, float* __restrict__ weights,
                                            uint32_t* masks, int bit, int lane) {
    uint32_t all[C];                                         // as read (the rounds clear the chosen)
#pragma unroll
    for (int c = 0; c < C; ++c) all[c] = key[c];
    uint32_t top = 0, mine = 0;
    int pick = -1;                                           // lane j: choice j
    for (int j = 0; j < k; ++j) {
        uint32_t best = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) best = max(best, key[c]);
        best = wave_umax(best);
        if (best == 0) break;                                // uniform: nothing left
        if (j == 0) top = best;
        int e = -1;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const unsigned long long has = __ballot(key[c] == best);
            if (e < 0 && has != 0) {                         // uniform
                const int l = __builtin_ctzll(has);
                e = 64 * c + l;
                if (lane == l) key[c] = 0;
            }
        }
        if (lane == j) {
            pick = e;
            mine = best;
        }
    }
    const float hi = key_logit(top);
    auto prob = [&](uint32_t q) __attribute__((always_inline)) {
        return q == 0 ? 0.f : (q == top ? 1.f : expf(key_logit(q) - hi));
    };
    const float p = prob(mine);
    float part = p;
    if (!renorm) {
        part = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) part += prob(all[c]);
    }
    const float total = wave_sum(part);
    if (lane < k) {
        experts[lane] = pick;
        weights[lane] = pick >= 0 ? p / total : 0.f;
        if (pick >= 0) atomicOr(&masks[pick], 1u << bit);
    }
}

// Tokens t0 + wave, + NW, ... of the n from t0 on, the next one's logits in
// flight while one is chosen for; token i's bits go to masks row i / 32.
template <typename LT, int C, int NW>
__device__ __forceinline__ void route_tokens_c(const LT* logits, int64_t t0, int n, int E, int k,
                                               bool renorm, int32_t* experts, float* weights,
                                               uint32_t* masks, int pitch, int wave, int lane) {
    uint32_t key[C], next[C];
    if (wave < n) load_keys<LT, C>(logits, t0 + wave, E, lane, key);
    for (int i = wave; i < n; i += NW) {                     // wave-uniform
        load_keys<LT, C>(logits, t0 + min(i + NW, n - 1), E, lane, next);
        route_token<C>(key, k, renorm, experts + (t0 + i) * k, weights + (t0 + i) * k,
                       masks + (i >> 5) * pitch, i & 31, lane);
#pragma unroll
        for (int c = 0; c < C; ++c) key[c] = next[c];
    }
}
template <typename LT, int NW>
__device__ __forceinline__ void route_tokens(const LT* logits, int64_t t0, int n, int E, int k, bool renorm,
                                             int32_t* experts, float* weights, uint32_t* masks, int pitch,
                                             int wave, int lane) {
#define MASQ_TOKENS(C) route_tokens_c<LT, C, NW>(logits, t0, n, E, k, renorm, experts, weights, masks, pitch, wave, lane)
    if (E <= 64) MASQ_TOKENS(1);
    else if (E <= 128) MASQ_TOKENS(2);
    else if (E <= 256) MASQ_TOKENS(4);
    else MASQ_TOKENS(8);
#undef MASQ_TOKENS
}

// Exclusive prefix of v over the workgroup's first kRouteMaxExperts threads
// (all NT threads call; the others give 0); *total: the sum.
template <int NT>
__device__ __forceinline__ int expert_prefix(int v, int* waves, int* total, int tid) {
    const int lane = tid & 63, wave = tid >> 6;
    int s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int p = __shfl_up(s, o);
        s += lane >= o ? p : 0;
    }
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const int x = waves[w];
        before += w < wave ? x : 0;
        all += x;
    }
    *total = all;
    return before + s - v;
}

// One workgroup for the whole batch (at most kRouteOneTokens tokens).
template <typename LT>
__global__ __launch_bounds__(kRouteOneThreads) void k_route_one(
    const LT* __restrict__ logits, const int32_t* __restrict__ mod, int T, int E, int k, bool renorm,
    int32_t* __restrict__ experts, float* __restrict__ weights, int32_t* __restrict__ offsets,
    int32_t* __restrict__ rows, int32_t* __restrict__ slots, int32_t* __restrict__ slot_mod) {
    constexpr int kWords = kRouteOneTokens / 32, NW = kRouteOneThreads / 64;
    __shared__ uint32_t masks[kWords][kRouteMaxExperts];
    __shared__ int base[kRouteMaxExperts];
    __shared__ int waves[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int words = (T + 31) >> 5;
    for (int i = tid; i < words * kRouteMaxExperts; i += kRouteOneThreads) (&masks[0][0])[i] = 0;
    __syncthreads();
    route_tokens<LT, NW>(logits, 0, T, E, k, renorm, experts, weights, &masks[0][0], kRouteMaxExperts, wave, lane);
    __syncthreads();
    int cnt = 0, total;
    if (tid < E)
        for (int w = 0; w < words; ++w) cnt += __popc(masks[w][tid]);
    const int first = expert_prefix<kRouteOneThreads>(cnt, waves, &total, tid);
    if (tid < E) {
        base[tid] = first;
        offsets[tid] = first;
    }
    if (tid == 0) offsets[E] = total;
    __syncthreads();
    for (int i = tid; i < T * k; i += kRouteOneThreads) {
        const int t = i / k;
        const int e = experts[i];                            // written by this workgroup before the barrier
        int slot = -1;
        if (e >= 0) {
            slot = base[e] + __popc(masks[t >> 5][e] & ((1u << (t & 31)) - 1u));
            for (int w = 0; w < (t >> 5); ++w) slot += __popc(masks[w][e]);
            rows[slot] = t;
            if (slot_mod != nullptr) slot_mod[slot] = mod[t];
        }
        slots[i] = slot;
        if (i >= total) {                                    // past the last choice
            rows[i] = -1;
            if (slot_mod != nullptr) slot_mod[i] = 0;
        }
    }
}

// Larger batches: the choices and the masks of every 32 tokens, then their
// places.  A workgroup of the second launch counts the choices of every expert
// before its tokens and in all from the masks; where there are more than
// kRouteFewBlocks of them, whose counting again in each would cost more than
// another launch, a launch between the two leaves the sums.
template <typename LT>
__global__ __launch_bounds__(kRouteChooseThreads) void k_route_choose(
    const LT* __restrict__ logits, int64_t T, int E, int k, bool renorm, int32_t* __restrict__ experts,
    float* __restrict__ weights, uint32_t* __restrict__ masks, int pitch) {
    __shared__ uint32_t sm[kRouteMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int e = tid; e < pitch; e += kRouteChooseThreads) sm[e] = 0;
    __syncthreads();
    const int64_t t0 = linear_block() * kRouteTokens;
    if (t0 >= T) return;
    const int n = static_cast<int>(min(T - t0, static_cast<int64_t>(kRouteTokens)));
    route_tokens<LT, kRouteChooseThreads / 64>(logits, t0, n, E, k, renorm, experts, weights, sm, 0, wave, lane);
    __syncthreads();
    for (int e = tid; e < pitch; e += kRouteChooseThreads) masks[linear_block() * pitch + e] = sm[e];
}

// A workgroup per 16 experts: 64 thread rows, each over a run of blocks.
constexpr int kScanCols = 16, kScanRows = 64;
__global__ __launch_bounds__(kScanCols * kScanRows) void k_route_scan(
    const uint32_t* __restrict__ masks, int64_t blocks, int pitch, int32_t* __restrict__ before,
    int32_t* __restrict__ totals) {
    __shared__ int part[kScanRows][kScanCols];
    const int col = threadIdx.x % kScanCols, row = threadIdx.x / kScanCols;
    const int e = blockIdx.x * kScanCols + col;
    const bool in = e < pitch;
    const int64_t per = (blocks + kScanRows - 1) / kScanRows;
    const int64_t b0 = min(blocks, row * per), b1 = min(blocks, b0 + per);
    int sum = 0;
    if (in)
        for (int64_t b = b0; b < b1; ++b) sum += __popc(masks[b * pitch + e]);
    part[row][col] = sum;
    __syncthreads();
    int at = 0, all = 0;
    for (int r = 0; r < kScanRows; ++r) {
        const int x = part[r][col];
        at += r < row ? x : 0;
        all += x;
    }
    if (!in) return;
    for (int64_t b = b0; b < b1; ++b) {
        before[b * pitch + e] = at;
        at += __popc(masks[b * pitch + e]);
    }
    if (row == 0) totals[e] = all;
}

__global__ __launch_bounds__(kRouteMaxExperts) void k_route_place(
    const int32_t* __restrict__ mod, int64_t T, int E, int k, const int32_t* __restrict__ experts,
    const uint32_t* __restrict__ masks, int pitch, int64_t blocks, const int32_t* __restrict__ before,
    const int32_t* __restrict__ totals, int32_t* __restrict__ offsets, int32_t* __restrict__ rows,
    int32_t* __restrict__ slots, int32_t* __restrict__ slot_mod) {
    constexpr int NT = kRouteMaxExperts;
    __shared__ int base[NT];
    __shared__ uint32_t sm[NT];
    __shared__ int waves[NT / 64];
    __shared__ __attribute__((aligned(16))) v4i sums[2][NT];
    const int tid = threadIdx.x;
    const int64_t b = linear_block(), t0 = b * kRouteTokens;
    if (t0 >= T) return;
    int mine = 0, all = 0;                                   // of expert tid: before this block, in all
    if (before != nullptr) {
        if (tid < E) {
            mine = before[b * pitch + tid];
            all = totals[tid];
        }
    } else {
        // thread (row, 4 experts): every rows-th block's masks
        const int quads = pitch >> 2, rows_ = NT / quads, row = tid / quads, qd = tid - row * quads;
        v4i lo = {0, 0, 0, 0}, sum = {0, 0, 0, 0};
        if (row < rows_) {
#pragma unroll 8
            for (int i = row; i < static_cast<int>(blocks); i += rows_) {
                const v4i w = *reinterpret_cast<const v4i*>(masks + static_cast<int64_t>(i) * pitch + 4 * qd);
                v4i c;
#pragma unroll
                for (int j = 0; j < 4; ++j) c[j] = static_cast<int>(__popc(static_cast<uint32_t>(w[j])));
                sum += c;
                if (i < b) lo += c;
            }
        }
        sums[0][tid] = lo;
        sums[1][tid] = sum;
        __syncthreads();
        if (tid < E)
            for (int g = 0; g < rows_; ++g) {
                mine += sums[0][g * quads + (tid >> 2)][tid & 3];
                all += sums[1][g * quads + (tid >> 2)][tid & 3];
            }
    }
    int total;
    const int first = expert_prefix<NT>(all, waves, &total, tid);
    if (tid < E) {
        base[tid] = first + mine;
        sm[tid] = masks[b * pitch + tid];
        if (b == 0) offsets[tid] = first;
    }
    if (b == 0 && tid == 0) offsets[E] = total;
    __syncthreads();
    const int n = static_cast<int>(min(T - t0, static_cast<int64_t>(kRouteTokens))) * k;
    for (int i = tid; i < n; i += NT) {
        const int t = i / k;
        const int e = experts[t0 * k + i];
        int slot = -1;
        if (e >= 0) {
            slot = base[e] + __popc(sm[e] & ((1u << t) - 1u));
            rows[slot] = static_cast<int32_t>(t0 + t);
            if (slot_mod != nullptr) slot_mod[slot] = mod[t0 + t];
        }
        slots[t0 * k + i] = slot;
        if (t0 * k + i >= total) {                           // past the last choice
            rows[t0 * k + i] = -1;
            if (slot_mod != nullptr) slot_mod[t0 * k + i] = 0;
        }
    }
}

// ================================================================ stage 1 of the experts' layer
// One launch for two independent pieces of work: workgroups below `downs` form
// u = (x S_m^-1) L1_e^m for the slots of modality m != text, those past them
// quantise x's rows (a row a workgroup for small batches, where a row's latency
// counts, else a row a wave).
//
// A down-projection workgroup takes 16 RG slots of one expert and 16 RB columns
// of the rank, its eight waves an eighth of the row each, U steps of 32 columns
// in flight, and the waves' sums are added in their order.  With bf16 factors
// the smoothed row enters as a hi + lo pair of bf16 terms, as in the layer;
// with fp32 factors the fp32 MFMA takes it whole.  Each modality is summed on
// its own, so that an infinite factor stays with its modality.
constexpr int kEdWaves = 8;

struct ExpertStage1 {
    const int32_t* mod;
    const float* inv_s;
    int64_t n_slots, T;
    int K, r, n_mod;
    float* u;
    uint8_t* u_hl;
    int8_t* q;
    float* x_scale;
    int64_t downs;
    bool row_group;       // a row a workgroup
    bool pair;            // q row-paired (code_row / code_col)
    int* zero_ints;       // cleared on the way (the layer's arrival counters)
    int n_zero;
};

// A fragment's 16 rows lie a row apart in memory, so a load in the MFMA's own
// order (lane l: row l % 16, columns 8 (l / 16) ..) asks for 64 pieces of 16
// bytes, one after the other.  The loads go by lane l: row l / 4, columns
// 8 (l % 4) .. instead, 64 contiguous bytes for four lanes, and the lanes trade
// their pieces through the LDS crossbar (32768 slots, half of them text, 2048
// columns, rank 32: 44 -> 40 us).
//
// The tile's slots of one modality come side by side first (a list in LDS), so
// that a group of 16 MFMA columns holds slots that count: a tile of which half
// is text costs half the loads and products.  A column's sums depend on its own
// row only, so the columns past the last slot may hold anything.
__device__ __forceinline__ v4i to_fragment(v4i v, int from) {
    return v4i{__builtin_amdgcn_ds_bpermute(from, v.x), __builtin_amdgcn_ds_bpermute(from, v.y),
               __builtin_amdgcn_ds_bpermute(from, v.z), __builtin_amdgcn_ds_bpermute(from, v.w)};
}
__device__ __forceinline__ void to_fragment(Raw8<bf16_t>& v, int from) { v.a = to_fragment(v.a, from); }
__device__ __forceinline__ void to_fragment(Raw8<float>& v, int from) {
    v.a = __builtin_bit_cast(v4f, to_fragment(__builtin_bit_cast(v4i, v.a), from));
    v.b = __builtin_bit_cast(v4f, to_fragment(__builtin_bit_cast(v4i, v.b), from));
}

template <typename XT, typename LT, int RG, int RB, int U>
__device__ __forceinline__ void expert_down_tile(const XT* __restrict__ x, const LT* __restrict__ l_down,
                                                 const ExpertStage1& a, const TileExtra& ex,
                                                 v4f (&red)[kEdWaves][RG * RB * 64], int (&list)[64]) {
    static_assert(RG <= 4, "a lane per slot");
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int K = a.K, r = a.r;
    const int chunks = (r + 16 * RB - 1) / (16 * RB);
    GroupTile gt;
    if (ex.offsets == nullptr) {                             // one expert of all slots
        const int64_t b = linear_block();
        gt.expert = 0;
        gt.tn = static_cast<int>(b % chunks);
        gt.first = b / chunks * (16 * RG);
        gt.end = min(gt.first + 16 * RG, a.n_slots);
        if (gt.first >= a.n_slots) return;
    } else if (!group_tile<16 * RG>(ex, a.n_slots, linear_block(), chunks, gt)) {
        return;
    }
    const int c0 = gt.tn * 16 * RB;
    const int nb = min(RB, (r - c0) >> 4);                   // 16-column blocks of the rank
    const int steps = (K + 31) >> 5, per = (steps + kEdWaves - 1) / kEdWaves;
    const int st0 = wave * per, st1 = min(steps, st0 + per);
    const int from = 4 * (4 * (lane & 15) + (lane >> 4));    // whose piece is this lane's (byte index)
    const int count = static_cast<int>(gt.end - gt.first);
    // lane l: slot l of the tile
    const int row_l = static_cast<int>(slot_row(ex, min(gt.first + lane, gt.end - 1)));
    const int md_l = lane < count ? sane_mod(a.mod[row_l], a.n_mod) : 0;
    for (int m = 1; m < a.n_mod; ++m) {
        const unsigned long long mask = __ballot(md_l == m);
        if (mask == 0ull) continue;                          // the same in every wave
        const int n = __builtin_popcountll(mask);
        if (wave == 0 && md_l == m) list[__builtin_popcountll(mask & ((1ull << lane) - 1ull))] = lane;
        __syncthreads();
        const LT* lm = l_down + (static_cast<int64_t>(gt.expert) * (a.n_mod - 1) + m - 1) * r * K;
        const float* im = a.inv_s + static_cast<int64_t>(m) * K;
        const XT* xp[RG];
#pragma unroll
        for (int g = 0; g < RG; ++g)                         // (places past n repeat the last slot)
            xp[g] = x + static_cast<int64_t>(__shfl(row_l, list[min(16 * g + (lane >> 2), n - 1)])) * K;
        v4f acc[RG][RB];
#pragma unroll
        for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int b = 0; b < RB; ++b) acc[g][b] = v4f{0.f, 0.f, 0.f, 0.f};
        // CNT steps from s0 on; TAIL: the last ones, which may end inside a step
        auto run = [&](int s0, auto cnt, auto tail) __attribute__((always_inline)) {
            constexpr int CNT = decltype(cnt)::value;
            constexpr bool TAIL = decltype(tail)::value;
            Raw8<LT> lv[CNT][RB];
            Raw8<XT> xv[CNT][RG];
            Raw8<float> sv[CNT];
            bool in[CNT];
#pragma unroll
            for (int i = 0; i < CNT; ++i) {
                const int kf = 32 * (s0 + i) + 8 * (lane >> 4), kl = 32 * (s0 + i) + 8 * (lane & 3);
                in[i] = !TAIL || kf < K;                     // K % 16 == 0: 8 columns in or out together
                const int kc = TAIL ? min(kl, K - 8) : kl;
#pragma unroll
                for (int b = 0; b < RB; ++b)
                    lv[i][b].load(lm + static_cast<int64_t>(c0 + 16 * min(b, nb - 1) + (lane >> 2)) * K + kc);
                sv[i].load(im + (TAIL ? min(kf, K - 8) : kf));
#pragma unroll
                for (int g = 0; g < RG; ++g)
                    if (16 * g < n) xv[i][g].load(xp[g] + kc);               // uniform
            }
#pragma unroll
            for (int i = 0; i < CNT; ++i) {
                float sm[8];
                sv[i].to_f32(sm);
#pragma unroll
                for (int b = 0; b < RB; ++b) to_fragment(lv[i][b], from);
#pragma unroll
                for (int g = 0; g < RG; ++g) {
                    if (16 * g >= n) break;                  // uniform
                    float xs[8];
                    to_fragment(xv[i][g], from);
                    xv[i][g].to_f32(xs);
#pragma unroll
                    for (int e = 0; e < 8; ++e) xs[e] = in[i] ? xs[e] * sm[e] : 0.f;
                    if constexpr (sizeof(LT) == 2) {
                        const v4i zero = {0, 0, 0, 0};
                        v4i hi, lo;
                        split_bf16x8(xs, hi, lo);
#pragma unroll
                        for (int b = 0; b < RB; ++b) {
                            const v8bf w = __builtin_bit_cast(v8bf, in[i] ? lv[i][b].a : zero);
                            acc[g][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(v8bf, hi), acc[g][b], 0, 0, 0);
                            acc[g][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(v8bf, lo), acc[g][b], 0, 0, 0);
                        }
                    } else {
#pragma unroll
                        for (int b = 0; b < RB; ++b) {
                            float w[8];
                            lv[i][b].to_f32(w);
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                acc[g][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(in[i] ? w[e] : 0.f, xs[e], acc[g][b], 0, 0, 0);
                        }
                    }
                }
            }
        };
        int s0 = st0;
        const int full = min(st1, K >> 5);                   // steps of 32 whole columns
        for (; s0 + U <= full; s0 += U) run(s0, std::integral_constant<int, U>{}, std::false_type{});
        for (; s0 < st1; ++s0) run(s0, std::integral_constant<int, 1>{}, std::true_type{});
#pragma unroll
        for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int b = 0; b < RB; ++b) red[wave][(g * RB + b) * 64 + lane] = acc[g][b];
        __syncthreads();
        // item 64 (RB g + b) + lane: columns 4 (lane / 16) .. of place 16 g + lane % 16
#pragma unroll
        for (int it = wave; it < RG * RB; it += kEdWaves) {
            const int g = it / RB, b = it % RB, j = 16 * g + (lane & 15);
            v4f v = red[0][it * 64 + lane];
#pragma unroll
            for (int w = 1; w < kEdWaves; ++w) v = v + red[w][it * 64 + lane];
            if (b >= nb || j >= n) continue;
            const int64_t slot = gt.first + list[j];
            const int c = c0 + 16 * b + 4 * (lane >> 4);
            *reinterpret_cast<v4f*>(a.u + slot * r + c) = v;
            if (a.u_hl == nullptr) continue;                 // rank <= 64: also as bf16 hi | lo
            uint8_t* p = a.u_hl + slot * 256 + 2 * c;
            const uint32_t h0 = pack_bf16x2(v.x, v.y), h1 = pack_bf16x2(v.z, v.w);
            const uint32_t l0 = pack_bf16x2(v.x - __uint_as_float(h0 << 16), v.y - __uint_as_float(h0 & 0xFFFF0000u));
            const uint32_t l1 = pack_bf16x2(v.z - __uint_as_float(h1 << 16), v.w - __uint_as_float(h1 & 0xFFFF0000u));
            *reinterpret_cast<v2i*>(p) = v2i{static_cast<int32_t>(h0), static_cast<int32_t>(h1)};
            *reinterpret_cast<v2i*>(p + 128) = v2i{static_cast<int32_t>(l0), static_cast<int32_t>(l1)};
        }
        __syncthreads();                                     // red and list are free for the next modality
    }
}

template <typename XT, typename LT, int RG, int RB, int U>
__global__ __launch_bounds__(64 * kEdWaves, 4) void k_expert_stage1(const XT* __restrict__ x,
                                                                 const LT* __restrict__ l_down,
                                                                 ExpertStage1 a, TileExtra ex) {
    __shared__ __attribute__((aligned(16))) v4f red[kEdWaves][RG * RB * 64];
    __shared__ int list[64];
    const int64_t b = linear_block() - a.downs;
    if (b == 0)
        for (int i = threadIdx.x; i < a.n_zero; i += 64 * kEdWaves) a.zero_ints[i] = 0;
    if (b < 0) {
        expert_down_tile<XT, LT, RG, RB, U>(x, l_down, a, ex, red, list);
    } else if (a.row_group) {
        if (b < a.T) sq_row<XT, 64 * kEdWaves, 2>(x, a.mod, a.inv_s, a.K, a.n_mod, a.q, a.x_scale, b, a.pair);
    } else {
        const int64_t t = b * kEdWaves + (threadIdx.x >> 6);
        if (t < a.T)
            quant_row_wave<XT, 4>(x, a.mod, a.inv_s, a.K, a.n_mod, a.q, a.x_scale, t, a.pair, threadIdx.x & 63,
                                  [](int) {});
    }
}

// ================================================================ combination
// y[t] = residual[t] + sum over j of weights[t][j] d[slots[t][j]], in fp32 in
// the order of j, rounded once.  8 columns a thread; a token's rows are read
// together (KB loads in flight).  A slot outside [0, n_slots) adds nothing.  Bound
// by its bytes: 4096 x 8 rows of 2048 in bf16, 160 MB, 34 us (4.7 TB/s; a large
// device copy moves 5.0).
template <typename DTy, int KB>
__global__ __launch_bounds__(256) void k_combine(const DTy* __restrict__ d,
                                                 const int32_t* __restrict__ slots,
                                                 const float* __restrict__ weights, int64_t T,
                                                 int64_t n_slots, int N, int k,
                                                 const DTy* residual, DTy* y) {
    const int per_row = N >> 3;
    const int64_t i = linear_block() * 256 + threadIdx.x;
    if (i >= T * per_row) return;
    const int64_t t = i / per_row;
    const int o = static_cast<int>(i - t * per_row) * 8;
    float v[8] = {};
    for (int j0 = 0; j0 < k; j0 += KB) {
        Raw8<DTy> raw[KB];
        float w[KB];
        bool in[KB];
#pragma unroll
        for (int j = 0; j < KB; ++j) {
            const int64_t at = t * k + min(j0 + j, k - 1);
            const int64_t s = slots[at];
            in[j] = j0 + j < k && s >= 0 && s < n_slots;
            w[j] = weights[at];
            if (in[j]) raw[j].load(d + s * N + o);
        }
#pragma unroll
        for (int j = 0; j < KB; ++j) {
            if (!in[j]) continue;
            float f[8];
            raw[j].to_f32(f);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(w[j], f[e], v[e]);
        }
    }
    if (residual != nullptr) {
        float q[8];
        Elem<DTy>::load8(residual + t * N + o, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += q[e];
    }
    store8(y + t * N + o, v);
}

}  // namespace

// ================================================================ launchers
hipError_t launch_gemm_tile_epilogue(const TileGemm& g, const TileExtra& ex) {
    if (g.K % 16 != 0 || g.N % (ex.gated ? 32 : 16) != 0 || g.plan.S < 1 || (g.w4 && g.K % 64 != 0) ||
        (g.a_pair && g.K % 64 != 0) || (g.plan.S > 1 && (g.part == nullptr || g.tickets == nullptr)) ||
        g.plan.shape < 0 || g.acc != nullptr)
        return hipErrorInvalidValue;
    const int bm = kTileShapes[g.plan.shape].bm;
    return launch_tile_any<kTileEpilogue>(g, ex, static_cast<int>((g.T + bm - 1) / bm));
}

hipError_t launch_gemm_stream_epilogue(const StreamGemm& g, const TileExtra& ex) {
    if (!small_path(g.T, g.K) || g.N % (ex.gated ? 32 : 16) != 0 || g.part == nullptr ||
        g.tickets == nullptr || g.only_mod >= 0)
        return hipErrorInvalidValue;
#define MASQ_STREAM(YT, LT) (g.w4 ? launch_stream_epi<YT, LT, true>(g, ex) : launch_stream_epi<YT, LT, false>(g, ex))
    if (g.y_dt == DT::BF16) return g.lr_dt == DT::BF16 ? MASQ_STREAM(bf16_t, bf16_t) : MASQ_STREAM(bf16_t, float);
    return g.lr_dt == DT::BF16 ? MASQ_STREAM(float, bf16_t) : MASQ_STREAM(float, float);
#undef MASQ_STREAM
}

hipError_t launch_gemm_experts(const TileGemm& g, const TileExtra& ex) {
    if (g.K % 16 != 0 || g.N % (ex.gated ? 32 : 16) != 0 || g.plan.S != 1 || (g.w4 && g.K % 64 != 0) ||
        g.a_pair || g.plan.shape < 0 || g.acc != nullptr)
        return hipErrorInvalidValue;
    return launch_tile_any<kTileExperts>(
        g, ex, static_cast<int>(expert_tiles(g.T, ex.n_experts, kTileShapes[g.plan.shape].bm)));
}

// Slots of a down-projection workgroup: 16 while that makes at most two
// workgroups a compute unit, 32 up to four, else 64 where the rank leaves the
// registers for it (L1 is read once a workgroup).
template <typename XT, typename LT, int RB>
static hipError_t launch_stage1_t(const void* x, const void* l_down, ExpertStage1 a, const TileExtra& ex,
                                  hipStream_t s) {
    const int64_t quant = a.row_group ? a.T : (a.T + kEdWaves - 1) / kEdWaves;
    const int chunks = (a.r + 16 * RB - 1) / (16 * RB);
    const int64_t most = expert_tiles(a.n_slots, ex.n_experts, 16) * chunks;
#define MASQ_STAGE1(RG, U)                                                                          \
    do {                                                                                            \
        a.downs = 8 * ((expert_tiles(a.n_slots, ex.n_experts, 16 * RG) * chunks + 7) / 8);          \
        hipLaunchKernelGGL((k_expert_stage1<XT, LT, RG, RB, U>), grid_of(a.downs + quant, 64 * kEdWaves), \
                           dim3(64 * kEdWaves), 0, s, static_cast<const XT*>(x),                    \
                           static_cast<const LT*>(l_down), a, ex);                                  \
    } while (0)
    constexpr bool kNarrow = sizeof(XT) == 2 && sizeof(LT) == 2;
    if (most <= 512) MASQ_STAGE1(1, (kNarrow ? 4 : 2));
    else if (most <= 1024 || RB > 2) MASQ_STAGE1(2, (kNarrow ? 2 : 1));
    else MASQ_STAGE1((RB > 2 ? 2 : 4), (kNarrow ? 2 : 1));
#undef MASQ_STAGE1
    return hipGetLastError();
}

hipError_t launch_expert_stage1(const void* x, DT x_dt, const int32_t* mod, const float* inv_s,
                                const void* l_down, DT lr_dt, int64_t T, int64_t n_slots, int64_t K,
                                int rank, int n_mod, float* u, uint8_t* u_hl, int8_t* q, float* x_scale,
                                const TileExtra& ex, bool pair, hipStream_t s, int* zero_ints,
                                int n_zero) {
    ExpertStage1 a{mod, inv_s, n_slots, T, static_cast<int>(K), rank, n_mod, u, u_hl, q, x_scale, 0,
                   T < kRowsPerWaveMinT, pair, zero_ints, n_zero};
#define MASQ_RB(XT, LT)                                                                             \
    (rank <= 16 ? launch_stage1_t<XT, LT, 1>(x, l_down, a, ex, s)                                   \
                : (rank <= 32 ? launch_stage1_t<XT, LT, 2>(x, l_down, a, ex, s)                     \
                              : launch_stage1_t<XT, LT, 4>(x, l_down, a, ex, s)))
    if (x_dt == DT::BF16) return lr_dt == DT::BF16 ? MASQ_RB(bf16_t, bf16_t) : MASQ_RB(bf16_t, float);
    return lr_dt == DT::BF16 ? MASQ_RB(float, bf16_t) : MASQ_RB(float, float);
#undef MASQ_RB
}

hipError_t launch_route(const void* logits, DT dt, const int32_t* mod, int64_t T, int E, int k,
                        bool renorm, int32_t* experts, float* weights, int32_t* offsets,
                        int32_t* rows, int32_t* slots, int32_t* slot_mod, const RouteWs& w,
                        hipStream_t s) {
    if (w.blocks == 0) {                                     // plan_route: one workgroup
#define MASQ_ROUTE(LT)                                                                              \
    hipLaunchKernelGGL(k_route_one<LT>, dim3(1), dim3(kRouteOneThreads), 0, s,                      \
                       static_cast<const LT*>(logits), mod, static_cast<int>(T), E, k, renorm,      \
                       experts, weights, offsets, rows, slots, slot_mod)
        if (dt == DT::BF16) MASQ_ROUTE(bf16_t);
        else MASQ_ROUTE(float);
#undef MASQ_ROUTE
        return hipGetLastError();
    }
    const int pitch = route_pitch(E);
    const dim3 grid = grid_of(w.blocks, kRouteChooseThreads);
#define MASQ_ROUTE(LT)                                                                              \
    hipLaunchKernelGGL(k_route_choose<LT>, grid, dim3(kRouteChooseThreads), 0, s,                   \
                       static_cast<const LT*>(logits), T, E, k, renorm, experts, weights, w.masks, pitch)
    if (dt == DT::BF16) MASQ_ROUTE(bf16_t);
    else MASQ_ROUTE(float);
#undef MASQ_ROUTE
    if (w.before != nullptr)
        hipLaunchKernelGGL(k_route_scan, dim3(static_cast<unsigned>((pitch + kScanCols - 1) / kScanCols)),
                           dim3(kScanCols * kScanRows), 0, s, w.masks, w.blocks, pitch, w.before, w.totals);
    hipLaunchKernelGGL(k_route_place, grid_of(w.blocks, kRouteMaxExperts), dim3(kRouteMaxExperts), 0, s,
                       mod, T, E, k, experts, w.masks, pitch, w.blocks, w.before, w.totals, offsets, rows,
                       slots, slot_mod);
    return hipGetLastError();
}

RouteWs plan_route(void* base, int64_t T, int E) {
    RouteWs w{};
    if (T <= kRouteOneTokens) return w;
    w.blocks = (T + kRouteTokens - 1) / kRouteTokens;
    const size_t table = (static_cast<size_t>(w.blocks) * route_pitch(E) * 4 + 255) / 256 * 256;
    const bool scan = w.blocks > kRouteFewBlocks;
    uint8_t* b = static_cast<uint8_t*>(base);
    if (b != nullptr) {
        w.masks = reinterpret_cast<uint32_t*>(b);
        if (scan) {
            w.before = reinterpret_cast<int32_t*>(b + table);
            w.totals = reinterpret_cast<int32_t*>(b + 2 * table);
        }
    }
    w.bytes = scan ? 2 * table + (static_cast<size_t>(route_pitch(E)) * 4 + 255) / 256 * 256 : table;
    return w;
}

hipError_t launch_combine(const void* d, DT dt, const int32_t* slots, const float* weights, int64_t T,
                          int64_t n_slots, int64_t N, int k, const void* residual, void* y,
                          hipStream_t s) {
    const dim3 grid = grid_of((T * (N / 8) + 255) / 256, 256);
#define MASQ_COMBINE(DTy, KB)                                                                       \
    hipLaunchKernelGGL((k_combine<DTy, KB>), grid, dim3(256), 0, s, static_cast<const DTy*>(d), slots, \
                       weights, T, n_slots, static_cast<int>(N), k,                                 \
                       static_cast<const DTy*>(residual), static_cast<DTy*>(y))
    if (dt == DT::BF16) {
        if (k > 4) MASQ_COMBINE(bf16_t, 8);
        else MASQ_COMBINE(bf16_t, 4);
    } else {
        MASQ_COMBINE(float, 4);
    }
#undef MASQ_COMBINE
    return hipGetLastError();
}

}  // namespace masq
