// 32-key tiles of a clean region in 4 bits, a wavefront's own, and the merge: what the 32-row attention bodies share
// (attend_kv4.hip, attend_kv4_f32.hip).
#pragma once

#include "attend_split.hpp"
#include "kv4.hpp"

// A head's rows: the codes of K and of V, how far behind them their scales are, the rows and their tiles.
struct FcCodesHead { const uint8_t *k, *v; int64_t to_scales; int L_clean, tiles; };

// One tile in registers: a lane has half a row of K and of V (row l32, half hh), W blocks of 32 codes with a scale each.  Step st of
// a contraction over the row's D elements is taken over elements hh D / 2 + 8 st .. + 8, so that a lane's codes are its operand.
template <int D>
struct FcCodes {
    static constexpr int W = D / 64;
    u32x4_native k[W], v[W];
    uint32_t ks, vs;
    __device__ __forceinline__ void fetch(const FcCodesHead& h, int tile, int l32, int hh) {
        tile = tile < h.tiles ? tile : h.tiles - 1;      // (past the end: fetched again, never used)
        const int left = h.L_clean - tile * 32 - 1;      // rows past the end: the last one
        const uint32_t row = (uint32_t)(l32 < left ? l32 : left);
        const uint8_t *kt = h.k + (int64_t)tile * (16 * D), *vt = h.v + (int64_t)tile * (16 * D);
        const uint8_t *kst = h.k + h.to_scales + (int64_t)tile * D, *vst = h.v + h.to_scales + (int64_t)tile * D;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            k[i] = *reinterpret_cast<const u32x4_native*>(kt + (row * (D / 2) + hh * (D / 4) + 16 * i));
            v[i] = *reinterpret_cast<const u32x4_native*>(vt + (row * (D / 2) + hh * (D / 4) + 16 * i));
        }
        const uint32_t at = row * (D / 32) + hh * W;
        if constexpr (W == 2) {
            ks = *reinterpret_cast<const uint16_t*>(kst + at);
            vs = *reinterpret_cast<const uint16_t*>(vst + at);
        } else {
            ks = kst[at];
            vs = vst[at];
        }
    }
    // eight bf16 values: elements hh D / 2 + 8 st .. + 8 of the lane's row
    __device__ __forceinline__ u32x4_native key(int st) const { return fc_kv4_to_bf16(k[st >> 2][st & 3], W == 1 ? ks : (ks >> (8 * (st >> 2))) & 255u); }
    __device__ __forceinline__ u32x4_native value(int st) const { return fc_kv4_to_bf16(v[st >> 2][st & 3], W == 1 ? vs : (vs >> (8 * (st >> 2))) & 255u); }
};

// V's tile in LDS as bf16 rows of D elements without padding: the place of 16-byte piece `piece` of row `row`.  Rows are 256
// bytes, all banks (128, half of them).  For one piece of both half rows, 8 neighbouring rows have 16 different places, and so have
// 16 rows for one half; an aligned pair of pieces of 8 neighbouring rows has 8 different pairs of places.  Row + 8 exchanges the
// two of a pair.
template <int D>
__device__ __forceinline__ int fc_swapped(int row, int piece) {
    const int b2 = (row >> 2) & 1, b3 = (row >> 3) & 1;
    return piece ^ (D == 128 ? ((row & 3) << 1 | (b2 << 3)) : ((row & 3) ^ b2) << 1) ^ b2 ^ b3;
}

namespace {

// The S <= MOST partials of every 32-row unit -> out and lse, as attend_merge_kernel does it but for few rows: a thread has four
// columns of one row, the factors of a row are computed once, and all of a row's partials are asked for at once, before those
// (12 x 128, one row on 61201 keys in 20 ranges 15.2 -> 6.4 us; 256 rows on 49201 in 20 ranges 17.9 -> 10.6).
constexpr int kMergeThreads = 256;
template <int D>
struct MergeShape {
    static constexpr int TPR = D / 4, RPB = kMergeThreads / TPR, BPU = kUnitRows / RPB;   // threads per row, rows per block, blocks per unit
};
template <typename T, int D, int MOST>
__global__ __launch_bounds__(kMergeThreads) void merge4_kernel(FcAttendArgs a, FcAttendPlan p, const float* parts) {
    constexpr int TPR = MergeShape<D>::TPR, RPB = MergeShape<D>::RPB, BPU = MergeShape<D>::BPU;
    __shared__ float m_s[MOST][RPB], l_s[MOST][RPB];
    const uint32_t valid = valid_blocks(a);
    const int R = __popc(valid);
    if (R == 0) return;
    const int S = p.splits[R - 1];
    if (S == 1) return;
    const int unit = blockIdx.x / BPU, row0 = blockIdx.x % BPU * RPB;
    int tile, r, h;
    if (!merge_unit(a, p, valid, R, S, unit, tile, r, h)) return;
    const int first_row = tile * kUnitRows + row0;
    if (first_row >= a.L_c) return;
    const int row = threadIdx.x / TPR, c0 = threadIdx.x % TPR * 4;
    const float4* src = reinterpret_cast<const float4*>(parts + ((int64_t)unit * S * kUnitRows + row0 + row) * D + c0);
    float4 v[MOST];
#pragma unroll
    for (int s = 0; s < MOST; ++s) v[s] = src[(int64_t)(s < S ? s : S - 1) * (kUnitRows * D / 4)];
    const float* ml = parts + (int64_t)p.parts * kUnitRows * D + (int64_t)unit * S * 2 * kUnitRows + row0;
    for (int i = threadIdx.x; i < S * RPB; i += kMergeThreads) {
        m_s[i / RPB][i % RPB] = ml[i / RPB * 2 * kUnitRows + i % RPB];
        l_s[i / RPB][i % RPB] = ml[(i / RPB * 2 + 1) * kUnitRows + i % RPB];
    }
    __syncthreads();
    float mt = kNegBig;
#pragma unroll
    for (int s = 0; s < MOST; ++s) mt = fmaxf(mt, s < S ? m_s[s][row] : kNegBig);
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
#pragma unroll
    for (int s = 0; s < MOST; ++s) {
        const float f = s < S ? __builtin_amdgcn_exp2f(m_s[s][row] - mt) : 0.f;
        l = fmaf(s < S ? l_s[s][row] : 0.f, f, l);
        acc[0] = fmaf(v[s].x, f, acc[0]);
        acc[1] = fmaf(v[s].y, f, acc[1]);
        acc[2] = fmaf(v[s].z, f, acc[2]);
        acc[3] = fmaf(v[s].w, f, acc[3]);
    }
    if (first_row + row >= a.L_c) return;
    const float inv = 1.0f / l;
    const int64_t grow = (int64_t)r * a.L_c + first_row + row;
    store_out((T*)a.out + (grow * a.H_q + h) * D + c0, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    if (a.lse && c0 == 0) a.lse[(int64_t)h * a.A * a.L_c + grow] = (mt + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D>
int launch_merge4(const FcAttendArgs& a, const FcAttendPlan& p, hipStream_t s) {
    if (p.merge_grid == 0) return FC_OK;
    const dim3 grid(p.merge_grid * MergeShape<D>::BPU);
    int most = 1;
    for (int R = 0; R < a.A; ++R) most = p.splits[R] > most ? p.splits[R] : most;
    if (most <= 4) merge4_kernel<T, D, 4><<<grid, kMergeThreads, 0, s>>>(a, p, (const float*)a.ws);
    else if (most <= 12) merge4_kernel<T, D, 12><<<grid, kMergeThreads, 0, s>>>(a, p, (const float*)a.ws);
    else merge4_kernel<T, D, kMaxSplits><<<grid, kMergeThreads, 0, s>>>(a, p, (const float*)a.ws);
    FC_LAUNCH_CHECK();
    return FC_OK;
}

}  // namespace
