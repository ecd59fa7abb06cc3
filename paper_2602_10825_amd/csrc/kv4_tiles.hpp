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

// The partials of every 32-row unit -> out and lse, as attend_merge_kernel does it but for few rows: a thread has four columns of
// one row and PER of its ranges, every G-th, whose partials, maxima and sums it asks for at once; the G threads of a column put theirs
// together in LDS.  (All ranges in one thread, 32 of them unrolled: the loads and the code itself, fetched once per launch, take
// longer, 12 x 128, one row on 61201 keys in 20 ranges 6.4 us instead of 4.0; attend_merge_kernel 15.)
constexpr int kMergeThreads = 256;
template <int D, int G>
struct MergeShape {
    static constexpr int TPR = D / 4, RPB = kMergeThreads / (TPR * G), BPU = kUnitRows / RPB;   // threads per row and group, rows per block, blocks per unit
};
template <typename T, int D, int PER, int G>
__global__ __launch_bounds__(kMergeThreads) void merge4_kernel(FcAttendArgs a, FcAttendPlan p, const float* parts) {
    constexpr int TPR = MergeShape<D, G>::TPR, RPB = MergeShape<D, G>::RPB, BPU = MergeShape<D, G>::BPU;
    __shared__ __attribute__((aligned(16))) float4 acc_s[G][RPB][TPR];
    __shared__ float m_s[G][RPB], l_s[G][RPB];
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
    const int row = threadIdx.x / (TPR * G), g = threadIdx.x / TPR % G, c = threadIdx.x % TPR;
    const float4* src = reinterpret_cast<const float4*>(parts + ((int64_t)unit * S * kUnitRows + row0 + row) * D) + c;
    const float* ml = parts + (int64_t)p.parts * kUnitRows * D + (int64_t)unit * S * 2 * kUnitRows + row0 + row;
    float4 v[PER];
    float m[PER], l_of[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int s = g + e * G < S ? g + e * G : S - 1;
        v[e] = src[(int64_t)s * (kUnitRows * D / 4)];
        m[e] = ml[s * 2 * kUnitRows];
        l_of[e] = ml[(s * 2 + 1) * kUnitRows];
    }
    float mt = kNegBig, l = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) mt = fmaxf(mt, m[e]);       // (the last range's, again, where there is none)
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float4& x, float lx, float f) {
        l = fmaf(lx, f, l);
        acc.x = fmaf(x.x, f, acc.x); acc.y = fmaf(x.y, f, acc.y); acc.z = fmaf(x.z, f, acc.z); acc.w = fmaf(x.w, f, acc.w);
    };
#pragma unroll
    for (int e = 0; e < PER; ++e) {                            // (... and nothing there: it may hold infinities, so no factor of zero)
        const bool there = g + e * G < S;
        const float4 x = there ? v[e] : make_float4(0.f, 0.f, 0.f, 0.f);
        add(x, there ? l_of[e] : 0.f, __builtin_amdgcn_exp2f(m[e] - mt));
    }
    if (G > 1) {
        acc_s[g][row][c] = acc;
        if (c == 0) { m_s[g][row] = mt; l_s[g][row] = l; }
        __syncthreads();
        if (g > 0) return;
#pragma unroll
        for (int o = 1; o < G; ++o) mt = fmaxf(mt, m_s[o][row]);
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
#pragma unroll
        for (int o = 0; o < G; ++o) add(acc_s[o][row][c], l_s[o][row], __builtin_amdgcn_exp2f(m_s[o][row] - mt));
    }
    if (first_row + row >= a.L_c) return;
    const float inv = 1.0f / l;
    const int64_t grow = (int64_t)r * a.L_c + first_row + row;
    store_out((T*)a.out + (grow * a.H_q + h) * D + 4 * c, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (a.lse && c == 0) a.lse[(int64_t)h * a.A * a.L_c + grow] = (mt + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D, int PER, int G>
void merge4(const FcAttendArgs& a, const FcAttendPlan& p, hipStream_t s) {
    merge4_kernel<T, D, PER, G><<<p.merge_grid * MergeShape<D, G>::BPU, kMergeThreads, 0, s>>>(a, p, (const float*)a.ws);
}
template <typename T, int D>
int launch_merge4(const FcAttendArgs& a, const FcAttendPlan& p, hipStream_t s) {
    if (p.merge_grid == 0) return FC_OK;
    int most = 1;
    for (int R = 0; R < a.A; ++R) most = p.splits[R] > most ? p.splits[R] : most;
    static_assert(kMaxSplits <= 32, "8 ranges for each of 4 threads");
    if (most <= 4) merge4<T, D, 4, 1>(a, p, s);
    else if (most <= 12) merge4<T, D, 3, 4>(a, p, s);
    else merge4<T, D, 8, 4>(a, p, s);
    FC_LAUNCH_CHECK();
    return FC_OK;
}

}  // namespace
